// What the products of the gated feed-forward blocks share (esp_ff_gemm.cu; esp_ff_vec.cu for single rows): bounded waits,
// operand descriptors, activations, tensor maps.
#pragma once

#include <type_traits>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "esp_ff_tiles.cuh"
#include "esp_tcgen.cuh"

namespace esp_moe_impl {

namespace {

// ---- waits, by the barrier's scope: one at which this CTA's copies, MMAs and threads arrive, or at which another CTA's
// warps hand tensor memory back (both sides relaxed at cluster scope: the tcgen05 fences around them order it).
enum Scope { OWN, HANDBACK };

template <int SCOPE>
__device__ __forceinline__ bool phase_done(uint32_t bar, uint32_t parity)
{
    uint32_t done;
    if (SCOPE == OWN)
        asm volatile(
            "{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.relaxed.cluster.shared::cta.b64 p, [%1], %2;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    return done != 0;
}

// Waits for at most `ms` milliseconds of the GPU's timer, which is read once in 256 polls.
template <int SCOPE>
__device__ __forceinline__ bool wait_ms(uint32_t bar, uint32_t parity, uint32_t ms, volatile int *dead)
{
    uint64_t end = 0;
    for (;;) {
        for (int i = 0; i < 256; ++i)
            if (phase_done<SCOPE>(bar, parity))
                return true;
        if (dead && *dead)
            return false;
        const uint64_t now = global_ns();
        if (end == 0)
            end = now + (uint64_t)ms * 1000000ull;
        else if (now >= end)
            return false;
    }
}

// Bounded wait of a whole warp; one that runs out ends the CTA's other waits and sets the error word.
template <int SCOPE = OWN>
__device__ __forceinline__ bool wait_phase(uint32_t bar, uint32_t parity, const GemmParams &p, volatile int *dead)
{
    bool ok = phase_done<SCOPE>(bar, parity) || wait_ms<SCOPE>(bar, parity, p.wait_ms, dead);
    ok = __all_sync(0xffffffffu, ok);
    if (!ok) {
        *dead = 1;
        *static_cast<volatile unsigned int *>(p.err) = 1u;   // in host memory
    }
    return ok;
}

__device__ __forceinline__ void arrive_relaxed(uint32_t cluster_addr)
{
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}

// Operand descriptors (version 1 in bits 46-47, 128-byte swizzle in bits 61-63). K-major: groups of 8 rows 1024 bytes
// apart; an MMA's 16 inner elements are 32 bytes. MN-major: 64 outer elements a row, the next 64 a half tile further
// (leading offset), groups of 8 inner indices 1024 bytes apart; 16 inner indices are 2048 bytes.
template <bool MN>
__device__ __forceinline__ uint64_t operand(uint32_t addr)
{
    return (uint64_t)((addr >> 4) & 0x3fffu) | ((uint64_t)(MN ? kHalfTile >> 4 : 1) << 16) |
           ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}

template <bool MN>
constexpr int kOperandStep = (MN ? 2048 : 32) >> 4;

// ---- activations: a = act(g), d = act'(g). The fast exponential's error (2 ulp and |x| 2^-24) and division (2 ulp) are
// far below the one rounding to 16 bits that follows.
__device__ __forceinline__ float logistic(float g)
{
    return __fdividef(1.0f, 1.0f + __expf(-g));
}

// The normal distribution's c = (1 + erf(g / sqrt 2)) / 2, and e = exp(-g^2 / 2), which its slope needs too. With x = |g| / sqrt 2
// and t = 1 / (1 + 0.42 x): erfc(x) = t Q(t) exp(-x^2), Q of degree 7 fitted by least squares whose weights are raised where
// the relative error over x < 6.5 is greatest, until it is even (4e-8; with the arithmetic 1.2e-6 down to g = -6 and 2e-7
// absolute). 1801 rows of 5 experts, 2056 x 1000: hidden rows, and the gradients of g and u, take 3 us less each than with erff.
__device__ __forceinline__ float normal(float g, float &e)
{
    const float t = __fdividef(1.0f, 1.0f + 0.29698485f * fabsf(g));
    e = __expf(-0.5f * g * g);
    float q = 0.0380021187f;
    q = fmaf(q, t, -0.172525816f);
    q = fmaf(q, t, 0.242480139f);
    q = fmaf(q, t, -0.0865336997f);
    q = fmaf(q, t, 0.146210648f);
    q = fmaf(q, t, 0.093552403f);
    q = fmaf(q, t, 0.120448583f);
    q = fmaf(q, t, 0.118365633f);
    q *= t * e;
    return g > 0.0f ? 1.0f - q : q;
}

template <int ACT>
__device__ __forceinline__ float act_of(float g)
{
    if (ACT == ESP_MOE_SILU)
        return g * logistic(g);
    if (ACT == ESP_MOE_GELU) {
        float e;
        return g * normal(g, e);
    }
    if (ACT == ESP_MOE_GELU_TANH)   // (1 + tanh t) / 2 = logistic(2 t)
        return g * logistic(1.59576912f * (g + 0.044715f * g * g * g));
    return g < 0.0f ? 0.0f : g;   // a maximum with 0 would drop NaN
}

template <int ACT>
__device__ __forceinline__ void act_and_slope(float g, float &a, float &d)
{
    if (ACT == ESP_MOE_SILU) {
        const float s = logistic(g);
        a = g * s;
        d = s * (1.0f + g * (1.0f - s));
    } else if (ACT == ESP_MOE_GELU) {
        float e;
        const float c = normal(g, e);
        a = g * c;
        d = c + g * 0.39894228f * e;
    } else if (ACT == ESP_MOE_GELU_TANH) {
        const float s = logistic(1.59576912f * (g + 0.044715f * g * g * g));
        a = g * s;
        d = s + a * (1.0f - s) * 1.59576912f * (1.0f + 0.134145f * g * g);
    } else {
        a = g < 0.0f ? 0.0f : g;
        d = g > 0.0f ? 1.0f : g <= 0.0f ? 0.0f : g;
    }
}

// Calls f with the activation as a constant.
template <typename F>
__device__ __forceinline__ void with_act(int act, F &&f)
{
    if (act == ESP_MOE_SILU)
        f(std::integral_constant<int, ESP_MOE_SILU>());
    else if (act == ESP_MOE_GELU)
        f(std::integral_constant<int, ESP_MOE_GELU>());
    else if (act == ESP_MOE_GELU_TANH)
        f(std::integral_constant<int, ESP_MOE_GELU_TANH>());
    else
        f(std::integral_constant<int, ESP_MOE_RELU>());
}

// Boxes of `bytes` (128 or 64) and `rows` of the second axis of a tensor of 2- or 4-byte elements: x elements contiguous, y and z
// ldy and ldz elements apart. What a load finds outside is zero, what a store has outside is dropped.
cudaError_t box_map3(CUtensorMap *map, const void *p, int size, int64_t x, int64_t y, int64_t ldy, int64_t z, int64_t ldz,
                     int rows, int bytes = 128)
{
    const EncodeTiled encode = encode_tiled();
    if (!encode)
        return cudaErrorNotSupported;
    const cuuint64_t dims[3] = {(cuuint64_t)x, (cuuint64_t)y, (cuuint64_t)z};
    const cuuint64_t strides[2] = {(cuuint64_t)ldy * size, (cuuint64_t)(z > 1 ? ldz : ldy) * size};
    const cuuint32_t box[3] = {(cuuint32_t)(bytes / size), (cuuint32_t)rows, 1}, step[3] = {1, 1, 1};
    const CUresult r = encode(map, size == 2 ? CU_TENSOR_MAP_DATA_TYPE_UINT16 : CU_TENSOR_MAP_DATA_TYPE_UINT32, 3,
                              const_cast<void *>(p), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                              bytes == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

// Calls f(T()) for a 16-bit type.
template <typename F>
cudaError_t with_16(int32_t dtype, F &&f)
{
    return dtype == ESP_MOE_BF16 ? f(__nv_bfloat16()) : f(__half());
}

FfParams common(esp_moe *m, const FfShape &s)
{
    FfParams p{};
    p.g.err = m->d_err;
    p.g.wait_ms = m->wait_ms;
    p.g.hold = m->hold_load ? 1 : 0;
    m->hold_load = false;   // the hook holds one launch only
    p.g.splits = 1;
    p.g.partial = s.partial;
    p.g.tickets = m->d_ticket + 1;
    p.g.M = (int32_t)s.M;
    p.g.E = s.E;
    p.g.offsets = s.offsets;
    p.halves = 1;
    p.act = s.act;
    p.half_f16 = s.dtype == ESP_MOE_F16;
    p.fp = s.fp;
    return p;
}

#define FF_TRY(call)                  \
    do {                              \
        const cudaError_t e_ = call;  \
        if (e_ != cudaSuccess)        \
            return e_;                \
    } while (0)

}  // namespace

}  // namespace esp_moe_impl
