// The forward products of one dense gated feed-forward block for one or two rows (single tokens), on the CUDA cores: every
// weight is loaded once, 16 bytes a lane, and multiplied with the rows in fp32. Bound by the weights' bytes; there is no
// tile to fill, no tensor memory and nothing to join, which is what a tensor-core kernel spends its time on here.
//
// A warp takes some weight rows at a time (HIDDEN: the same ones of G and of U) over the whole inner axis, and the rows of
// x, which lie in L1; the next weights are on their way while these are multiplied, across rows too. Weight rows go round
// over the CTAs, so that every SM streams the same bytes.

#include <algorithm>

#include "esp_ff.cuh"
#include "esp_moe_launch.cuh"
#include "esp_moe_load.cuh"

namespace esp_moe_impl {

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;

struct VecParams {
    int32_t M, T, N, K;          // M: at most 2; N: weight rows (HIDDEN: of G), K: inner axis
    const int32_t *offsets, *rows;
    const void *w, *x;
    int64_t ldw, ldx;
    void *out;
    int64_t ldo;
    float *pre;                  // HIDDEN: kept (or null)
    int64_t fp;
    int32_t act;
    bool early;                  // this call's own launch is the one before
};

__device__ __forceinline__ uint4 load_stream(const void *p)
{
    uint4 r;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w)
                 : "l"(p));
    return r;
}

// Elements 8 g .. 8 g + 7 of a row of K; those past its end are 0 and not read.
template <bool STREAM>
__device__ __forceinline__ uint4 load_group(const uint16_t *row, int g, int K)
{
    if (8 * g + 8 <= K)
        return STREAM ? load_stream(row + 8 * g) : *reinterpret_cast<const uint4 *>(row + 8 * g);
    uint32_t r[4] = {};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (8 * g + i < K)
            r[i / 2] |= (uint32_t)row[8 * g + i] << (16 * (i & 1));
    return make_uint4(r[0], r[1], r[2], r[3]);
}

template <typename T>
__device__ __forceinline__ uint64_t pair_of(uint32_t v);
template <>
__device__ __forceinline__ uint64_t pair_of<__nv_bfloat16>(uint32_t v)
{
    return (uint64_t)(v << 16) | (uint64_t)(v & 0xffff0000u) << 32;
}
template <>
__device__ __forceinline__ uint64_t pair_of<__half>(uint32_t v)
{
    __half2 h;
    memcpy(&h, &v, 4);
    const float2 f = __half22float2(h);
    return (uint64_t)__float_as_uint(f.x) | (uint64_t)__float_as_uint(f.y) << 32;
}

__device__ __forceinline__ uint32_t part_of(const uint4 &v, int i)
{
    return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w;
}

// c += a * b, two fp32 at a time.
__device__ __forceinline__ void fma2(uint64_t &c, uint64_t a, uint64_t b)
{
    asm("fma.rn.f32x2 %0, %1, %2, %0;" : "+l"(c) : "l"(a), "l"(b));
}

// R rows of x, NF weight rows (HIDDEN: of each of G and U). U groups of 8 elements of each at a time, the next ones on their
// way while these are multiplied.
template <int KIND, int R, int NF, typename T>
__global__ void __launch_bounds__(kThreads, 2) k_ff_vec(const VecParams p)
{
    constexpr int W = KIND == HIDDEN ? 2 * NF : NF;       // weight rows
    constexpr int U = 8 / W;
    const int lane = threadIdx.x & 31;
    if (!p.early) {
        wait_for_launch_before();
        let_next_launch_start();
    }
    const int groups = (p.K + 7) / 8, step = gridDim.x * kWarps * NF;
    const uint16_t *w[W], *x[R];
    const auto rows_from = [&](int n0) {   // rows past the last are its copies
#pragma unroll
        for (int f = 0; f < W; ++f)
            w[f] = static_cast<const uint16_t *>(p.w) +
                   ((int64_t)(KIND == HIDDEN && f >= NF ? p.N : 0) + min(n0 + f % NF, p.N - 1)) * p.ldw;
    };
    uint4 v[2][W][U];
    const auto load = [&](uint4 (&to)[W][U], int g0) {
#pragma unroll
        for (int f = 0; f < W; ++f)
#pragma unroll
            for (int j = 0; j < U; ++j) {
                const int g = g0 + 32 * j + lane;
                to[f][j] = g < groups ? load_group<true>(w[f], g, p.K) : make_uint4(0, 0, 0, 0);
            }
    };
    int n0 = (blockIdx.x + gridDim.x * (threadIdx.x >> 5)) * NF;
    if (n0 < p.N) {
        rows_from(n0);
        load(v[0], 0);
    }
    if (p.early) {
        // the first weights are on their way; what the launch before writes (the rows) comes after this
        wait_for_launch_before();
        let_next_launch_start();
    }
    const int lo = p.offsets ? max(0, min(p.M, p.offsets[0])) : 0, hi = p.offsets ? max(lo, min(p.M, p.offsets[1])) : p.M;
    bool there[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int64_t from = r < p.M ? (p.rows ? p.rows[r] : r) : -1;
        there[r] = from >= 0 && from < p.T;
        x[r] = static_cast<const uint16_t *>(p.x) + (there[r] ? from : 0) * p.ldx;
    }
    for (; n0 < p.N; n0 += step) {
        uint64_t sum[W][R] = {};
        const auto multiply = [&](const uint4 (&by)[W][U], int g0) {
#pragma unroll
            for (int j = 0; j < U; ++j) {
                const int g = g0 + 32 * j + lane;
                if (g >= groups)
                    break;
                uint4 xv[R];
#pragma unroll
                for (int r = 0; r < R; ++r)
                    xv[r] = there[r] ? load_group<false>(x[r], g, p.K) : make_uint4(0, 0, 0, 0);
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    uint64_t xp[R];
#pragma unroll
                    for (int r = 0; r < R; ++r)
                        xp[r] = pair_of<T>(part_of(xv[r], q));
#pragma unroll
                    for (int f = 0; f < W; ++f) {
                        const uint64_t wp = pair_of<T>(part_of(by[f][j], q));
#pragma unroll
                        for (int r = 0; r < R; ++r)
                            fma2(sum[f][r], wp, xp[r]);
                    }
                }
            }
        };
        for (int g0 = 0; g0 < groups; g0 += 64 * U) {
            load(v[1], g0 + 32 * U);
            multiply(v[0], g0);
            if (g0 + 64 * U < groups)
                load(v[0], g0 + 64 * U);
            else if (n0 + step < p.N) {   // the next rows' first weights
                rows_from(n0 + step);
                load(v[0], 0);
            }
            multiply(v[1], g0 + 32 * U);
        }
        // every lane gets every sum; lane f R + r stores feature f of row r
        float mine = 0.0f, up = 0.0f;
#pragma unroll
        for (int f = 0; f < W; ++f)
#pragma unroll
            for (int r = 0; r < R; ++r) {
                float s = __uint_as_float((uint32_t)sum[f][r]) + __uint_as_float((uint32_t)(sum[f][r] >> 32));
#pragma unroll
                for (int o = 16; o > 0; o >>= 1)
                    s += __shfl_xor_sync(0xffffffffu, s, o);
                if (lane == f % NF * R + r)
                    (f < NF ? mine : up) = s;
            }
        const int f = lane / R, r = lane % R, n = n0 + f;
        if (f < NF && r >= lo && r < hi && n < p.N) {
            if (KIND == HIDDEN) {
                if (p.pre) {
                    p.pre[r * 2 * p.fp + n] = mine;
                    p.pre[r * 2 * p.fp + p.fp + n] = up;
                }
                with_act(p.act, [&](auto kind) { mine = act_of<decltype(kind)::value>(mine) * up; });
            }
            static_cast<T *>(p.out)[r * p.ldo + n] = from_f32<T>(mine);
        }
    }
}

template <int KIND, int R, typename T>
cudaError_t launch(esp_moe *m, const VecParams &p)
{
    const int ctas = 2 * m->sm_count;
    m->launches += 1;
    // two weight rows (HIDDEN: of each matrix) at a time where there are enough for every warp, else one
    constexpr int NF = KIND == HIDDEN ? 2 : 4;
    if (p.N >= ctas * kWarps * NF / 2)
        return launch_after(k_ff_vec<KIND, R, NF, T>, dim3((unsigned)std::min<int64_t>(ctas, ceil_div(p.N, NF))), kThreads, 0,
                            m->stream, p);
    return launch_after(k_ff_vec<KIND, R, NF / 2, T>, dim3((unsigned)std::min<int64_t>(ctas, ceil_div(p.N, NF / 2))), kThreads,
                        0, m->stream, p);
}

template <int KIND>
cudaError_t by_rows(esp_moe *m, int32_t dtype, const VecParams &p)
{
    return with_16(dtype, [&](auto elem) -> cudaError_t {
        using T = decltype(elem);
        return p.M == 1 ? launch<KIND, 1, T>(m, p) : launch<KIND, 2, T>(m, p);
    });
}

}  // namespace

bool use_vec(int64_t M, int32_t E)
{
    return E == 1 && M <= 2;
}

cudaError_t launch_vec(esp_moe *m, const FfShape &s, const void *x, int64_t ldx, int64_t T, const int32_t *rows, void *hidden,
                       void *pre, void *y, int64_t ldy)
{
    VecParams p{};
    p.M = (int32_t)s.M;
    p.T = (int32_t)T;
    p.N = s.F;
    p.K = s.H;
    p.offsets = s.offsets;
    p.rows = rows;
    p.w = s.inner;
    p.ldw = s.ld_inner;
    p.x = x;
    p.ldx = ldx;
    p.out = hidden;
    p.ldo = p.fp = s.fp;
    p.pre = static_cast<float *>(pre);
    p.act = s.act;
    const cudaError_t e = by_rows<HIDDEN>(m, s.dtype, p);
    if (e != cudaSuccess)
        return e;
    p.T = p.M;
    p.N = s.H;
    p.K = s.F;
    p.rows = nullptr;
    p.w = s.outer;
    p.ldw = s.ld_outer;
    p.x = hidden;
    p.ldx = s.fp;
    p.out = y;
    p.ldo = ldy;
    p.early = true;   // no weights are written by the launch before, which began after everything before it
    return by_rows<OUT>(m, s.dtype, p);
}

}  // namespace esp_moe_impl
