// 8-bit codes with a scale per block (include/esp_moe.h): rows of activations (1 x 128 blocks, gathered),
// columns of activations for the weights' gradient (128 x 1 blocks inside an expert's rows, transposed),
// and weights (128 x 128 blocks, with their transposed copy).
//
// A block's codes are e4m3(x * inv), inv = 448 / a, and its scale a / 448 with a = max(max |x|, 2^-100):
// the floor keeps inv finite and an all-zero block needs no case of its own. A maximum that is not
// finite makes inv 0 and the scale NaN, so that every result that reads the block shows it.

#include <algorithm>

#include <cuda_fp8.h>

#include "esp_moe_impl.h"
#include "esp_moe_load.cuh"

namespace esp_moe_impl {

namespace {

constexpr float kMaxCode = 448.0f;
constexpr float kFloor = 7.888609052210118e-31f;   // 2^-100

__device__ __forceinline__ void block_scale(float amax, bool finite, float &scale, float &inv)
{
    const float a = fmaxf(amax, kFloor);
    scale = finite ? __fdiv_rn(a, kMaxCode) : __int_as_float(0x7fffffff);
    inv = finite ? __fdiv_rn(kMaxCode, a) : 0.0f;
}

// Four values as codes, the first in the lowest byte (rounded to nearest even, saturated at 448).
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d, float inv)
{
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(__fmul_rn(a, inv), __fmul_rn(b, inv)), __NV_SATFINITE,
                                                 __NV_E4M3);
    const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(__fmul_rn(c, inv), __fmul_rn(d, inv)), __NV_SATFINITE,
                                                 __NV_E4M3);
    return lo | (hi << 16);
}

__device__ __forceinline__ bool is_finite(float v)
{
    return fabsf(v) <= 3.4028234663852886e38f;
}

// ---- rows: 16 lanes per block of 128, 8 elements per lane

constexpr int kRowThreads = 256;

template <typename T>
__global__ void __launch_bounds__(kRowThreads) k_quant_rows(const QuantRowsArgs a, int blocks_k, bool aligned)
{
    const int lane16 = threadIdx.x & 15;
    const int64_t total = a.M * blocks_k;
    const int64_t stride = (int64_t)gridDim.x * (kRowThreads / 16);
    const int64_t rounds = (total + stride - 1) / stride;   // whole warps take every turn of the loop
    int64_t i = (int64_t)blockIdx.x * (kRowThreads / 16) + (threadIdx.x >> 4);
    for (int64_t turn = 0; turn < rounds; ++turn, i += stride) {
        const bool on = i < total;
        const int64_t row = on ? i / blocks_k : 0;
        const int kb = on ? (int)(i - row * blocks_k) : 0;
        int64_t src = row;
        if (on && a.rows)
            src = a.rows[row];
        const bool there = on && src >= 0 && src < a.T;
        const int k0 = kb * kBlock + lane16 * 8;
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)
            v[j] = 0.0f;
        if (there) {
            const T *p = static_cast<const T *>(a.x) + src * a.ldx + k0;
            constexpr int W = 16 / (int)sizeof(T) < 8 ? 16 / (int)sizeof(T) : 8;
            if (aligned && k0 + 8 <= a.K) {
#pragma unroll
                for (int c = 0; c < 8 / W; ++c)
                    load_pack<T, W>(p + c * W, v + c * W);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (k0 + j < a.K)
                        v[j] = to_f32(p[j]);
            }
        }
        float amax = 0.0f;
        bool finite = true;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            amax = fmaxf(amax, fabsf(v[j]));
            finite = finite && is_finite(v[j]);
        }
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) {
            amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
            finite = __shfl_xor_sync(0xffffffffu, (int)finite, o) && finite;
        }
        float scale, inv;
        block_scale(amax, finite, scale, inv);
        if (!on)
            continue;
        if (!finite) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                v[j] = 0.0f;
        }
        // codes past K (up to the padded row) are zero
        uint2 q;
        q.x = codes4(v[0], v[1], v[2], v[3], inv);
        q.y = codes4(v[4], v[5], v[6], v[7], inv);
        if (k0 < a.ldq)
            *reinterpret_cast<uint2 *>(a.q + row * a.ldq + k0) = q;
        if (lane16 == 0)
            a.scale[row * a.lds + kb] = scale;
    }
}

// ---- columns: a CTA takes 128 positions of an expert's run and 64 columns

constexpr int kColTile = 64;
constexpr int kColThreads = 256;

// Expert and first source row of the run of 128 positions number `tile` (false past the last). The
// offsets are read by every thread in turn: at most 1024 experts.
__device__ bool find_run(const int32_t *offsets, int E, int64_t M, int64_t tile, int64_t &row0, int &n)
{
    int64_t base = 0;
    for (int e = 0; e < E; ++e) {
        const int64_t a = offsets ? max((int64_t)0, min(M, (int64_t)offsets[e])) : 0;
        const int64_t b = offsets ? max(a, min(M, (int64_t)offsets[e + 1])) : M;
        const int64_t runs = (b - a + kBlock - 1) / kBlock;
        if (tile < base + runs) {
            row0 = a + (tile - base) * kBlock;
            n = (int)min((int64_t)kBlock, b - row0);
            return true;
        }
        base += runs;
    }
    return false;
}

template <typename T>
__global__ void __launch_bounds__(kColThreads) k_quant_cols(const QuantColsArgs a)
{
    __shared__ float tile[kBlock][kColTile + 1];
    __shared__ int64_t s_row0;
    __shared__ int s_n;
    if (threadIdx.x == 0) {
        int64_t row0 = 0;
        int n = 0;
        s_n = find_run(a.offsets, a.E, a.M, blockIdx.x, row0, n) ? n : 0;
        s_row0 = row0;
    }
    __syncthreads();
    const int n = s_n;
    if (n == 0)
        return;
    const int c0 = blockIdx.y * kColTile;
    for (int i = threadIdx.x; i < kBlock * kColTile; i += kColThreads) {
        const int r = i / kColTile, c = i % kColTile;
        float v = 0.0f;
        if (r < n && c0 + c < a.K) {
            const int64_t src = a.rows ? a.rows[s_row0 + r] : s_row0 + r;
            if (src >= 0 && src < a.T)
                v = to_f32(static_cast<const T *>(a.x)[src * a.ldx + c0 + c]);
        }
        tile[r][c] = v;
    }
    __syncthreads();
    // four threads per column, 32 positions each
    const int c = threadIdx.x >> 2, part = threadIdx.x & 3;
    float amax = 0.0f;
    bool finite = true;
    for (int r = 0; r < 32; ++r) {
        const float v = tile[part * 32 + r][c];
        amax = fmaxf(amax, fabsf(v));
        finite = finite && is_finite(v);
    }
#pragma unroll
    for (int o = 1; o < 4; o <<= 1) {
        amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
        finite = __shfl_xor_sync(0xffffffffu, (int)finite, o) && finite;
    }
    float scale, inv;
    block_scale(amax, finite, scale, inv);
    if (c0 + c >= a.K)
        return;
    uint32_t q[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        float v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            v[i] = finite ? tile[part * 32 + 4 * j + i][c] : 0.0f;
        q[j] = codes4(v[0], v[1], v[2], v[3], inv);
    }
    uint4 *dst = reinterpret_cast<uint4 *>(a.q + (int64_t)(c0 + c) * a.ldq + (int64_t)blockIdx.x * kBlock + part * 32);
    dst[0] = make_uint4(q[0], q[1], q[2], q[3]);
    dst[1] = make_uint4(q[4], q[5], q[6], q[7]);
    if (part == 0)
        a.scale[(int64_t)blockIdx.x * a.lds + c0 + c] = scale;
}

// ---- weights: a CTA per block of 128 x 128

constexpr int kWThreads = 512;

template <typename T>
__global__ void __launch_bounds__(kWThreads) k_quant_weight(const T *w, int64_t ldw, const esp_moe_weight o, bool aligned)
{
    __shared__ float red[kWThreads / 32];
    __shared__ int bad;
    __shared__ uint32_t codes[kBlock][kBlock / 4 + 1];
    const int kb = blockIdx.x, nb = blockIdx.y, e = blockIdx.z;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (threadIdx.x == 0)
        bad = 0;
    __syncthreads();
    // thread: 4 columns (4 * lane) of the rows warp, warp + 16, ...
    constexpr int kRows = kBlock / (kWThreads / 32);
    float v[kRows][4];
    const int k0 = kb * kBlock + 4 * lane;
    float amax = 0.0f;
    bool finite = true;
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        const int n = nb * kBlock + warp + r * (kWThreads / 32);
#pragma unroll
        for (int j = 0; j < 4; ++j)
            v[r][j] = 0.0f;
        if (n < o.N) {
            const T *p = w + ((int64_t)e * o.N + n) * ldw + k0;
            if (aligned && k0 + 4 <= o.K) {
                load_pack<T, 4>(p, v[r]);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (k0 + j < o.K)
                        v[r][j] = to_f32(p[j]);
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            amax = fmaxf(amax, fabsf(v[r][j]));
            finite = finite && is_finite(v[r][j]);
        }
    }
#pragma unroll
    for (int s = 16; s > 0; s >>= 1)
        amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, s));
    if (lane == 0)
        red[warp] = amax;
    if (!finite)
        bad = 1;
    __syncthreads();
    finite = bad == 0;
    amax = 0.0f;
#pragma unroll
    for (int i = 0; i < kWThreads / 32; ++i)
        amax = fmaxf(amax, red[i]);
    float scale, inv;
    block_scale(amax, finite, scale, inv);
    if (threadIdx.x == 0)
        o.scale[((int64_t)e * gridDim.y + nb) * gridDim.x + kb] = scale;
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        const int i = warp + r * (kWThreads / 32), n = nb * kBlock + i;
        const uint32_t q = finite ? codes4(v[r][0], v[r][1], v[r][2], v[r][3], inv) : 0u;
        codes[i][lane] = q;
        if (n < o.N && k0 < o.ld)
            *reinterpret_cast<uint32_t *>(o.q + ((int64_t)e * o.N + n) * o.ld + k0) = q;
    }
    if (!o.qt)
        return;
    __syncthreads();
    // transposed: a word holds four consecutive n of one k
    for (int i = threadIdx.x; i < kBlock * kBlock / 4; i += kWThreads) {
        const int k = i / (kBlock / 4), n4 = 4 * (i % (kBlock / 4));
        if (kb * kBlock + k >= o.K || nb * kBlock + n4 >= o.ldt)
            continue;
        uint32_t q = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            q |= ((codes[n4 + j][k >> 2] >> (8 * (k & 3))) & 0xffu) << (8 * j);
        *reinterpret_cast<uint32_t *>(o.qt + ((int64_t)e * o.K + kb * kBlock + k) * o.ldt + nb * kBlock + n4) = q;
    }
}

}  // namespace

cudaError_t launch_quant_rows(esp_moe *m, int32_t dtype, const QuantRowsArgs &a)
{
    const int blocks_k = (int)ceil_div(a.K, kBlock);
    const int64_t total = a.M * blocks_k;
    if (total == 0)
        return cudaSuccess;
    return with_dtype(dtype, [&](auto elem) -> cudaError_t {
        using T = decltype(elem);
        const int64_t ctas = ceil_div(total, kRowThreads / 16);
        k_quant_rows<T><<<(unsigned)std::min<int64_t>(ctas, (int64_t)m->sm_count * 32), kRowThreads, 0, m->stream>>>(
            a, blocks_k, rows_aligned(a.x, a.ldx, sizeof(T), 16));
        m->launches += 1;
        return cudaGetLastError();
    });
}

cudaError_t launch_quant_cols(esp_moe *m, int32_t dtype, const QuantColsArgs &a)
{
    if (a.M == 0)
        return cudaSuccess;
    return with_dtype(dtype, [&](auto elem) -> cudaError_t {
        using T = decltype(elem);
        // runs of 128 positions: at most this many, some past the last
        const int64_t runs = a.M / kBlock + a.E;
        const dim3 grid((unsigned)runs, (unsigned)ceil_div(a.K, kColTile));
        k_quant_cols<T><<<grid, kColThreads, 0, m->stream>>>(a);
        m->launches += 1;
        return cudaGetLastError();
    });
}

cudaError_t launch_quant_weight(esp_moe *m, int32_t dtype, const void *w, int64_t ldw, const esp_moe_weight &o)
{
    return with_dtype(dtype, [&](auto elem) -> cudaError_t {
        using T = decltype(elem);
        const dim3 grid((unsigned)ceil_div(o.K, kBlock), (unsigned)ceil_div(o.N, kBlock), (unsigned)o.E);
        k_quant_weight<T><<<grid, kWThreads, 0, m->stream>>>(static_cast<const T *>(w), ldw, o,
                                                             rows_aligned(w, ldw, sizeof(T), 4 * sizeof(T)));
        m->launches += 1;
        return cudaGetLastError();
    });
}

}  // namespace esp_moe_impl
