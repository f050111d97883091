// 8-bit codes with a scale per block (include/esp_moe.h): rows of activations (1 x 128 blocks, gathered),
// columns of activations for the weights' gradient (128 x 1 blocks inside an expert's rows, transposed),
// and weights (128 x 128 blocks, with their transposed copy).
//
// A block's codes are e4m3(x * inv), inv = 448 / a, and its scale a / 448 with a = max(max |x|, 2^-100):
// the floor keeps inv finite and an all-zero block needs no case of its own. A maximum that is not
// finite makes inv 0 and the scale NaN, so that every result that reads the block shows it.

#include <algorithm>
#include <cstring>
#include <type_traits>

#include <cuda_fp8.h>

#include "esp_moe_impl.h"
#include "esp_moe_launch.cuh"
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

// Magnitudes compare as integers: a value's bits without the sign, NaN above infinity above all others.
template <typename T>
__device__ __forceinline__ float magnitude_value(uint32_t bits);
template <>
__device__ __forceinline__ float magnitude_value<float>(uint32_t bits) { return __uint_as_float(bits); }
template <>
__device__ __forceinline__ float magnitude_value<__nv_bfloat16>(uint32_t bits) { return __uint_as_float(bits << 16); }
template <>
__device__ __forceinline__ float magnitude_value<__half>(uint32_t bits)
{
    return __half2float(__ushort_as_half((unsigned short)bits));
}

// Eight consecutive elements of a row, as stored.
template <typename T>
struct Eight {
    static constexpr int kWords = (int)sizeof(T) * 2;
    uint32_t w[kWords];

    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int i = 0; i < kWords; ++i)
            w[i] = 0;
    }
    // n of them exist (others become zero); aligned: p is a multiple of 16 bytes
    __device__ __forceinline__ void load(const T *p, int n, bool aligned)
    {
        if (aligned && n >= 8) {
#pragma unroll
            for (int i = 0; i < kWords; i += 4) {
                const uint4 v = *reinterpret_cast<const uint4 *>(reinterpret_cast<const uint32_t *>(p) + i);
                w[i] = v.x;
                w[i + 1] = v.y;
                w[i + 2] = v.z;
                w[i + 3] = v.w;
            }
            return;
        }
        T v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i)
            v[i] = i < n ? p[i] : from_f32<T>(0.0f);
        memcpy(w, v, sizeof(v));
    }
    __device__ __forceinline__ float get(int i) const
    {
        if constexpr (sizeof(T) == 4)
            return __uint_as_float(w[i]);
        else if constexpr (std::is_same<T, __half>::value)
            return __half2float(__ushort_as_half((unsigned short)(w[i / 2] >> (16 * (i & 1)))));
        else
            return __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
    }
    // words of magnitudes: one per element, or two elements in the halves of a word
    __device__ __forceinline__ uint32_t magnitudes(int i) const
    {
        return w[i] & (sizeof(T) == 4 ? 0x7fffffffu : 0x7fff7fffu);
    }
    static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b)
    {
        return sizeof(T) == 4 ? max(a, b) : __vmaxu2(a, b);
    }
    // the larger of a word's halves
    static __device__ __forceinline__ uint32_t flat(uint32_t m)
    {
        return sizeof(T) == 4 ? m : max(m & 0xffffu, m >> 16);
    }
    __device__ __forceinline__ uint32_t largest() const
    {
        uint32_t m = magnitudes(0);
#pragma unroll
        for (int i = 1; i < kWords; ++i)
            m = larger(m, magnitudes(i));
        return m;
    }
};

// Scale and inverse of a block from the bits of its greatest magnitude.
template <typename T>
__device__ __forceinline__ void scale_of(uint32_t bits, float &scale, float &inv)
{
    const float amax = magnitude_value<T>(bits);
    block_scale(amax, amax <= 3.4028234663852886e38f, scale, inv);
}

// In a block that is not finite the inverse is 0 and the codes are 0 or NaN: its scale makes every result that
// reads them NaN either way.
template <typename T>
__device__ __forceinline__ uint2 codes8(const Eight<T> &x, float inv)
{
    return make_uint2(codes4(x.get(0), x.get(1), x.get(2), x.get(3), inv),
                      codes4(x.get(4), x.get(5), x.get(6), x.get(7), inv));
}

// ---- rows: 4 lanes per block of 128, four times 8 elements per lane. Bound by the bytes; a block's two
// divisions are done by its 4 lanes only, and a lane's four loads are in flight at once.

constexpr int kRowThreads = 256;
constexpr int kRowBlocks = kRowThreads / 4;   // of a CTA

template <typename T>
__global__ void __launch_bounds__(kRowThreads) k_quant_rows(const QuantRowsArgs a, int blocks_k, bool aligned)
{
    let_next_launch_start();
    wait_for_launch_before();
    const int lane4 = threadIdx.x & 3;
    const int64_t total = a.M * blocks_k, i = (int64_t)blockIdx.x * kRowBlocks + (threadIdx.x >> 2);
    const bool on = i < total;
    const int64_t row = !on ? 0 : total <= 0x7fffffff ? (int64_t)((uint32_t)i / (uint32_t)blocks_k) : i / blocks_k;
    const int kb = (int)(i - row * blocks_k);
    int64_t src = row;
    if (on && a.rows)
        src = a.rows[row];
    const bool there = on && src >= 0 && src < a.T;
    const int k0 = kb * kBlock + lane4 * 8;
    const T *p = static_cast<const T *>(a.x) + src * a.ldx + k0;
    Eight<T> x[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        x[c].zero();
        if (there)
            x[c].load(p + 32 * c, a.K - k0 - 32 * c, aligned);
    }
    uint32_t m = x[0].largest();
#pragma unroll
    for (int c = 1; c < 4; ++c)
        m = Eight<T>::larger(m, x[c].largest());
    m = Eight<T>::flat(m);
    m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
    m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
    if (!on)
        return;
    float scale, inv;
    scale_of<T>(m, scale, inv);
    uint8_t *q = a.q + row * a.ldq + k0;
#pragma unroll
    for (int c = 0; c < 4; ++c)
        if (k0 + 32 * c < a.ldq)   // codes past K, up to the padded row, are zero
            *reinterpret_cast<uint2 *>(q + 32 * c) = codes8<T>(x[c], inv);
    if (lane4 == 0)
        a.scale[row * a.lds + kb] = scale;
}

// A warp copies a row: 512 bytes of codes at a time, then the scales.
__global__ void __launch_bounds__(kRowThreads) k_pick_rows(const PickRowsArgs a)
{
    let_next_launch_start();
    wait_for_launch_before();
    const int lane = threadIdx.x & 31;
    const int64_t row = (int64_t)blockIdx.x * (kRowThreads / 32) + (threadIdx.x >> 5);
    if (row >= a.M)
        return;
    int64_t src = a.rows[row];
    src = src >= 0 && src < a.T ? src : a.T;
    const uint4 *from = reinterpret_cast<const uint4 *>(a.from_q + src * a.ldq);
    uint4 *to = reinterpret_cast<uint4 *>(a.q + row * a.ldq);
    const int n = (int)(a.ldq / 16);
    for (int i = lane; i < n; i += 128) {
        uint4 v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (i + 32 * j < n)
                v[j] = from[i + 32 * j];
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (i + 32 * j < n)
                to[i + 32 * j] = v[j];
    }
    for (int i = lane; i < a.lds; i += 32)
        a.scale[row * a.lds + i] = a.from_scale[src * a.lds + i];
}

// ---- tiles of 128 x 128: thread (r, c) of 16 x 16 holds 8 consecutive columns of every 16th row

constexpr int kTileThreads = 256;
constexpr int kPitch = kBlock / 4 + 2;   // words of a row of codes in shared memory (pairs stay aligned)
constexpr int kTurnedPitch = kBlock / 4 + 4;   // rows that are read 16 bytes at a time

struct alignas(16) TileSmem {
    uint32_t turned[kBlock][kTurnedPitch];
    uint32_t high[16][kBlock];           // greatest magnitudes by thread row and column
    float inv[kBlock];
    uint32_t codes[kBlock][kPitch];
};

// codes -> turned: bytes (row, column) exchanged, in 4 x 4 squares. Called by the whole CTA between barriers.
__device__ __forceinline__ void turn_codes(TileSmem &s)
{
    for (int i = threadIdx.x; i < 32 * 32; i += kTileThreads) {
        // 8 x 4 squares per warp: its reads fall on 32 banks
        const int a = (i & 7) | ((i >> 5) & 3) << 3, b = ((i >> 3) & 3) | (i >> 7) << 2;
        uint32_t r[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
            r[j] = s.codes[4 * a + j][b];
        const uint32_t lo01 = __byte_perm(r[0], r[1], 0x5140), lo23 = __byte_perm(r[2], r[3], 0x5140);
        const uint32_t hi01 = __byte_perm(r[0], r[1], 0x7362), hi23 = __byte_perm(r[2], r[3], 0x7362);
        s.turned[4 * b][a] = __byte_perm(lo01, lo23, 0x5410);
        s.turned[4 * b + 1][a] = __byte_perm(lo01, lo23, 0x7632);
        s.turned[4 * b + 2][a] = __byte_perm(hi01, hi23, 0x5410);
        s.turned[4 * b + 3][a] = __byte_perm(hi01, hi23, 0x7632);
    }
}

// Rows [0, rows) of the turned codes to dst, ld bytes apart, the first `bytes` (a multiple of 16) of each.
__device__ __forceinline__ void store_turned(const TileSmem &s, uint8_t *dst, int64_t ld, int rows, int bytes)
{
    for (int i = threadIdx.x; i < kBlock * 8; i += kTileThreads) {
        const int r = i >> 3, w = (i & 7) * 4;
        if (r < rows && 4 * w < bytes)
            *reinterpret_cast<uint4 *>(dst + r * ld + 4 * w) = *reinterpret_cast<const uint4 *>(&s.turned[r][w]);
    }
}

// A block of 128 x 128 of the weights: one scale, codes and (qt) transposed codes from one read.
template <typename T>
__global__ void __launch_bounds__(kTileThreads) k_quant_weight(const T *w, int64_t ldw, const esp_moe_weight o,
                                                               bool aligned)
{
    __shared__ TileSmem s;
    __shared__ uint32_t high[kTileThreads / 32];
    let_next_launch_start();
    wait_for_launch_before();
    const int kb = blockIdx.x, nb = blockIdx.y, e = blockIdx.z;
    const int c = threadIdx.x & 15, r0 = threadIdx.x >> 4;
    const int k0 = kb * kBlock + 8 * c, n0 = nb * kBlock;
    Eight<T> x[8];
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int n = n0 + r0 + 16 * i;
        x[i].zero();
        if (n < o.N && k0 < o.K)
            x[i].load(w + ((int64_t)e * o.N + n) * ldw + k0, o.K - k0, aligned);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        m = Eight<T>::larger(m, x[i].largest());
    m = __reduce_max_sync(0xffffffffu, Eight<T>::flat(m));
    if ((threadIdx.x & 31) == 0)
        high[threadIdx.x >> 5] = m;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kTileThreads / 32; ++i)
        m = max(m, high[i]);
    float scale, inv;
    scale_of<T>(m, scale, inv);
    if (threadIdx.x == 0)
        o.scale[((int64_t)e * gridDim.y + nb) * gridDim.x + kb] = scale;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int r = r0 + 16 * i;
        const uint2 q = codes8<T>(x[i], inv);
        *reinterpret_cast<uint2 *>(&s.codes[r][2 * c]) = q;
        if (n0 + r < o.N && k0 < o.ld)
            *reinterpret_cast<uint2 *>(o.q + ((int64_t)e * o.N + n0 + r) * o.ld + k0) = q;
    }
    if (!o.qt)
        return;
    __syncthreads();
    turn_codes(s);
    __syncthreads();
    store_turned(s, o.qt + ((int64_t)e * o.K + kb * kBlock) * o.ldt + n0, o.ldt, o.K - kb * kBlock,
                 (int)min((int64_t)kBlock, o.ldt - n0));
}

// First source row and row count of the experts' run of 128 positions number `tile` (n = 0 past the last).
// Called by the whole CTA (256 threads).
__device__ void find_run(const int32_t *offsets, int E, int64_t M, int tile, int &row0, int &n)
{
    __shared__ int s_row0, s_n;
    if (threadIdx.x < 32) {
        const int lane = threadIdx.x;
        int carry = 0;
        if (lane == 0)
            s_n = 0;
        __syncwarp();
        for (int e0 = 0; e0 < E; e0 += 32) {
            int a = 0, b = 0;
            if (e0 + lane < E) {
                a = offsets ? max(0, min((int)M, offsets[e0 + lane])) : 0;
                b = offsets ? max(a, min((int)M, offsets[e0 + lane + 1])) : (int)M;
            }
            const int runs = (b - a) / kBlock + ((b - a) % kBlock != 0);
            int sum = runs;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int y = __shfl_up_sync(0xffffffffu, sum, o);
                if (lane >= o)
                    sum += y;
            }
            const int first = carry + sum - runs;
            if (tile >= first && tile < first + runs) {
                s_row0 = a + (tile - first) * kBlock;
                s_n = min(kBlock, b - s_row0);
            }
            carry += __shfl_sync(0xffffffffu, sum, 31);
            if (carry > tile)
                break;
        }
    }
    __syncthreads();
    row0 = s_row0;
    n = s_n;
}

// A run of up to 128 rows of an expert and 128 columns: a scale per column, codes transposed. The four CTAs
// of an SM overlap their loads, rounding and turning: 16384 gathered rows of 4096 bf16 (200 MB) take 45 us,
// with several tiles per CTA, or the next tile's rows fetched ahead, 50 to 59. ROWS: the rows' own codes and
// scales (a tile is one block of each row) from the same read.
template <typename T, bool ROWS>
__global__ void __launch_bounds__(kTileThreads, sizeof(T) == 4 ? 2 : 4) k_quant_cols(const QuantColsArgs a, bool aligned)
{
    __shared__ TileSmem s;
    __shared__ int64_t source[kBlock];   // element offset of each row (negative: zeros)
    __shared__ uint32_t row_high[ROWS ? kBlock : 1];
    __shared__ float row_inv[ROWS ? kBlock : 1];
    let_next_launch_start();
    wait_for_launch_before();
    const int tiles_k = (a.K + kBlock - 1) / kBlock, run = blockIdx.x / tiles_k;
    int row0, n;
    find_run(a.offsets, a.E, a.M, run, row0, n);
    if (n == 0)
        return;
    if (threadIdx.x < kBlock) {
        int64_t src = -1;
        if ((int)threadIdx.x < n) {
            src = a.rows ? a.rows[row0 + threadIdx.x] : row0 + (int)threadIdx.x;
            src = src >= 0 && src < a.T ? src * a.ldx : -1;
        }
        source[threadIdx.x] = src;
    }
    __syncthreads();
    const int c = threadIdx.x & 15, r0 = threadIdx.x >> 4;
    const T *in = static_cast<const T *>(a.x);
    const int c0 = (blockIdx.x - run * tiles_k) * kBlock, k0 = c0 + 8 * c;
    Eight<T> x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int64_t src = source[r0 + 16 * i];
        x[i].zero();
        if (src >= 0 && k0 < a.K)
            x[i].load(in + src + k0, a.K - k0, aligned);
    }
    // greatest magnitudes: over the thread's rows, then over the thread rows
    uint32_t high[8];
#pragma unroll
    for (int w = 0; w < Eight<T>::kWords; ++w) {
        uint32_t m = x[0].magnitudes(w);
#pragma unroll
        for (int i = 1; i < 8; ++i)
            m = Eight<T>::larger(m, x[i].magnitudes(w));
        if (sizeof(T) == 4) {
            high[w] = m;
        } else {
            high[2 * w] = m & 0xffffu;
            high[2 * w + 1] = m >> 16;
        }
    }
    uint4 *hp = reinterpret_cast<uint4 *>(&s.high[r0][8 * c]);
    hp[0] = make_uint4(high[0], high[1], high[2], high[3]);
    hp[1] = make_uint4(high[4], high[5], high[6], high[7]);
    if (ROWS) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            uint32_t m = Eight<T>::flat(x[i].largest());
#pragma unroll
            for (int o = 1; o < 16; o <<= 1)
                m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
            if (c == 0)
                row_high[r0 + 16 * i] = m;
        }
    }
    __syncthreads();
    float scale, inv_of;
    if (threadIdx.x < kBlock) {
        uint32_t m = 0;
#pragma unroll
        for (int r = 0; r < 16; ++r)
            m = max(m, s.high[r][threadIdx.x]);
        scale_of<T>(m, scale, inv_of);
        s.inv[threadIdx.x] = inv_of;
        if (c0 + (int)threadIdx.x < a.K)
            a.scale[(int64_t)run * a.lds + c0 + threadIdx.x] = scale;
    } else if (ROWS) {
        const int r = threadIdx.x - kBlock;
        scale_of<T>(row_high[r], scale, inv_of);
        row_inv[r] = inv_of;
        if (r < n)
            a.row_scale[(int64_t)(row0 + r) * a.row_lds + c0 / kBlock] = scale;
    }
    __syncthreads();
    if (ROWS) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int r = r0 + 16 * i;
            if (r < n && k0 < a.row_ldq)
                *reinterpret_cast<uint2 *>(a.row_q + (int64_t)(row0 + r) * a.row_ldq + k0) = codes8<T>(x[i], row_inv[r]);
        }
    }
    const float4 i0 = *reinterpret_cast<const float4 *>(&s.inv[8 * c]);
    const float4 i1 = *reinterpret_cast<const float4 *>(&s.inv[8 * c + 4]);
    const float inv[8] = {i0.x, i0.y, i0.z, i0.w, i1.x, i1.y, i1.z, i1.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)
            v[j] = __fmul_rn(x[i].get(j), inv[j]);
        *reinterpret_cast<uint2 *>(&s.codes[r0 + 16 * i][2 * c]) =
            make_uint2(codes4(v[0], v[1], v[2], v[3], 1.0f), codes4(v[4], v[5], v[6], v[7], 1.0f));
    }
    __syncthreads();
    turn_codes(s);
    __syncthreads();
    store_turned(s, a.q + (int64_t)c0 * a.ldq + (int64_t)run * kBlock, a.ldq, a.K - c0, kBlock);
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
        m->launches += 1;
        return launch_after(k_quant_rows<T>, dim3((unsigned)ceil_div(total, kRowBlocks)), kRowThreads, 0, m->stream, a,
                            blocks_k, rows_aligned(a.x, a.ldx, sizeof(T), 16));
    });
}

cudaError_t launch_pick_rows(esp_moe *m, const PickRowsArgs &a)
{
    m->launches += 1;
    return launch_after(k_pick_rows, dim3((unsigned)ceil_div(a.M, kRowThreads / 32)), kRowThreads, 0, m->stream, a);
}

cudaError_t launch_quant_cols(esp_moe *m, int32_t dtype, const QuantColsArgs &a)
{
    if (a.M == 0)
        return cudaSuccess;
    return with_dtype(dtype, [&](auto elem) -> cudaError_t {
        using T = decltype(elem);
        // runs of 128 positions: at most this many, some past the last
        const int64_t runs = a.M / kBlock + a.E;
        m->launches += 1;
        return launch_after(a.row_q ? k_quant_cols<T, true> : k_quant_cols<T, false>,
                            dim3((unsigned)(runs * ceil_div(a.K, kBlock))), kTileThreads, 0, m->stream, a,
                            rows_aligned(a.x, a.ldx, sizeof(T), 16));
    });
}

cudaError_t launch_quant_weight(esp_moe *m, int32_t dtype, const void *w, int64_t ldw, const esp_moe_weight &o)
{
    return with_dtype(dtype, [&](auto elem) -> cudaError_t {
        using T = decltype(elem);
        const dim3 grid((unsigned)ceil_div(o.K, kBlock), (unsigned)ceil_div(o.N, kBlock), (unsigned)o.E);
        m->launches += 1;
        return launch_after(k_quant_weight<T>, grid, kTileThreads, 0, m->stream, static_cast<const T *>(w), ldw, o,
                            rows_aligned(w, ldw, sizeof(T), 16));
    });
}

}  // namespace esp_moe_impl
