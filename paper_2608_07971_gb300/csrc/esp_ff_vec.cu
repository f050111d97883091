// The forward products of one dense gated feed-forward block for up to eight rows (single tokens), on the CUDA cores: every
// weight is loaded once, 16 bytes a lane, and multiplied with the rows in fp32. Bound by the weights' bytes; there is no
// tile to fill, no tensor memory and nothing to join, which is what a tensor-core kernel spends its time on here.
//
// A CTA takes a few weight rows at a time (HIDDEN: the same ones of G and of U), each thread some 16-byte groups of all of
// them and the same groups of x in registers; the next rows are on their way while these are multiplied, and a sum over
// the CTA ends each. Items go round over the CTAs, so that every SM streams the same bytes. Four CTAs of an SM and four
// groups of a thread: two CTAs and eight groups took 11% longer, warps that take rows of their own, x from L1, 6%.
// Registers hold the loads of one item ahead; the rows of the item after that are on their way to L2. One token of 4096 x
// 8192 (201 MB) takes 34.9 us in a graph, 41.0 without this; 2, 4 and 8 rows of 2048 x 4096 14.7, 20.5 and 32 (15.9, 21.8 and
// 32). One item further ahead: 34.9, 15.4, 20.9.

#include <algorithm>

#include "esp_ff.cuh"
#include "esp_moe_launch.cuh"
#include "esp_moe_load.cuh"

namespace esp_moe_impl {

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;

struct VecParams {
    int32_t M, T, N, K;          // M: at most 8; N: weight rows (HIDDEN: of G), K: inner axis
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

// Asks L2 for a row of K elements (what does not fill its last 16 bytes comes with the load).
__device__ __forceinline__ void prefetch_row(const uint16_t *row, int K)
{
    if (K >= 8)
        asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(row), "r"((uint32_t)(K & ~7) * 2) : "memory");
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

// CTAs of an SM: what their registers leave room for.
template <int R>
constexpr int kCtas = R == 1 ? 4 : R == 2 ? 3 : 2;
template <int R>
constexpr int kLoads = R == 8 ? 2 : 4;

// R rows of x; a thread has J groups of 8 elements of a weight row's 256 J in a step (a row longer than that takes several
// steps), and W weight rows: four loads in flight, with eight rows two.
template <int KIND, int R, int J, typename T>
__global__ void __launch_bounds__(kThreads, kCtas<R>) k_ff_vec(const VecParams p)
{
    constexpr int W = kLoads<R> / J, NF = KIND == HIDDEN ? W / 2 : W;
    __shared__ float part[2][W * R][kWarps];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (!p.early) {
        wait_for_launch_before();
        let_next_launch_start();
    }
    const int groups = (p.K + 7) / 8, segs = (groups + kThreads * J - 1) / (kThreads * J);
    const int items = (p.N + NF - 1) / NF;
    // weight row f of an item; rows past the last are its copies
    const auto weight_row = [&](int item, int f) {
        const int64_t n = (KIND == HIDDEN && f >= NF ? p.N : 0) + min(item * NF + f % NF, p.N - 1);
        return static_cast<const uint16_t *>(p.w) + n * p.ldw;
    };
    // the groups of an item's rows in step `seg`
    const auto load = [&](uint4 (&to)[W][J], int item, int seg) {
#pragma unroll
        for (int f = 0; f < W; ++f) {
            const uint16_t *w = weight_row(item, f);
#pragma unroll
            for (int j = 0; j < J; ++j) {
                const int g = (seg * J + j) * kThreads + threadIdx.x;
                to[f][j] = g < groups ? load_group<true>(w, g, p.K) : make_uint4(0, 0, 0, 0);
            }
        }
    };
    // registers hold the loads of one item ahead; the item after it is on its way to L2
    const auto prefetch = [&](int64_t item) {
        if (threadIdx.x < W && item < items)
            prefetch_row(weight_row((int)item, threadIdx.x), p.K);
    };
    uint4 now[W][J], next[W][J], x[R][J];
    int item = blockIdx.x, seg = 0;
    if (item < items)
        load(now, item, 0);
    prefetch((int64_t)item + gridDim.x);
    if (p.early) {
        // the first weights are on their way; what the launch before writes (the rows) comes after this
        wait_for_launch_before();
        let_next_launch_start();
    }
    const int lo = p.offsets ? max(0, min(p.M, p.offsets[0])) : 0, hi = p.offsets ? max(lo, min(p.M, p.offsets[1])) : p.M;
    const auto load_x = [&](int s) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int64_t from = r < p.M ? (p.rows ? p.rows[r] : r) : -1;
            const bool there = from >= 0 && from < p.T;
            const uint16_t *row = static_cast<const uint16_t *>(p.x) + (there ? from : 0) * p.ldx;
#pragma unroll
            for (int j = 0; j < J; ++j) {
                const int g = (s * J + j) * kThreads + threadIdx.x;
                x[r][j] = there && g < groups ? load_group<false>(row, g, p.K) : make_uint4(0, 0, 0, 0);
            }
        }
    };
    load_x(0);
    uint64_t sum[W][R] = {};
    int turn = 0;
    while (item < items) {
        const int item1 = seg + 1 < segs ? item : item + (int)gridDim.x, seg1 = seg + 1 < segs ? seg + 1 : 0;
        if (item1 < items)
            load(next, item1, seg1);
        if (seg == 0)
            prefetch((int64_t)item + 2 * gridDim.x);
#pragma unroll
        for (int j = 0; j < J; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                uint64_t xp[R];
#pragma unroll
                for (int r = 0; r < R; ++r)
                    xp[r] = pair_of<T>(part_of(x[r][j], q));
#pragma unroll
                for (int f = 0; f < W; ++f) {
                    const uint64_t wp = pair_of<T>(part_of(now[f][j], q));
#pragma unroll
                    for (int r = 0; r < R; ++r)
                        fma2(sum[f][r], wp, xp[r]);
                }
            }
        if (segs > 1)
            load_x(seg1);
        if (seg1 == 0) {
            // the rows are done: over the warp, then over the CTA
#pragma unroll
            for (int f = 0; f < W; ++f)
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    float s = __uint_as_float((uint32_t)sum[f][r]) + __uint_as_float((uint32_t)(sum[f][r] >> 32));
#pragma unroll
                    for (int o = 16; o > 0; o >>= 1)
                        s += __shfl_xor_sync(0xffffffffu, s, o);
                    if (lane == 0)
                        part[turn][f * R + r][warp] = s;
                    sum[f][r] = 0;
                }
            __syncthreads();
            const int f = threadIdx.x / R, r = threadIdx.x % R, n = item * NF + f;
            if (f < NF && r >= lo && r < hi && n < p.N) {
                float y = 0.0f, up = 0.0f;
#pragma unroll
                for (int w = 0; w < kWarps; ++w) {
                    y += part[turn][f * R + r][w];
                    if (KIND == HIDDEN)
                        up += part[turn][(NF + f) * R + r][w];
                }
                if (KIND == HIDDEN) {
                    if (p.pre) {
                        p.pre[r * 2 * p.fp + n] = y;
                        p.pre[r * 2 * p.fp + p.fp + n] = up;
                    }
                    with_act(p.act, [&](auto kind) { y = act_of<decltype(kind)::value>(y) * up; });
                }
                static_cast<T *>(p.out)[r * p.ldo + n] = from_f32<T>(y);
            }
            turn ^= 1;   // read before the next barrier, written after it
        }
#pragma unroll
        for (int f = 0; f < W; ++f)
#pragma unroll
            for (int j = 0; j < J; ++j)
                now[f][j] = next[f][j];
        item = item1;
        seg = seg1;
    }
}

template <int KIND, int R, int J, typename T>
cudaError_t launch(esp_moe *m, const VecParams &p)
{
    constexpr int W = kLoads<R> / J, NF = KIND == HIDDEN ? W / 2 : W;
    m->launches += 1;
    return launch_after(k_ff_vec<KIND, R, J, T>, dim3((unsigned)std::min<int64_t>(kCtas<R> * m->sm_count, ceil_div(p.N, NF))), kThreads,
                        0, m->stream, p);
}

// A weight row in one step where it can be; HIDDEN has rows of both matrices.
template <int KIND, int R, typename T>
cudaError_t by_length(esp_moe *m, const VecParams &p)
{
    constexpr int kMost = KIND == HIDDEN ? kLoads<R> / 2 : kLoads<R>;   // J
    if (kMost == 1 || p.K <= 8 * kThreads)
        return launch<KIND, R, 1, T>(m, p);
    if (kMost == 2 || p.K <= 16 * kThreads)
        return launch<KIND, R, std::min(2, kMost), T>(m, p);
    return launch<KIND, R, kMost, T>(m, p);
}

template <int KIND>
cudaError_t by_rows(esp_moe *m, int32_t dtype, const VecParams &p)
{
    return with_16(dtype, [&](auto elem) -> cudaError_t {
        using T = decltype(elem);
        return p.M == 1   ? by_length<KIND, 1, T>(m, p)
               : p.M == 2 ? by_length<KIND, 2, T>(m, p)
               : p.M <= 4 ? by_length<KIND, 4, T>(m, p)
                          : by_length<KIND, 8, T>(m, p);
    });
}

}  // namespace

bool use_vec(int64_t M, int32_t E, int32_t F, int32_t H)
{
    // Times of both products in a graph, weights not in L2 (us), here and on the tensor cores, whose kernels take 12 before the
    // weights' bytes count:
    //   rows  512 x 512  1024 x 2048  2048 x 2048  2048 x 4096  4096 x 4096  4096 x 8192  8192 x 8192  6144 x 16384 (604 MB)
    //   1     3.3  13.4    6.1  22.4    7.6  27.3   12.2  32.0   19.1  48     34.9  67      72  95      121  127
    //   2     3.4  13.4    7.3  22.4    8.9  27.3   14.7  32.0   23.1  48     45.2  67      94  95      170  127
    //   4     5.1  13.4   10.0  22.4   12.5  27.3   20.5  32.0   34.3  48     65.7  67     152  95      295  127
    //   8     6.9  13.4   16.0  22.4   20.2  27.3   32.0  32.0   76.8  48      179  67     335  95      498  127
    const int64_t bytes = 6 * (int64_t)F * H;
    return E == 1 && (M == 1 || (M == 2 && bytes <= 384 << 20) || (M <= 4 && bytes <= 160 << 20) || (M <= 8 && bytes <= 32 << 20));
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
