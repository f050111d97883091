// Products of the gated feed-forward blocks for few rows (single tokens, a row or two for each expert, and sizes that fill
// the tiles of esp_ff_gemm.cu badly): HIDDEN, OUT, DPRE and DX as named there, with the operands' roles exchanged.
//
// The weights are the MMA's 128 rows, the rows of x its NT columns (16 to 128). A tile is two blocks of 128 weight rows,
// each with an accumulator of its own (HIDDEN: the same 128 rows of G and of U, so that both halves of a hidden element
// meet in one thread), and NT rows of one expert. Every weight is loaded once for NT rows: bound by HBM until NT rows
// need more tensor time than the weights' bytes.
//
// Work is split evenly over the CTAs, one per SM, in blocks of the inner axis: all blocks of all tiles in one line, an
// equal run of it to each CTA. A tile whose blocks belong to several CTAs is joined by the last of them to finish, from
// sums in memory, added in the order of the line.
//
// Warps 0-3 own the accumulators (a thread a weight row), warp 4 loads by TMA, warp 5 issues the MMAs. Every wait is
// bounded, as in esp_fp8_gemm.cu.

#include <algorithm>

#include "esp_ff.cuh"
#include "esp_moe_launch.cuh"
#include "esp_moe_load.cuh"

namespace esp_moe_impl {

namespace {

constexpr int kThreads = 192;
constexpr int kEpilogueThreads = 128;
constexpr int kWeights = 2 * 128 * 128;   // bytes of a stage: two blocks of 128 weight rows
constexpr int kTable = (ESP_MOE_MAX_EXPERTS + 1) * 4 + 12;
constexpr int kLeast = 4;                 // blocks that a CTA takes at least

template <int NT>
struct Few {
    static constexpr int kStage = kWeights + NT * 128;
    static constexpr int kStages = std::min(6, (232448 - kTable - 256 - 1024) / kStage);
    static constexpr int kSmem = kStages * kStage + kTable + 256 + 1024;
    static constexpr uint32_t kTmem = 4 * NT;   // two tiles' accumulators in turn
    static constexpr int64_t kPart = 2 * 128 * NT;
    static_assert((2 * kStages + 5) * 8 + 16 <= 256, "barriers");
};

// Barrier of the epilogue's threads that also ANDs a predicate over them.
__device__ __forceinline__ bool all_of_epilogue(bool v)
{
    uint32_t r;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %1, 0;\n\tbar.red.and.pred q, 1, %2, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
        : "=r"(r)
        : "r"((uint32_t)v), "n"(kEpilogueThreads)
        : "memory");
    return r != 0;
}

__device__ __forceinline__ void load_box1(uint32_t dst, const CUtensorMap *map, int x, int y, int z, uint32_t bar)
{
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], "
        "[%5];" ::"r"(dst),
        "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
        : "memory");
}

__device__ __forceinline__ void mma16_one(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
        : "memory");
}

// The line of blocks: `units` of them, `per` for each tile; CTA c of `ctas` owns [units c / ctas, units (c + 1) / ctas).
struct Line {
    int64_t units;
    int per, ctas;
    __device__ int64_t first(int c) const { return units * c / ctas; }
    // the CTA that owns unit x
    __device__ int owner(int64_t x) const { return (int)(((x + 1) * ctas - 1) / units); }
};

// A CTA's part of a tile: blocks k0 .. k1 - 1 of rows m0 .. m0 + rows - 1 of expert e and weight rows n0 ..
struct Piece {
    int e, m0, rows, n0, k0, k1;
    int64_t unit;   // of the tile's first block
};

// table[e]: row chunks of the experts before e.
template <int KIND, int NT>
__device__ __forceinline__ bool piece_at(const FfParams &p, const int *table, const Line &l, int64_t u, int64_t end, Piece &t)
{
    if (u >= end)
        return false;
    const int64_t tile = u / l.per;
    t.unit = tile * l.per;
    t.k0 = (int)(u - t.unit);
    t.k1 = (int)min((int64_t)l.per, end - t.unit);
    const int ft = (p.g.N + (KIND == HIDDEN ? 127 : 255)) / (KIND == HIDDEN ? 128 : 256);
    int lo = 0, hi = p.g.E;   // the expert whose tiles hold this one
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if ((int64_t)table[mid] * ft <= tile)
            lo = mid;
        else
            hi = mid;
    }
    t.e = lo;
    const int chunks = table[lo + 1] - table[lo], i = (int)(tile - (int64_t)table[lo] * ft);
    int a, b;
    expert_rows(p.g, lo, a, b);
    t.m0 = a + (i % chunks) * NT;
    t.rows = min(NT, b - t.m0);
    t.n0 = (i / chunks) * (KIND == HIDDEN ? 128 : 256);
    return true;
}

// 16 rows' results of this thread's weight row: a, b are the two accumulators.
template <int KIND, typename T>
__device__ __forceinline__ void finish(const FfParams &p, const Piece &t, int first, const uint32_t (&a)[16],
                                       const uint32_t (&b)[16])
{
    const int n = t.n0 + (int)threadIdx.x, rows = min(16, t.rows - first);
    const int64_t y = t.m0 + first;
    if (KIND == HIDDEN) {
        if (n >= p.g.N)
            return;
        T *out = static_cast<T *>(p.g.out) + y * p.g.ldo + n;
        float *pre = static_cast<float *>(p.out2) + y * 2 * p.fp + n;
        with_act(p.act, [&](auto kind) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (i < rows) {
                    const float g = __uint_as_float(a[i]), u = __uint_as_float(b[i]);
                    out[i * p.g.ldo] = from_f32<T>(act_of<decltype(kind)::value>(g) * u);
                    if (p.out2) {
                        pre[i * 2 * p.fp] = g;
                        pre[i * 2 * p.fp + p.fp] = u;
                    }
                }
        });
        return;
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t(&v)[16] = h == 0 ? a : b;
        const int c = n + 128 * h;
        if (c >= p.g.N)
            return;
        if (KIND == DPRE) {
            const float *pre = static_cast<const float *>(p.pre) + y * 2 * p.fp + c;
            T *out = static_cast<T *>(p.g.out) + y * 2 * p.fp + c;
            with_act(p.act, [&](auto kind) {
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (i < rows) {
                        const float dh = __uint_as_float(v[i]), g = pre[i * 2 * p.fp], u = pre[i * 2 * p.fp + p.fp];
                        float act, slope;
                        act_and_slope<decltype(kind)::value>(g, act, slope);
                        out[i * 2 * p.fp] = from_f32<T>(dh * u * slope);
                        out[i * 2 * p.fp + p.fp] = from_f32<T>(dh * act);
                    }
            });
        } else {
            T *out = static_cast<T *>(p.g.out) + y * p.g.ldo + c;
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (i < rows)
                    out[i * p.g.ldo] = from_f32<T>(__uint_as_float(v[i]));
        }
    }
}

template <int KIND, int NT, typename T>
__global__ void __launch_bounds__(kThreads, 1)
    k_ff_few(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x, const FfParams p)
{
    using S = Few<NT>;
    constexpr bool W_MN = KIND == DPRE || KIND == DX;
    extern __shared__ unsigned char smem_raw[];
    unsigned char *sm = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                                          ~static_cast<uintptr_t>(1023));
    int *table = reinterpret_cast<int *>(sm + S::kStages * S::kStage);
    uint64_t *bars = reinterpret_cast<uint64_t *>(reinterpret_cast<unsigned char *>(table) + kTable);
    const uint32_t full = smem_u32(bars), empty = full + 8 * S::kStages, tfull = empty + 8 * S::kStages, tempty = tfull + 16,
                   drain = tempty + 16;
    uint32_t *slot = reinterpret_cast<uint32_t *>(bars + 2 * S::kStages + 5);
    volatile int *dead = reinterpret_cast<volatile int *>(slot + 1), *last = dead + 1;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        *dead = 0;
        for (int i = 0; i < S::kStages; ++i) {
            mbar_init(full + 8 * i, 1);
            mbar_init(empty + 8 * i, 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(tfull + 8 * i, 1);
            mbar_init(tempty + 8 * i, kEpilogueThreads / 32);
        }
        mbar_init(drain, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 5) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(slot)),
                     "r"(S::kTmem)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    wait_for_launch_before();
    if (warp == 4) {
        // the experts' row chunks before each: one warp's scan
        int carry = 0;
        for (int e0 = 0; e0 < p.g.E; e0 += 32) {
            int n = 0;
            if (e0 + lane < p.g.E) {
                int a, b;
                expert_rows(p.g, e0 + lane, a, b);
                n = (b - a) / NT + ((b - a) % NT != 0);
            }
            int s = n;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int y = __shfl_up_sync(0xffffffffu, s, o);
                if (lane >= o)
                    s += y;
            }
            if (e0 + lane < p.g.E)
                table[e0 + lane] = min(p.g.most, carry + s - n);
            carry = min(p.g.most, carry + __shfl_sync(0xffffffffu, s, 31));
        }
        if (lane == 0)
            table[p.g.E] = carry;
    }
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tmem = *slot;
    Line line;
    line.per = p.blocks * p.halves;
    line.units = (int64_t)table[p.g.E] * ((p.g.N + (KIND == HIDDEN ? 127 : 255)) / (KIND == HIDDEN ? 128 : 256)) * line.per;
    line.ctas = (int)max((int64_t)1, min((int64_t)gridDim.x, line.units / kLeast));
    const int c = blockIdx.x;
    const int64_t begin = c < line.ctas ? line.first(c) : line.units, end = c < line.ctas ? line.first(c + 1) : line.units;
    uint32_t issued = 0;
    Piece t;

    if (warp == 4) {
        int s = 0;
        uint32_t ph = 1;
        bool ok = true;
        for (int64_t u = begin; ok && piece_at<KIND, NT>(p, table, line, u, end, t); u = t.unit + t.k1)
            for (int kb = t.k0; kb < t.k1; ++kb) {
                if (!(ok = wait_phase(empty + 8 * s, ph, p.g, dead)))
                    break;
                const uint32_t w = smem_u32(sm + s * S::kStage), bar = full + 8 * s;
                const int half = KIND == DX && kb >= p.blocks ? 1 : 0, k = (kb - half * p.blocks) * kInner;
                if (elect_one()) {
                    mbar_expect(bar, S::kStage);
                    if (!(p.g.hold && issued == 2)) {
                        if (W_MN) {
                            const int z = KIND == DX ? 2 * t.e + half : t.e;
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                load_box1(w + i * kHalfTile, &map_w, t.n0 + 64 * i, k, z, bar);
                        } else {
                            load_box1(w, &map_w, k, t.n0, KIND == HIDDEN ? 2 * t.e : t.e, bar);
                            load_box1(w + kWeights / 2, &map_w, k, KIND == HIDDEN ? t.n0 : t.n0 + 128,
                                      KIND == HIDDEN ? 2 * t.e + 1 : t.e, bar);
                        }
                        load_box1(w + kWeights, &map_x, k, t.m0, half, bar);
                    }
                }
                __syncwarp();
                ++issued;
                if (++s == S::kStages) {
                    s = 0;
                    ph ^= 1;
                }
            }
    } else if (warp == 5) {
        const uint32_t format = p.half_f16 ? 0u : (1u << 7) | (1u << 10);
        const uint32_t idesc = (1u << 4) | format | (W_MN ? 1u << 15 : 0u) | ((uint32_t)(NT >> 3) << 17) |
                               ((uint32_t)(128 >> 4) << 24);
        int s = 0, acc = 0;
        uint32_t ph = 0, aph = 1;
        bool ok = true;
        for (int64_t u = begin; ok && piece_at<KIND, NT>(p, table, line, u, end, t); u = t.unit + t.k1) {
            if (!(ok = wait_phase(tempty + 8 * acc, aph, p.g, dead)))
                break;
            for (int kb = t.k0; kb < t.k1; ++kb) {
                if (!(ok = wait_phase(full + 8 * s, ph, p.g, dead)))
                    break;
                fence_after();
                const uint32_t w = smem_u32(sm + s * S::kStage);
                const uint64_t a0 = operand<W_MN>(w), a1 = operand<W_MN>(w + kWeights / 2), b = operand<false>(w + kWeights);
                if (elect_one()) {
#pragma unroll
                    for (int k = 0; k < kInner / 16; ++k) {
                        const uint32_t d = tmem + acc * 2 * NT;
                        mma16_one(d, a0 + k * kOperandStep<W_MN>, b + k * kOperandStep<false>, idesc, kb > t.k0 || k > 0);
                        mma16_one(d + NT, a1 + k * kOperandStep<W_MN>, b + k * kOperandStep<false>, idesc, kb > t.k0 || k > 0);
                    }
                    mma_commit<1>(empty + 8 * s);
                    if (kb == t.k1 - 1)
                        mma_commit<1>(tfull + 8 * acc);
                }
                __syncwarp();
                if (++s == S::kStages) {
                    s = 0;
                    ph ^= 1;
                }
            }
            acc ^= 1;
            aph ^= acc == 0;
        }
    } else {
        int acc = 0;
        uint32_t aph = 0;
        for (int64_t u = begin; piece_at<KIND, NT>(p, table, line, u, end, t); u = t.unit + t.k1) {
            // all four warps go on, or none: those that join a tile meet at a barrier
            if (!all_of_epilogue(wait_phase(tfull + 8 * acc, aph, p.g, dead)))
                break;
            fence_after();
            const uint32_t src = tmem + ((uint32_t)(32 * warp) << 16) + (uint32_t)(acc * 2 * NT);
            const bool whole = t.k1 - t.k0 == line.per;
            // its sums' place where it is a part: a CTA's run begins inside one tile and ends inside another
            float *mine = p.g.partial + (2 * c + (u == begin ? 0 : 1)) * S::kPart + threadIdx.x;
            uint32_t v[2][16];
            for (int i = 0; i < NT && i < t.rows; i += 16) {
                tmem_ld16(src + i, v[0]);
                tmem_ld16(src + NT + i, v[1]);
                tmem_wait(v);
                if (whole) {
                    finish<KIND, T>(p, t, i, v[0], v[1]);
                } else {
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        __stcg(mine + (i + j) * 128, __uint_as_float(v[0][j]));
                        __stcg(mine + (NT + i + j) * 128, __uint_as_float(v[1][j]));
                    }
                }
            }
            fence_before();
            __syncwarp();
            if (lane == 0)
                mbar_arrive_cta(tempty + 8 * acc);
            acc ^= 1;
            aph ^= acc == 0;
            if (whole)
                continue;
            const int from = line.owner(t.unit), to = line.owner(t.unit + line.per - 1);
            __threadfence();
            all_of_epilogue(true);
            if (threadIdx.x == 0) {
                // a CTA is the first of at most one tile that it shares
                const bool l = atomicAdd(p.g.tickets + from, 1u) == (unsigned)(to - from);
                if (l)
                    p.g.tickets[from] = 0u;
                *last = l;
                __threadfence();
            }
            all_of_epilogue(true);
            if (*last) {
                for (int i = 0; i < NT && i < t.rows; i += 16) {
                    float sum[2][16] = {};
                    for (int q = from; q <= to; ++q) {
                        const float *part =
                            p.g.partial + (2 * q + (q == from && line.first(q) != t.unit ? 1 : 0)) * S::kPart + threadIdx.x;
#pragma unroll
                        for (int j = 0; j < 16; ++j) {
                            sum[0][j] += __ldcg(part + (i + j) * 128);
                            sum[1][j] += __ldcg(part + (NT + i + j) * 128);
                        }
                    }
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        v[0][j] = __float_as_uint(sum[0][j]);
                        v[1][j] = __float_as_uint(sum[1][j]);
                    }
                    finish<KIND, T>(p, t, i, v[0], v[1]);
                }
            }
            all_of_epilogue(true);   // `last` has been read
        }
    }
    fence_before();
    __syncthreads();
    fence_after();
    if (*dead) {
        // nothing may still land in this CTA's memory: copies first, then MMAs
        if (warp == 4 && lane == 0)
            for (uint32_t i = issued < S::kStages ? 0 : issued - S::kStages; i < issued; ++i)
                wait_ms<OWN>(full + 8 * (i % S::kStages), (i / S::kStages) & 1, 20, nullptr);
        if (warp == 5 && elect_one()) {
            mma_commit<1>(drain);
            wait_ms<OWN>(drain, 0, 1000, nullptr);
        }
    }
    fence_before();
    __syncthreads();
    fence_after();
    if (warp == 5)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(S::kTmem) : "memory");
}

template <int KIND, int NT, typename T>
cudaError_t launch(esp_moe *m, const CUtensorMap &w, const CUtensorMap &x, const FfParams &p, int64_t blocks)
{
    const cudaError_t e = allow_smem<k_ff_few<KIND, NT, T>, Few<NT>::kSmem>(m->device);
    if (e != cudaSuccess)
        return e;
    const unsigned grid = (unsigned)std::max<int64_t>(1, std::min<int64_t>(few_ctas(m), blocks / kLeast));
    m->launches += 1;
    return launch_after(k_ff_few<KIND, NT, T>, dim3(grid), kThreads, Few<NT>::kSmem, m->stream, w, x, p);
}

template <int KIND>
cudaError_t by_chunk(esp_moe *m, int32_t dtype, int chunk, const CUtensorMap &w, const CUtensorMap &x, const FfParams &p,
                     int64_t blocks)
{
    return with_16(dtype, [&](auto elem) -> cudaError_t {
        using T = decltype(elem);
        if (chunk == 16)
            return launch<KIND, 16, T>(m, w, x, p, blocks);
        if (chunk == 32)
            return launch<KIND, 32, T>(m, w, x, p, blocks);
        if (chunk == 64)
            return launch<KIND, 64, T>(m, w, x, p, blocks);
        return launch<KIND, 128, T>(m, w, x, p, blocks);
    });
}

}  // namespace

int few_ctas(const esp_moe *m)
{
    return std::min(m->sm_count, kTickets - 1);
}

size_t few_partial_floats(const esp_moe *m, int chunk)
{
    return (size_t)few_ctas(m) * 2 * 2 * 128 * chunk;
}

cudaError_t launch_few(esp_moe *m, const FfShape &s, int kind, int chunk, const void *w, const void *x, const void *params)
{
    FfParams p = *static_cast<const FfParams *>(params);
    const CUtensorMap &mw = *static_cast<const CUtensorMap *>(w), &mx = *static_cast<const CUtensorMap *>(x);
    // at most this many chunks of rows: every expert with rows has one that is not full
    const int64_t chunks = s.E == 1 ? ceil_div(s.M, chunk) : s.M / chunk + std::min<int64_t>(s.E, s.M);
    p.g.most = (int32_t)chunks;
    const int64_t blocks = chunks * ceil_div(p.g.N, kind == HIDDEN ? 128 : 256) * p.blocks * p.halves;
    if (kind == HIDDEN)
        return by_chunk<HIDDEN>(m, s.dtype, chunk, mw, mx, p, blocks);
    if (kind == OUT)
        return by_chunk<OUT>(m, s.dtype, chunk, mw, mx, p, blocks);
    if (kind == DPRE)
        return by_chunk<DPRE>(m, s.dtype, chunk, mw, mx, p, blocks);
    return by_chunk<DX>(m, s.dtype, chunk, mw, mx, p, blocks);
}

}  // namespace esp_moe_impl
