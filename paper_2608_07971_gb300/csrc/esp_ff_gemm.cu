// Products of the gated feed-forward blocks (include/esp_moe.h) on the tensor cores: 16-bit operands (tcgen05.mma
// kind::f16), sums over the whole inner axis in tensor memory.
//
//   HIDDEN  rows x [G; U]^T, and from both accumulators act(g) * u: projections, activation and product in one kernel
//   OUT     hidden x O^T
//   DPRE    dy x O, and from it and the kept g, u the gradients of g and u
//   DX      dpre x [G; U]
//   DW      dpre^T x rows and dy^T x hidden: the inner axis is an expert's rows; its last ones, where they do not fill a
//           block of 64, come from copies padded with zeros (Tails), so that no other expert's rows, NaN included, reach
//           the sums
//
// Every operand is read as it lies in memory: where the inner axis is the contiguous one, a tile is K-major (rows of 64
// inner elements, 128 bytes, 128-byte swizzle), else MN-major (rows of 64 outer elements, one for each inner index; an
// MMA's operand then is two such tiles side by side). No transposed copies are made.
//
// A tile is 256 rows of two CTAs (cta_group::2, each holding 128 rows of A and half of B's 256 columns; HIDDEN: one CTA
// loads 128 columns of G, the other the same ones of U, so that both halves of a hidden element meet in one thread).
// Two accumulators of 256 columns: warps 0-7 empty one while the tensor core fills the other. Warp 8 loads by TMA,
// warp 9 issues the MMAs. CTAs are persistent.
//
// Bound by the tensor pipe where it can be kept fed, and under a long load by the card's power: 8192 rows x 4096 x 8192
// (HIDDEN and OUT) takes 861 us in a burst (1.92 PFLOP/s, the library's bf16 product 1.88) and 990 to 1020 after a second
// of load. What else the kernels move is nearly on top of that, as the operands already take 64 bytes of L2 a clock and
// SM: with half of the operands' loads left out, the same takes 790 us; with g and u kept in 32 bits, HIDDEN of 9728 rows x
// 2048 x 2048 takes 22 us more, their bytes at HBM's rate. Experts' rows are the other loss: tiles of 256 rows are half
// empty at each expert's end (16384 rows over 16 experts of uneven load as if they were 18400).
//   single CTAs: 128 rows x 256 columns, 48 instead of 32 KB for the same MMAs (8192 x 2048 x 2048: 137 us, pairs 119); for
//     few tiles, or many experts of few rows (8 x 256 rows, 2048 x 1024: 37 us, pairs 46)
//   split inner axes: a tile's parts meet in memory (one of 16 rows, 4096 x 8192: 58 us, whole 82, pairs 71)
// What did not help: gathering rows of A by the kernel itself with 16-byte asynchronous copies (64 experts of 1024 rows,
// 2048 x 1024: 1490 us, with a copy of the rows before 530 + 55), a third box for DPRE's g and u at the cost of a stage (234 us,
// 210 with two), g and u in 16 bits with block scales (15 us less in HIDDEN of a training step, 25 more in ragged small ones).
//
// Every wait is bounded, as in esp_fp8_gemm.cu.

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "esp_ff.cuh"
#include "esp_moe_launch.cuh"
#include "esp_moe_load.cuh"

namespace esp_moe_impl {

namespace {

constexpr int kThreads = 320;
constexpr int kEpilogueWarps = 8;
constexpr int kTileBytes = kRowsA * 128;             // 128 rows of one operand in a stage
constexpr int kBoxBytes = 128, kBox = 32 * kBoxBytes;
constexpr uint32_t kTmemCols = 512;
constexpr int kAccCols = 256;
constexpr int kBars = 256;
constexpr int kOrdered = 512;                        // experts that DW can put in order

// CG: CTAs that share a tile. An epilogue warp stages its stores in boxes; DPRE's g and u arrive in two (a third one, for
// the next g and u, at the cost of a stage of the operands: 16384 x 2048 x 4096 234 us, 210 with two).
template <int CG, int KIND>
struct Shape {
    static constexpr int kStageB = CG == 2 ? kTileBytes : 2 * kTileBytes;
    static constexpr int kStage = kTileBytes + kStageB;
    static constexpr int kStages = (CG == 2 ? 5 : 4) - (KIND == DPRE && CG == 1 ? 1 : 0);
    static constexpr int kBoxes = KIND == DPRE || CG == 2 ? 2 : 1;
    static constexpr int kSmem = kStages * kStage + kEpilogueWarps * kBoxes * kBox + kBars + 2 * kOrdered + 1024;
    static_assert((2 * kStages + 2 * 2 + 1 + kEpilogueWarps) * 8 + 16 <= kBars, "barriers");
    static_assert(kSmem <= 232448, "shared memory");
};

// A box into this CTA's shared memory; its bytes arrive at a barrier of this CTA or of the other one of a pair.
template <int CG>
__device__ __forceinline__ void load_box(uint32_t dst, const CUtensorMap *map, int x, int y, int z, uint32_t bar)
{
    if (CG == 2)
        asm volatile(
            "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, "
            "{%2, %3, %4}], [%5];" ::"r"(dst),
            "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
            : "memory");
    else
        asm volatile(
            "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], "
            "[%5];" ::"r"(dst),
            "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
            : "memory");
}

__device__ __forceinline__ void prefetch_map(const CUtensorMap *map)
{
    asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
}

template <int CG>
__device__ __forceinline__ void mma16(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate)
{
    if (CG == 2)
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
            "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
            : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
            "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
            : "memory");
}

// ---- a warp's staged box: 128 bytes of 32 rows, 16-byte chunk j of row r at place j ^ (r & 7) (the 128-byte swizzle), or
// half a box: 64 bytes of 32 rows, chunk j at place j ^ (r / 2 & 3) (the 64-byte swizzle).
template <int BYTES>
__device__ __forceinline__ int box_place(int r, int j)
{
    return r * BYTES + (BYTES == 128 ? j ^ (r & 7) : j ^ (r >> 1 & 3)) * 16;
}

// N boxes, used in turn.
template <int N>
class Staging {
public:
    __device__ explicit Staging(unsigned char *at) : at_(at) {}
    // The next box, once its last store has been read (each box's stores are one bulk group).
    __device__ __forceinline__ unsigned char *next()
    {
        asm volatile("cp.async.bulk.commit_group;\n\tcp.async.bulk.wait_group.read %0;" ::"n"(N - 1) : "memory");
        __syncwarp();
        turn_ = turn_ == N - 1 ? 0 : turn_ + 1;
        return at_ + turn_ * kBox;
    }

    // Waits until the stores of all boxes have been read.
    __device__ __forceinline__ void drain()
    {
        asm volatile("cp.async.bulk.commit_group;\n\tcp.async.bulk.wait_group.read 0;" ::: "memory");
        __syncwarp();
    }

private:
    unsigned char *at_;
    int turn_ = 0;
};

// Values of this lane's row into and out of chunk j.
template <typename T, int BYTES>
__device__ __forceinline__ void box_put(unsigned char *box, int lane, int j, const float *v)
{
    store_pack<T, 16 / (int)sizeof(T)>(reinterpret_cast<T *>(box + box_place<BYTES>(lane, j)), v);
}

__device__ __forceinline__ void box_get(const unsigned char *box, int lane, int j, float *v)
{
    load_pack<float, 4>(reinterpret_cast<const float *>(box + box_place<128>(lane, j)), v);
}

template <typename T>
__device__ __forceinline__ bool rows_aligned4(const T *p, int64_t ld)
{
    return ((reinterpret_cast<uintptr_t>(p) | (uintptr_t)ld * sizeof(T)) & 3) == 0;
}

// The box leaves: by one TMA store where all its rows are there to be written (columns past the matrix are dropped by the
// store), else by the lanes: rows at or past `rows`, columns at or past `cols` are dropped.
template <typename T, int BYTES>
__device__ __forceinline__ void box_store(const CUtensorMap *map, int x, int y, int z, T *out, int64_t ldo, int rows,
                                          int cols, bool wide, const unsigned char *box, int lane)
{
    constexpr int V = 16 / (int)sizeof(T), C = BYTES / (int)sizeof(T), J = BYTES / 16;
    if (wide && rows >= 32) {
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0)
            asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%1, %2, %3}], [%4];" ::"l"(map),
                         "r"(x), "r"(y), "r"(z), "r"(smem_u32(box))
                         : "memory");
        return;
    }
    __syncwarp();
    if (wide && cols >= C) {
        const int j = lane % J;
#pragma unroll
        for (int i = 0; i < J; ++i) {
            const int r = lane / J + i * (32 / J);
            if (r < rows)
                *reinterpret_cast<uint4 *>(out + r * ldo + j * V) =
                    *reinterpret_cast<const uint4 *>(box + box_place<BYTES>(r, j));
        }
    } else if (BYTES == 128 && cols >= C && rows_aligned4(out, ldo)) {   // a lane 4 bytes of every row
#pragma unroll 8
        for (int r = 0; r < 32; ++r)
            if (r < rows)
                reinterpret_cast<uint32_t *>(out + r * ldo)[lane] =
                    *reinterpret_cast<const uint32_t *>(box + box_place<BYTES>(r, lane / 4) + lane % 4 * 4);
    } else {
#pragma unroll
        for (int c0 = 0; c0 < C; c0 += 32) {
            const int c = c0 + lane;
#pragma unroll 8
            for (int r = 0; r < 32; ++r)
                if (r < rows && c < cols)
                    out[r * ldo + c] = reinterpret_cast<const T *>(box + box_place<BYTES>(r, c / V))[c % V];
        }
    }
    __syncwarp();
}

// Barrier of the epilogue's threads that also ANDs a predicate over them.
__device__ __forceinline__ bool all_of_epilogue(bool v)
{
    uint32_t r;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %1, 0;\n\tbar.red.and.pred q, 1, %2, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
        : "=r"(r)
        : "r"((uint32_t)v), "n"(32 * kEpilogueWarps)
        : "memory");
    return r != 0;
}

// s + c = s + c + v, what s rounds off kept in c.
__device__ __forceinline__ void add_exactly(float &s, float &c, float v)
{
    const float t = s + v, z = t - s;
    c += (s - (t - z)) + (v - z);
    s = t;
}

// A warp's product of two rows of n 16-bit elements on 16 bytes, to within 2^-24 of itself and about n 2^-48 of the sum of its
// terms' magnitudes: the terms are exact in 32 bits, their sums are kept in two numbers.
template <typename T>
__device__ __noinline__ float exact_dot(const T *a, const T *b, int n)
{
    const int lane = threadIdx.x & 31;
    float s = 0.0f, c = 0.0f;
    constexpr int kAhead = 4;   // loads in flight: one after the other a dot of 8192 takes 30 us next to the tensor core's loads
    const uint4 none = {0u, 0u, 0u, 0u};
    for (int i = 8 * lane; i < n; i += 256 * kAhead) {
        uint4 va[kAhead], vb[kAhead];
#pragma unroll
        for (int q = 0; q < kAhead; ++q) {
            const bool in = i + 256 * q + 8 <= n;
            va[q] = in ? __ldcg(reinterpret_cast<const uint4 *>(a + i + 256 * q)) : none;
            vb[q] = in ? __ldcg(reinterpret_cast<const uint4 *>(b + i + 256 * q)) : none;
        }
#pragma unroll
        for (int q = 0; q < kAhead; ++q) {
            const T *ea = reinterpret_cast<const T *>(&va[q]), *eb = reinterpret_cast<const T *>(&vb[q]);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                add_exactly(s, c, float(ea[j]) * float(eb[j]));
        }
    }
    if (const int j = (n & ~7) + lane; j < n)   // fewer than 8 are left
        add_exactly(s, c, float(__ldcg(a + j)) * float(__ldcg(b + j)));
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
        const float other = __shfl_xor_sync(0xffffffffu, s, d);
        c += __shfl_xor_sync(0xffffffffu, c, d);
        add_exactly(s, c, other);
    }
    return s + c;
}

// Tensor maps of a product. a2, b2: DW's tails; a2: HIDDEN's and DPRE's pre.
struct OneMaps {
    CUtensorMap a, b, out, a2, b2;
};

template <int KIND>
struct FfMaps {
    OneMaps of[KIND == DW ? 2 : 1];   // DW: of each gradient
};

// T: operands; O: output.
template <int CG, int KIND, typename T, typename O>
__global__ void __launch_bounds__(kThreads, 1)
    k_ff(const __grid_constant__ FfMaps<KIND> maps, const FfParams p)
{
    using S = Shape<CG, KIND>;
    constexpr int kStages = S::kStages, kStage = S::kStage;
    constexpr bool A_MN = KIND == DW, B_MN = KIND == DPRE || KIND == DX || KIND == DW;
    extern __shared__ unsigned char smem_raw[];
    unsigned char *sm = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                                          ~static_cast<uintptr_t>(1023));
    unsigned char *staging = sm + kStages * kStage;
    uint64_t *bars = reinterpret_cast<uint64_t *>(staging + kEpilogueWarps * S::kBoxes * kBox);
    const uint32_t full = smem_u32(bars), empty = full + 8 * kStages, tfull = empty + 8 * kStages, tempty = tfull + 16,
                   drain = tempty + 16, landed = drain + 8;
    uint16_t *order = reinterpret_cast<uint16_t *>(bars + kBars / 8);
    uint32_t *slot = reinterpret_cast<uint32_t *>(bars + 2 * kStages + 5 + kEpilogueWarps);
    volatile int *dead = reinterpret_cast<volatile int *>(slot + 1), *last = dead + 1;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = CG == 1 ? 0 : cluster_rank();

    if (threadIdx.x == 0) {
        *dead = 0;
        for (int i = 0; i < kStages; ++i) {
            mbar_init(full + 8 * i, 1);
            mbar_init(empty + 8 * i, 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(tfull + 8 * i, 1);
            mbar_init(tempty + 8 * i, CG * kEpilogueWarps);
        }
        mbar_init(drain, 1);
        for (int i = 0; i < kEpilogueWarps; ++i)
            mbar_init(landed + 8 * i, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 8 && lane == 0) {
        prefetch_map(&maps.of[0].a);
        prefetch_map(&maps.of[0].b);
        prefetch_map(&maps.of[0].out);
    }
    if (warp == 9) {
        if (CG == 2) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(slot)),
                         "r"(kTmemCols)
                         : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(slot)),
                         "r"(kTmemCols)
                         : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        }
    }
    fence_before();
    __syncthreads();
    if (CG == 2)
        cluster_sync();
    fence_after();
    wait_for_launch_before();
    // The launch after starts on SMs that are free (40 rows of 64 x 64: both products 9.4 us in a graph, 11.7 without). Where
    // few are, its waiting CTAs keep an SM from this one's (a ragged training step 174 us, 203 with it always).
    if (p.few_ctas)
        let_next_launch_start();
    const uint32_t tmem = *slot;
    uint32_t issued = 0;   // loads of this CTA's loading warp
    const int me = blockIdx.x / CG, n = gridDim.x / CG;
    FfTile t;
    Walk<CG, KIND> walk;
    if (KIND == DW && p.g.E > 1 && p.g.E <= kOrdered) {
        // longest inner axes first, so that the list ends with short items (dinner and douter of 16384 rows over 16 uneven experts,
        // 4096 x 2048: a launch each 328 and 170 us; in the experts' own order 345 and 178)
        int *blocks = reinterpret_cast<int *>(sm);   // nothing is loaded yet
        for (int e = threadIdx.x; e < p.g.E; e += kThreads) {
            int lo, hi;
            expert_rows(p.g, e, lo, hi);
            blocks[e] = (hi - lo + kInner - 1) / kInner;
        }
        __syncthreads();
        for (int e = threadIdx.x; e < p.g.E; e += kThreads) {
            int at = 0;
            for (int f = 0; f < p.g.E; ++f)
                at += blocks[f] > blocks[e] || (blocks[f] == blocks[e] && f < e);
            order[at] = (uint16_t)e;
        }
        // the loads that follow write the same memory through the other proxy
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncthreads();
        if (CG == 2)
            cluster_sync();
        walk.order = order;
    }

    if (warp == 8) {
        const uint32_t full0 = CG == 1 ? full : map_rank(full, 0);
        int s = 0;
        uint32_t ph = 1;
        bool ok = true;
        while (ok && walk.next(p, me, n, t)) {
            const OneMaps &map = maps.of[KIND == DW ? t.q : 0];
            const int outer_a = t.m0 + (int)rank * kRowsA;
            const int outer_b = t.n0 + (KIND == HIDDEN ? 0 : (int)rank * 128);
            for (int kb = t.k0; kb < t.k1; ++kb) {
                if (!(ok = wait_phase(empty + 8 * s, ph, p.g, dead)))
                    break;
                const uint32_t a = smem_u32(sm + s * kStage), b = a + kTileBytes;
                const int half = KIND == DX && kb >= p.blocks ? 1 : 0, k = (kb - half * p.blocks) * kInner;
                const bool cut = KIND == DW && t.cut && kb == t.k1 - 1;
                if (elect_one()) {
                    const uint32_t bar = full0 + 8 * s;
                    if (rank == 0)
                        mbar_expect(full + 8 * s, CG * kStage);
                    if (!(p.g.hold && issued == 2)) {
                        constexpr int kHalves = S::kStageB / kHalfTile;   // MN-major halves of B
                        // DW: the inner axis' first row, and the tensors that hold it
                        const int y = KIND == DW ? (cut ? t.e * kInner : t.lo + k) : k;
                        const CUtensorMap *const a_map = KIND == DW && cut ? &map.a2 : &map.a;
                        const CUtensorMap *const b_map = KIND == DW && cut ? &map.b2 : &map.b;
                        if (A_MN) {
                            load_box<CG>(a, a_map, outer_a, y, t.z, bar);
                            load_box<CG>(a + kHalfTile, a_map, outer_a + 64, y, t.z, bar);
                        } else {
                            load_box<CG>(a, &map.a, k, outer_a, half, bar);
                        }
                        if (B_MN) {
                            const int z = KIND == DW ? 0 : KIND == DX ? 2 * t.e + half : t.e;
#pragma unroll
                            for (int i = 0; i < kHalves; ++i)
                                load_box<CG>(b + i * kHalfTile, b_map, outer_b + 64 * i, y, z, bar);
                        } else if (KIND == HIDDEN) {
                            load_box<CG>(b, &map.b, k, outer_b, 2 * t.e + (int)rank, bar);
                            if (CG == 1)
                                load_box<CG>(b + kTileBytes, &map.b, k, outer_b, 2 * t.e + 1, bar);
                        } else {
                            load_box<CG>(b, &map.b, k, outer_b, t.e, bar);
                            if (CG == 1)
                                load_box<CG>(b + kTileBytes, &map.b, k, outer_b + 128, t.e, bar);
                        }
                    }
                }
                __syncwarp();
                ++issued;
                if (++s == kStages) {
                    s = 0;
                    ph ^= 1;
                }
            }
        }
    } else if (warp == 9) {
        if (rank == 0) {
            const uint32_t format = p.half_f16 ? 0u : (1u << 7) | (1u << 10);
            const uint32_t idesc = (1u << 4) | format | (A_MN ? 1u << 15 : 0u) | (B_MN ? 1u << 16 : 0u) |
                                   ((uint32_t)(kAccCols >> 3) << 17) | ((uint32_t)(128 * CG >> 4) << 24);
            int s = 0, acc = 0;
            uint32_t ph = 0, aph = 1;
            bool ok = true;
            while (ok && walk.next(p, me, n, t)) {
                if (t.k0 == t.k1)
                    continue;
                if (!(ok = wait_phase<CG == 2 ? HANDBACK : OWN>(tempty + 8 * acc, aph, p.g, dead)))
                    break;
                for (int kb = t.k0; kb < t.k1; ++kb) {
                    if (!(ok = wait_phase(full + 8 * s, ph, p.g, dead)))
                        break;
                    fence_after();
                    const uint64_t a = operand<A_MN>(smem_u32(sm + s * kStage));
                    const uint64_t b = operand<B_MN>(smem_u32(sm + s * kStage + kTileBytes));
                    if (elect_one()) {
#pragma unroll
                        for (int k = 0; k < kInner / 16; ++k)
                            mma16<CG>(tmem + acc * kAccCols, a + k * kOperandStep<A_MN>, b + k * kOperandStep<B_MN>, idesc,
                                  kb > t.k0 || k > 0);
                        mma_commit<CG>(empty + 8 * s);
                        if (kb == t.k1 - 1)
                            mma_commit<CG>(tfull + 8 * acc);
                    }
                    __syncwarp();
                    if (++s == kStages) {
                        s = 0;
                        ph ^= 1;
                    }
                }
                acc ^= 1;
                aph ^= acc == 0;
            }
        }
    } else if (warp < kEpilogueWarps) {
        const int wg = warp >> 2, quarter = warp & 3;
        const uint32_t tempty0 = CG == 1 ? tempty : map_rank(tempty, 0);
        unsigned char *const gbox = staging + warp * S::kBoxes * kBox, *const ubox = gbox + kBox;   // DPRE
        Staging<S::kBoxes> boxes(gbox);
        int acc = 0;
        uint32_t aph = 0, lph = 0;
        bool loading = false;   // DPRE: g and u are on their way to the staging boxes
        while (walk.next(p, me, n, t)) {
            const OneMaps &map = maps.of[KIND == DW ? t.q : 0];
            const int N = KIND == DW ? p.dw[t.q].N : p.g.N;   // columns of the output
            const int rows = t.rows - (int)rank * kRowsA - 32 * quarter;   // of this warp's 32 that exist, from the first
            const int y = t.m0 + (int)rank * kRowsA + 32 * quarter;        // the first
            const bool split = CG == 1 && p.g.splits > 1, some = t.k0 < t.k1;
            const uint32_t src = tmem + ((uint32_t)(32 * quarter) << 16) + (uint32_t)(acc * kAccCols);
            // DPRE: 32 columns of g and u at a time, from column c of the tile on, into two boxes; they arrive together. The
            // fence: the lanes' own reads and writes of the boxes come before the copies, which write through the other proxy
            const auto load_pre = [&](int c) {
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) {
                    mbar_expect(landed + 8 * warp, 2 * kBox);
                    load_box<CG>(smem_u32(gbox), &map.a2, t.n0 + c, y, 0, landed + 8 * warp);
                    load_box<CG>(smem_u32(ubox), &map.a2, t.n0 + c, y, 1, landed + 8 * warp);
                }
                loading = true;
            };
            const int first = 128 * wg, columns = min(128, N - t.n0 - first);   // of this warp (not HIDDEN)
            if (KIND == DPRE && !split && rows > 0 && columns > 0) {
                boxes.drain();
                load_pre(first);
            }
            bool ok = !some || wait_phase(tfull + 8 * acc, aph, p.g, dead);
            if (split)   // all warps go on, or none: those that join a tile meet at a barrier
                ok = all_of_epilogue(ok);
            if (!ok)
                break;
            fence_after();
            bool joined = false, skip = rows <= 0;
            // 16 columns of this thread's row from each of four places
            const float *parts = nullptr;
            uint32_t v[4][16];
            const auto fetch = [&](int c0, int c1, int c2, int c3) {
                const int c[4] = {c0, c1, c2, c3};
                if (joined) {
#pragma unroll
                    for (int i = 0; i < 64; ++i)
                        v[i / 16][i % 16] = 0u;
                    for (int q = 0; q < p.g.splits; ++q) {
                        float one[64];   // all on their way before the first is added
#pragma unroll
                        for (int i = 0; i < 64; ++i)
                            one[i] = __ldcg(parts + ((int64_t)q * kAccCols + c[i / 16] + i % 16) * kRowsA);
#pragma unroll
                        for (int i = 0; i < 64; ++i)
                            v[i / 16][i % 16] = __float_as_uint(__uint_as_float(v[i / 16][i % 16]) + one[i]);
                    }
                } else if (some) {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        tmem_ld16(src + c[i], v[i]);
                    tmem_wait(v);
                } else {
#pragma unroll
                    for (int i = 0; i < 64; ++i)
                        v[i / 16][i % 16] = 0u;
                }
            };
            const auto release = [&] {   // the accumulator has been read
                if (!some)
                    return;
                fence_before();
                __syncwarp();
                if (lane == 0) {
                    if (CG == 2)
                        arrive_relaxed(tempty0 + 8 * acc);
                    else
                        mbar_arrive_cta(tempty0 + 8 * acc);
                }
            };
            if (split) {
                // this part's sums go to memory; the last part of the tile to arrive adds all of them up, in order
                const int tile = t.item / p.g.splits;
                float *const of_tile =
                    p.g.partial + (int64_t)tile * p.g.splits * kAccCols * kRowsA + 32 * quarter + lane;
                float *const mine = of_tile + (int64_t)(t.item - tile * p.g.splits) * kAccCols * kRowsA;
                if (!skip)
                    for (int b = 0; b < 2; ++b) {
                        const int c = KIND == HIDDEN ? 128 * b + 64 * wg : first + 64 * b;
                        fetch(c, c + 16, c + 32, c + 48);
#pragma unroll
                        for (int i = 0; i < 64; ++i)
                            __stcg(mine + (int64_t)(c + i) * kRowsA, __uint_as_float(v[i / 16][i % 16]));
                    }
                release();
                __threadfence();
                all_of_epilogue(true);
                if (threadIdx.x == 0) {
                    const bool l = atomicAdd(p.g.tickets + tile, 1u) == (unsigned)p.g.splits - 1;
                    if (l)
                        p.g.tickets[tile] = 0u;
                    *last = l;
                    __threadfence();
                }
                all_of_epilogue(true);
                joined = true;
                parts = of_tile;
                skip = skip || !*last;
                all_of_epilogue(true);   // `last` has been read
                if (KIND == DPRE && !skip && columns > 0) {
                    boxes.drain();
                    load_pre(first);
                }
            }
            if (!skip) {
                if (KIND == HIDDEN) {
                    const int c = 64 * wg, n = t.n0 + c, cols = N - n;
                    if (cols > 0) {
                        if (p.out2) {
#pragma unroll 1
                            for (int half = 0; half < 2; ++half) {   // g, u
                                const int at = 128 * half + c;
                                const bool again = half == 0 && p.lengths;
                                float mine = 0.0f, length[2] = {0.0f, 0.0f};   // of this lane's row and columns; 0: not there
                                if (again) {
                                    const float *const of = p.lengths + p.g.M + (int64_t)t.e * N + n;
                                    mine = lane < rows ? p.near_zero * __ldcg(p.lengths + y + lane) : 0.0f;
#pragma unroll
                                    for (int i = 0; i < 2; ++i)
                                        length[i] = 32 * i + lane < cols ? __ldcg(of + 32 * i + lane) : 0.0f;
                                }
                                fetch(at, at + 16, at + 32, at + 48);
                                if (again) {
                                    // the g whose sign the tensor core's sum leaves open
                                    const float most = __uint_as_float(
                                        __reduce_max_sync(0xffffffffu, __float_as_uint(fmaxf(length[0], length[1]))));
                                    float least = INFINITY;
#pragma unroll
                                    for (int i = 0; i < 64; ++i)
                                        if (i < cols)
                                            least = fminf(least, fabsf(__uint_as_float(v[i / 16][i % 16])));
                                    uint64_t open = 0;
                                    if (__any_sync(0xffffffffu, least < mine * most)) {
                                        uint64_t zeros = 0;
#pragma unroll
                                        for (int i = 0; i < 64; ++i) {
                                            const float g = fabsf(__uint_as_float(v[i / 16][i % 16]));
                                            if (g < mine * __shfl_sync(0xffffffffu, length[i / 32], i % 32)) {
                                                open |= 1ull << i;
                                                zeros |= (uint64_t)(g == 0.0f) << i;
                                            }
                                        }
                                        // many of exactly 0 are of operands that have no common elements, not of what is cut off
                                        if (__reduce_add_sync(0xffffffffu, (unsigned)__popcll(zeros)) > 64)
                                            open &= ~zeros;
                                    }
                                    for (unsigned left; (left = __ballot_sync(0xffffffffu, open != 0)) != 0;) {
                                        const int r = __ffs(left) - 1, at0 = __shfl_sync(0xffffffffu, __ffsll(open) - 1, r);
                                        const float g = exact_dot(
                                            static_cast<const T *>(p.x) + (int64_t)(y + r) * p.ldx,
                                            static_cast<const T *>(p.inner) + ((int64_t)2 * t.e * N + n + at0) * p.ld_inner,
                                            p.g.K);
                                        if (lane == r) {
                                            open &= open - 1;
#pragma unroll
                                            for (int i = 0; i < 64; ++i)
                                                if (i == at0)
                                                    v[i / 16][i % 16] = __float_as_uint(g);
                                        }
                                    }
                                }
#pragma unroll
                                for (int b = 0; b < 2; ++b) {
                                    if (32 * b >= cols)
                                        break;
                                    unsigned char *box = boxes.next();
#pragma unroll
                                    for (int j = 0; j < 8; ++j)
                                        box_put<float, 128>(box, lane, j,
                                                            reinterpret_cast<const float *>(&v[2 * b + j / 4][4 * (j & 3)]));
                                    box_store<float, 128>(
                                        &map.a2, n + 32 * b, y, half,
                                        static_cast<float *>(p.out2) + y * 2 * p.fp + half * p.fp + n + 32 * b, 2 * p.fp, rows,
                                        cols - 32 * b, true, box, lane);
                                }
                            }
                        }
                        unsigned char *box = boxes.next();
                        // A loop, as is the one above: where there is one round of tiles this runs once, from a cold
                        // instruction cache (1801 rows of 5 experts, 2050 x 999, gelu: both products 50 us, unrolled 56).
                        with_act(p.act, [&](auto kind) {
#pragma unroll 1
                            for (int h = 0; h < 2; ++h) {
                                fetch(c + 32 * h, c + 32 * h + 16, 128 + c + 32 * h, 128 + c + 32 * h + 16);
#pragma unroll
                                for (int j = 0; j < 4; ++j) {
                                    float r[8];
#pragma unroll
                                    for (int i = 0; i < 8; ++i)
                                        r[i] = act_of<decltype(kind)::value>(__uint_as_float(v[j / 2][8 * (j & 1) + i])) *
                                               __uint_as_float(v[2 + j / 2][8 * (j & 1) + i]);
                                    box_put<T, 128>(box, lane, 4 * h + j, r);
                                }
                            }
                        });
                        box_store<T, 128>(&map.out, n, y, 0, static_cast<T *>(p.g.out) + y * p.g.ldo + n, p.g.ldo, rows, cols,
                                          true, box, lane);
                    }
                } else if (KIND == DPRE) {
                    bool landed_all = true;
                    for (int c = first; c < first + columns; c += 32) {
                        const int h = (c - first) & 32;   // columns come 64 at a time
                        if (h == 0)
                            fetch(c, c + 16, c + 32, c + 48);
                        if (!(landed_all = wait_phase(landed + 8 * warp, lph, p.g, dead)))
                            break;
                        loading = false;
                        lph ^= 1;
                        float g[32], u[32];
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            box_get(gbox, lane, j, g + 4 * j);
                            box_get(ubox, lane, j, u + 4 * j);
                        }
                        __syncwarp();
                        with_act(p.act, [&](auto kind) {
#pragma unroll
                            for (int i = 0; i < 32; ++i) {
                                const float dh = __uint_as_float(h == 0 ? v[i / 16][i % 16] : v[2 + i / 16][i % 16]);
                                float a, slope;
                                act_and_slope<decltype(kind)::value>(g[i], a, slope);
                                g[i] = dh * u[i] * slope;
                                u[i] = dh * a;
                            }
                        });
                        // both results, 64 bytes of every row, in the box that u came in
                        const int n = t.n0 + c;
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            box_put<T, 64>(ubox, lane, j, g + 8 * j);
                            box_put<T, 64>(ubox + kBox / 2, lane, j, u + 8 * j);
                        }
                        T *out = static_cast<T *>(p.g.out) + y * 2 * p.fp + n;
                        box_store<T, 64>(&map.out, n, y, 0, out, 2 * p.fp, rows, N - n, true, ubox, lane);
                        box_store<T, 64>(&map.out, n, y, 1, out + p.fp, 2 * p.fp, rows, N - n, true, ubox + kBox / 2, lane);
                        if (c + 32 < first + columns) {
                            boxes.drain();
                            load_pre(c + 32);
                        }
                    }
                    if (!landed_all)
                        break;
                } else {
                    constexpr int C = kBoxBytes / (int)sizeof(O), V = 16 / (int)sizeof(O);
                    const int z = KIND == DW ? t.e * p.dw[t.q].planes + t.z : 0;
                    const int64_t ldo = KIND == DW ? N : p.g.ldo;
                    const bool wide = KIND == DW ? p.dw[t.q].wide : p.g.wide_store;
                    O *out = KIND == DW ? static_cast<O *>(p.dw[t.q].out) + ((int64_t)z * p.dw[t.q].out_rows + y) * ldo + t.n0
                                        : static_cast<O *>(p.g.out) + y * ldo + t.n0;
                    for (int c = first; c < first + columns; c += 64) {
                        fetch(c, c + 16, c + 32, c + 48);
#pragma unroll
                        for (int b = 0; b < 64 / C; ++b) {
                            const int n = c + b * C, cols = N - t.n0 - n;
                            if (cols <= 0)
                                break;
                            unsigned char *box = boxes.next();
#pragma unroll
                            for (int j = 0; j < 8; ++j) {
                                const int i = b * C + j * V;
                                box_put<O, 128>(box, lane, j, reinterpret_cast<const float *>(&v[i / 16][i % 16]));
                            }
                            // rows past the plane's last are dropped by a TMA store
                            box_store<O, 128>(&map.out, t.n0 + n, y, z, out + n, ldo, KIND == DW && wide ? 32 : rows, cols,
                                              wide, box, lane);
                        }
                    }
                }
            }
            if (!split)
                release();
            if (some) {
                acc ^= 1;
                aph ^= acc == 0;
            }
        }
        if (loading)   // given up: nothing may still land in this CTA's memory
            wait_ms<OWN>(landed + 8 * warp, lph, 20, nullptr);
        asm volatile("cp.async.bulk.commit_group;\n\tcp.async.bulk.wait_group 0;" ::: "memory");
    }
    fence_before();
    __syncthreads();
    fence_after();
    if (*dead) {
        // nothing may still land in this CTA's memory: copies first (the leader's barriers count both CTAs'), then MMAs
        if (warp == 8 && lane == 0 && rank == 0)
            for (uint32_t i = issued < kStages ? 0 : issued - kStages; i < issued; ++i)
                wait_ms<OWN>(full + 8 * (i % kStages), (i / kStages) & 1, 20, nullptr);
        if (warp == 9 && rank == 0 && elect_one()) {
            mma_commit<CG>(drain);
            wait_ms<OWN>(drain, 0, 1000, nullptr);
        }
    }
    fence_before();
    __syncthreads();
    if (CG == 2)
        cluster_sync();
    fence_after();
    if (warp == 9) {
        if (CG == 2)
            asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
        else
            asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
    }
}

// ---- launches

// Row tiles over all experts, at most: each with rows has one that is not full.
int64_t row_tiles(const FfShape &s, int rows)
{
    return s.E == 1 ? ceil_div(s.M, rows) : s.M / rows + std::min<int64_t>(s.E, s.M);
}

template <int CG, int KIND, typename T, typename O>
cudaError_t launch(esp_moe *m, const FfMaps<KIND> &maps, FfParams p, int64_t tiles)
{
    constexpr int kSmem = Shape<CG, KIND>::kSmem;
    auto kernel = k_ff<CG, KIND, T, O>;
    cudaError_t e = allow_smem<k_ff<CG, KIND, T, O>, kSmem>(m->device);
    if (e != cudaSuccess)
        return e;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[2];
    attr[0] = after_launch_before();
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = kSmem;
    cfg.stream = m->stream;
    int groups = m->sm_count;
    if (CG == 2) {
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = 2;
        attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
        cfg.numAttrs = 2;
        if (m->max_pairs == 0) {   // any product kernel's: they all take an SM for a CTA
            cfg.gridDim = dim3((unsigned)(m->sm_count / 2 * 2));
            e = cudaOccupancyMaxActiveClusters(&m->max_pairs, kernel, &cfg);
            if (e != cudaSuccess)
                return e;
        }
        groups = std::max(1, m->max_pairs);
    }
    cfg.gridDim = dim3((unsigned)(CG * std::max<int64_t>(1, std::min<int64_t>(groups, tiles))));
    p.few_ctas = 2 * (int64_t)cfg.gridDim.x <= m->sm_count;
    m->launches += 1;
    return cudaLaunchKernelEx(&cfg, kernel, maps, p);
}

// Which tiles a product takes: pairs of CTAs with 256 x 256, or single ones with 128 x 256 whose inner axis may be split
// into parts. Times in blocks of the inner axis (0.27 us of a pair's MMAs): a tile's start and end take about four, a single
// CTA's block 1.17, joining parts 12 and 5 for each (5000 x 64 x 72: both weights' gradients 25 us in parts, 34 whole).
struct Choice {
    bool pair;
    int splits;
};

// rounds(tile's rows, parts): how many rounds of tiles there are, in the mean.
template <typename R>
Choice choose_tiles(const esp_moe *m, R &&rounds, int64_t most_one, double blocks)
{
    Choice best{true, 1};
    double t_best = rounds(256, 1) * (blocks + 4.0);
    for (int splits = 1; splits <= 16; ++splits) {
        // parts fill at most one round and keep four blocks each
        if (splits > 1 && (most_one * splits > m->sm_count || blocks < 4 * splits))
            break;
        const double t = rounds(128, splits) * (1.17 * std::ceil(blocks / splits) + 4.0) +
                         (splits > 1 ? 12.0 + 5.0 * splits : 0.0);
        if (t < t_best) {
            t_best = t;
            best = Choice{false, splits};
        }
    }
    return best;
}

template <int KIND, typename T>
cudaError_t rows_launch(esp_moe *m, const FfShape &s, const CUtensorMap &a, const CUtensorMap &b, const CUtensorMap &o,
                        const CUtensorMap &o2, FfParams &p)
{
    const FfMaps<KIND> maps = {{{a, b, o, o2, b}}};
    const int64_t nt = ceil_div(p.g.N, kTileCols<KIND>), pairs = row_tiles(s, 256), ones = row_tiles(s, 128);
    // The experts' rows are not known here: each one's last tile is half full in the mean, with a deviation of 12^-1/2 of a tile.
    // One round where 1.2 deviations more fit, else half a round more than the tiles (hidden rows and outer product of 921 rows
    // of 8 experts, 2048 x 1024: 36 us, 40 with half a round more everywhere; all rounds counted so, with mean and deviation:
    // 7372 rows of 16 experts that may be 8192, 2048 x 1024: 101 us, 91).
    const double experts = s.E == 1 ? 0.0 : (double)std::min<int64_t>(s.E, s.M);
    const auto rounds = [&](int rows, int parts) {
        const double tiles = s.E == 1 ? (double)ceil_div(s.M, rows) : (double)s.M / rows + 0.5 * experts;
        const double most = std::min(tiles + 0.35 * std::sqrt(experts), (double)row_tiles(s, rows));
        const int at_once = rows == 256 ? m->sm_count / 2 : m->sm_count;
        if (s.E == 1)
            return std::ceil(tiles * nt * parts / at_once);
        return most * nt * parts <= at_once ? 1.0 : std::max(1.0, tiles * nt * parts / at_once + 0.5);
    };
    const Choice c = choose_tiles(m, rounds, ones * nt, (double)p.blocks * p.halves);
    p.g.most = (int32_t)(c.pair ? pairs : ones);
    p.g.splits = c.splits;
    return c.pair ? launch<2, KIND, T, T>(m, maps, p, pairs * nt)
                  : launch<1, KIND, T, T>(m, maps, p, ones * nt * c.splits);
}

template <typename T, typename O>
cudaError_t weights_launch(esp_moe *m, const FfShape &s, FfMaps<DW> &maps, FfParams &p)
{
    int64_t pairs = 0, ones = 0;
    for (int q = 0; q < p.dws; ++q) {
        DwOut &d = p.dw[q];
        d.wide = rows_aligned(d.out, d.N, sizeof(O), 16);
        maps.of[q].out = maps.of[q].a;   // not used where the output is not aligned
        if (d.wide)
            FF_TRY(box_map3(&maps.of[q].out, d.out, sizeof(O), d.N, d.out_rows, d.N, (int64_t)s.E * d.planes,
                            (int64_t)d.out_rows * d.N, 32));
        const int64_t per = (int64_t)s.E * d.planes * ceil_div(d.N, 256);
        pairs += per * ceil_div(d.out_rows, 256);
        ones += per * ceil_div(d.out_rows, 128);
    }
    if (p.dws == 1)
        maps.of[1] = maps.of[0];
    // items differ with the experts' rows: half a round more
    const auto rounds = [&](int rows, int parts) {
        const double r = rows == 256 ? (double)pairs / (m->sm_count / 2) : (double)(ones * parts) / m->sm_count;
        return s.E == 1 ? std::ceil(r) : std::max(1.0, r + 0.5);
    };
    const Choice c = choose_tiles(m, rounds, ones, (double)s.M / s.E / kInner);
    p.g.splits = c.splits;
    return c.pair ? launch<2, DW, T, O>(m, maps, p, pairs) : launch<1, DW, T, O>(m, maps, p, ones * c.splits);
}

// ---- tails
constexpr int kTailRows = 4;   // of a CTA, a warp for each

// A warp copies a row, 16 bytes a lane, eight of them in flight; rows behind an expert's last are zeros. Elements past a
// row's `width` are not read, and zeros up to `ld_out`.
__global__ void __launch_bounds__(32 * kTailRows) k_tails(const TailArgs a)
{
    wait_for_launch_before();
    let_next_launch_start();
    const TailArgs::Part &p = a.part[blockIdx.y];
    const int e = blockIdx.x / (kInner / kTailRows), lane = threadIdx.x & 31;
    const int r = blockIdx.x % (kInner / kTailRows) * kTailRows + (threadIdx.x >> 5);
    const int lo = a.offsets ? max(0, min(a.M, a.offsets[e])) : 0;
    const int hi = a.offsets ? max(lo, min(a.M, a.offsets[e + 1])) : a.M;
    const int rows = (hi - lo) % kInner;
    if (rows == 0)
        return;
    const uint16_t *x = static_cast<const uint16_t *>(p.x) + (int64_t)(hi - rows + min(r, rows - 1)) * p.ldx;
    uint16_t *out = static_cast<uint16_t *>(p.out) + ((int64_t)e * kInner + r) * p.ld_out;
    constexpr int U = 8;
    for (int h0 = lane * 8; h0 < p.ld_out; h0 += 256 * U) {
        Pack<uint16_t, 8> v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int h = h0 + 256 * u;
            v[u] = {};
            if (r < rows && h + 8 <= p.width)
                v[u] = *reinterpret_cast<const Pack<uint16_t, 8> *>(x + h);
            else if (r < rows && h < p.width)
                for (int j = 0; h + j < p.width; ++j)
                    v[u].v[j] = x[h + j];
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (h0 + 256 * u < p.ld_out)
                *reinterpret_cast<Pack<uint16_t, 8> *>(out + h0 + 256 * u) = v[u];
    }
}

// ---- lengths of rows
constexpr int kLengthRows = 8;   // of a CTA, a warp for each

struct LengthArgs {
    int64_t M;
    int32_t E, F, H;
    int64_t ldx, ld_inner;
    const void *x, *inner;       // rows on 16 bytes
    float *out;                  // M + E F
};

// Lengths of the rows of x, and of G's of each expert; 0 for a row with NaN. Bound by the rows' bytes. Squares that leave
// fp32's range are summed again of scaled elements.
template <typename T>
__global__ void __launch_bounds__(32 * kLengthRows) k_lengths(const LengthArgs a)
{
    wait_for_launch_before();
    let_next_launch_start();
    const int64_t i = (int64_t)blockIdx.x * kLengthRows + (threadIdx.x >> 5), j = i - a.M;
    const int lane = threadIdx.x & 31;
    if (j >= (int64_t)a.E * a.F)
        return;
    // U's rows lie behind G's
    const T *row = j < 0 ? static_cast<const T *>(a.x) + i * a.ldx
                         : static_cast<const T *>(a.inner) + (j + j / a.F * a.F) * a.ld_inner;
    const auto squares = [&](float scale) {
        constexpr int U = 4;
        float s = 0.0f;
        for (int h0 = 8 * lane; h0 < a.H; h0 += 256 * U) {
            Pack<T, 8> r[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int h = h0 + 256 * u;
                r[u] = {};
                if (h + 8 <= a.H)
                    r[u] = *reinterpret_cast<const Pack<T, 8> *>(row + h);
                else
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        if (h + k < a.H)
                            r[u].v[k] = row[h + k];
            }
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const float f = to_f32(r[u].v[k]) * scale;
                    s = fmaf(f, f, s);
                }
        }
#pragma unroll
        for (int d = 16; d > 0; d >>= 1)
            s += __shfl_xor_sync(0xffffffffu, s, d);
        return s;
    };
    float s = squares(1.0f), back = 1.0f;
    if (!(s > 0x1p-90f && s < 0x1p120f)) {
        back = s > 1.0f ? 0x1p80f : 0x1p-80f;
        s = squares(1.0f / back);
    }
    if (lane == 0)
        a.out[i] = s >= 0.0f ? sqrtf(s) * back : 0.0f;
}

}  // namespace

size_t ff_partial_floats(const esp_moe *m)
{
    return (size_t)m->sm_count * kRowsA * kAccCols;   // parts fill at most one round
}

cudaError_t launch_ff_hidden(esp_moe *m, const FfShape &s, const void *x, int64_t ldx, void *hidden, void *pre)
{
    FfParams p = common(m, s);
    p.g.N = p.g.rows_b = s.F;
    p.g.K = s.H;
    p.blocks = (int32_t)ceil_div(s.H, kInner);
    p.g.out = hidden;
    p.g.ldo = s.fp;
    p.out2 = pre;
    if (s.lengths) {
        // The tensor core cuts off what it adds below its accumulator's last bit, at every step of 16: of 8192 products a g is off
        // by ten times an ordinary 32-bit sum (9e-6 rms of products whose sum is around 1), and the sign of one in half a million
        // is wrong, which takes a whole gradient away or adds one. The error goes with the sums on the way, not with g: of
        // terms in no order those are around S = |x||w| / sqrt H (lengths of the two rows), whatever g itself is. Measured: an
        // error of 0.08 to 0.16 H/16 2^-23 S (rms), of a rounding's size in g below that; the bound is 2 (H/16 + 4) 2^-23 S.
        // Sums on the way that are far above S (terms that are sorted by sign) are not covered. 8192 rows x 2048 x 2048 with g and u
        // kept: 148 us (silu 135); 4416 x 8192 x 1024: 179 (140); 11 and 18 of it are k_lengths.
        p.x = x;
        p.ldx = ldx;
        p.inner = s.inner;
        p.ld_inner = s.ld_inner;
        p.near_zero = (float)(2.0 * (s.H / 16 + 4) * 0x1p-23 / std::sqrt((double)s.H));
        p.lengths = s.lengths;
        const LengthArgs l{s.M, s.E, s.F, s.H, ldx, s.ld_inner, x, s.inner, s.lengths};
        FF_TRY(with_16(s.dtype, [&](auto elem) {
            m->launches += 1;
            return launch_after(k_lengths<decltype(elem)>, dim3((unsigned)ceil_div(s.M + (int64_t)s.E * s.F, kLengthRows)),
                                32 * kLengthRows, 0, m->stream, l);
        }));
    }
    CUtensorMap a, b, o, o2;
    FF_TRY(box_map3(&a, x, 2, s.H, s.M, ldx, 1, 0, kRowsA));
    FF_TRY(box_map3(&b, s.inner, 2, s.H, s.F, s.ld_inner, 2 * (int64_t)s.E, s.F * s.ld_inner, kRowsA));
    FF_TRY(box_map3(&o, hidden, 2, s.F, s.M, s.fp, 1, 0, 32));
    o2 = o;
    if (pre)
        FF_TRY(box_map3(&o2, pre, 4, s.F, s.M, 2 * s.fp, 2, s.fp, 32));
    return with_16(s.dtype, [&](auto elem) { return rows_launch<HIDDEN, decltype(elem)>(m, s, a, b, o, o2, p); });
}

cudaError_t launch_ff_out(esp_moe *m, const FfShape &s, const void *hidden, void *y, int64_t ldy)
{
    FfParams p = common(m, s);
    p.g.N = p.g.rows_b = s.H;
    p.g.K = s.F;
    p.blocks = (int32_t)ceil_div(s.F, kInner);
    p.g.out = y;
    p.g.ldo = ldy;
    p.g.wide_store = rows_aligned(y, ldy, 2, 16);
    CUtensorMap a, b, o;
    FF_TRY(box_map3(&a, hidden, 2, s.F, s.M, s.fp, 1, 0, kRowsA));
    FF_TRY(box_map3(&b, s.outer, 2, s.F, s.H, s.ld_outer, s.E, s.H * s.ld_outer, kRowsA));
    o = a;
    if (p.g.wide_store)
        FF_TRY(box_map3(&o, y, 2, s.H, s.M, ldy, 1, 0, 32));
    return with_16(s.dtype, [&](auto elem) { return rows_launch<OUT, decltype(elem)>(m, s, a, b, o, o, p); });
}

cudaError_t launch_ff_dpre(esp_moe *m, const FfShape &s, const void *dy, int64_t lddy, const void *pre, void *dpre)
{
    FfParams p = common(m, s);
    p.g.N = p.g.rows_b = s.F;
    p.g.K = s.H;
    p.blocks = (int32_t)ceil_div(s.H, kInner);
    p.g.out = dpre;
    p.g.ldo = 2 * s.fp;
    CUtensorMap a, b, o, g;
    FF_TRY(box_map3(&a, dy, 2, s.H, s.M, lddy, 1, 0, kRowsA));
    FF_TRY(box_map3(&b, s.outer, 2, s.F, s.H, s.ld_outer, s.E, s.H * s.ld_outer, kInner));
    FF_TRY(box_map3(&o, dpre, 2, s.F, s.M, 2 * s.fp, 2, s.fp, 32, 64));
    FF_TRY(box_map3(&g, pre, 4, s.F, s.M, 2 * s.fp, 2, s.fp, 32));
    return with_16(s.dtype, [&](auto elem) { return rows_launch<DPRE, decltype(elem)>(m, s, a, b, o, g, p); });
}

cudaError_t launch_ff_dx(esp_moe *m, const FfShape &s, const void *dpre, void *dx, int64_t lddx)
{
    FfParams p = common(m, s);
    p.g.N = p.g.rows_b = s.H;
    p.g.K = s.F;
    p.blocks = (int32_t)ceil_div(s.F, kInner);
    p.halves = 2;
    p.g.out = dx;
    p.g.ldo = lddx;
    p.g.wide_store = rows_aligned(dx, lddx, 2, 16);
    CUtensorMap a, b, o;
    FF_TRY(box_map3(&a, dpre, 2, s.F, s.M, 2 * s.fp, 2, s.fp, kRowsA));
    FF_TRY(box_map3(&b, s.inner, 2, s.H, s.F, s.ld_inner, 2 * (int64_t)s.E, s.F * s.ld_inner, kInner));
    o = a;
    if (p.g.wide_store)
        FF_TRY(box_map3(&o, dx, 2, s.H, s.M, lddx, 1, 0, 32));
    return with_16(s.dtype, [&](auto elem) { return rows_launch<DX, decltype(elem)>(m, s, a, b, o, o, p); });
}

cudaError_t launch_tails(esp_moe *m, const TailArgs &a, int32_t E)
{
    m->launches += 1;
    return launch_after(k_tails, dim3((unsigned)(E * (kInner / kTailRows)), (unsigned)a.parts), 32 * kTailRows, 0, m->stream, a);
}

cudaError_t launch_ff_weights(esp_moe *m, const FfShape &s, const FfWeightArgs &a)
{
    FfParams p = common(m, s);
    FfMaps<DW> maps;
    const int64_t tails = (int64_t)s.E * kInner;
    p.tails = a.tails;
    if (a.dinner) {   // dpre^T x
        OneMaps &w = maps.of[p.dws];
        p.dw[p.dws++] = DwOut{2, s.F, s.H, false, a.dinner};
        FF_TRY(box_map3(&w.a, a.dpre, 2, s.F, s.M, 2 * s.fp, 2, s.fp, kInner));
        FF_TRY(box_map3(&w.b, a.x, 2, s.H, s.M, a.ldx, 1, 0, kInner));
        w.a2 = w.a;
        w.b2 = w.b;
        if (a.tails) {
            FF_TRY(box_map3(&w.a2, a.dpre_tails, 2, s.F, tails, 2 * s.fp, 2, s.fp, kInner));
            FF_TRY(box_map3(&w.b2, a.x_tails, 2, s.H, tails, s.hp, 1, 0, kInner));
        }
    }
    if (a.douter) {   // dy^T hidden
        OneMaps &w = maps.of[p.dws];
        p.dw[p.dws++] = DwOut{1, s.H, s.F, false, a.douter};
        FF_TRY(box_map3(&w.a, a.dy, 2, s.H, s.M, a.lddy, 1, 0, kInner));
        FF_TRY(box_map3(&w.b, a.hidden, 2, s.F, s.M, s.fp, 1, 0, kInner));
        w.a2 = w.a;
        w.b2 = w.b;
        if (a.tails) {
            FF_TRY(box_map3(&w.a2, a.dy_tails, 2, s.H, tails, s.hp, 1, 0, kInner));
            FF_TRY(box_map3(&w.b2, a.hidden_tails, 2, s.F, tails, s.fp, 1, 0, kInner));
        }
    }
    return with_16(s.dtype, [&](auto elem) -> cudaError_t {
        using T = decltype(elem);
        return a.f32 ? weights_launch<T, float>(m, s, maps, p) : weights_launch<T, T>(m, s, maps, p);
    });
}

}  // namespace esp_moe_impl
