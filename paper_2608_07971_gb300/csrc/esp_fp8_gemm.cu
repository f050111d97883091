// Products of 8-bit codes with a scale per block of 128 (include/esp_moe.h) on the tensor cores.
//
// out[m][n] = sum over blocks b of sa[m][b] sb[n][b] (sum over the 128 codes of block b of A[m] B[n]). The
// scales change from block to block, so a block's products (four tcgen05.mma kind::f8f6f4 of K = 32)
// go into an accumulator stage of tensor memory of their own; the epilogue warps read it, scale it and
// add it to fp32 sums in registers, while the tensor core works on the next stage.
//
// A tile is 128 rows (CG = 1: one CTA) or 256 rows (CG = 2: two CTAs of a cluster that share the MMAs,
// each holding 128 rows of A and half of B) times BN columns; one block of K per shared-memory stage
// (128 codes = one 128-byte swizzled row). Warps 0-3 own the first half of the columns, warps 4-7 the
// second, a thread one row (its TMEM lane) of its half; warp 8 loads tiles by TMA, warps 9 and 11 issue
// the MMAs in turn, warp 10 brings the scales of the weight gradient to shared memory. CTAs are persistent:
// every role walks the same list of tiles, so loads and MMAs of the next tile run during a tile's stores.
//
// GROUPED ROWS (forward, row gradient): expert e's rows times its own B; a tile never spans two experts,
// rows past the expert's end are computed and dropped. sb is one value per 128 columns.
// GROUPED INNER AXIS (weight gradient): expert e's blocks of 128 positions; sb is a value per column.
//
// Bound by a block's turn: issue, MMAs, epilogue and the hand-back of the stage take longer than the two stages of
// 256 columns hide. 8192 x 8192 x 4096 takes 222 us (2.48 PFLOP/s), 166 with the loads and MMAs alone; 65536 rows
// over 64 experts x 4096 x 2048 515 us; the weight gradient of 16384 rows x 2048 x 4096 over 16 experts 257 us.
// Tiles of 128 columns with four stages are 1.1 to 1.25 times slower (they load and read more of A for each
// column), single CTAs with 256 columns 1.01 to 1.03 times, 16 epilogue warps 1.1 to 1.2 times.
//
// Every wait is bounded; one that runs out sets a flag that ends the CTA's other waits, the error word
// reports it, and the CTA drains its copies and MMAs (bounded) before it frees its tensor memory.

#include <algorithm>

#include "esp_fp8_tiles.cuh"
#include "esp_moe_impl.h"
#include "esp_moe_launch.cuh"
#include "esp_moe_load.cuh"
#include "esp_tcgen.cuh"

namespace esp_moe_impl {

namespace {

constexpr int kThreads = 384;                // 8 epilogue warps, loads, MMAs, scales (COLS), MMAs
// registers per thread of the epilogue and of the other warpgroup: 2 * 216 + 72 = 3 * 168, the launch's
constexpr int kEpilogueRegs = 216, kOtherRegs = 72;
constexpr int kEpilogueWarps = 8;
constexpr int kStageA = kRowsA * kBlock;     // bytes
constexpr uint32_t kTmemCols = 512;
constexpr int kBoxBytes = 128, kBox = 32 * kBoxBytes;   // a warp's staged store: 128 bytes of 32 rows
constexpr int kStageBoxes = 2;               // of a warp
constexpr int kSmemLimit = 232448;

template <int CG, int BN>
struct Shape {
    static constexpr int kRowsB = BN / CG;   // rows of B that a CTA holds
    static constexpr int kStage = kStageA + kRowsB * kBlock;
    static constexpr int kAcc = (int)kTmemCols / BN;
    static constexpr int kWGCols = BN / 2;   // columns of a warpgroup
    // after the stages: store staging, tile table, scales, barriers
    static constexpr int kTable = (ESP_MOE_MAX_EXPERTS + 1) * 4 + 12;   // a multiple of 16
    static constexpr int kStaging = kEpilogueWarps * kStageBoxes * kBox;
    static constexpr int kScaleFloats = kRowsA + BN;   // of a stage: row and column scales (COLS)
    static constexpr int kScales = kAcc * kScaleFloats * 4;
    static constexpr int kBars = 256;
    static constexpr int kFixed = kTable + kStaging + kScales + kBars + 1024;
    static constexpr int kStages = std::min(8, (kSmemLimit - kFixed) / kStage);
    static constexpr int kSmem = kStages * kStage + kFixed;
    static_assert((2 * kStages + 3 * kAcc + 1) * 8 + 16 <= kBars, "barriers");
};

// Arrival on a barrier of this CTA or, through its cluster address, of another. Relaxed: it orders the
// tensor-memory loads before it, which have completed; a release would wait for unrelated stores.
__device__ __forceinline__ void mbar_arrive(uint32_t cluster_addr)
{
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}

// PAIR: a barrier at which another CTA's threads arrive (mbar_arrive); what orders their tensor-memory loads before the
// MMAs that follow are the tcgen05 fences around a relaxed arrival and wait of the same, cluster, scope.
template <bool PAIR>
__device__ __forceinline__ bool mbar_try(uint32_t bar, uint32_t parity)
{
    uint32_t done;
    if (PAIR)
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "mbarrier.try_wait.parity.relaxed.cluster.shared::cta.b64 p, [%1], %2;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(done)
            : "r"(bar), "r"(parity)
            : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(done)
            : "r"(bar), "r"(parity)
            : "memory");
    return done != 0;
}

// Waits for a phase for at most `ms` milliseconds of the GPU's timer, which is read once in 256 polls.
template <bool PAIR = false>
__device__ __forceinline__ bool mbar_wait_ms(uint32_t bar, uint32_t parity, uint32_t ms, volatile int *dead)
{
    uint64_t end = 0;
    for (;;) {
        for (int i = 0; i < 256; ++i)
            if (mbar_try<PAIR>(bar, parity))
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

// Bounded wait of a role; gives up early once another wait of the CTA did. On running out it sets the CTA's
// flag and the error word.
template <bool PAIR = false>
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity, const GemmParams &p, volatile int *dead)
{
    if (mbar_try<PAIR>(bar, parity) || mbar_wait_ms<PAIR>(bar, parity, p.wait_ms, dead))
        return true;
    *dead = 1;
    *static_cast<volatile unsigned int *>(p.err) = 1u;   // in host memory
    return false;
}

template <int CG>
__device__ __forceinline__ void tma_tile(uint32_t dst, const CUtensorMap *map, int x, int y, uint32_t bar)
{
    if (CG == 1)
        asm volatile(
            "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], "
            "[%4];" ::"r"(dst),
            "l"(map), "r"(x), "r"(y), "r"(bar)
            : "memory");
    else
        asm volatile(
            "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, "
            "{%2, %3}], [%4];" ::"r"(dst),
            "l"(map), "r"(x), "r"(y), "r"(bar)
            : "memory");
}

// Shared-memory operand of 128-byte rows in the 128-byte swizzle: groups of 8 rows 1024 bytes apart
// (stride offset), descriptor version 1 (bits 46-47), swizzle mode 2 (bits 61-63).
__device__ __forceinline__ uint64_t operand_desc(uint32_t addr)
{
    return (uint64_t)((addr >> 4) & 0x3fffu) | (1ull << 16) | ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) |
           (2ull << 61);
}

template <int CG>
__device__ __forceinline__ void mma_codes(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate)
{
    if (CG == 1)
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
            "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
            : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
            "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
            : "memory");
}

// (c, d) += (a, b) * (s, t) and (a, b) *= s, each one instruction on pairs of registers.
__device__ __forceinline__ void fma_pair(float &c, float &d, float a, float b, float s, float t)
{
    asm("{\n\t.reg .b64 x, y, z;\n\t"
        "mov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmov.b64 z, {%0, %1};\n\t"
        "fma.rn.f32x2 z, x, y, z;\n\tmov.b64 {%0, %1}, z;\n\t}"
        : "+f"(c), "+f"(d)
        : "f"(a), "f"(b), "f"(s), "f"(t));
}

__device__ __forceinline__ void mul_pair(float &a, float &b, float s)
{
    asm("{\n\t.reg .b64 x, y;\n\t"
        "mov.b64 x, {%0, %1};\n\tmov.b64 y, {%2, %2};\n\t"
        "mul.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;\n\t}"
        : "+f"(a), "+f"(b)
        : "f"(s));
}

// Barrier of N threads that also ANDs a predicate over them.
template <int N>
__device__ __forceinline__ bool sync_and(int id, bool v)
{
    uint32_t r;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.b32 p, %1, 0;\n\t"
        "bar.red.and.pred q, %2, %3, p;\n\t"
        "selp.u32 %0, 1, 0, q;\n\t}"
        : "=r"(r)
        : "r"((uint32_t)v), "r"(id), "n"(N)
        : "memory");
    return r != 0;
}

// A warp's 32 rows of one box of the output: 128 bytes of every row (a lane holds a row's values), staged in
// the 128-byte swizzle (16-byte chunk j of row r at place j ^ (r & 7): no bank conflicts). Whole boxes leave
// by one TMA store, so that the warp goes on while they are written; with a bulk copy for every row instead,
// 65536 x 4096 x 2048 takes 596 us, and 514 without the copies. Boxes that reach past the expert's last row,
// and outputs that are not 16-byte aligned, are stored by the lanes: rows at or past `rows` and columns at
// or past `cols` are dropped.
template <typename T>
__device__ __forceinline__ void store_box(const CUtensorMap *map, int x, int y, T *out, int64_t ldo, int rows, int cols,
                                          bool wide, const float *v, unsigned char *box, int lane)
{
    constexpr int V = 16 / (int)sizeof(T), C = kBoxBytes / (int)sizeof(T);
#pragma unroll
    for (int i = 0; i < C; i += V)
        store_pack<T, V>(reinterpret_cast<T *>(box + lane * kBoxBytes + (((i / V) ^ (lane & 7)) * 16)), v + i);
    if (wide && rows >= 32) {
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0)
            asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];" ::"l"(map),
                         "r"(x), "r"(y), "r"(smem_u32(box))
                         : "memory");
        return;
    }
    __syncwarp();
    if (wide && cols >= C) {
        const int j = lane & 7;
        for (int r = lane >> 3; r < 32 && r < rows; r += 4)
            *reinterpret_cast<uint4 *>(out + r * ldo + j * V) =
                *reinterpret_cast<const uint4 *>(box + r * kBoxBytes + ((j ^ (r & 7)) * 16));
    } else {
        for (int r = 0; r < 32 && r < rows; ++r)
            for (int c = lane; c < C && c < cols; c += 32)
                out[r * ldo + c] =
                    reinterpret_cast<const T *>(box + r * kBoxBytes + (((c / V) ^ (r & 7)) * 16))[c % V];
    }
}

// Joins the parts of a split tile: every part's sums go to memory, and the CTA whose part is the last to
// arrive gets back true and the sums over all parts, in their order. Called by all epilogue threads, those
// whose waits ran out (ok false) too: then ok is false for all.
template <int BN, int C>
__device__ __forceinline__ bool join_parts(const GemmParams &p, int item, int row, int rows, int col, float (&sum)[C],
                                           volatile int *last, bool &ok)
{
    const int tile = item / p.splits;
    constexpr int64_t kPart = (int64_t)kRowsA * BN;
    float4 *mine = reinterpret_cast<float4 *>(p.partial + item * kPart) + (col / 4) * kRowsA + row;
    if (row < rows)
#pragma unroll
        for (int i = 0; i < C / 4; ++i)
            __stcg(mine + i * kRowsA, make_float4(sum[4 * i], sum[4 * i + 1], sum[4 * i + 2], sum[4 * i + 3]));
    __threadfence();
    ok = sync_and<32 * kEpilogueWarps>(7, ok);
    if (!ok)
        return false;
    if (threadIdx.x == 0) {
        const bool l = atomicAdd(p.tickets + tile, 1u) == (unsigned)p.splits - 1;
        if (l)
            p.tickets[tile] = 0u;
        *last = l;
        __threadfence();
    }
    asm volatile("bar.sync 7, %0;" ::"n"(32 * kEpilogueWarps) : "memory");
    if (!*last)
        return false;
    const float4 *all =
        reinterpret_cast<const float4 *>(p.partial + tile * (int64_t)p.splits * kPart) + (col / 4) * kRowsA + row;
    if (row < rows) {
#pragma unroll
        for (int i = 0; i < C; ++i)
            sum[i] = 0.0f;
        for (int q = 0; q < p.splits; ++q)
#pragma unroll
            for (int i = 0; i < C / 4; ++i) {
                const float4 v = __ldcg(all + q * (kPart / 4) + i * kRowsA);
                sum[4 * i] += v.x;
                sum[4 * i + 1] += v.y;
                sum[4 * i + 2] += v.z;
                sum[4 * i + 3] += v.w;
            }
    }
    return true;
}

template <int CG, int BN, bool COLS, typename T>
__global__ void __launch_bounds__(kThreads, 1)
    k_gemm(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
           const __grid_constant__ CUtensorMap map_out, const GemmParams p)
{
    using S = Shape<CG, BN>;
    extern __shared__ unsigned char smem_raw[];
    unsigned char *sm = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                                          ~static_cast<uintptr_t>(1023));
    unsigned char *staging = sm + S::kStages * S::kStage;   // its boxes are 1024-byte aligned
    int *table = reinterpret_cast<int *>(staging + S::kStaging);
    float *scales = reinterpret_cast<float *>(reinterpret_cast<unsigned char *>(table) + S::kTable);
    uint64_t *bars = reinterpret_cast<uint64_t *>(
        (reinterpret_cast<uintptr_t>(scales + S::kScales / 4) + 15) & ~static_cast<uintptr_t>(15));
    const uint32_t full = smem_u32(bars), empty = full + 8 * S::kStages, tfull = empty + 8 * S::kStages,
                   tempty = tfull + 8 * S::kAcc, sempty = tempty + 8 * S::kAcc, drain = sempty + 8 * S::kAcc;
    uint32_t *slot = reinterpret_cast<uint32_t *>(bars + 2 * S::kStages + 3 * S::kAcc + 1);
    volatile int *dead = reinterpret_cast<volatile int *>(slot + 1), *last = dead + 1;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = CG == 1 ? 0 : cluster_rank();

    if (threadIdx.x == 0) {
        *dead = 0;
        for (int i = 0; i < S::kStages; ++i) {
            mbar_init(full + 8 * i, 1);
            mbar_init(empty + 8 * i, 1);
        }
        for (int i = 0; i < S::kAcc; ++i) {
            mbar_init(tfull + 8 * i, COLS ? 2 : 1);   // the stage's MMAs, and (COLS) its scales
            mbar_init(tempty + 8 * i, CG * kEpilogueWarps);
            mbar_init(sempty + 8 * i, kEpilogueWarps);
        }
        mbar_init(drain, 2);   // both issuing threads
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 9) {
        if (CG == 1) {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(slot)),
                         "r"(kTmemCols)
                         : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(slot)),
                         "r"(kTmemCols)
                         : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        }
    }
    // What follows reads what the launch before wrote (the codes) or is ordered after it. The launch after is
    // not let start early: its waiting CTAs slow this kernel's tail (1001 x 1999 x 2050: 24.1 us, 19.3 without).
    wait_for_launch_before();
    if (warp == 8) {
        // the experts' row tiles (blocks) before each: one warp's scan
        int carry = 0;
        for (int e0 = 0; e0 < p.E; e0 += 32) {
            const int n = e0 + lane < p.E ? tiles_of<CG, COLS>(p, e0 + lane) : 0;
            int s = n;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int y = __shfl_up_sync(0xffffffffu, s, o);
                if (lane >= o)
                    s += y;
            }
            if (e0 + lane < p.E)
                table[e0 + lane] = min(p.most, carry + s - n);
            carry = min(p.most, carry + __shfl_sync(0xffffffffu, s, 31));
        }
        if (lane == 0)
            table[p.E] = carry;
    }
    fence_before();
    __syncthreads();
    if (CG == 2)
        cluster_sync();
    fence_after();
    const uint32_t tmem = *slot;
    const int w0 = blockIdx.x / CG, dw = gridDim.x / CG;
    uint32_t issued = 0;   // loads issued by this CTA's producer

    if (warp >= kEpilogueWarps) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
        if (warp == 8) {
            const uint32_t full0 = CG == 1 ? full : map_rank(full, 0);
            int s = 0;
            uint32_t ph = 1;
            bool ok = true;
            Tile t;
            for (int w = w0; ok && tile_at<CG, BN, COLS>(p, table, w, t); w += dw) {
                const int ya = t.m0 + (int)rank * kRowsA;
                const int yb = (COLS ? 0 : t.e * p.rows_b) + t.n0 + (int)rank * S::kRowsB;
                for (int kb = t.kb0; kb < t.kb1; ++kb) {
                    if (!(ok = __all_sync(0xffffffffu, mbar_wait(empty + 8 * s, ph, p, dead))))
                        break;
                    const uint32_t dst = smem_u32(sm + s * S::kStage);
                    if (elect_one()) {
                        if (rank == 0)
                            mbar_expect(full + 8 * s, CG * S::kStage);
                        if (!(p.hold && issued == 2)) {
                            tma_tile<CG>(dst, &map_a, kb * kBlock, ya, full0 + 8 * s);
                            tma_tile<CG>(dst + kStageA, &map_b, kb * kBlock, yb, full0 + 8 * s);
                        }
                    }
                    __syncwarp();
                    ++issued;
                    if (++s == S::kStages) {
                        s = 0;
                        ph ^= 1;
                    }
                }
            }
        }
        if ((warp == 9 || warp == 11) && rank == 0) {
            // Two warps issue in turn, a block each: a single thread took about 490 cycles for a block's waits and
            // commits and 60 for each MMA, more than the MMAs themselves (128 each); 8192 x 8192 x 4096 took 230 us.
            const bool odd = warp == 11;
            constexpr uint32_t idesc = (1u << 4) | ((uint32_t)(BN >> 3) << 17) | ((uint32_t)(kRowsA * CG >> 4) << 24);
            int s = 0, acc = 0;
            uint32_t ph = 0, aph = 1;
            bool ok = true;
            Tile t;
            for (int w = w0; ok && tile_at<CG, BN, COLS>(p, table, w, t); w += dw)
                for (int kb = t.kb0; kb < t.kb1; ++kb) {
                    if ((bool)(acc & 1) == odd) {
                        ok = __all_sync(0xffffffffu, mbar_wait(full + 8 * s, ph, p, dead) &&
                                                         mbar_wait<CG == 2>(tempty + 8 * acc, aph, p, dead));
                        if (!ok)
                            break;
                        fence_after();
                        const uint64_t a = operand_desc(smem_u32(sm + s * S::kStage));
                        const uint64_t b = operand_desc(smem_u32(sm + s * S::kStage + kStageA));
                        if (elect_one()) {
#pragma unroll
                            for (int k = 0; k < kBlock / 32; ++k)   // 32 bytes = 2 units of the descriptor's address
                                mma_codes<CG>(tmem + acc * BN, a + 2 * k, b + 2 * k, idesc, k > 0);
                            mma_commit<CG>(tfull + 8 * acc);
                            mma_commit<CG>(empty + 8 * s);
                        }
                        __syncwarp();
                    }
                    if (++s == S::kStages) {
                        s = 0;
                        ph ^= 1;
                    }
                    if (++acc == S::kAcc) {
                        acc = 0;
                        aph ^= 1;
                    }
                }
        }
        if (COLS && warp == 10) {
            // a lane brings the scales of rows 4 l .. 4 l + 3 and of columns BN / 32 * l ..; the next block's,
            // of the next tile too, are on their way while a stage is waited for
            constexpr int R = kRowsA / 32, C = BN / 32;
            int acc = 0, w = w0, left = 0;
            uint32_t aph = 1;
            Tile t;
            const float *pa[R], *pb[C];
            float a[R], b[C];
            auto next = [&]() -> bool {   // moves to the next block, if there is one
                if (left > 0) {
#pragma unroll
                    for (int i = 0; i < R; ++i)
                        pa[i] += p.sa_k;
#pragma unroll
                    for (int i = 0; i < C; ++i)
                        pb[i] += p.sb_k;
                }
                for (; left == 0; w += dw) {   // tiles may have no blocks
                    if (!tile_at<CG, BN, COLS>(p, table, w, t))
                        return false;
                    left = t.kb1 - t.kb0;
#pragma unroll
                    for (int i = 0; i < R; ++i)   // rows past the end take the last one's
                        pa[i] = p.scale_a + (t.m0 + min((int)rank * kRowsA + R * lane + i, t.rows - 1)) * p.sa_row +
                                t.kb0 * p.sa_k;
#pragma unroll
                    for (int i = 0; i < C; ++i)
                        pb[i] = p.scale_b + t.kb0 * p.sb_k + min(t.n0 + C * lane + i, p.N - 1);
                }
#pragma unroll
                for (int i = 0; i < R; ++i)
                    a[i] = *pa[i];
#pragma unroll
                for (int i = 0; i < C; ++i)
                    b[i] = *pb[i];
                return true;
            };
            for (bool more = next(); more;) {
                if (!__all_sync(0xffffffffu, mbar_wait(sempty + 8 * acc, aph, p, dead)))
                    break;
                float *to = scales + acc * S::kScaleFloats;
#pragma unroll
                for (int i = 0; i < R; ++i)
                    to[R * lane + i] = a[i];
#pragma unroll
                for (int i = 0; i < C; ++i)
                    to[kRowsA + C * lane + i] = b[i];
                __syncwarp();
                if (lane == 0)
                    mbar_arrive_cta(tfull + 8 * acc);
                --left;
                more = next();
                if (++acc == S::kAcc) {
                    acc = 0;
                    aph ^= 1;
                }
            }
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kEpilogueRegs));
        const int wg = warp >> 2, quarter = warp & 3;
        const uint32_t lane_cols = ((uint32_t)(32 * quarter) << 16) + (uint32_t)(wg * S::kWGCols);
        const uint32_t tempty0 = CG == 1 ? tempty : map_rank(tempty, 0);
        unsigned char *stage = staging + warp * kStageBoxes * kBox;
        int acc = 0;
        uint32_t aph = 0;
        bool ok = true;
        Tile t;
        for (int w = w0; ok && tile_at<CG, BN, COLS>(p, table, w, t); w += dw) {
            const int row = 32 * quarter + lane;                    // of this CTA's 128
            const int rows = t.rows - (int)rank * kRowsA;           // that exist
            const bool some = 32 * quarter < rows;                  // a row of this warp exists
            const int c0 = t.n0 + wg * S::kWGCols;
            float sum[S::kWGCols];
#pragma unroll
            for (int i = 0; i < S::kWGCols; ++i)
                sum[i] = 0.0f;
            // FWD: a row's scale (of the last row past the end) and the one of this warpgroup's columns, fetched a
            // block ahead
            const int ra = t.m0 + min((int)rank * kRowsA + row, t.rows - 1);
            const float *pa = p.scale_a + ra * p.sa_row;
            const float *pb = p.scale_b + t.e * p.sb_e + min(c0, p.N - 1) / kBlock * p.sb_n + t.kb0 * p.sb_k;
            float next_a = 0.0f, next_b = 0.0f;
            if (!COLS) {
                pa += t.kb0 * p.sa_k;
                next_a = *pa;
                next_b = *pb;
            }
            for (int left = t.kb1 - t.kb0; left > 0; --left) {
                float scale = next_a * next_b;
                if (!COLS && left > 1) {
                    pa += p.sa_k;
                    pb += p.sb_k;
                    next_a = *pa;
                    next_b = *pb;
                }
                ok = __all_sync(0xffffffffu, mbar_wait(tfull + 8 * acc, aph, p, dead));
                if (!ok)
                    break;
                fence_after();
                // The stage is given back as soon as its last columns are in registers: the MMAs of the block
                // after next wait for it, and what the stage's turn takes beyond the other stage's MMAs
                // is time that the tensor core stands still.
                if (some) {
                    const uint32_t src = tmem + acc * BN + lane_cols;
                    const float *csb = scales + acc * S::kScaleFloats + kRowsA + wg * S::kWGCols;
                    if (COLS)
                        scale = scales[acc * S::kScaleFloats + row];
                    constexpr int D = COLS ? 4 : 3, chunks = S::kWGCols / 16;   // loads in flight, loads in all
                    uint32_t v[D][16];
#pragma unroll
                    for (int c = 0; c < D; ++c)
                        tmem_ld16(src + 16 * c, v[c]);
// chunk c is held in v[c % D] until it is added
                    auto add = [&](int c) {
                        const uint32_t(&x)[16] = v[c % D];
#pragma unroll
                        for (int i = 0; i < 16; i += 4) {
                            float *to = sum + 16 * c + i;
                            float a = __uint_as_float(x[i]), b = __uint_as_float(x[i + 1]);
                            float d = __uint_as_float(x[i + 2]), f = __uint_as_float(x[i + 3]);
                            if (COLS) {
                                const float4 s4 = *reinterpret_cast<const float4 *>(csb + 16 * c + i);
                                mul_pair(a, b, scale);
                                mul_pair(d, f, scale);
                                fma_pair(to[0], to[1], a, b, s4.x, s4.y);
                                fma_pair(to[2], to[3], d, f, s4.z, s4.w);
                            } else {
                                fma_pair(to[0], to[1], a, b, scale, scale);
                                fma_pair(to[2], to[3], d, f, scale, scale);
                            }
                        }
                    };
#pragma unroll
                    for (int c0 = 0; c0 + D < chunks; c0 += D) {
                        tmem_wait(v);
#pragma unroll
                        for (int c = c0; c < c0 + D && c + D < chunks; ++c) {
                            add(c);
                            tmem_ld16(src + 16 * (c + D), v[c % D]);
                        }
                    }
                    tmem_wait(v);
                    fence_before();
                    __syncwarp();
                    if (lane == 0)
                        mbar_arrive(tempty0 + 8 * acc);
#pragma unroll
                    for (int c = chunks - D; c < chunks; ++c)
                        add(c);
                } else if (lane == 0) {
                    mbar_arrive(tempty0 + 8 * acc);
                }
                if (COLS) {
                    __syncwarp();
                    if (lane == 0)
                        mbar_arrive_cta(sempty + 8 * acc);
                }
                if (++acc == S::kAcc) {
                    acc = 0;
                    aph ^= 1;
                }
            }
            if (CG == 1 && p.splits > 1) {
                if (!join_parts<BN, S::kWGCols>(p, w, row, rows, wg * S::kWGCols, sum, last, ok))
                    continue;
            }
            if (!ok || !some)
                continue;
            const int y = (COLS ? t.e * p.rows_b : 0) + t.m0 + (int)rank * kRowsA + 32 * quarter;
            T *out = static_cast<T *>(p.out) + y * p.ldo + c0;
            constexpr int C = kBoxBytes / (int)sizeof(T);
#pragma unroll
            for (int c = 0; c < S::kWGCols; c += C) {
                if (c / C % kStageBoxes == 0) {   // the boxes before have been read
                    asm volatile("cp.async.bulk.commit_group;\n\tcp.async.bulk.wait_group.read 0;" ::: "memory");
                    __syncwarp();
                }
                if (c0 + c < p.N)
                    store_box<T>(&map_out, c0 + c, y, out + c, p.ldo, rows - 32 * quarter, p.N - c0 - c, p.wide_store,
                                 sum + c, stage + c / C % kStageBoxes * kBox, lane);
            }
            asm volatile("cp.async.bulk.commit_group;" ::: "memory");
        }
        asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");   // the last boxes are read from this CTA's memory
    }
    fence_before();
    __syncthreads();
    fence_after();
    if (*dead) {
        // nothing may still land in this CTA's memory: copies first (the leader's barriers count both
        // CTAs'), then the MMAs
        if (warp == 8 && lane == 0 && rank == 0)
            for (uint32_t i = issued < S::kStages ? 0 : issued - S::kStages; i < issued; ++i)
                mbar_wait_ms(full + 8 * (i % S::kStages), (i / S::kStages) & 1, 20, nullptr);
        if ((warp == 9 || warp == 11) && rank == 0 && elect_one()) {   // the threads that issued
            mma_commit<CG>(drain);
            mbar_wait_ms(drain, 0, 1000, nullptr);
        }
    }
    fence_before();
    __syncthreads();
    if (CG == 2)
        cluster_sync();
    fence_after();
    if (warp == 9) {
        if (CG == 1)
            asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
        else
            asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
    }
}

// ---- launches

// Boxes of box_rows rows and 128 bytes of a matrix of elements of 1, 2 or 4 bytes; what a load finds outside
// is zero, what a store has outside is dropped.
cudaError_t box_map(CUtensorMap *map, const void *p, int size, int64_t rows, int64_t cols, int64_t ld, int box_rows)
{
    const EncodeTiled encode = encode_tiled();
    if (!encode)
        return cudaErrorNotSupported;
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)ld * size};
    const cuuint32_t box[2] = {(cuuint32_t)(128 / size), (cuuint32_t)box_rows}, step[2] = {1, 1};
    const CUtensorMapDataType type = size == 1   ? CU_TENSOR_MAP_DATA_TYPE_UINT8
                                     : size == 2 ? CU_TENSOR_MAP_DATA_TYPE_UINT16
                                                 : CU_TENSOR_MAP_DATA_TYPE_UINT32;
    const CUresult r = encode(map, type, 2, const_cast<void *>(p), dims, strides, box, step,
                              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

template <int CG, int BN, bool COLS, typename T>
cudaError_t launch(esp_moe *m, const CUtensorMap &a, const CUtensorMap &b, const CUtensorMap &o, const GemmParams &p,
                   int64_t tiles)
{
    using S = Shape<CG, BN>;
    auto kernel = k_gemm<CG, BN, COLS, T>;
    cudaError_t e = allow_smem<k_gemm<CG, BN, COLS, T>, S::kSmem>(m->device);
    if (e != cudaSuccess)
        return e;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[2];
    attr[0] = after_launch_before();
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = S::kSmem;
    cfg.stream = m->stream;
    int groups = m->sm_count;
    if (CG == 2) {
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = CG;
        attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
        cfg.numAttrs = 2;
        if (m->max_pairs == 0) {
            cfg.gridDim = dim3((unsigned)(m->sm_count / CG * CG));
            e = cudaOccupancyMaxActiveClusters(&m->max_pairs, kernel, &cfg);
            if (e != cudaSuccess)
                return e;
        }
        groups = std::max(1, m->max_pairs);
    }
    cfg.gridDim = dim3((unsigned)(CG * std::max<int64_t>(1, std::min<int64_t>(groups, tiles))));
    m->launches += 1;
    return cudaLaunchKernelEx(&cfg, kernel, a, b, o, p);
}

template <int CG, int BN, bool COLS, typename T>
cudaError_t encode_and_launch(esp_moe *m, const uint8_t *A, int64_t rows_a, int64_t inner, int64_t lda, const uint8_t *B,
                              int64_t rows_b, int64_t ldb, const GemmParams &p, int64_t tiles)
{
    CUtensorMap a, b, o;
    cudaError_t e = box_map(&a, A, 1, rows_a, inner, lda, kRowsA);
    if (e == cudaSuccess)
        e = box_map(&b, B, 1, rows_b, inner, ldb, Shape<CG, BN>::kRowsB);
    o = a;   // not used where the output is not aligned
    if (e == cudaSuccess && p.wide_store)
        e = box_map(&o, p.out, sizeof(T), COLS ? (int64_t)p.E * p.rows_b : p.M, p.N, p.ldo, 32);
    return e != cudaSuccess ? e : launch<CG, BN, COLS, T>(m, a, b, o, p, tiles);
}

GemmParams common(esp_moe *m)
{
    GemmParams p{};
    p.err = m->d_err;
    p.wait_ms = m->wait_ms;
    p.hold = m->hold_load ? 1 : 0;
    m->hold_load = false;   // the hook holds one launch only
    p.splits = 1;
    p.tickets = m->d_ticket + 1;
    return p;
}

// Which tiles a product takes: pairs of CTAs with 256 x 256, or single CTAs with 128 x 128 whose inner axis
// may be split into parts. Times in units of a single CTA's block (about 0.4 us): rounds of tiles over the
// SMs times the blocks of each. A pair's block takes 1.35 units (4096 x 4096 x 4096 as pairs 67 us, as
// single CTAs 74; 1000 x 2000 x 2050: 14.9 and 13.3); joining parts takes 8 and 1 to 1.5 for each part
// (16 x 2048 x 4096 in parts 12.6 us, whole 16.3; 128 x 4096 x 4096 16.6 and 17.4).
struct Choice {
    bool pair;
    int splits;
};

Choice choose_tiles(const esp_moe *m, int64_t tiles_pair, int64_t tiles_one, int64_t blocks, int64_t rows)
{
    const double t_pair = 1.35 * (double)(ceil_div(tiles_pair, std::max(1, m->sm_count / 2)) * blocks);
    Choice best{true, 1};
    double t_best = t_pair;
    for (int splits = 1; splits <= 16; ++splits) {
        // parts fill at most one round and keep four blocks each
        if (splits > 1 && (tiles_one * splits > m->sm_count || blocks < 4 * splits))
            break;
        double t = (double)(ceil_div(tiles_one * splits, m->sm_count) * ceil_div(blocks, splits));
        if (splits > 1)
            t += 8.0 + splits * std::max(1.0, 1.5 * (double)std::min<int64_t>(rows, kRowsA) / kRowsA);
        if (t < t_best) {
            t_best = t;
            best = Choice{false, splits};
        }
    }
    return best;
}

}  // namespace

size_t gemm_partial_floats(const esp_moe *m)
{
    return (size_t)m->sm_count * kRowsA * 128;   // parts fill at most one round
}

cudaError_t launch_gemm_rows(esp_moe *m, int32_t dtype, const GemmRowsArgs &a)
{
    return with_dtype(dtype, [&](auto elem) -> cudaError_t {
        using T = decltype(elem);
        GemmParams p = common(m);
        p.M = (int32_t)a.M;
        p.sa_row = a.lds;
        p.sa_k = 1;
        p.E = a.E;
        p.N = p.rows_b = a.N;
        p.K = a.K;
        p.scale_a = a.scale_a;
        p.scale_b = a.scale_b;
        p.sb_e = a.sb_e;
        p.sb_n = a.sb_n;
        p.sb_k = a.sb_k;
        p.offsets = a.offsets;
        p.out = a.out;
        p.ldo = a.ldo;
        p.wide_store = rows_aligned(a.out, a.ldo, sizeof(T), 16);
        p.partial = a.partial;
        // at most this many tiles: every expert with rows has one that is not full
        const auto row_tiles = [&](int rows) {
            return a.E == 1 ? ceil_div(a.M, rows) : a.M / rows + std::min<int64_t>(a.E, a.M);
        };
        const int64_t pair = row_tiles(256) * ceil_div(a.N, 256), one = row_tiles(128) * ceil_div(a.N, 128);
        const Choice c = choose_tiles(m, pair, one, ceil_div(a.K, kBlock), a.M / a.E);
        p.most = (int32_t)row_tiles(c.pair ? 256 : 128);
        if (c.pair)
            return encode_and_launch<2, 256, false, T>(m, a.A, a.M, a.K, a.lda, a.B, (int64_t)a.E * a.N, a.ldb, p, pair);
        p.splits = c.splits;
        return encode_and_launch<1, 128, false, T>(m, a.A, a.M, a.K, a.lda, a.B, (int64_t)a.E * a.N, a.ldb, p,
                                                   one * c.splits);
    });
}

cudaError_t launch_gemm_cols(esp_moe *m, const GemmColsArgs &a)
{
    GemmParams p = common(m);
    p.M = (int32_t)a.M;
    p.sa_row = 1;
    p.sa_k = a.lds_a;
    p.E = a.E;
    p.N = a.K;
    p.rows_b = a.N;
    p.scale_a = a.scale_a;
    p.scale_b = a.scale_b;
    p.sb_k = a.lds_b;
    p.offsets = a.offsets;
    p.out = a.out;
    p.ldo = a.ldo;
    p.wide_store = rows_aligned(a.out, a.ldo, 4, 16);
    p.partial = a.partial;
    p.most = (int32_t)(a.M / kBlock + a.E);
    const int64_t positions = (int64_t)p.most * kBlock;
    const int64_t pair = (int64_t)a.E * ceil_div(a.N, 256) * ceil_div(a.K, 256);
    const int64_t one = (int64_t)a.E * ceil_div(a.N, 128) * ceil_div(a.K, 128);
    const Choice c = choose_tiles(m, pair, one, ceil_div(a.M, kBlock * a.E), a.N);   // blocks: the experts' mean
    if (c.pair)
        return encode_and_launch<2, 256, true, float>(m, a.A, a.N, positions, a.lda, a.B, a.K, a.ldb, p, pair);
    p.splits = c.splits;
    return encode_and_launch<1, 128, true, float>(m, a.A, a.N, positions, a.lda, a.B, a.K, a.ldb, p, one * c.splits);
}

}  // namespace esp_moe_impl
