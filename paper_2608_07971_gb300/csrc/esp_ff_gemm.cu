// Products of the gated feed-forward blocks (include/esp_moe.h) on the tensor cores: 16-bit operands (tcgen05.mma
// kind::f16), sums over the whole inner axis in tensor memory.
//
//   HIDDEN  rows x [G; U]^T, and from both accumulators act(g) * u: projections, activation and product in one kernel
//   OUT     hidden x O^T
//   DPRE    dy x O, and from it and the kept g, u the gradients of g and u
//   DX      dpre x [G; U]
//   DW      dpre^T x rows and dy^T x hidden: the inner axis is an expert's rows
//
// Every operand is read as it lies in memory: where the inner axis is the contiguous one, a tile is K-major (rows of 64
// inner elements, 128 bytes, 128-byte swizzle), else MN-major (rows of 64 outer elements, one for each inner index; an
// MMA's operand then is two such tiles side by side). No transposed copies are made.
//
// A tile is 256 rows of two CTAs (cta_group::2, each holding 128 rows of A and half of B's 256 columns; HIDDEN: one CTA
// loads 128 columns of G, the other the same ones of U, so that both halves of a hidden element meet in one thread).
// Two accumulators of 256 columns: warps 0-7 empty one while the tensor core fills the other. Warp 8 loads by TMA,
// warp 9 issues the MMAs, warp 10 clears the rows behind an expert's last in its last block (DW). CTAs are persistent.
//
// Every wait is bounded, as in esp_fp8_gemm.cu.

#include <algorithm>
#include <type_traits>

#include "esp_ff.cuh"
#include "esp_moe_launch.cuh"
#include "esp_moe_load.cuh"

namespace esp_moe_impl {

namespace {

constexpr int kThreads = 384;
constexpr int kEpilogueWarps = 8;
constexpr int kStages = 5;
constexpr int kTileBytes = kRowsA * 128;             // one operand's share of a stage in a CTA
constexpr int kStage = 2 * kTileBytes;
constexpr int kBoxBytes = 128, kBox = 32 * kBoxBytes;
constexpr uint32_t kTmemCols = 512;
constexpr int kAccCols = 256;
constexpr int kTable = (ESP_MOE_MAX_EXPERTS + 1) * 4 + 12;
constexpr int kBars = 192;
constexpr int kSmem = kStages * kStage + kEpilogueWarps * kBox + kTable + kBars + 1024;
static_assert((3 * kStages + 2 * 2 + 1) * 8 + 16 <= kBars, "barriers");
static_assert(kSmem <= 232448, "shared memory");

// One item of the list. Row kinds: rows m0 .. m0 + rows - 1 of expert e, columns n0 ..; DW: output rows m0 .. of plane z,
// over the rows lo .. hi - 1.
struct FfTile {
    int e, m0, rows, n0, blocks, z, lo, hi;
};

template <int KIND>
constexpr int kTileCols = KIND == HIDDEN ? 128 : 256;

template <int KIND>
__device__ __forceinline__ bool ff_tile(const FfParams &p, const int *table, int item, FfTile &t)
{
    if (KIND != DW) {
        Tile r;
        if (!tile_at<2, kTileCols<KIND>, false>(p.g, table, item, r))
            return false;
        t.e = r.e;
        t.m0 = r.m0;
        t.rows = r.rows;
        t.n0 = r.n0;
        t.blocks = p.blocks * p.halves;
        return true;
    }
    const int mt = (p.out_rows + 255) / 256, nt = (p.g.N + 255) / 256, per = mt * nt * p.planes;
    if (item >= per * p.g.E)
        return false;
    t.e = item / per;
    int i = item - t.e * per;
    t.z = i / (mt * nt);
    i -= t.z * (mt * nt);
    t.m0 = (i % mt) * 256;
    t.n0 = (i / mt) * 256;
    t.rows = min(256, p.out_rows - t.m0);
    expert_rows(p.g, t.e, t.lo, t.hi);
    t.blocks = (t.hi - t.lo) / kInner + ((t.hi - t.lo) % kInner != 0);
    return true;
}

// A box into this CTA's shared memory; its bytes arrive at a barrier of either CTA of the pair.
__device__ __forceinline__ void load_box(uint32_t dst, const CUtensorMap *map, int x, int y, int z, uint32_t bar)
{
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, "
        "%3, %4}], [%5];" ::"r"(dst),
        "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
        : "memory");
}

__device__ __forceinline__ void mma16(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
        : "memory");
}

// ---- a warp's staged box: 128 bytes of 32 rows, 16-byte chunk j of row r at place j ^ (r & 7).

// Waits until the box's last store has been read.
__device__ __forceinline__ void box_free()
{
    asm volatile("cp.async.bulk.commit_group;\n\tcp.async.bulk.wait_group.read 0;" ::: "memory");
    __syncwarp();
}

// V values of this lane's row into chunk j.
template <typename T>
__device__ __forceinline__ void box_put(unsigned char *box, int lane, int j, const float *v)
{
    store_pack<T, 16 / (int)sizeof(T)>(reinterpret_cast<T *>(box + lane * kBoxBytes + ((j ^ (lane & 7)) * 16)), v);
}

// The box leaves: by one TMA store where all its rows are there to be written (columns past the matrix are dropped by the
// store), else by the lanes: rows at or past `rows`, columns at or past `cols` are dropped.
template <typename T>
__device__ __forceinline__ void box_store(const CUtensorMap *map, int x, int y, int z, T *out, int64_t ldo, int rows,
                                          int cols, bool wide, const unsigned char *box, int lane)
{
    constexpr int V = 16 / (int)sizeof(T), C = kBoxBytes / (int)sizeof(T);
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
    __syncwarp();
}

// 64 columns of this thread's lane of tensor memory.
__device__ __forceinline__ void tmem_ld64(uint32_t addr, uint32_t (&v)[4][16])
{
#pragma unroll
    for (int i = 0; i < 4; ++i)
        tmem_ld16(addr + 16 * i, v[i]);
}

// T: operands; O: output.
template <int KIND, typename T, typename O>
__global__ void __launch_bounds__(kThreads, 1)
    k_ff(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
         const __grid_constant__ CUtensorMap map_out, const __grid_constant__ CUtensorMap map_out2, const FfParams p)
{
    constexpr bool A_MN = KIND == DW, B_MN = KIND == DPRE || KIND == DX || KIND == DW;
    extern __shared__ unsigned char smem_raw[];
    unsigned char *sm = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                                          ~static_cast<uintptr_t>(1023));
    unsigned char *staging = sm + kStages * kStage;
    int *table = reinterpret_cast<int *>(staging + kEpilogueWarps * kBox);
    uint64_t *bars = reinterpret_cast<uint64_t *>(reinterpret_cast<unsigned char *>(table) + kTable);
    const uint32_t full = smem_u32(bars), empty = full + 8 * kStages, tfull = empty + 8 * kStages, tempty = tfull + 16,
                   tail = tempty + 16, drain = tail + 8 * kStages;
    uint32_t *slot = reinterpret_cast<uint32_t *>(bars + 3 * kStages + 5);
    volatile int *dead = reinterpret_cast<volatile int *>(slot + 1);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();

    if (threadIdx.x == 0) {
        *dead = 0;
        for (int i = 0; i < kStages; ++i) {
            mbar_init(full + 8 * i, KIND == DW ? 2 : 1);   // DW: one arrival of each CTA
            mbar_init(empty + 8 * i, 1);
            mbar_init(tail + 8 * i, 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(tfull + 8 * i, 1);
            mbar_init(tempty + 8 * i, 2 * kEpilogueWarps);
        }
        mbar_init(drain, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 9) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(slot)),
                     "r"(kTmemCols)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    wait_for_launch_before();
    if (KIND != DW && warp == 8) {
        // the experts' row tiles before each: one warp's scan
        int carry = 0;
        for (int e0 = 0; e0 < p.g.E; e0 += 32) {
            const int n = e0 + lane < p.g.E ? tiles_of<2, false>(p.g, e0 + lane) : 0;
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
    cluster_sync();
    fence_after();
    const uint32_t tmem = *slot;
    const int w0 = blockIdx.x / 2, dw = gridDim.x / 2;
    // of this CTA's loading warp: its loads, the stages whose tail barrier it used, and those barriers' next phases
    uint32_t issued = 0, tail_used = 0, tail_phase = 0;
    FfTile t;

    if (warp == 8) {
        const uint32_t full0 = map_rank(full, 0);
        int s = 0;
        uint32_t ph = 1;
        bool ok = true;
        for (int w = w0; ok && ff_tile<KIND>(p, table, w, t); w += dw) {
            const int outer_a = t.m0 + (int)rank * kRowsA;
            const int outer_b = t.n0 + (KIND == HIDDEN ? 0 : (int)rank * kRowsA);
            for (int kb = 0; kb < t.blocks; ++kb) {
                if (!(ok = wait_phase(empty + 8 * s, ph, p.g, dead)))
                    break;
                const uint32_t a = smem_u32(sm + s * kStage), b = a + kTileBytes;
                const int half = KIND == DX && kb >= p.blocks ? 1 : 0, k = (kb - half * p.blocks) * kInner;
                const bool cut = KIND == DW && kb == t.blocks - 1 && (t.hi - t.lo) % kInner != 0;
                if (elect_one()) {
                    uint32_t bar = full0 + 8 * s;
                    if (cut) {   // arrives here first: warp 10 clears what is not the expert's
                        bar = map_rank(tail + 8 * s, rank);
                        mbar_expect(tail + 8 * s, kStage);
                    } else if (rank == 0) {
                        mbar_expect(full + 8 * s, 2 * kStage);
                    } else if (KIND == DW) {
                        arrive_relaxed(bar);
                    }
                    if (!(p.g.hold && issued == 2)) {
                        if (A_MN) {
                            load_box(a, &map_a, outer_a, t.lo + k, t.z, bar);
                            load_box(a + kHalfTile, &map_a, outer_a + 64, t.lo + k, t.z, bar);
                        } else {
                            load_box(a, &map_a, k, outer_a, half, bar);
                        }
                        if (KIND == DW) {
                            load_box(b, &map_b, outer_b, t.lo + k, 0, bar);
                            load_box(b + kHalfTile, &map_b, outer_b + 64, t.lo + k, 0, bar);
                        } else if (B_MN) {
                            const int z = KIND == DX ? 2 * t.e + half : t.e;
                            load_box(b, &map_b, outer_b, k, z, bar);
                            load_box(b + kHalfTile, &map_b, outer_b + 64, k, z, bar);
                        } else {
                            load_box(b, &map_b, k, outer_b, KIND == HIDDEN ? 2 * t.e + (int)rank : t.e, bar);
                        }
                    }
                }
                __syncwarp();
                ++issued;
                tail_used |= (uint32_t)cut << s;
                tail_phase ^= (uint32_t)cut << s;
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
                                   ((uint32_t)(kAccCols >> 3) << 17) | ((uint32_t)(256 >> 4) << 24);
            int s = 0, acc = 0;
            uint32_t ph = 0, aph = 1;
            bool ok = true;
            for (int w = w0; ok && ff_tile<KIND>(p, table, w, t); w += dw) {
                if (t.blocks == 0)
                    continue;
                if (!(ok = wait_phase<HANDBACK>(tempty + 8 * acc, aph, p.g, dead)))
                    break;
                for (int kb = 0; kb < t.blocks; ++kb) {
                    if (!(ok = wait_phase<KIND == DW ? PAIR : OWN>(full + 8 * s, ph, p.g, dead)))
                        break;
                    fence_after();
                    const uint64_t a = operand<A_MN>(smem_u32(sm + s * kStage));
                    const uint64_t b = operand<B_MN>(smem_u32(sm + s * kStage + kTileBytes));
                    if (elect_one()) {
#pragma unroll
                        for (int k = 0; k < kInner / 16; ++k)
                            mma16(tmem + acc * kAccCols, a + k * kOperandStep<A_MN>, b + k * kOperandStep<B_MN>, idesc,
                                  kb > 0 || k > 0);
                        mma_commit<2>(empty + 8 * s);
                        if (kb == t.blocks - 1)
                            mma_commit<2>(tfull + 8 * acc);
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
    } else if (KIND == DW && warp == 10) {
        // rows of the next expert in this one's last block: zeros in both operands, so that nothing of theirs, NaN
        // included, reaches the sums
        const uint32_t full0 = map_rank(full, 0);
        int s = 0;
        uint32_t tph = 0;   // a bit for each stage
        for (int w = w0; ff_tile<KIND>(p, table, w, t); w += dw) {
            const int rows = (t.hi - t.lo) % kInner;
            if (rows != 0) {
                const int at = (s + t.blocks - 1) % kStages;
                if (!wait_phase(tail + 8 * at, tph >> at & 1, p.g, dead))
                    break;
                tph ^= 1u << at;
                unsigned char *stage = sm + at * kStage;
                for (int i = lane; i < 4 * (kInner - rows) * 8; i += 32) {
                    const int part = i & 3, chunk = (i >> 2) & 7, row = rows + (i >> 5);
                    *reinterpret_cast<uint4 *>(stage + part * kHalfTile + row * 128 + chunk * 16) = make_uint4(0, 0, 0, 0);
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0)
                    arrive_release(full0 + 8 * at);
            }
            s = (s + t.blocks) % kStages;
        }
    } else if (warp < kEpilogueWarps) {
        const int wg = warp >> 2, quarter = warp & 3;
        const uint32_t tempty0 = map_rank(tempty, 0);
        unsigned char *box = staging + warp * kBox;
        int acc = 0;
        uint32_t aph = 0;
        for (int w = w0; ff_tile<KIND>(p, table, w, t); w += dw) {
            const int rows = t.rows - (int)rank * kRowsA - 32 * quarter;   // of this warp's 32 that exist, from the first
            const int y = t.m0 + (int)rank * kRowsA + 32 * quarter;        // the first
            if (t.blocks > 0) {
                if (!wait_phase(tfull + 8 * acc, aph, p.g, dead))
                    break;
                fence_after();
            }
            const uint32_t src = tmem + ((uint32_t)(32 * quarter) << 16) + (uint32_t)(acc * kAccCols);
            if (rows > 0) {
                uint32_t v[4][16];
                if (KIND == HIDDEN) {
                    const int c = 64 * wg, n = t.n0 + c, cols = p.g.N - n;
                    if (cols > 0) {
                        if (p.out2) {
                            for (int part = 0; part < 4; ++part) {   // 32 columns of g, 32 more, and of u
                                const int half = part >> 1, off = 32 * (part & 1);
                                if (off >= cols)
                                    continue;
                                tmem_ld16(src + 128 * half + c + off, v[0]);
                                tmem_ld16(src + 128 * half + c + off + 16, v[1]);
                                tmem_wait(v);
                                box_free();
#pragma unroll
                                for (int j = 0; j < 8; ++j)
                                    box_put<float>(box, lane, j, reinterpret_cast<const float *>(&v[j / 4][4 * (j & 3)]));
                                box_store<float>(&map_out2, n + off, y, half,
                                                 static_cast<float *>(p.out2) + y * 2 * p.fp + half * p.fp + n + off, 2 * p.fp,
                                                 rows, cols - off, true, box, lane);
                            }
                        }
                        box_free();
                        with_act(p.act, [&](auto kind) {
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                tmem_ld16(src + c + 32 * h, v[0]);
                                tmem_ld16(src + c + 32 * h + 16, v[1]);
                                tmem_ld16(src + 128 + c + 32 * h, v[2]);
                                tmem_ld16(src + 128 + c + 32 * h + 16, v[3]);
                                tmem_wait(v);
#pragma unroll
                                for (int j = 0; j < 4; ++j) {
                                    float r[8];
#pragma unroll
                                    for (int i = 0; i < 8; ++i)
                                        r[i] = act_of<decltype(kind)::value>(__uint_as_float(v[j / 2][8 * (j & 1) + i])) *
                                               __uint_as_float(v[2 + j / 2][8 * (j & 1) + i]);
                                    box_put<T>(box, lane, 4 * h + j, r);
                                }
                            }
                        });
                        box_store<T>(&map_out, n, y, 0, static_cast<T *>(p.g.out) + y * p.g.ldo + n, p.g.ldo, rows, cols, true,
                                     box, lane);
                    }
                } else if (KIND == DPRE) {
                    for (int c = 128 * wg; c < 128 * wg + 128 && t.n0 + c < p.g.N; c += 64) {
                        const int n = t.n0 + c, cols = p.g.N - n;
                        tmem_ld64(src + c, v);
                        const float *g = static_cast<const float *>(p.pre) + (y + min(lane, rows - 1)) * 2 * p.fp + n;
                        const float *u = g + p.fp;
                        tmem_wait(v);
                        box_free();
                        with_act(p.act, [&](auto kind) {
#pragma unroll
                            for (int j = 0; j < 8; ++j) {
                                float gv[8] = {}, uv[8] = {}, dg[8];
                                if (8 * j < cols) {   // a half's rows are whole groups of 8
                                    load_pack<float, 4>(g + 8 * j, gv);
                                    load_pack<float, 4>(g + 8 * j + 4, gv + 4);
                                    load_pack<float, 4>(u + 8 * j, uv);
                                    load_pack<float, 4>(u + 8 * j + 4, uv + 4);
                                }
#pragma unroll
                                for (int i = 0; i < 8; ++i) {
                                    uint32_t &d = v[j / 2][8 * (j & 1) + i];
                                    const float dh = __uint_as_float(d);
                                    float a, slope;
                                    act_and_slope<decltype(kind)::value>(gv[i], a, slope);
                                    dg[i] = dh * uv[i] * slope;
                                    d = __float_as_uint(dh * a);
                                }
                                box_put<T>(box, lane, j, dg);
                            }
                        });
                        for (int half = 0; half < 2; ++half) {
                            if (half == 1) {
                                box_free();
#pragma unroll
                                for (int j = 0; j < 8; ++j)
                                    box_put<T>(box, lane, j, reinterpret_cast<const float *>(&v[j / 2][8 * (j & 1)]));
                            }
                            box_store<T>(&map_out, n, y, half, static_cast<T *>(p.g.out) + y * 2 * p.fp + half * p.fp + n,
                                         2 * p.fp, rows, cols, true, box, lane);
                        }
                    }
                } else {
                    constexpr int C = kBoxBytes / (int)sizeof(O), V = 16 / (int)sizeof(O);
                    const int z = KIND == DW ? t.e * p.planes + t.z : 0;
                    O *out = static_cast<O *>(p.g.out) + ((int64_t)z * p.out_rows + y) * p.g.ldo + t.n0;
                    for (int c = 128 * wg; c < 128 * wg + 128 && t.n0 + c < p.g.N; c += 64) {
                        if (t.blocks > 0) {
                            tmem_ld64(src + c, v);
                            tmem_wait(v);
                        } else {
#pragma unroll
                            for (int i = 0; i < 64; ++i)
                                v[i / 16][i % 16] = 0u;
                        }
#pragma unroll
                        for (int b = 0; b < 64 / C; ++b) {
                            const int n = c + b * C, cols = p.g.N - t.n0 - n;
                            if (cols <= 0)
                                break;
                            box_free();
#pragma unroll
                            for (int j = 0; j < 8; ++j) {
                                const int i = b * C + j * V;
                                box_put<O>(box, lane, j, reinterpret_cast<const float *>(&v[i / 16][i % 16]));
                            }
                            // rows past the plane's last are dropped by a TMA store
                            box_store<O>(&map_out, t.n0 + n, y, z, out + n, p.g.ldo, KIND == DW && p.g.wide_store ? 32 : rows,
                                         cols, p.g.wide_store, box, lane);
                        }
                    }
                }
            }
            if (t.blocks > 0) {
                fence_before();
                __syncwarp();
                if (lane == 0)
                    arrive_relaxed(tempty0 + 8 * acc);
                acc ^= 1;
                aph ^= acc == 0;
            }
        }
        asm volatile("cp.async.bulk.commit_group;\n\tcp.async.bulk.wait_group 0;" ::: "memory");
    }
    fence_before();
    __syncthreads();
    fence_after();
    if (*dead) {
        // nothing may still land in this CTA's memory: copies first (the leader's barriers count both CTAs'), then MMAs
        if (warp == 8 && lane == 0) {
            if (rank == 0)
                for (uint32_t i = issued < kStages ? 0 : issued - kStages; i < issued; ++i)
                    wait_ms<OWN>(full + 8 * (i % kStages), (i / kStages) & 1, 20, nullptr);
            for (int i = 0; i < kStages; ++i)
                if (tail_used >> i & 1)
                    wait_ms<OWN>(tail + 8 * i, (tail_phase >> i & 1) ^ 1, 20, nullptr);
        }
        if (warp == 9 && rank == 0 && elect_one()) {
            mma_commit<2>(drain);
            wait_ms<OWN>(drain, 0, 1000, nullptr);
        }
    }
    fence_before();
    __syncthreads();
    cluster_sync();
    fence_after();
    if (warp == 9)
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
}

// ---- launches

// Row tiles of 256 over all experts, at most: each with rows has one that is not full.
int64_t row_tiles(const FfShape &s)
{
    return s.E == 1 ? ceil_div(s.M, 256) : s.M / 256 + std::min<int64_t>(s.E, s.M);
}

template <int KIND, typename T, typename O>
cudaError_t launch(esp_moe *m, const CUtensorMap &a, const CUtensorMap &b, const CUtensorMap &o, const CUtensorMap &o2,
                   FfParams p, int64_t tiles)
{
    auto kernel = k_ff<KIND, T, O>;
    cudaError_t e = allow_smem<k_ff<KIND, T, O>, kSmem>(m->device);
    if (e != cudaSuccess)
        return e;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[2];
    attr[0] = after_launch_before();
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = 2;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = kSmem;
    cfg.stream = m->stream;
    if (m->max_pairs == 0) {   // any product kernel's: they all take an SM for a CTA
        cfg.gridDim = dim3((unsigned)(m->sm_count / 2 * 2));
        e = cudaOccupancyMaxActiveClusters(&m->max_pairs, kernel, &cfg);
        if (e != cudaSuccess)
            return e;
    }
    cfg.gridDim = dim3((unsigned)(2 * std::max<int64_t>(1, std::min<int64_t>(std::max(1, m->max_pairs), tiles))));
    m->launches += 1;
    return cudaLaunchKernelEx(&cfg, kernel, a, b, o, o2, p);
}

template <int KIND, typename T>
cudaError_t rows_launch(esp_moe *m, const FfShape &s, const CUtensorMap &a, const CUtensorMap &b, const CUtensorMap &o,
                        const CUtensorMap &o2, FfParams &p)
{
    const int64_t tiles = row_tiles(s);
    p.g.most = (int32_t)tiles;
    return launch<KIND, T, T>(m, a, b, o, o2, p, tiles * ceil_div(p.g.N, kTileCols<KIND>));
}

template <int KIND>
cudaError_t weights_launch(esp_moe *m, const FfShape &s, const CUtensorMap &a, const CUtensorMap &b, FfParams &p, void *out,
                           bool f32)
{
    const int size = f32 ? 4 : 2;
    p.g.out = out;
    p.g.ldo = p.g.N;
    p.g.wide_store = rows_aligned(out, p.g.N, size, 16);
    CUtensorMap o = a;   // not used where the output is not aligned
    if (p.g.wide_store)
        FF_TRY(box_map3(&o, out, size, p.g.N, p.out_rows, p.g.N, (int64_t)s.E * p.planes, (int64_t)p.out_rows * p.g.N, 32));
    const int64_t tiles = (int64_t)s.E * p.planes * ceil_div(p.out_rows, 256) * ceil_div(p.g.N, 256);
    return with_16(s.dtype, [&](auto elem) -> cudaError_t {
        using T = decltype(elem);
        return f32 ? launch<KIND, T, float>(m, a, b, o, o, p, tiles) : launch<KIND, T, T>(m, a, b, o, o, p, tiles);
    });
}

}  // namespace

int few_chunk(const esp_moe *m, int64_t M, int32_t E)
{
    const int64_t rows = ceil_div(M, E);
    return rows > 128 ? 0 : rows > 64 ? 128 : rows > 32 ? 64 : rows > 16 ? 32 : 16;
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
    CUtensorMap a, b, o, o2;
    FF_TRY(box_map3(&a, x, 2, s.H, s.M, ldx, 1, 0, s.chunk ? s.chunk : kRowsA));
    FF_TRY(box_map3(&b, s.inner, 2, s.H, s.F, s.ld_inner, 2 * (int64_t)s.E, s.F * s.ld_inner, kRowsA));
    if (s.chunk)
        return launch_few(m, s, HIDDEN, s.chunk, &b, &a, &p);
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
    FF_TRY(box_map3(&a, hidden, 2, s.F, s.M, s.fp, 1, 0, s.chunk ? s.chunk : kRowsA));
    FF_TRY(box_map3(&b, s.outer, 2, s.F, s.H, s.ld_outer, s.E, s.H * s.ld_outer, kRowsA));
    if (s.chunk)
        return launch_few(m, s, OUT, s.chunk, &b, &a, &p);
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
    p.pre = pre;
    CUtensorMap a, b, o;
    FF_TRY(box_map3(&a, dy, 2, s.H, s.M, lddy, 1, 0, s.chunk ? s.chunk : kRowsA));
    FF_TRY(box_map3(&b, s.outer, 2, s.F, s.H, s.ld_outer, s.E, s.H * s.ld_outer, kInner));
    if (s.chunk)
        return launch_few(m, s, DPRE, s.chunk, &b, &a, &p);
    FF_TRY(box_map3(&o, dpre, 2, s.F, s.M, 2 * s.fp, 2, s.fp, 32));
    return with_16(s.dtype, [&](auto elem) { return rows_launch<DPRE, decltype(elem)>(m, s, a, b, o, o, p); });
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
    FF_TRY(box_map3(&a, dpre, 2, s.F, s.M, 2 * s.fp, 2, s.fp, s.chunk ? s.chunk : kRowsA));
    FF_TRY(box_map3(&b, s.inner, 2, s.H, s.F, s.ld_inner, 2 * (int64_t)s.E, s.F * s.ld_inner, kInner));
    if (s.chunk)
        return launch_few(m, s, DX, s.chunk, &b, &a, &p);
    o = a;
    if (p.g.wide_store)
        FF_TRY(box_map3(&o, dx, 2, s.H, s.M, lddx, 1, 0, 32));
    return with_16(s.dtype, [&](auto elem) { return rows_launch<DX, decltype(elem)>(m, s, a, b, o, o, p); });
}

cudaError_t launch_ff_dinner(esp_moe *m, const FfShape &s, const void *dpre, const void *x, int64_t ldx, void *dinner,
                             bool f32)
{
    FfParams p = common(m, s);
    p.g.N = s.H;
    p.planes = 2;
    p.out_rows = s.F;
    CUtensorMap a, b;
    FF_TRY(box_map3(&a, dpre, 2, s.F, s.M, 2 * s.fp, 2, s.fp, kInner));
    FF_TRY(box_map3(&b, x, 2, s.H, s.M, ldx, 1, 0, kInner));
    return weights_launch<DW>(m, s, a, b, p, dinner, f32);
}

cudaError_t launch_ff_douter(esp_moe *m, const FfShape &s, const void *dy, int64_t lddy, const void *hidden, void *douter,
                             bool f32)
{
    FfParams p = common(m, s);
    p.g.N = s.F;
    p.planes = 1;
    p.out_rows = s.H;
    CUtensorMap a, b;
    FF_TRY(box_map3(&a, dy, 2, s.H, s.M, lddy, 1, 0, kInner));
    FF_TRY(box_map3(&b, hidden, 2, s.F, s.M, s.fp, 1, 0, kInner));
    return weights_launch<DW>(m, s, a, b, p, douter, f32);
}

}  // namespace esp_moe_impl
