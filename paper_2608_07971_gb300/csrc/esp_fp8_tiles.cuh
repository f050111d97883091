// The list of work items of the 8-bit products (esp_fp8_gemm.cu): which rows, columns and blocks of the inner axis an
// item is. Every role of a CTA walks it by itself. Host code can walk it too.
#pragma once

#include <algorithm>

#include <cuda_runtime.h>

#include "esp_moe_impl.h"

namespace esp_moe_impl {

namespace {

constexpr int kRowsA = 128;                  // rows of A that a CTA holds

struct GemmParams {
    int32_t M, E, N, K;              // rows over all experts; N: the output's columns; K: of the inner axis (FWD)
    int64_t sa_row, sa_k;            // steps of A's scales by row and block
    int32_t rows_b;                  // rows of B per expert (FWD)
    const float *scale_a, *scale_b;
    int64_t sb_e, sb_n, sb_k;
    const int32_t *offsets;
    void *out;
    int64_t ldo;
    bool wide_store;
    unsigned int *err;               // set to 1 where a wait runs out
    uint32_t wait_ms;
    // parts of every tile's inner axis, each a work item of its own (CG = 1); their sums meet in
    // partial[item][BN / 4][128][4] (lanes hold rows: consecutive rows, four columns each, lie together), and
    // the last part of a tile to arrive adds them up in order
    int32_t splits;
    float *partial;
    unsigned int *tickets;           // one per tile, zero between launches
    // the most row tiles (COLS: blocks) that experts whose offsets ascend have in all; more are left out, so that
    // offsets that do not ascend reach nothing beyond the codes, scales and parts
    int32_t most;
    int32_t hold;                    // leave out the CTAs' third load (failure detection)
};

// Expert e's rows [lo, hi).
__host__ __device__ __forceinline__ void expert_rows(const GemmParams &p, int e, int &lo, int &hi)
{
    lo = p.offsets ? std::max(0, std::min(p.M, p.offsets[e])) : 0;
    hi = p.offsets ? std::max(lo, std::min(p.M, p.offsets[e + 1])) : p.M;
}

// Row tiles (COLS: blocks) of expert e.
template <int CG, bool COLS>
__host__ __device__ __forceinline__ int tiles_of(const GemmParams &p, int e)
{
    constexpr int per = COLS ? kBlock : kRowsA * CG;
    int lo, hi;
    expert_rows(p, e, lo, hi);
    return (hi - lo) / per + ((hi - lo) % per != 0);
}

// One item of the list: rows m0 .. m0 + rows - 1 of expert e (COLS: of its output), columns n0 .., blocks
// kb0 .. kb1 - 1 (of a tile's, where its inner axis is split).
struct Tile {
    int e, m0, rows, n0, kb0, kb1;
};

// Part number `part` of the tile's blocks.
template <int CG>
__host__ __device__ __forceinline__ void take_part(const GemmParams &p, int part, Tile &t)
{
    if (CG == 2 || p.splits == 1)
        return;
    const int first = t.kb0, n = t.kb1 - t.kb0;
    t.kb0 = first + (int)((int64_t)n * part / p.splits);
    t.kb1 = first + (int)((int64_t)n * (part + 1) / p.splits);
}

// table[e]: row tiles (COLS: blocks) of the experts before e. Tiles run over an expert's rows first, so that
// the tiles in flight share columns of B.
template <int CG, int BN, bool COLS>
__host__ __device__ __forceinline__ bool tile_at(const GemmParams &p, const int *table, int item, Tile &t)
{
    constexpr int BM = kRowsA * CG;
    int w = item, part = 0;
    if (CG == 1 && p.splits > 1) {
        w = item / p.splits;
        part = item - w * p.splits;
    }
    const int nt = (p.N + BN - 1) / BN;
    if (!COLS) {
        if (w >= table[p.E] * nt)
            return false;
        int lo = 0, hi = p.E;   // the expert whose tiles hold w
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (table[mid] * nt <= w)
                lo = mid;
            else
                hi = mid;
        }
        t.e = lo;
        const int mt = table[lo + 1] - table[lo], i = w - table[lo] * nt;
        int a, b;
        expert_rows(p, lo, a, b);
        t.m0 = a + (i % mt) * BM;
        t.rows = std::min(BM, b - t.m0);
        t.n0 = (i / mt) * BN;
        t.kb0 = 0;
        t.kb1 = (p.K + kBlock - 1) / kBlock;
        take_part<CG>(p, part, t);
        return true;
    }
    const int mt = (p.rows_b + BM - 1) / BM;   // rows_b: output rows per expert
    const int per = mt * nt;
    if (w >= per * p.E)
        return false;
    t.e = w / per;
    const int i = w % per;
    t.m0 = (i % mt) * BM;
    t.rows = std::min(BM, p.rows_b - t.m0);
    t.n0 = (i / mt) * BN;
    t.kb0 = table[t.e];
    t.kb1 = table[t.e + 1];
    take_part<CG>(p, part, t);
    return true;
}

}  // namespace

}  // namespace esp_moe_impl
