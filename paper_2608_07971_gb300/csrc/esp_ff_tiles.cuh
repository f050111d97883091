// The list of work items of the gated feed-forward blocks' products (esp_ff_gemm.cu): which rows, columns and blocks of the
// inner axis an item is. Every role of a CTA walks it by itself. Host code can walk it too.
#pragma once

#include <algorithm>

#include <cuda_runtime.h>

#include "esp_fp8_tiles.cuh"
#include "esp_moe_ff_impl.h"

namespace esp_moe_impl {

namespace {

enum Kind { HIDDEN, OUT, DPRE, DX, DW };

constexpr int kHalfTile = 64 * 128;   // MN-major: 64 inner indices of 64 outer elements

// DW: one of a launch's weight gradients, E x planes matrices of out_rows x N.
struct DwOut {
    int32_t planes, out_rows, N;
    bool wide;                // rows on 16 bytes
    void *out;
};

struct FfParams {
    GemmParams g;             // rows, experts, N (columns of the output), waits
    int32_t blocks, halves;   // blocks of the inner axis in a half, halves (DX: G and U)
    DwOut dw[2];              // DW (the second one of a launch with one: zeros)
    int32_t dws;              // how many
    bool tails;               // DW: a block that an expert's rows do not fill is read from the tails
    int32_t act;
    bool few_ctas;            // most SMs are free
    int32_t half_f16;         // operands are fp16 (else bf16)
    int64_t fp;
    void *out2;               // HIDDEN: pre (or null)
    // HIDDEN with pre and a kinked activation: the operands, their rows' lengths (null: no g is summed again), and below which
    // part of the product of two of them a g is
    const void *x, *inner;
    int64_t ldx, ld_inner;
    const float *lengths;     // M rows of x, E x F rows of G
    float near_zero;
};

// One item of the list: blocks k0 .. k1 - 1 of the inner axis of a tile. Row kinds: rows m0 .. m0 + rows - 1 of expert e,
// columns n0 ..; DW: output rows m0 .. of plane z of gradient q, over the rows lo .. hi - 1, the last block from the tails where `cut` is set.
struct FfTile {
    int item, e, m0, rows, n0, k0, k1, q, z, lo, hi;
    bool cut;
};

template <int KIND>
constexpr int kTileCols = KIND == HIDDEN ? 128 : 256;

// A role's way through the list, in rounds of an item for every CTA (pair), every second round backwards, so that nobody
// gets the longer item of every round (experts' rows differ). Tiles run over an expert's rows first, so that the tiles in
// flight share columns of B. Items ascend: the row kinds' expert is kept from one to the next.
template <int CG, int KIND>
class Walk {
public:
    const uint16_t *order = nullptr;   // DW: the experts in the order of the list

    // The next item of CTA (pair) `me` of n.
    __host__ __device__ __forceinline__ bool next(const FfParams &p, int me, int n, FfTile &t)
    {
        const int item = round_ * n + (round_ & 1 ? n - 1 - me : me);
        ++round_;
        t.item = item;
        if (CG == 2 || p.g.splits == 1)
            return tile(p, item, t);
        const int part = item % p.g.splits;
        if (!tile(p, item / p.g.splits, t))
            return false;
        const int blocks = t.k1;
        t.k0 = (int)((int64_t)blocks * part / p.g.splits);
        t.k1 = (int)((int64_t)blocks * (part + 1) / p.g.splits);
        t.cut = t.cut && t.k0 < t.k1 && t.k1 == blocks;
        return true;
    }

private:
    __host__ __device__ __forceinline__ bool tile(const FfParams &p, int item, FfTile &t)
    {
        constexpr int kRows = 128 * CG;
        t.k0 = 0;
        t.cut = false;
        if (KIND != DW) {
            const int nt = (p.g.N + kTileCols<KIND> - 1) / kTileCols<KIND>;
            while (item >= (before_ + tiles_) * nt) {
                before_ += tiles_;
                if (++e_ >= p.g.E)
                    return false;
                expert_rows(p.g, e_, lo_, hi_);
                // offsets that do not ascend have more tiles than the list
                tiles_ = std::min((hi_ - lo_) / kRows + ((hi_ - lo_) % kRows != 0), p.g.most - before_);
            }
            const int i = item - before_ * nt;
            t.e = e_;
            t.m0 = lo_ + (i % tiles_) * kRows;
            t.rows = std::min(kRows, hi_ - t.m0);
            t.n0 = (i / tiles_) * kTileCols<KIND>;
            t.k1 = p.blocks * p.halves;
            return true;
        }
        // an expert's tiles of both gradients together
        const int mt0 = (p.dw[0].out_rows + kRows - 1) / kRows, per0 = mt0 * ((p.dw[0].N + 255) / 256) * p.dw[0].planes;
        const int mt1 = (p.dw[1].out_rows + kRows - 1) / kRows, per1 = mt1 * ((p.dw[1].N + 255) / 256) * p.dw[1].planes;
        if (item >= (per0 + per1) * p.g.E)
            return false;
        t.e = item / (per0 + per1);
        int i = item - t.e * (per0 + per1);
        if (order)
            t.e = order[t.e];
        t.q = i >= per0;
        i -= t.q ? per0 : 0;
        const int m = t.q ? mt1 : mt0, plane = t.q ? per1 / p.dw[1].planes : per0 / p.dw[0].planes;
        t.z = i / plane;
        i -= t.z * plane;
        t.m0 = (i % m) * kRows;
        t.n0 = (i / m) * 256;
        t.rows = std::min(kRows, (t.q ? p.dw[1].out_rows : p.dw[0].out_rows) - t.m0);
        expert_rows(p.g, t.e, t.lo, t.hi);
        const bool part = (t.hi - t.lo) % kInner != 0;   // without tails, what follows the last row is outside: zeros
        t.cut = part && p.tails;
        t.k1 = (t.hi - t.lo) / kInner + part;
        return true;
    }

    int round_ = 0;
    int e_ = -1, before_ = 0, tiles_ = 0, lo_ = 0, hi_ = 0;   // expert, row tiles of those before it, its own, its rows
};

}  // namespace

}  // namespace esp_moe_impl
