// The gated feed-forward products' list of work items (csrc/esp_ff_tiles.cuh) walked on the host, by every CTA of a launch:
// with offsets that ascend every row of every expert meets every column once, with every block of the inner axis in one
// part; the weight gradient's outputs are covered once, over all blocks of their expert, in any order of the experts. With
// other offsets no item reaches beyond the rows, or the items that there is room for.

#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "esp_ff_tiles.cuh"

using namespace esp_moe_impl;

namespace {

std::mt19937 rng(1);

int pick(int lo, int hi) { return std::uniform_int_distribution<int>(lo, hi)(rng); }

[[noreturn]] void fault(const char *what, const FfParams &p)
{
    printf("%s: M %d E %d N %d gradients %d splits %d\n", what, p.g.M, p.g.E, p.g.N, p.dws, p.g.splits);
    std::exit(1);
}

FfParams some(std::vector<int32_t> &off, bool ascending, int parts)
{
    FfParams p{};
    p.g.M = pick(1, 3000);
    p.g.E = pick(1, 40);
    p.g.N = pick(1, 900);
    p.g.splits = parts;
    off.resize(p.g.E + 1);
    for (int32_t &o : off)
        o = ascending ? pick(0, p.g.M) : pick(-100, 2 * p.g.M);
    if (ascending)
        std::sort(off.begin(), off.end());
    p.g.offsets = off.data();
    return p;
}

template <int CG, int KIND>
void rows(bool ascending)
{
    std::vector<int32_t> off;
    FfParams p = some(off, ascending, CG == 1 ? pick(1, 4) : 1);
    p.blocks = pick(1, 40);
    p.halves = KIND == DX ? 2 : 1;
    constexpr int kRows = 128 * CG, kCols = kTileCols<KIND>;
    p.g.most = p.g.E == 1 ? (p.g.M + kRows - 1) / kRows : p.g.M / kRows + std::min(p.g.E, p.g.M);
    const int nt = (p.g.N + kCols - 1) / kCols, blocks = p.blocks * p.halves, ctas = pick(1, 160);
    std::vector<int> seen((size_t)p.g.M * nt, 0), items((size_t)p.g.most * nt * p.g.splits, 0);
    for (int me = 0; me < ctas; ++me) {
        Walk<CG, KIND> walk;
        for (FfTile t; walk.next(p, me, ctas, t);) {
            if (t.item < 0 || t.item >= (int)items.size() || items[t.item]++)
                fault("items", p);
            if (t.e < 0 || t.e >= p.g.E || t.m0 < 0 || t.rows < 1 || t.rows > kRows || t.m0 + t.rows > p.g.M || t.n0 < 0 ||
                t.n0 >= p.g.N || t.n0 % kCols || t.k0 < 0 || t.k1 < t.k0 || t.k1 > blocks || t.cut)
                fault("item out of range", p);
            for (int i = 0; i < t.rows; ++i)
                seen[(size_t)(t.m0 + i) * nt + t.n0 / kCols] += t.k1 - t.k0;
        }
    }
    for (int r = 0; ascending && r < p.g.M; ++r)
        for (int c = 0; c < nt; ++c)
            if (seen[(size_t)r * nt + c] != (r >= off[0] && r < off[p.g.E] ? blocks : 0))
                fault("row not in one tile", p);
}

template <int CG>
void weights(bool ascending)
{
    std::vector<int32_t> off;
    FfParams p = some(off, ascending, CG == 1 ? pick(1, 4) : 1);
    p.dws = pick(1, 2);
    for (int q = 0; q < p.dws; ++q)
        p.dw[q] = DwOut{pick(1, 2), pick(1, 700), pick(1, 900), false, nullptr};
    p.tails = pick(0, 1);
    std::vector<uint16_t> order(p.g.E);
    for (int e = 0; e < p.g.E; ++e)
        order[e] = (uint16_t)e;
    std::shuffle(order.begin(), order.end(), rng);
    const bool ordered = pick(0, 1);
    const int ctas = pick(1, 160);
    int nt[2] = {};
    std::vector<int> seen[2];
    for (int q = 0; q < p.dws; ++q) {
        nt[q] = (p.dw[q].N + 255) / 256;
        seen[q].assign((size_t)p.g.E * p.dw[q].planes * p.dw[q].out_rows * nt[q], 0);
    }
    for (int me = 0; me < ctas; ++me) {
        Walk<CG, DW> walk;
        if (ordered)
            walk.order = order.data();
        for (FfTile t; walk.next(p, me, ctas, t);) {
            if (t.q < 0 || t.q >= p.dws)
                fault("item of no gradient", p);
            const DwOut &d = p.dw[t.q];
            if (t.e < 0 || t.e >= p.g.E || t.z < 0 || t.z >= d.planes || t.m0 < 0 || t.rows < 1 || t.rows > 128 * CG ||
                t.m0 + t.rows > d.out_rows || t.n0 < 0 || t.n0 >= d.N || t.n0 % 256 || t.k0 < 0 || t.k1 < t.k0 ||
                t.lo < 0 || t.hi < t.lo || t.hi > p.g.M || t.k1 > (t.hi - t.lo + kInner - 1) / kInner)
                fault("item out of range", p);
            const int last = (t.hi - t.lo + kInner - 1) / kInner;
            if (t.cut != (p.tails && (t.hi - t.lo) % kInner != 0 && t.k1 == last && t.k0 < t.k1))
                fault("the block that is not full", p);
            for (int i = 0; i < t.rows; ++i)   // an expert without rows has its output all the same
                seen[t.q][(((size_t)t.e * d.planes + t.z) * d.out_rows + t.m0 + i) * nt[t.q] + t.n0 / 256] +=
                    last ? t.k1 - t.k0 : (t.item % p.g.splits == 0);
        }
    }
    for (int e = 0; e < p.g.E; ++e) {
        int lo, hi;
        expert_rows(p.g, e, lo, hi);
        const int want = std::max(1, (hi - lo + kInner - 1) / kInner);
        for (int q = 0; q < p.dws; ++q) {
            const int n = p.dw[q].planes * p.dw[q].out_rows * nt[q];
            for (int i = 0; i < n; ++i)
                if (seen[q][(size_t)e * n + i] != want)
                    fault("an output not covered once", p);
        }
    }
}

}  // namespace

int main()
{
    for (int i = 0; i < 100; ++i)
        for (bool ascending : {true, false}) {
            rows<1, HIDDEN>(ascending);
            rows<2, HIDDEN>(ascending);
            rows<1, OUT>(ascending);
            rows<2, DX>(ascending);
            weights<1>(ascending);
            weights<2>(ascending);
        }
    printf("ok\n");
    return 0;
}
