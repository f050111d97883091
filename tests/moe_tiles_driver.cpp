// The products' list of work items (csrc/esp_fp8_tiles.cuh) walked on the host: with offsets that ascend every row of
// every expert and every column lies in one tile (with parts: every block in one part); with any others no item
// reaches beyond the rows, the blocks, or the items that there is room for.

#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "esp_fp8_tiles.cuh"

using namespace esp_moe_impl;

namespace {

std::mt19937 rng(1);

int pick(int lo, int hi) { return std::uniform_int_distribution<int>(lo, hi)(rng); }

[[noreturn]] void fault(const char *what, const GemmParams &p)
{
    printf("%s: M %d E %d N %d K %d splits %d\n", what, p.M, p.E, p.N, p.K, p.splits);
    std::exit(1);
}

// As the kernel's scan, saturating at each step.
template <int CG, bool COLS>
std::vector<int> table_of(const GemmParams &p)
{
    std::vector<int> t(1, 0);
    for (int e = 0; e < p.E; ++e)
        t.push_back((int)std::min<int64_t>(p.most, (int64_t)t.back() + tiles_of<CG, COLS>(p, e)));
    return t;
}

template <int CG, int BN>
void rows(bool ascending)
{
    GemmParams p{};
    p.M = pick(1, 3000);
    p.E = pick(1, 40);
    p.N = pick(1, 700);
    p.K = pick(1, 2000);
    p.splits = CG == 1 ? pick(1, 4) : 1;
    std::vector<int32_t> off(p.E + 1);
    for (int32_t &o : off)
        o = ascending ? pick(0, p.M) : pick(-100, 2 * p.M);
    if (ascending)
        std::sort(off.begin(), off.end());
    p.offsets = off.data();
    p.most = p.E == 1 ? (p.M + kRowsA * CG - 1) / (kRowsA * CG) : p.M / (kRowsA * CG) + std::min(p.E, p.M);
    const std::vector<int> table = table_of<CG, false>(p);
    const int blocks = (p.K + kBlock - 1) / kBlock, nt = (p.N + BN - 1) / BN;
    std::vector<int> seen((size_t)p.M * nt, 0);
    Tile t;
    int item = 0;
    for (; tile_at<CG, BN, false>(p, table.data(), item, t); ++item) {
        if (t.e < 0 || t.e >= p.E || t.m0 < 0 || t.rows < 1 || t.rows > kRowsA * CG || t.m0 + t.rows > p.M ||
            t.n0 < 0 || t.n0 >= p.N || t.n0 % BN || t.kb0 < 0 || t.kb1 < t.kb0 || t.kb1 > blocks)
            fault("item out of range", p);
        for (int i = 0; i < t.rows; ++i)
            seen[(size_t)(t.m0 + i) * nt + t.n0 / BN] += t.kb1 - t.kb0;
    }
    if (item > p.most * nt * p.splits)
        fault("more items than there is room for", p);
    if (!ascending)
        return;
    for (int r = 0; r < p.M; ++r)
        for (int c = 0; c < nt; ++c)
            if (seen[(size_t)r * nt + c] != (r >= off[0] && r < off[p.E] ? blocks : 0))
                fault("row not in one tile", p);
}

template <int CG, int BN>
void columns(bool ascending)
{
    GemmParams p{};
    p.M = pick(0, 3000);
    p.E = pick(1, 20);
    p.rows_b = pick(1, 500);
    p.N = pick(1, 500);
    p.splits = CG == 1 ? pick(1, 4) : 1;
    std::vector<int32_t> off(p.E + 1);
    for (int32_t &o : off)
        o = ascending ? pick(0, p.M) : pick(-100, 2 * p.M);
    if (ascending)
        std::sort(off.begin(), off.end());
    p.offsets = off.data();
    p.most = p.M / kBlock + p.E;
    const std::vector<int> table = table_of<CG, true>(p);
    const int mt = (p.rows_b + kRowsA * CG - 1) / (kRowsA * CG), nt = (p.N + BN - 1) / BN;
    std::vector<int> blocks(p.E, 0), first(p.E, 1 << 30);
    Tile t;
    int item = 0;
    for (; tile_at<CG, BN, true>(p, table.data(), item, t); ++item) {
        if (t.e < 0 || t.e >= p.E || t.m0 < 0 || t.rows < 1 || t.m0 + t.rows > p.rows_b || t.n0 < 0 || t.n0 >= p.N ||
            t.kb0 < 0 || t.kb1 < t.kb0 || t.kb1 > p.most)
            fault("item out of range", p);
        blocks[t.e] += t.kb1 - t.kb0;
        first[t.e] = std::min(first[t.e], t.kb0);
    }
    if (item != mt * nt * p.E * p.splits)
        fault("items", p);
    int before = 0;
    for (int e = 0; ascending && e < p.E; ++e) {
        const int n = (off[e + 1] - off[e] + kBlock - 1) / kBlock;
        if (blocks[e] != n * mt * nt || first[e] != before)
            fault("an expert's blocks", p);
        before += n;
    }
}

}  // namespace

int main()
{
    for (int i = 0; i < 3000; ++i)
        for (bool ascending : {true, false}) {
            rows<1, 128>(ascending);
            rows<2, 256>(ascending);
            columns<1, 128>(ascending);
            columns<2, 256>(ascending);
        }
    printf("ok\n");
    return 0;
}
