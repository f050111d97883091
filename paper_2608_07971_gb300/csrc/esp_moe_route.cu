// Router of the expert layer (include/esp_moe.h): the choice of experts at shadow prices, the plan that
// sorts rows by expert, the balance and logit losses, the gradient of the logits and the price step.
//
// A warp holds one token's row in registers, lane l the elements c * 32 V + l V .. + V - 1 of chunk c (V
// elements = one load of up to 16 bytes), so a row is read once, coalesced, and the statistics are
// warp reductions. The bytes are few (16384 x 256 bf16: 8.4 MB, 1.3 us). At that size and k = 8 the choice takes
// 15 us, its plan 5: 783 warp instructions per token fill 52% of the issue slots, the rest goes to a token's chain of
// dependent reductions (half of the SM's warps are there to hide it) and to the barriers around a CTA's tokens. The
// losses (10 us and 6 to join the parts) and the gradients (8 us from the weights, 12 from the losses) are bound by the
// chain of a warp's tokens, each fetched while the one before is worked on (issue slots 29 to 37% full).

#include <algorithm>
#include <cfloat>
#include <cmath>

#include "esp_moe_impl.h"
#include "esp_moe_launch.cuh"
#include "esp_moe_load.cuh"

namespace esp_moe_impl {

namespace {

constexpr uint32_t kFull = 0xffffffffu;
constexpr int kThreads = 1024;           // k_balance_sum, k_step_prices
constexpr int kWarps = kThreads / 32;
constexpr int kLeastChunk = 16;          // tokens of a CTA
// T * k up to which one CTA routes and plans in a single launch
constexpr int kFusedSlots = 512;

template <typename T, int VPT>
struct RowShape {
    static constexpr int kMaxV = 16 / (int)sizeof(T);
    static constexpr int V = VPT < kMaxV ? VPT : kMaxV;
    static __device__ __forceinline__ int element(int i, int lane) { return (i / V) * 32 * V + lane * V + i % V; }
    // Place of an element in a row of shared memory that lanes read value by value: 32 i + lane, no bank
    // conflicts (in the elements' own order the lanes would be V words apart).
    static __device__ __forceinline__ int place(int e) { return ((e / (32 * V)) * V + e % V) * 32 + e / V % 32; }
};

// A gate's reading of a logit: +inf as the largest finite value, NaN as -inf.
__device__ __forceinline__ float clean(float z)
{
    return fminf(fmaxf(z, -INFINITY), FLT_MAX);   // fmaxf of a NaN and a number is the number
}

// What a price adds to a logit: its negative, with +0 for both zeros (then a sum of 0 is +0, whatever the
// logit's sign).
__device__ __forceinline__ float price_term(float price)
{
    return price == 0.0f ? 0.0f : -price;
}

template <typename T, int VPT>
__device__ __forceinline__ void load_row(const T *row, int E, bool aligned, int lane, float (&z)[VPT])
{
    using S = RowShape<T, VPT>;
#pragma unroll
    for (int c = 0; c < VPT / S::V; ++c) {
        const int e0 = c * 32 * S::V + lane * S::V;
        if (aligned && e0 + S::V <= E) {
            load_pack<T, S::V>(row + e0, z + c * S::V);
        } else {
#pragma unroll
            for (int j = 0; j < S::V; ++j)
                z[c * S::V + j] = e0 + j < E ? to_f32(row[e0 + j]) : -INFINITY;
        }
    }
}

template <typename T, int VPT>
__device__ __forceinline__ void store_row(T *row, int E, bool aligned, int lane, const float (&d)[VPT])
{
    using S = RowShape<T, VPT>;
#pragma unroll
    for (int c = 0; c < VPT / S::V; ++c) {
        const int e0 = c * 32 * S::V + lane * S::V;
        if (aligned && e0 + S::V <= E) {
            store_pack<T, S::V>(row + e0, d + c * S::V);
        } else {
#pragma unroll
            for (int j = 0; j < S::V; ++j)
                if (e0 + j < E)
                    row[e0 + j] = from_f32<T>(d[c * S::V + j]);
        }
    }
}

__device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        v += __shfl_xor_sync(kFull, v, o);
    return v;
}

// Order-preserving key of a float that is neither NaN nor -0; kClosed is -inf's.
constexpr uint32_t kClosed = 0x007fffffu;

__device__ __forceinline__ uint32_t order_key(float v)
{
    const uint32_t u = __float_as_uint(v);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}

__device__ __forceinline__ float key_value(uint32_t k)
{
    return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}

// Largest value over the warp (no NaN among them; -0 counts as less than +0).
__device__ __forceinline__ float warp_max(float v)
{
    return key_value(__reduce_max_sync(kFull, order_key(v)));
}

__device__ __forceinline__ float sigmoid_f(float z)
{
    return 1.0f / (1.0f + expf(-z));
}

// log sigmoid(z) = min(z, 0) - log(1 + exp(-|z|)); -inf at -inf.
__device__ __forceinline__ float log_sigmoid(float z)
{
    return fminf(z, 0.0f) - log1pf(expf(-fabsf(z)));
}

// softmax of a row held in registers (max-subtracted); a row without a finite value gives zeros. Returns
// its log-sum-exp.
template <int VPT>
__device__ __forceinline__ float row_softmax(const float (&a)[VPT], float (&p)[VPT])
{
    float m = a[0];
#pragma unroll
    for (int i = 1; i < VPT; ++i)
        m = fmaxf(m, a[i]);
    m = warp_max(m);
    if (m == -INFINITY) {
#pragma unroll
        for (int i = 0; i < VPT; ++i)
            p[i] = 0.0f;
        return -INFINITY;
    }
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        p[i] = expf(a[i] - m);
        s += p[i];
    }
    s = warp_sum(s);
    const float inv = 1.0f / s;
#pragma unroll
    for (int i = 0; i < VPT; ++i)
        p[i] *= inv;
    return m + logf(s);
}

// Gate weight before `scale` of the choice in this lane (on: there is one) with logit zj; m and zsum are the
// row's maximum and sum of exponentials (softmax over all experts).
__device__ __forceinline__ float gate_weight(const Gate &g, bool on, float zj, float m, float zsum)
{
    if (g.renorm) {
        const float a = on ? (g.sigmoid ? log_sigmoid(zj) : zj) : -INFINITY;
        const float top = warp_max(a);
        const float e = on ? expf(a - top) : 0.0f;
        const float s = warp_sum(e);
        return on ? e / s : 0.0f;
    }
    if (!on)
        return 0.0f;
    return g.sigmoid ? sigmoid_f(zj) : expf(zj - m) / zsum;
}

// Exclusive scan of v[0..E) in shared memory into out[0..E] by the whole CTA (at least E threads, or E in
// steps of its threads); sums: a word per warp. Barriers before and after are inside.
__device__ __forceinline__ void block_scan(const int *v, int E, int *out, int *sums)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    int carry = 0;
    for (int e0 = 0; e0 < E; e0 += blockDim.x) {
        __syncthreads();
        const int e = e0 + threadIdx.x, x = e < E ? v[e] : 0;
        int s = x;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(kFull, s, o);
            if (lane >= o)
                s += y;
        }
        if (lane == 31)
            sums[warp] = s;
        __syncthreads();
        const int part = lane < warps ? sums[lane] : 0;
        const int before = __reduce_add_sync(kFull, lane < warp ? part : 0);
        if (e < E)
            out[e] = carry + before + s - x;
        carry += __reduce_add_sync(kFull, part);
    }
    if (threadIdx.x == 0)
        out[E] = carry;
    __syncthreads();
}

// ---- route

// The chunks' demands between k_route and k_plan, in 16 bits where a chunk's tokens fit: k_plan reads all of
// them in every CTA.
__device__ __forceinline__ void store_demand(const RouteArgs &a, int64_t i, int n)
{
    if (a.hist16)
        reinterpret_cast<uint16_t *>(a.hist)[i] = (uint16_t)n;
    else
        a.hist[i] = n;
}

// Threads of k_route's CTAs: every SM holds one, and 32 warps hide the chain of a token's k rounds; rows of
// more than 256 experts keep up to 32 values a lane, and the registers of 16 warps.
template <int VPT>
constexpr int kRouteThreads = VPT <= 8 ? 1024 : 512;

// Bytes of dynamic shared memory of k_route and of k_balance for E experts; E is at most 32 VPT.
template <int VPT>
constexpr size_t route_smem(int E)
{
    return (size_t)(32 * VPT + (kRouteThreads<VPT> / 32 + 2) * E + 1) * sizeof(int);
}

template <int VPT>
constexpr size_t balance_smem(int E)
{
    return ((size_t)kRouteThreads<VPT> * VPT + E) * sizeof(float);
}

// A lane's values in descending order of key, equal keys in their order (Batcher's odd-even merge sort), so
// that a round of the choice looks at the lanes' first values only; packed: the sorted values' places
// before, four bits each, the first in the lowest.
template <int VPT>
__device__ __forceinline__ uint32_t sort_lane(uint32_t (&key)[VPT])
{
    uint32_t at[VPT];
#pragma unroll
    for (int i = 0; i < VPT; ++i)
        at[i] = i;
#pragma unroll
    for (int p = 1; p < VPT; p <<= 1)
#pragma unroll
        for (int k = p; k >= 1; k >>= 1)
#pragma unroll
            for (int j = k % p; j + k < VPT; j += 2 * k)
#pragma unroll
                for (int i = 0; i < k; ++i)
                    if (i + j + k < VPT && (i + j) / (2 * p) == (i + j + k) / (2 * p)) {
                        const int x = i + j, y = i + j + k;
                        const bool swap = key[x] < key[y] || (key[x] == key[y] && at[x] > at[y]);
                        const uint32_t kx = key[x], ax = at[x];
                        key[x] = swap ? key[y] : kx;
                        at[x] = swap ? at[y] : ax;
                        key[y] = swap ? kx : key[y];
                        at[y] = swap ? ax : at[y];
                    }
    uint32_t packed = 0;
#pragma unroll
    for (int i = 0; i < VPT; ++i)
        packed |= at[i] << (4 * i);
    return packed;
}

// The k elements of greatest key of a row (kClosed or less: cannot be chosen), ties to the lower element:
// lane j gets the j-th, or -1.
template <typename T, int VPT>
__device__ __forceinline__ int choose(uint32_t (&key)[VPT], int k, int lane)
{
    using S = RowShape<T, VPT>;
    int sel = -1;
    if constexpr (VPT <= 8) {
        uint32_t places = sort_lane<VPT>(key);
        for (int j = 0; j < k; ++j) {
            const uint32_t top = __reduce_max_sync(kFull, key[0]);
            if (top <= kClosed)
                break;
            const int i = places & 15u;
            const unsigned el = (unsigned)((i / S::V) * 32 * S::V + lane * S::V + i % S::V);
            const bool tied = key[0] == top;
            const unsigned e = __reduce_min_sync(kFull, tied ? el : 0xffffffffu);
            if (lane == j)
                sel = (int)e;
            if (tied && el == e) {
#pragma unroll
                for (int q = 0; q < VPT; ++q)
                    key[q] = q + 1 < VPT ? key[q + 1 < VPT ? q + 1 : q] : 0u;
                places >>= 4;
            }
        }
    } else {
        for (int j = 0; j < k; ++j) {
            uint32_t best = key[0];
#pragma unroll
            for (int i = 1; i < VPT; ++i)
                best = max(best, key[i]);
            const uint32_t top = __reduce_max_sync(kFull, best);
            if (top <= kClosed)
                break;
            unsigned cand = 0xffffffffu;
#pragma unroll
            for (int i = VPT - 1; i >= 0; --i)
                if (key[i] == top)
                    cand = (unsigned)S::element(i, lane);
            const int e = (int)__reduce_min_sync(kFull, cand);
#pragma unroll
            for (int i = 0; i < VPT; ++i)
                if (S::element(i, lane) == e)
                    key[i] = 0u;
            if (lane == j)
                sel = e;
        }
    }
    return sel;
}

// Tokens [blockIdx.x * chunk, ...) of one CTA, a run of consecutive ones per warp. A choice's rank among its
// CTA's choices of the same expert (in the order of the tokens) is the expert's count in its warp so far,
// plus the counts of the warps before. FUSED (one CTA in all): counts, offsets and the plan too; otherwise
// the ranks go to pos and the CTA's demand per expert to hist[blockIdx.x], for k_plan.
template <typename T, int VPT, bool FUSED>
__global__ void __launch_bounds__(kRouteThreads<VPT>) k_route(const RouteArgs a, int64_t chunk, bool aligned)
{
    using S = RowShape<T, VPT>;
    const int threads = blockDim.x, W = blockDim.x >> 5;   // FUSED: as many warps as tokens, at least four
    extern __shared__ int sm[];
    let_next_launch_start();
    wait_for_launch_before();
    constexpr int kPadded = 32 * VPT;                  // E rounded up to the lanes' elements
    float *price = reinterpret_cast<float *>(sm);      // kPadded price terms
    int *wcount = sm + kPadded;                        // W x E
    int *hist = wcount + W * a.E;                      // E
    int *offs = hist + a.E;                            // E + 1 (FUSED)
    __shared__ int sums[kRouteThreads<VPT> / 32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int E = a.E, k = a.k;
    const bool plan = a.offsets != nullptr;
    const int64_t t0 = blockIdx.x * chunk, t1 = min(a.T, t0 + chunk);
    const int64_t per = (t1 - t0 + W - 1) / W, ta = min(t1, t0 + warp * per), tb = min(t1, ta + per);
    const T *logits = static_cast<const T *>(a.logits);
    float next[VPT];
    if (ta < tb)
        load_row<T, VPT>(logits + ta * a.ld, E, aligned, lane, next);
    int last_e = -1, last_rank = -1;   // this lane's choice and rank for the warp's last token
    int *mine = wcount + warp * E;
    for (int e = lane; e < E; e += 32)
        mine[e] = 0;
    for (int e = threadIdx.x; e < kPadded; e += threads)
        price[S::place(e)] = a.prices && e < E ? price_term(a.prices[e]) : 0.0f;
    __syncthreads();
    for (int64_t t = ta; t < tb; ++t) {
        const T *row = logits + t * a.ld;
        const bool open = !a.valid || a.valid[t] != 0;
        float z[VPT];
        uint32_t key[VPT];
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            z[i] = next[i];
            // the logit as it is minus the price; a NaN closes the expert as -inf does
            key[i] = order_key(fmaxf(__fadd_rn(z[i], price[32 * i + lane]), -INFINITY));
        }
        if (t + 1 < tb)
            load_row<T, VPT>(row + a.ld, E, aligned, lane, next);
        float m = -INFINITY, zsum = 0.0f;
        if (!a.gate.renorm && !a.gate.sigmoid) {
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                z[i] = clean(z[i]);
                m = fmaxf(m, z[i]);
            }
            m = warp_max(m);
            if (m > -INFINITY) {
#pragma unroll
                for (int i = 0; i < VPT; ++i)
                    zsum += expf(z[i] - m);
                zsum = warp_sum(zsum);
            }
        }
        const int sel = open ? choose<T, VPT>(key, k, lane) : -1;   // the same for every lane
        const float zsel = sel >= 0 ? clean(to_f32(row[sel])) : 0.0f;
        const float w = gate_weight(a.gate, sel >= 0, zsel, m, zsum);
        if (lane < k) {
            a.idx[t * k + lane] = sel;
            a.weight[t * k + lane] = __fmul_rn(a.gate.scale, w);
            int rank = -1;
            if (sel >= 0)
                rank = mine[sel]++;   // a token's choices differ: no two lanes meet
            if (plan && t + 1 < tb)
                a.pos[t * k + lane] = rank;
            last_e = sel;
            last_rank = rank;
        }
        __syncwarp();
    }
    __syncthreads();
    // counts of the warps before, and the CTA's
    for (int e = threadIdx.x; e < E; e += threads) {
        int run = 0;
#pragma unroll 8
        for (int w = 0; w < W; ++w) {
            const int c = wcount[w * E + e];
            wcount[w * E + e] = run;
            run += c;
        }
        if (!FUSED)
            store_demand(a, (int64_t)blockIdx.x * E + e, run);
        else
            a.counts[e] = hist[e] = run;
    }
    if (!plan)
        return;
    if (!FUSED)
        __syncthreads();
    if (FUSED) {
        block_scan(hist, E, offs, sums);
        for (int e = threadIdx.x; e <= E; e += threads)
            a.offsets[e] = offs[e];
        for (int64_t p = offs[E] + threadIdx.x; p < a.T * k; p += threads)
            a.rows[p] = -1;
    }
    // the warps before count too: the last token's choices are still at hand
    auto place = [&](int64_t i, int e, int rank) {
        int p = -1;
        if (e >= 0) {
            p = rank + mine[e] + (FUSED ? offs[e] : 0);
            if (FUSED)
                a.rows[p] = (int32_t)((uint32_t)i / (uint32_t)k);
        }
        a.pos[i] = p;
    };
    for (int64_t i = ta * k + lane; i < (tb - 1) * k; i += 32)
        place(i, a.idx[i], a.pos[i]);
    if (ta < tb && lane < k)
        place((tb - 1) * k + lane, last_e, last_rank);
}

// Counts and offsets from the chunks' demands hist[nb][E]; the ranks in pos become rows. A CTA takes one chunk
// and sums the columns over all chunks and over those before its own.
constexpr int kPlanThreads = 1024;

// D: a demand; a thread adds V columns (one load) of every groups-th chunk.
template <typename D, int V>
__device__ __forceinline__ void sum_columns(const D *hist, int E, int nb, int c0, int *total, int *before)
{
    struct alignas(sizeof(D) * V) Row {
        D v[V];
    };
    const int cols = E / V, groups = max(1, kPlanThreads / cols);
    for (int i = threadIdx.x; i < groups * cols; i += kPlanThreads) {
        const int c = i % cols, g = i / cols;
        int all[V] = {}, bef[V] = {};
#pragma unroll 8
        for (int b = g; b < nb; b += groups) {
            const Row r = *reinterpret_cast<const Row *>(hist + (int64_t)b * E + c * V);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                all[j] += r.v[j];
                bef[j] += b < c0 ? r.v[j] : 0;
            }
        }
#pragma unroll
        for (int j = 0; j < V; ++j) {
            atomicAdd(total + c * V + j, all[j]);
            atomicAdd(before + c * V + j, bef[j]);
        }
    }
}

__global__ void __launch_bounds__(kPlanThreads) k_plan(const RouteArgs a, int64_t chunk, int nb)
{
    extern __shared__ int sm[];
    __shared__ int sums[kPlanThreads / 32];
    const int E = a.E, k = a.k, c0 = blockIdx.x;
    int *total = sm, *before = sm + E, *offs = sm + 2 * E;
    for (int e = threadIdx.x; e < E; e += kPlanThreads)
        total[e] = before[e] = 0;
    let_next_launch_start();
    wait_for_launch_before();
    // the first slots' ranks are on their way while the columns are summed
    const int64_t s0 = c0 * chunk * k, s1 = a.offsets ? min(a.T * k, s0 + chunk * k) : s0;
    int64_t i = s0 + threadIdx.x;
    int e = i < s1 ? a.idx[i] : -1, rank = i < s1 ? a.pos[i] : 0;
    __syncthreads();
    if (!a.hist16)
        sum_columns<int32_t, 1>(a.hist, E, nb, c0, total, before);
    else if (E % 4 == 0)
        sum_columns<uint16_t, 4>(reinterpret_cast<const uint16_t *>(a.hist), E, nb, c0, total, before);
    else
        sum_columns<uint16_t, 1>(reinterpret_cast<const uint16_t *>(a.hist), E, nb, c0, total, before);
    block_scan(total, E, offs, sums);
    if (blockIdx.x == 0)
        for (int q = threadIdx.x; q < E; q += kPlanThreads)
            a.counts[q] = total[q];
    if (!a.offsets)
        return;
    if (blockIdx.x == 0)
        for (int q = threadIdx.x; q <= E; q += kPlanThreads)
            a.offsets[q] = offs[q];
    for (; i < s1;) {
        if (e >= 0) {
            const int p = rank + offs[e] + before[e];
            a.pos[i] = p;
            a.rows[p] = (int32_t)((uint32_t)i / (uint32_t)k);
        }
        i += kPlanThreads;
        e = i < s1 ? a.idx[i] : -1;
        rank = i < s1 ? a.pos[i] : 0;
    }
    for (int64_t p = offs[E] + (int64_t)blockIdx.x * kPlanThreads + threadIdx.x; p < a.T * k;
         p += (int64_t)gridDim.x * kPlanThreads)
        a.rows[p] = -1;
}

// ---- balance

__device__ __forceinline__ int seq_bound(const int32_t *seq, int b, int64_t T)
{
    return (int)max((int64_t)0, min(T, (int64_t)seq[b]));
}

// First sequence whose end lies beyond token t (B if none). A whole warp looks: 32 ends at a time, so that up
// to 32 sequences take one trip to memory and 65536 take four.
__device__ __forceinline__ int seq_of(const int32_t *seq, int B, int64_t t, int lane)
{
    int lo = 0, hi = B;
    while (lo < hi) {
        const int step = (hi - lo + 31) / 32, probe = min(lo + (lane + 1) * step, hi) - 1;
        const uint32_t beyond = __ballot_sync(kFull, (int64_t)seq[probe + 1] > t);
        if (beyond == 0)
            return hi;
        const int first = __ffs(beyond) - 1;
        if (step == 1)
            return min(lo + first, hi - 1);
        lo += first * step;
        hi = min(hi, lo + step);
    }
    return lo;
}

template <typename T, int VPT>
__global__ void __launch_bounds__(kRouteThreads<VPT>) k_balance(const BalanceArgs a, int64_t chunk, bool aligned)
{
    using S = RowShape<T, VPT>;
    constexpr int kThr = kRouteThreads<VPT>, W = kThr / 32;
    extern __shared__ float smf[];
    const int E = a.E, k = a.k;
    constexpr int kRow = 32 * VPT;
    float *red = smf;                                       // W rows of kRow, by place
    int *hist = reinterpret_cast<int *>(red + W * kRow);    // E
    let_next_launch_start();
    wait_for_launch_before();
    __shared__ float lse_w[W];
    __shared__ int tok_w[W];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t c0 = blockIdx.x * chunk, c1 = min(a.T, c0 + chunk);
    for (int s = a.seq ? seq_of(a.seq, a.B, c0, lane) : 0; s < a.B; ++s) {
        const int64_t lo = a.seq ? max(c0, (int64_t)seq_bound(a.seq, s, a.T)) : c0;
        const int64_t hi = a.seq ? min(c1, (int64_t)seq_bound(a.seq, s + 1, a.T)) : c1;
        if (lo >= c1)
            break;
        if (lo >= hi)
            continue;
        __syncthreads();
        for (int e = threadIdx.x; e < E; e += kThr)
            hist[e] = 0;
        __syncthreads();
        float acc[VPT];
#pragma unroll
        for (int i = 0; i < VPT; ++i)
            acc[i] = 0.0f;
        float lse2 = 0.0f;
        int tokens = 0;
        // the next token's row and choices are on their way while a token is summed
        float next[VPT];
        int next_idx = -1;
        auto fetch = [&](int64_t t) {
            if (t < hi) {
                next_idx = lane < k ? a.idx[t * k + lane] : -1;
                load_row<T, VPT>(static_cast<const T *>(a.logits) + t * a.ld, E, aligned, lane, next);
            }
        };
        fetch(lo + warp);
        for (int64_t t = lo + warp; t < hi; t += W) {
            const int mine = next_idx;
            float z[VPT], p[VPT];
#pragma unroll
            for (int i = 0; i < VPT; ++i)
                z[i] = clean(next[i]);
            fetch(t + W);
            if (__shfl_sync(kFull, mine, 0) < 0)
                continue;
            if (mine >= 0 && mine < E)
                atomicAdd(hist + mine, 1);
            ++tokens;
            const float lse = row_softmax<VPT>(z, p);
            lse2 += lse * lse;
            if (a.gate.sigmoid) {
#pragma unroll
                for (int i = 0; i < VPT; ++i)
                    z[i] = log_sigmoid(z[i]);
                row_softmax<VPT>(z, p);
            }
#pragma unroll
            for (int i = 0; i < VPT; ++i)
                acc[i] += p[i];
        }
#pragma unroll
        for (int i = 0; i < VPT; ++i)
            red[warp * kRow + 32 * i + lane] = acc[i];
        if (lane == 0) {
            lse_w[warp] = lse2;
            tok_w[warp] = tokens;
        }
        __syncthreads();
        const int64_t slot = (int64_t)blockIdx.x + s;
        for (int q = threadIdx.x; q < kRow; q += kThr) {
            const int e = S::element(q / 32, q % 32);
            if (e >= E)
                continue;
            float v = 0.0f;
#pragma unroll
            for (int w = 0; w < W; ++w)
                v += red[w * kRow + q];
            a.part_share[slot * E + e] = v;
            a.part_count[slot * E + e] = hist[e];
        }
        if (warp == W - 1) {
            const float l = warp_sum(lane < W ? lse_w[lane] : 0.0f);
            const int n = __reduce_add_sync(kFull, lane < W ? tok_w[lane] : 0);
            if (lane == 0) {
                a.part_lse[slot] = l;
                a.part_tokens[slot] = n;
            }
        }
    }
}

// Sums over a CTA of kThreads in a fixed order (warp trees, then the warps in turn); every thread gets them.
// buf: N words per warp, not read by the CTA since its last barrier.
template <int N>
__device__ __forceinline__ void block_sums(float (&v)[N], float (*buf)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i)
        v[i] = warp_sum(v[i]);
    if ((threadIdx.x & 31) == 0)
#pragma unroll
        for (int i = 0; i < N; ++i)
            buf[threadIdx.x >> 5][i] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        v[i] = 0.0f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w)
            v[i] += buf[w][i];
    }
}

// One CTA per sequence: the chunks' parts in order; the last CTA to finish sums the sequences' losses.
__global__ void __launch_bounds__(kThreads) k_balance_sum(const BalanceArgs a, int chunk)
{
    extern __shared__ float smf[];
    __shared__ float buf1[kWarps][1], buf2[kWarps][1], buf4[kWarps][4];
    __shared__ int nbuf[kWarps];
    __shared__ bool last;
    const int E = a.E, s = blockIdx.x;
    const int groups = max(1, kThreads / E);
    float *share = smf;                                          // groups x E
    int *count = reinterpret_cast<int *>(smf + groups * E);      // groups x E
    let_next_launch_start();
    wait_for_launch_before();
    const int lo = a.seq ? seq_bound(a.seq, s, a.T) : 0, hi = a.seq ? seq_bound(a.seq, s + 1, a.T) : (int)a.T;
    const int b0 = lo / chunk, b1 = lo < hi ? (hi - 1) / chunk + 1 : b0;
    int n = 0;
    float lse[1] = {0.0f};
    for (int b = b0 + threadIdx.x; b < b1; b += kThreads) {
        n += a.part_tokens[b + s];
        lse[0] += a.part_lse[b + s];
    }
    for (int i = threadIdx.x; i < groups * E; i += kThreads) {
        const int e = i % E, g = i / E;
        float v = 0.0f;
        int c = 0;
        const int64_t step = (int64_t)groups * E;
        const float *ps = a.part_share + (int64_t)(b0 + g + s) * E + e;
        const int32_t *pc = a.part_count + (int64_t)(b0 + g + s) * E + e;
#pragma unroll 8
        for (int b = b0 + g; b < b1; b += groups, ps += step, pc += step) {
            v += *ps;
            c += *pc;
        }
        share[i] = v;
        count[i] = c;
    }
    n = __reduce_add_sync(kFull, n);
    if ((threadIdx.x & 31) == 0)
        nbuf[threadIdx.x >> 5] = n;
    block_sums<1>(lse, buf1);   // its barrier publishes the parts too
    n = 0;
    for (int w = 0; w < kWarps; ++w)
        n += nbuf[w];
    float dot[1] = {0.0f};
    for (int e = threadIdx.x; e < E; e += kThreads) {
        float v = 0.0f;
        int c = 0;
        for (int g = 0; g < groups; ++g) {
            v += share[g * E + e];
            c += count[g * E + e];
        }
        const float mean = n > 0 ? v / (float)n : 0.0f;
        a.share[(int64_t)s * E + e] = mean;
        a.counts[(int64_t)s * E + e] = c;
        dot[0] += (float)c * mean;
    }
    block_sums<1>(dot, buf2);
    if (threadIdx.x == 0) {
        a.tokens[s] = n;
        float *mine = a.seq_loss + 3 * s;
        mine[0] = n > 0 ? (float)E * dot[0] / ((float)a.k * (float)n) : 0.0f;
        mine[1] = lse[0];
        mine[2] = (float)n;
        __threadfence();
        last = atomicAdd(a.ticket, 1u) == gridDim.x - 1;
    }
    __syncthreads();
    if (!last)
        return;
    __threadfence();
    // balance losses, squares, sequences in use, tokens
    float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int b = threadIdx.x; b < a.B; b += kThreads) {
        const float n_b = __ldcg(a.seq_loss + 3 * b + 2);
        sum[0] += __ldcg(a.seq_loss + 3 * b);
        sum[1] += __ldcg(a.seq_loss + 3 * b + 1);
        sum[2] += n_b > 0.0f ? 1.0f : 0.0f;
        sum[3] += n_b;
    }
    block_sums<4>(sum, buf4);
    if (threadIdx.x == 0) {
        a.loss[0] = sum[2] > 0.0f ? sum[0] / sum[2] : 0.0f;
        a.loss[1] = sum[3] > 0.0f ? sum[1] / sum[3] : 0.0f;
        *a.ticket = 0u;
    }
}

// ---- gradient of the logits

constexpr int kBwdThreads = 256;

// BALANCE: with the losses' gradient. A warp takes consecutive tokens; the next token's row, choices and
// gradients are on their way while a token is worked on.
template <typename T, int VPT, bool BALANCE>
__global__ void __launch_bounds__(kBwdThreads) k_route_backward(const RouteBackwardArgs a, int64_t per_warp,
                                                                 bool aligned, bool aligned_out)
{
    using S = RowShape<T, VPT>;
    extern __shared__ float smf[];
    const int E = a.E, k = a.k, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    float *row = smf + warp * 32 * VPT;   // the chosen experts' part by place, zero elsewhere
#pragma unroll
    for (int i = 0; i < VPT; ++i)
        row[32 * i + lane] = 0.0f;
    let_next_launch_start();
    wait_for_launch_before();
    const int64_t w = (int64_t)blockIdx.x * (kBwdThreads / 32) + warp;
    const int64_t t0 = w * per_warp, t1 = min(a.T, t0 + per_warp);
    const T *logits = static_cast<const T *>(a.logits);
    float next[VPT], next_g = 0.0f;
    int next_e = -1;
    auto fetch = [&](int64_t t) {
        if (t < t1) {
            load_row<T, VPT>(logits + t * a.ld, E, aligned, lane, next);
            next_e = lane < k ? a.idx[t * k + lane] : -1;
            if (a.dweight)
                next_g = lane < k ? a.dweight[t * k + lane] : 0.0f;
        }
    };
    fetch(t0);
    float g0 = 0.0f, g1 = 0.0f;
    if (BALANCE) {
        float used = 0.0f, tok = 0.0f;
        for (int b = lane; b < a.B; b += 32) {
            const int64_t n = a.tokens[b];
            used += n > 0 ? 1.0f : 0.0f;
            tok += (float)n;
        }
        used = warp_sum(used);
        tok = warp_sum(tok);
        g0 = used > 0.0f ? a.dloss[0] * (float)E / ((float)k * used) : 0.0f;
        g1 = tok > 0.0f ? 2.0f * a.dloss[1] / tok : 0.0f;
    }
    const bool dense_softmax = !a.gate.sigmoid && !a.gate.renorm;
    float coef[BALANCE ? VPT : 1];   // gradient of a counted token's r, for the sequence `held`
    int held = -1;
    int64_t held_end = 0;   // the first token past the stretch that `held` describes (-1: in no sequence)
    __syncwarp();
    for (int64_t t = t0; t < t1; ++t) {
        T *drow = static_cast<T *>(a.dlogits) + t * a.ld_out;
        const int e = next_e;
        const float gw = next_g;
        float z[VPT], p[VPT], d[VPT];
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            z[i] = clean(next[i]);
            d[i] = 0.0f;
        }
        fetch(t + 1);
        if (__shfl_sync(kFull, e, 0) < 0) {
            store_row<T, VPT>(drow, E, aligned_out, lane, d);
            continue;
        }
        const bool on = e >= 0 && e < E;
        float lse = 0.0f;
        if (dense_softmax || BALANCE)
            lse = row_softmax<VPT>(z, p);
        if (a.dweight) {
            const float g = on ? a.gate.scale * gw : 0.0f;
            float dj = g;
            if (!dense_softmax) {
                const float zj = on ? clean(to_f32(logits[t * a.ld + e])) : 0.0f;
                if (a.gate.renorm) {
                    const float pj = gate_weight(a.gate, on, zj, 0.0f, 1.0f);
                    const float dot = warp_sum(g * pj);
                    dj = pj * (g - dot) * (a.gate.sigmoid ? sigmoid_f(-zj) : 1.0f);
                } else {
                    dj = g * sigmoid_f(zj) * sigmoid_f(-zj);
                }
            }
            const int at = on ? S::place(e) : 0;
            if (on)
                row[at] = dj;
            __syncwarp();
#pragma unroll
            for (int i = 0; i < VPT; ++i)
                d[i] = row[32 * i + lane];
            __syncwarp();
            if (on)
                row[at] = 0.0f;
            if (dense_softmax) {
                float dot = 0.0f;
#pragma unroll
                for (int i = 0; i < VPT; ++i)
                    dot += p[i] * d[i];
                dot = warp_sum(dot);
#pragma unroll
                for (int i = 0; i < VPT; ++i)
                    d[i] = p[i] * (d[i] - dot);
            }
            __syncwarp();
        }
        if constexpr (BALANCE) {
            if (t >= held_end) {   // the token's sequence, if it lies in one
                const int s = a.seq ? seq_of(a.seq, a.B, t, lane) : 0;
                const bool in = s < a.B && (!a.seq || t >= a.seq[s]);
                held_end = a.seq ? (in ? (int64_t)a.seq[s + 1] : s < a.B ? (int64_t)a.seq[s] : a.T) : a.T;
                if (!in)
                    held = -1;
                if (in && s != held) {
                    held = s;
                    const float n = (float)a.tokens[s];
                    const float c = n > 0.0f ? g0 / (n * n) : 0.0f;
#pragma unroll
                    for (int i = 0; i < VPT; ++i) {
                        const int q = S::element(i, lane);
                        coef[i] = q < E ? c * (float)(int32_t)a.counts[(int64_t)s * E + q] : 0.0f;   // below 2^31
                    }
                }
            }
            if (held >= 0) {
                const float gz = g1 * lse;
                if (!a.gate.sigmoid) {
                    float dot = 0.0f;
#pragma unroll
                    for (int i = 0; i < VPT; ++i)
                        dot += coef[i] * p[i];
                    dot = warp_sum(dot);
#pragma unroll
                    for (int i = 0; i < VPT; ++i)
                        d[i] += p[i] * (coef[i] - dot + gz);
                } else {
                    float r[VPT], la[VPT];
#pragma unroll
                    for (int i = 0; i < VPT; ++i)
                        la[i] = log_sigmoid(z[i]);
                    row_softmax<VPT>(la, r);
                    float dot = 0.0f;
#pragma unroll
                    for (int i = 0; i < VPT; ++i)
                        dot += coef[i] * r[i];
                    dot = warp_sum(dot);
#pragma unroll
                    for (int i = 0; i < VPT; ++i)
                        d[i] += r[i] * (coef[i] - dot) * sigmoid_f(-z[i]) + p[i] * gz;
                }
            }
        }
        store_row<T, VPT>(drow, E, aligned_out, lane, d);
    }
}

__global__ void __launch_bounds__(kThreads) k_step_prices(int32_t E, const int64_t *counts, double eta, double slack,
                                                          float *prices)
{
    __shared__ unsigned long long total;
    let_next_launch_start();
    wait_for_launch_before();
    if (threadIdx.x == 0)
        total = 0;
    __syncthreads();
    unsigned long long s = 0;
    for (int e = threadIdx.x; e < E; e += kThreads)
        s += (unsigned long long)counts[e];
    atomicAdd(&total, s);
    __syncthreads();
    if (total == 0)
        return;
    const double cap = slack * (double)total / (double)E;
    for (int e = threadIdx.x; e < E; e += kThreads)
        prices[e] = (float)fmax(0.0, (double)prices[e] + eta * (((double)counts[e] - cap) / cap));
}

// ---- launches

// Tokens of a CTA: one CTA for every SM, kLeastChunk at least.
int64_t route_chunk(int64_t T)
{
    return std::max<int64_t>(kLeastChunk, ceil_div(T, 152));
}

bool fused(int64_t T, int32_t k)
{
    return T * k <= kFusedSlots;
}

// Calls f.template run<VPT>() for the row length.
template <typename F>
cudaError_t with_vpt(int32_t E, F &&f)
{
    if (E <= 32)
        return f(std::integral_constant<int, 1>());
    if (E <= 64)
        return f(std::integral_constant<int, 2>());
    if (E <= 128)
        return f(std::integral_constant<int, 4>());
    if (E <= 256)
        return f(std::integral_constant<int, 8>());
    if (E <= 512)
        return f(std::integral_constant<int, 16>());
    return f(std::integral_constant<int, 32>());
}

}  // namespace

size_t route_hist_ints(int64_t T, int32_t E, int32_t k)
{
    return fused(T, k) ? 0 : (size_t)ceil_div(T, route_chunk(T)) * E;
}

cudaError_t launch_route(esp_moe *m, int32_t dtype, const RouteArgs &args)
{
    RouteArgs a = args;
    a.hist16 = route_chunk(a.T) < 65536;
    return with_dtype(dtype, [&](auto elem) {
        using T = decltype(elem);
        return with_vpt(a.E, [&](auto vpt) -> cudaError_t {
            constexpr int VPT = decltype(vpt)::value;
            using S = RowShape<T, VPT>;
            const bool aligned = rows_aligned(a.logits, a.ld, sizeof(T), S::V * sizeof(T));
            constexpr int kThr = kRouteThreads<VPT>;
            const size_t smem = route_smem<VPT>(a.E);
            constexpr size_t kMost = route_smem<VPT>(32 * VPT);
            if (fused(a.T, a.k)) {
                const cudaError_t e = allow_smem<k_route<T, VPT, true>, kMost>(m->device);
                if (e != cudaSuccess)
                    return e;
                const int warps = std::min(kThr / 32, std::max(4, (int)a.T));
                m->launches += 1;
                return launch_after(k_route<T, VPT, true>, dim3(1), 32 * warps, smem, m->stream, a, a.T, aligned);
            }
            const int64_t chunk = route_chunk(a.T);
            const int nb = (int)ceil_div(a.T, chunk);
            cudaError_t e = allow_smem<k_route<T, VPT, false>, kMost>(m->device);
            if (e == cudaSuccess)
                e = launch_after(k_route<T, VPT, false>, dim3((unsigned)nb), kThr, smem, m->stream, a, chunk, aligned);
            if (e != cudaSuccess)
                return e;
            m->launches += 2;
            return launch_after(k_plan, dim3(a.offsets ? (unsigned)nb : 1u), kPlanThreads,
                                (size_t)(3 * a.E + 1) * sizeof(int), m->stream, a, chunk, nb);
        });
    });
}

int64_t balance_slots(int64_t T, int32_t B)
{
    return ceil_div(T, route_chunk(T)) + B;
}

cudaError_t launch_balance(esp_moe *m, int32_t dtype, const BalanceArgs &a)
{
    const int64_t chunk = route_chunk(a.T);
    if (a.T > 0) {
        const cudaError_t e = with_dtype(dtype, [&](auto elem) {
            using T = decltype(elem);
            return with_vpt(a.E, [&](auto vpt) -> cudaError_t {
                constexpr int VPT = decltype(vpt)::value;
                using S = RowShape<T, VPT>;
                constexpr int kThr = kRouteThreads<VPT>;
                const size_t smem = balance_smem<VPT>(a.E);
                const cudaError_t e2 = allow_smem<k_balance<T, VPT>, balance_smem<VPT>(32 * VPT)>(m->device);
                if (e2 != cudaSuccess)
                    return e2;
                m->launches += 1;
                return launch_after(k_balance<T, VPT>, dim3((unsigned)ceil_div(a.T, chunk)), kThr, smem, m->stream, a, chunk,
                                    rows_aligned(a.logits, a.ld, sizeof(T), S::V * sizeof(T)));
            });
        });
        if (e != cudaSuccess)
            return e;
    }
    const size_t smem = (size_t)std::max(1, kThreads / a.E) * a.E * (sizeof(float) + sizeof(int));
    m->launches += 1;
    return launch_after(k_balance_sum, dim3((unsigned)a.B), kThreads, smem, m->stream, a, (int)chunk);
}

cudaError_t launch_route_backward(esp_moe *m, int32_t dtype, const RouteBackwardArgs &a)
{
    if (a.T == 0)
        return cudaSuccess;
    return with_dtype(dtype, [&](auto elem) {
        using T = decltype(elem);
        return with_vpt(a.E, [&](auto vpt) -> cudaError_t {
            constexpr int VPT = decltype(vpt)::value;
            using S = RowShape<T, VPT>;
            constexpr int kW = kBwdThreads / 32;
            // resident at once: with the losses a warp first reads its sequence's counts, so it takes more tokens
            const int64_t warps = std::min<int64_t>(a.T, (int64_t)m->sm_count * (a.dloss ? 2 : 4) * kW);
            const int64_t per = ceil_div(a.T, warps);
            const int grid = (int)ceil_div(ceil_div(a.T, per), kW);
            const size_t smem = (size_t)kW * 32 * VPT * sizeof(float);
            const bool in = rows_aligned(a.logits, a.ld, sizeof(T), S::V * sizeof(T));
            const bool out = rows_aligned(a.dlogits, a.ld_out, sizeof(T), S::V * sizeof(T));
            m->launches += 1;
            return launch_after(a.dloss ? k_route_backward<T, VPT, true> : k_route_backward<T, VPT, false>,
                                dim3((unsigned)grid), kBwdThreads, smem, m->stream, a, per, in, out);
        });
    });
}

cudaError_t launch_step_prices(esp_moe *m, int32_t E, const int64_t *counts, double eta, double slack, float *prices)
{
    m->launches += 1;
    return launch_after(k_step_prices, dim3(1), kThreads, 0, m->stream, E, counts, eta, slack, prices);
}

}  // namespace esp_moe_impl
