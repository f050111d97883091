// Router of the expert layer (include/esp_moe.h): the choice of experts at shadow prices, the plan that
// sorts rows by expert, the balance and logit losses, the gradient of the logits and the price step.
//
// A warp holds one token's row in registers, lane l the elements c * 32 V + l V .. + V - 1 of chunk c (V
// elements = one load of up to 16 bytes), so a row is read once, coalesced, and the statistics are
// warp reductions.

#include <algorithm>
#include <cfloat>
#include <cmath>

#include "esp_moe_impl.h"
#include "esp_moe_load.cuh"

namespace esp_moe_impl {

namespace {

constexpr uint32_t kFull = 0xffffffffu;
constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;
// T * k up to which one CTA routes and plans in a single launch
constexpr int kFusedSlots = 512;

template <typename T, int VPT>
struct RowShape {
    static constexpr int kMaxV = 16 / (int)sizeof(T);
    static constexpr int V = VPT < kMaxV ? VPT : kMaxV;
    static __device__ __forceinline__ int element(int i, int lane) { return (i / V) * 32 * V + lane * V + i % V; }
};

// A gate's reading of a logit: +inf as the largest finite value, NaN as -inf.
__device__ __forceinline__ float clean(float z)
{
    return z > -INFINITY ? fminf(z, FLT_MAX) : -INFINITY;
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
#pragma unroll
    for (int i = 0; i < VPT; ++i)
        z[i] = clean(z[i]);
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

// Order-preserving key of a float; 0 for NaN and -inf (below every other key), one key for both zeros.
__device__ __forceinline__ uint32_t order_key(float v)
{
    if (!(v > -INFINITY))
        return 0u;
    const uint32_t u = __float_as_uint(v + 0.0f);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}

__device__ __forceinline__ float key_value(uint32_t k)
{
    return k == 0u ? -INFINITY : __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}

// Largest value over the warp (values cleaned: no NaN).
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

// Exclusive scan of v[0..E) in shared memory into out[0..E] by one warp.
__device__ __forceinline__ void warp_scan(const int *v, int E, int *out, int lane)
{
    int carry = 0;
    for (int e0 = 0; e0 < E; e0 += 32) {
        const int x = e0 + lane < E ? v[e0 + lane] : 0;
        int s = x;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(kFull, s, o);
            if (lane >= o)
                s += y;
        }
        if (e0 + lane < E)
            out[e0 + lane] = carry + s - x;
        carry += __shfl_sync(kFull, s, 31);
    }
    if (lane == 0)
        out[E] = carry;
}

// ---- route

// Threads of k_route's CTAs: every SM holds one, and 32 warps hide the chain of a token's k rounds; rows of
// more than 256 experts keep up to 32 values a lane, and the registers of 16 warps.
template <int VPT>
constexpr int kRouteThreads = VPT <= 8 ? 1024 : 512;

// A lane's values in descending order of key, equal keys in ascending order of element (Batcher's odd-even
// merge sort), so that a round of the choice looks at the lanes' first values only.
template <int VPT>
__device__ __forceinline__ void sort_lane(uint32_t (&key)[VPT], int (&el)[VPT])
{
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
                        const bool swap = key[x] < key[y] || (key[x] == key[y] && el[x] > el[y]);
                        const uint32_t kx = key[x];
                        const int ex = el[x];
                        key[x] = swap ? key[y] : kx;
                        el[x] = swap ? el[y] : ex;
                        key[y] = swap ? kx : key[y];
                        el[y] = swap ? ex : el[y];
                    }
}

// The k elements of greatest key of a row (0: cannot be chosen), ties to the lower element: lane j gets the
// j-th, or -1.
template <typename T, int VPT>
__device__ __forceinline__ int choose(uint32_t (&key)[VPT], int k, int lane)
{
    using S = RowShape<T, VPT>;
    int sel = -1;
    if constexpr (VPT <= 8) {
        int el[VPT];
#pragma unroll
        for (int i = 0; i < VPT; ++i)
            el[i] = S::element(i, lane);
        sort_lane<VPT>(key, el);
        for (int j = 0; j < k; ++j) {
            const uint32_t top = __reduce_max_sync(kFull, key[0]);
            if (top == 0u)
                break;
            const int e = (int)__reduce_min_sync(kFull, key[0] == top ? (unsigned)el[0] : 0xffffffffu);
            const bool mine = key[0] == top && el[0] == e;
            if (lane == j)
                sel = e;
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                key[i] = !mine ? key[i] : i + 1 < VPT ? key[i + 1 < VPT ? i + 1 : i] : 0u;
                el[i] = mine && i + 1 < VPT ? el[i + 1 < VPT ? i + 1 : i] : el[i];
            }
        }
    } else {
        for (int j = 0; j < k; ++j) {
            uint32_t best = key[0];
#pragma unroll
            for (int i = 1; i < VPT; ++i)
                best = max(best, key[i]);
            const uint32_t top = __reduce_max_sync(kFull, best);
            if (top == 0u)
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
    constexpr int kThr = kRouteThreads<VPT>, W = kThr / 32;
    extern __shared__ int sm[];
    int *wcount = sm;               // W x E
    int *hist = sm + W * a.E;       // E
    int *offs = hist + a.E;         // E + 1 (FUSED)
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int E = a.E, k = a.k;
    const bool plan = a.offsets != nullptr;
    const int64_t t0 = blockIdx.x * chunk, t1 = min(a.T, t0 + chunk);
    const int64_t per = (t1 - t0 + W - 1) / W, ta = min(t1, t0 + warp * per), tb = min(t1, ta + per);
    const T *logits = static_cast<const T *>(a.logits);
    float next[VPT];
    if (ta < tb)
        load_row<T, VPT>(logits + ta * a.ld, E, aligned, lane, next);
    int *mine = wcount + warp * E;
    for (int e = lane; e < E; e += 32)
        mine[e] = 0;
    __syncwarp();
    for (int64_t t = ta; t < tb; ++t) {
        const T *row = logits + t * a.ld;
        const bool open = !a.valid || a.valid[t] != 0;
        float z[VPT];
        uint32_t key[VPT];
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            z[i] = next[i];
            const int e = S::element(i, lane);
            const float price = a.prices && e < E ? __ldg(a.prices + e) : 0.0f;
            key[i] = open ? order_key(__fsub_rn(z[i], price)) : 0u;
        }
        if (t + 1 < tb)
            load_row<T, VPT>(row + a.ld, E, aligned, lane, next);
        float m = -INFINITY, zsum = 0.0f;
        if (!a.gate.renorm && !a.gate.sigmoid) {
#pragma unroll
            for (int i = 0; i < VPT; ++i)
                m = fmaxf(m, z[i]);
            m = warp_max(m);
            if (m > -INFINITY) {
#pragma unroll
                for (int i = 0; i < VPT; ++i)
                    zsum += expf(z[i] - m);
                zsum = warp_sum(zsum);
            }
        }
        const int sel = choose<T, VPT>(key, k, lane);
        const float zsel = sel >= 0 ? clean(to_f32(row[sel])) : 0.0f;
        const float w = gate_weight(a.gate, sel >= 0, zsel, m, zsum);
        if (lane < k) {
            a.idx[t * k + lane] = sel;
            a.weight[t * k + lane] = __fmul_rn(a.gate.scale, w);
            int rank = -1;
            if (sel >= 0)
                rank = mine[sel]++;   // a token's choices differ: no two lanes meet
            if (plan)
                a.pos[t * k + lane] = rank;
        }
        __syncwarp();
    }
    __syncthreads();
    // counts of the warps before, and the CTA's
    for (int e = threadIdx.x; e < E; e += kThr) {
        int run = 0;
#pragma unroll 8
        for (int w = 0; w < W; ++w) {
            const int c = wcount[w * E + e];
            wcount[w * E + e] = run;
            run += c;
        }
        if (!FUSED)
            a.hist[(int64_t)blockIdx.x * E + e] = run;
        else
            a.counts[e] = hist[e] = run;
    }
    if (!plan)
        return;
    __syncthreads();
    if (FUSED) {
        if (warp == 0)
            warp_scan(hist, E, offs, lane);
        __syncthreads();
        for (int e = threadIdx.x; e <= E; e += kThr)
            a.offsets[e] = offs[e];
        for (int64_t p = offs[E] + threadIdx.x; p < a.T * k; p += kThr)
            a.rows[p] = -1;
    }
    for (int64_t i = ta * k + lane; i < tb * k; i += 32) {
        const int e = a.idx[i];
        if (e < 0)
            continue;
        const int p = a.pos[i] + mine[e] + (FUSED ? offs[e] : 0);
        a.pos[i] = p;
        if (FUSED)
            a.rows[p] = (int32_t)(i / k);
    }
}

// Counts and offsets from the CTAs' demands hist[nb][E]; the ranks in pos become rows: every CTA sums the
// columns (all, and those of the chunks before its own).
constexpr int kPlanThreads = 1024;

__global__ void __launch_bounds__(kPlanThreads) k_plan(const RouteArgs a, int64_t chunk, int nb)
{
    extern __shared__ int sm[];
    const int E = a.E, k = a.k;
    int *total = sm, *before = sm + E, *offs = sm + 2 * E;
    for (int e = threadIdx.x; e < E; e += kPlanThreads)
        total[e] = before[e] = 0;
    __syncthreads();
    const int groups = max(1, kPlanThreads / E);
    for (int i = threadIdx.x; i < groups * E; i += kPlanThreads) {
        const int e = i % E, g = i / E;
        int all = 0, bef = 0;
#pragma unroll 16
        for (int b = g; b < nb; b += groups) {
            const int h = a.hist[(int64_t)b * E + e];
            all += h;
            bef += b < (int)blockIdx.x ? h : 0;
        }
        atomicAdd(total + e, all);
        atomicAdd(before + e, bef);
    }
    __syncthreads();
    if (threadIdx.x < 32)
        warp_scan(total, E, offs, threadIdx.x);
    __syncthreads();
    if (blockIdx.x == 0) {
        for (int e = threadIdx.x; e < E; e += kPlanThreads)
            a.counts[e] = total[e];
        if (a.offsets)
            for (int e = threadIdx.x; e <= E; e += kPlanThreads)
                a.offsets[e] = offs[e];
    }
    if (!a.offsets)
        return;
    for (int64_t p = offs[E] + (int64_t)blockIdx.x * kPlanThreads + threadIdx.x; p < a.T * k;
         p += (int64_t)gridDim.x * kPlanThreads)
        a.rows[p] = -1;
    const int64_t s0 = blockIdx.x * chunk * k, s1 = min(a.T * k, s0 + chunk * k);
    for (int64_t i = s0 + threadIdx.x; i < s1; i += kPlanThreads) {
        const int e = a.idx[i];
        if (e < 0)
            continue;
        const int p = a.pos[i] + offs[e] + before[e];
        a.pos[i] = p;
        a.rows[p] = (int32_t)(i / k);
    }
}

// ---- balance

__device__ __forceinline__ int seq_bound(const int32_t *seq, int b, int64_t T)
{
    return (int)max((int64_t)0, min(T, (int64_t)seq[b]));
}

// First sequence whose end lies beyond token t (B if none).
__device__ __forceinline__ int seq_of(const int32_t *seq, int B, int64_t t)
{
    int lo = 0, hi = B;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if ((int64_t)seq[mid + 1] > t)
            hi = mid;
        else
            lo = mid + 1;
    }
    return lo;
}

template <typename T, int VPT>
__global__ void __launch_bounds__(kThreads) k_balance(const BalanceArgs a, int64_t chunk, bool aligned)
{
    using S = RowShape<T, VPT>;
    extern __shared__ float smf[];
    const int E = a.E, k = a.k;
    float *red = smf;                                      // warps x E
    int *hist = reinterpret_cast<int *>(red + kWarps * E); // E
    __shared__ float lse_w[kWarps];
    __shared__ int tok_w[kWarps];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t c0 = blockIdx.x * chunk, c1 = min(a.T, c0 + chunk);
    for (int s = a.seq ? seq_of(a.seq, a.B, c0) : 0; s < a.B; ++s) {
        const int64_t lo = a.seq ? max(c0, (int64_t)seq_bound(a.seq, s, a.T)) : c0;
        const int64_t hi = a.seq ? min(c1, (int64_t)seq_bound(a.seq, s + 1, a.T)) : c1;
        if (lo >= c1)
            break;
        if (lo >= hi)
            continue;
        __syncthreads();
        for (int e = threadIdx.x; e < E; e += kThreads)
            hist[e] = 0;
        __syncthreads();
        float acc[VPT];
#pragma unroll
        for (int i = 0; i < VPT; ++i)
            acc[i] = 0.0f;
        float lse2 = 0.0f;
        int tokens = 0;
        for (int64_t t = lo + warp; t < hi; t += kWarps) {
            const int mine = lane < k ? a.idx[t * k + lane] : -1;
            if (__shfl_sync(kFull, mine, 0) < 0)
                continue;
            if (mine >= 0 && mine < E)
                atomicAdd(hist + mine, 1);
            ++tokens;
            float z[VPT], p[VPT];
            load_row<T, VPT>(static_cast<const T *>(a.logits) + t * a.ld, E, aligned, lane, z);
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
        for (int i = 0; i < VPT; ++i) {
            const int e = S::element(i, lane);
            if (e < E)
                red[warp * E + e] = acc[i];
        }
        if (lane == 0) {
            lse_w[warp] = lse2;
            tok_w[warp] = tokens;
        }
        __syncthreads();
        const int64_t slot = (int64_t)blockIdx.x + s;
        for (int e = threadIdx.x; e < E; e += kThreads) {
            float v = 0.0f;
            for (int w = 0; w < kWarps; ++w)
                v += red[w * E + e];
            a.part_share[slot * E + e] = v;
            a.part_count[slot * E + e] = hist[e];
        }
        if (threadIdx.x == 0) {
            float l = 0.0f;
            int n = 0;
            for (int w = 0; w < kWarps; ++w) {
                l += lse_w[w];
                n += tok_w[w];
            }
            a.part_lse[slot] = l;
            a.part_tokens[slot] = n;
        }
    }
}

// Sum over a CTA in a fixed order (warp trees, then the warps in turn); every thread gets it.
__device__ float block_sum(float v, float *buf)
{
    v = warp_sum(v);
    __syncthreads();
    if ((threadIdx.x & 31) == 0)
        buf[threadIdx.x >> 5] = v;
    __syncthreads();
    float s = 0.0f;
    for (int w = 0; w < (int)(blockDim.x >> 5); ++w)
        s += buf[w];
    return s;
}

// One CTA per sequence: the chunks' parts in order; the last CTA to finish sums the sequences' losses.
__global__ void __launch_bounds__(kThreads) k_balance_sum(const BalanceArgs a, int64_t chunk)
{
    extern __shared__ float smf[];
    __shared__ float buf[kWarps];
    __shared__ bool last;
    const int E = a.E, s = blockIdx.x;
    const int groups = max(1, kThreads / E);
    float *share = smf;                                          // groups x E
    int *count = reinterpret_cast<int *>(smf + groups * E);      // groups x E
    const int64_t lo = a.seq ? seq_bound(a.seq, s, a.T) : 0, hi = a.seq ? seq_bound(a.seq, s + 1, a.T) : a.T;
    const int64_t b0 = lo / chunk, b1 = lo < hi ? (hi - 1) / chunk + 1 : b0;
    int n = 0;
    float lse = 0.0f;
    for (int64_t b = b0; b < b1; ++b) {
        n += a.part_tokens[b + s];
        lse += a.part_lse[b + s];
    }
    for (int i = threadIdx.x; i < groups * E; i += kThreads) {
        const int e = i % E, g = i / E;
        float v = 0.0f;
        int c = 0;
#pragma unroll 4
        for (int64_t b = b0 + g; b < b1; b += groups) {
            v += a.part_share[(b + s) * E + e];
            c += a.part_count[(b + s) * E + e];
        }
        share[i] = v;
        count[i] = c;
    }
    __syncthreads();
    float dot = 0.0f;
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
        dot += (float)c * mean;
    }
    dot = block_sum(dot, buf);
    if (threadIdx.x == 0) {
        a.tokens[s] = n;
        a.seq_loss[2 * s] = n > 0 ? (float)E * dot / ((float)a.k * (float)n) : 0.0f;
        a.seq_loss[2 * s + 1] = lse;
        __threadfence();
        last = atomicAdd(a.ticket, 1u) == gridDim.x - 1;
    }
    __syncthreads();
    if (!last)
        return;
    __threadfence();
    float bal = 0.0f, zl = 0.0f, used = 0.0f;
    double tok = 0.0;
    for (int b = threadIdx.x; b < a.B; b += kThreads) {
        bal += __ldcg(a.seq_loss + 2 * b);
        zl += __ldcg(a.seq_loss + 2 * b + 1);
        const long long nb = __ldcg(reinterpret_cast<const long long *>(a.tokens) + b);
        used += nb > 0 ? 1.0f : 0.0f;
        tok += (double)nb;
    }
    bal = block_sum(bal, buf);
    zl = block_sum(zl, buf);
    used = block_sum(used, buf);
    const float total = block_sum((float)tok, buf);
    if (threadIdx.x == 0) {
        a.loss[0] = used > 0.0f ? bal / used : 0.0f;
        a.loss[1] = total > 0.0f ? zl / total : 0.0f;
        *a.ticket = 0u;
    }
}

// ---- gradient of the logits

constexpr int kBwdThreads = 256;

template <typename T, int VPT>
__global__ void __launch_bounds__(kBwdThreads) k_route_backward(const RouteBackwardArgs a, int64_t per_warp,
                                                                 bool aligned, bool aligned_out)
{
    using S = RowShape<T, VPT>;
    extern __shared__ float smf[];
    __shared__ float buf[kBwdThreads / 32];
    const int E = a.E, k = a.k, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    float *row = smf + warp * E;   // the chosen experts' part, zero elsewhere
    for (int e = lane; e < E; e += 32)
        row[e] = 0.0f;
    float g0 = 0.0f, g1 = 0.0f;
    if (a.dloss) {
        float used = 0.0f, tok = 0.0f;
        for (int b = threadIdx.x; b < a.B; b += kBwdThreads) {
            const int64_t n = a.tokens[b];
            used += n > 0 ? 1.0f : 0.0f;
            tok += (float)n;
        }
        used = block_sum(used, buf);
        tok = block_sum(tok, buf);
        g0 = used > 0.0f ? a.dloss[0] * (float)E / ((float)k * used) : 0.0f;
        g1 = tok > 0.0f ? 2.0f * a.dloss[1] / tok : 0.0f;
    }
    __syncwarp();
    const bool dense_softmax = !a.gate.sigmoid && !a.gate.renorm;
    float coef[VPT];   // gradient of a counted token's r, for the sequence `held`
    int held = -1;
#pragma unroll
    for (int i = 0; i < VPT; ++i)
        coef[i] = 0.0f;
    const int64_t w = (int64_t)blockIdx.x * (kBwdThreads / 32) + warp;
    const int64_t t0 = w * per_warp, t1 = min(a.T, t0 + per_warp);
    for (int64_t t = t0; t < t1; ++t) {
        const T *zrow = static_cast<const T *>(a.logits) + t * a.ld;
        T *drow = static_cast<T *>(a.dlogits) + t * a.ld_out;
        int e = lane < k ? a.idx[t * k + lane] : -1;
        float d[VPT];
#pragma unroll
        for (int i = 0; i < VPT; ++i)
            d[i] = 0.0f;
        if (__shfl_sync(kFull, e, 0) < 0) {
            store_row<T, VPT>(drow, E, aligned_out, lane, d);
            continue;
        }
        const bool on = e >= 0 && e < E;
        float z[VPT], p[VPT];
        load_row<T, VPT>(zrow, E, aligned, lane, z);
        const float zj = on ? clean(to_f32(zrow[e])) : 0.0f;
        float lse = 0.0f;
        if (dense_softmax || a.dloss)
            lse = row_softmax<VPT>(z, p);
        if (a.dweight) {
            const float g = on ? a.gate.scale * a.dweight[t * k + lane] : 0.0f;
            if (dense_softmax) {
                if (on)
                    row[e] = g;
                __syncwarp();
                float dot = 0.0f;
#pragma unroll
                for (int i = 0; i < VPT; ++i) {
                    const int q = S::element(i, lane);
                    d[i] = q < E ? row[q] : 0.0f;
                    dot += p[i] * d[i];
                }
                dot = warp_sum(dot);
#pragma unroll
                for (int i = 0; i < VPT; ++i)
                    d[i] = p[i] * (d[i] - dot);
            } else {
                float dj;
                if (a.gate.renorm) {
                    const float pj = gate_weight(a.gate, on, zj, 0.0f, 1.0f);
                    const float dot = warp_sum(g * pj);
                    dj = pj * (g - dot) * (a.gate.sigmoid ? sigmoid_f(-zj) : 1.0f);
                } else {
                    const float s = sigmoid_f(zj);
                    dj = g * s * sigmoid_f(-zj);
                }
                if (on)
                    row[e] = dj;
                __syncwarp();
#pragma unroll
                for (int i = 0; i < VPT; ++i) {
                    const int q = S::element(i, lane);
                    d[i] = q < E ? row[q] : 0.0f;
                }
            }
            __syncwarp();
            if (on)
                row[e] = 0.0f;
            __syncwarp();
        }
        const int s = !a.dloss ? a.B : (a.seq ? seq_of(a.seq, a.B, t) : 0);
        if (a.dloss && s < a.B && (!a.seq || t >= a.seq[s])) {
            if (s != held) {
                held = s;
                const float n = (float)a.tokens[s];
                const float c = n > 0.0f ? g0 / (n * n) : 0.0f;
#pragma unroll
                for (int i = 0; i < VPT; ++i) {
                    const int q = S::element(i, lane);
                    coef[i] = q < E ? c * (float)a.counts[(int64_t)s * E + q] : 0.0f;
                }
            }
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
        store_row<T, VPT>(drow, E, aligned_out, lane, d);
    }
}

__global__ void __launch_bounds__(kThreads) k_step_prices(int32_t E, const int64_t *counts, double eta, double slack,
                                                          float *prices)
{
    __shared__ unsigned long long total;
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

// Tokens of a CTA: one CTA for every SM, a token for each of its warps at least.
int64_t route_chunk(int64_t T)
{
    return std::max<int64_t>(kWarps, ceil_div(T, 152));
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

template <typename K>
cudaError_t allow_smem(K kernel, size_t bytes)
{
    return bytes > 48 * 1024
               ? cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes)
               : cudaSuccess;
}

}  // namespace

size_t route_hist_ints(int64_t T, int32_t E, int32_t k)
{
    return fused(T, k) ? 0 : (size_t)ceil_div(T, route_chunk(T)) * E;
}

cudaError_t launch_route(esp_moe *m, int32_t dtype, const RouteArgs &a)
{
    return with_dtype(dtype, [&](auto elem) {
        using T = decltype(elem);
        return with_vpt(a.E, [&](auto vpt) -> cudaError_t {
            constexpr int VPT = decltype(vpt)::value;
            using S = RowShape<T, VPT>;
            const bool aligned = rows_aligned(a.logits, a.ld, sizeof(T), S::V * sizeof(T));
            constexpr int kThr = kRouteThreads<VPT>;
            const size_t route_smem = (size_t)((kThr / 32 + 2) * a.E + 1) * sizeof(int);
            if (fused(a.T, a.k)) {
                const cudaError_t e = allow_smem(k_route<T, VPT, true>, route_smem);
                if (e != cudaSuccess)
                    return e;
                k_route<T, VPT, true><<<1, kThr, route_smem, m->stream>>>(a, a.T, aligned);
                m->launches += 1;
                return cudaGetLastError();
            }
            const int64_t chunk = route_chunk(a.T);
            const int nb = (int)ceil_div(a.T, chunk);
            const cudaError_t e = allow_smem(k_route<T, VPT, false>, route_smem);
            if (e != cudaSuccess)
                return e;
            k_route<T, VPT, false><<<nb, kThr, route_smem, m->stream>>>(a, chunk, aligned);
            k_plan<<<a.offsets ? nb : 1, kPlanThreads, (size_t)(3 * a.E + 1) * sizeof(int), m->stream>>>(a, chunk, nb);
            m->launches += 2;
            return cudaGetLastError();
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
                const size_t smem = (size_t)(kWarps + 1) * a.E * sizeof(float);
                const cudaError_t e2 = allow_smem(k_balance<T, VPT>, smem);
                if (e2 != cudaSuccess)
                    return e2;
                k_balance<T, VPT><<<(int)ceil_div(a.T, chunk), kThreads, smem, m->stream>>>(
                    a, chunk, rows_aligned(a.logits, a.ld, sizeof(T), S::V * sizeof(T)));
                m->launches += 1;
                return cudaGetLastError();
            });
        });
        if (e != cudaSuccess)
            return e;
    }
    const size_t smem = (size_t)std::max(1, kThreads / a.E) * a.E * (sizeof(float) + sizeof(int));
    k_balance_sum<<<a.B, kThreads, smem, m->stream>>>(a, chunk);
    m->launches += 1;
    return cudaGetLastError();
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
            const int64_t warps = std::min<int64_t>(a.T, (int64_t)m->sm_count * 6 * kW);
            const int64_t per = ceil_div(a.T, warps);
            const int grid = (int)ceil_div(ceil_div(a.T, per), kW);
            k_route_backward<T, VPT><<<grid, kBwdThreads, (size_t)kW * a.E * sizeof(float), m->stream>>>(
                a, per, rows_aligned(a.logits, a.ld, sizeof(T), S::V * sizeof(T)),
                rows_aligned(a.dlogits, a.ld_out, sizeof(T), S::V * sizeof(T)));
            m->launches += 1;
            return cudaGetLastError();
        });
    });
}

cudaError_t launch_step_prices(esp_moe *m, int32_t E, const int64_t *counts, double eta, double slack, float *prices)
{
    k_step_prices<<<1, kThreads, 0, m->stream>>>(E, counts, eta, slack, prices);
    m->launches += 1;
    return cudaGetLastError();
}

}  // namespace esp_moe_impl
