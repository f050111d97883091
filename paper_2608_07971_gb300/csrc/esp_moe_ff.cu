// C entry points of the gated feed-forward blocks (include/esp_moe.h), and the copy of rows that tensor maps cannot read
// where they lie.

#include <algorithm>

#include "esp_moe_ff_impl.h"
#include "esp_moe_launch.cuh"
#include "esp_moe_load.cuh"
#include "esp_moe_spans.h"

namespace esp_moe_impl {

namespace {

constexpr int kCopyRows = 4;   // of a CTA, a warp for each

// A warp copies a row's 16-byte groups, eight in flight; bound by HBM's writes (65536 rows of 2048 from 8192: 53 us, 268 MB).
// V: elements that a source row allows to load at once.
template <int V>
__global__ void __launch_bounds__(32 * kCopyRows) k_copy_rows(const CopyRowsArgs a)
{
    wait_for_launch_before();
    let_next_launch_start();
    const int64_t i = (int64_t)blockIdx.x * kCopyRows + (threadIdx.x >> 5);
    const int lane = threadIdx.x & 31;
    if (i >= a.M)
        return;
    const int64_t from = a.rows ? a.rows[i] : i;
    const bool there = from >= 0 && from < a.T;
    const uint16_t *x = static_cast<const uint16_t *>(a.x) + (there ? from : 0) * a.ldx;
    uint16_t *out = static_cast<uint16_t *>(a.out) + i * a.ldo;
    constexpr int U = V == 8 ? 8 : 2;
    for (int h0 = lane * 8; h0 < a.H; h0 += 256 * U) {
        Pack<uint16_t, 8> r[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int h = h0 + 256 * u;
            r[u] = {};
            if (V == 8) {
                if (there && h < a.H)
                    r[u] = *reinterpret_cast<const Pack<uint16_t, 8> *>(x + h);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (there && h + j < a.H)
                        r[u].v[j] = x[h + j];
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (h0 + 256 * u < a.H)   // a row of `out` is whole groups of 8
                *reinterpret_cast<Pack<uint16_t, 8> *>(out + h0 + 256 * u) = r[u];
    }
}

// Rows of intermediate matrices start at multiples of 128 bytes: a tile's 128-byte rows then are whole lines.
int64_t up64(int64_t n)
{
    return (n + 63) / 64 * 64;
}

bool aligned_to(const void *p, size_t bytes)
{
    return reinterpret_cast<uintptr_t>(p) % bytes == 0;
}

bool good_blocks(const esp_moe_gated *w)
{
    constexpr int64_t kMostBytes = (int64_t)1 << 40;   // steps of a tensor map
    return w && (w->dtype == ESP_MOE_BF16 || w->dtype == ESP_MOE_F16) && w->activation >= ESP_MOE_SILU &&
           w->activation <= ESP_MOE_RELU && w->E >= 1 && w->E <= ESP_MOE_MAX_EXPERTS && w->F >= 1 && w->H >= 1 &&
           w->F <= (1 << 22) && w->H <= (1 << 22) && (int64_t)w->E * w->F <= kMaxRows / 2 &&
           (int64_t)w->E * w->H <= kMaxRows && w->inner && w->outer && w->ld_inner >= w->H && w->ld_outer >= w->F &&
           w->ld_inner % 8 == 0 && w->ld_outer % 8 == 0 && aligned_to(w->inner, 16) && aligned_to(w->outer, 16) &&
           w->ld_inner < kMostBytes / 2 / w->F && w->ld_outer < kMostBytes / 2 / w->H;
}

bool good_rows(const esp_moe_gated *w, int64_t T, int64_t ldx, const void *x, int64_t M, const int32_t *rows,
               const int32_t *offsets)
{
    if (!good_blocks(w) || T < 0 || M < 0 || T > kMaxRows || M > kMaxRows || (!rows && M != T) ||
        (!offsets && w->E != 1) || ldx < w->H || ldx >= (int64_t)1 << 39 || (M > 0 && T > 0 && !x) || !aligned_to(x, 2))
        return false;
    return (M / 256 + w->E) * ceil_div(std::max(w->F, w->H), 128) <= kMaxTiles &&
           2 * (int64_t)w->E * ceil_div(w->F, 256) * ceil_div(w->H, 256) <= kMaxTiles;
}

bool good_kept(const esp_moe_kept *k, bool copied)
{
    return k->pre && k->hidden && aligned_to(k->pre, 16) && aligned_to(k->hidden, 16) &&
           (!copied || (k->rows && aligned_to(k->rows, 16)));
}

// Whether a tensor map can read the rows in place.
bool mappable(const void *x, int64_t ldx)
{
    return rows_aligned(x, ldx, 2, 16);
}

// Rows of 16-bit elements, and the weights.
Span rows16(const void *p, int64_t rows, int64_t ld, int64_t width)
{
    return Span{p, rows, 2 * ld, 2 * width};
}

Span inner_of(const esp_moe_gated *w)
{
    return rows16(w->inner, 2 * (int64_t)w->E * w->F, w->ld_inner, w->H);
}

Span outer_of(const esp_moe_gated *w)
{
    return rows16(w->outer, (int64_t)w->E * w->H, w->ld_outer, w->F);
}

Span pre_of(const esp_moe_gated *w, const esp_moe_kept *k, int64_t M)
{
    return rows16(k->pre, M, 4 * up64(w->F), 4 * up64(w->F));
}

Span hidden_of(const esp_moe_gated *w, const esp_moe_kept *k, int64_t M)
{
    return rows16(k->hidden, M, up64(w->F), up64(w->F));
}

Span rows_of(const esp_moe_gated *w, const esp_moe_kept *k, int64_t M, bool copied)
{
    return rows16(copied ? k->rows : nullptr, M, up64(w->H), up64(w->H));
}

// Whether the forward pass would write over what it, or its gradients, still read.
bool forward_meets(const esp_moe_gated *w, const Span &x, const Span &y, const esp_moe_kept *k, int64_t M, bool copied)
{
    const Span inner = inner_of(w), outer = outer_of(w);
    if (!k)
        return written_over({y}, {inner, outer});   // x has been read before y is written
    const Span pre = pre_of(w, k, M), hidden = hidden_of(w, k, M), rows = rows_of(w, k, M, copied);
    return written_over({y, pre, hidden, rows}, {inner, outer}) || written_over({pre, hidden, rows}, {x}) || (!copied && meet(y, x));
}

FfShape shape_of(const esp_moe_gated *w, int64_t M, const int32_t *offsets)
{
    return FfShape{w->dtype, w->activation, w->E, w->F, w->H, M, offsets, w->inner, w->outer, w->ld_inner, w->ld_outer,
                   up64(w->H), nullptr, up64(w->F), nullptr};
}

}  // namespace

cudaError_t launch_copy_rows(esp_moe *m, const CopyRowsArgs &a)
{
    if (a.M == 0)
        return cudaSuccess;
    const bool wide = rows_aligned(a.x, a.ldx, 2, 16) && a.H % 8 == 0;
    const dim3 grid((unsigned)ceil_div(a.M, kCopyRows));
    m->launches += 1;
    return wide ? launch_after(k_copy_rows<8>, grid, 32 * kCopyRows, 0, m->stream, a)
                : launch_after(k_copy_rows<1>, grid, 32 * kCopyRows, 0, m->stream, a);
}

}  // namespace esp_moe_impl

using namespace esp_moe_impl;

#define MOE_CUDA(call)               \
    do {                             \
        if ((call) != cudaSuccess)   \
            return fail_call(m);     \
    } while (0)

extern "C" {

esp_status esp_moe_feed_forward(esp_moe *m, const esp_moe_gated *w, int64_t T, int64_t ldx, const void *x, int64_t M,
                                const int32_t *rows, const int32_t *offsets, int64_t ldy, void *y, esp_moe_kept *kept)
{
    esp_status st = begin_call(m);
    if (st != ESP_OK)
        return st;
    const bool copied = rows || !mappable(x, ldx);
    if (!good_rows(w, T, ldx, x, M, rows, offsets) || ldy < w->H || ldy >= (int64_t)1 << 39 || (M > 0 && !y) ||
        !aligned_to(y, 2) || (kept && M > 0 && !good_kept(kept, copied)) ||
        (M > 0 && forward_meets(w, rows16(x, T, ldx, w->H), rows16(y, M, ldy, w->H), kept, M, copied)))
        return ESP_ERR_INVALID_ARG;
    if (kept)
        kept->copied = copied;
    if (M == 0)
        return ESP_OK;
    FfShape s = shape_of(w, M, offsets);
    const int64_t hp = up64(w->H);
    // a few rows: gathered by the products themselves, unless they are kept for the gradients
    const bool vec = use_vec(M, w->E, w->F, w->H);
    const bool copy = copied && !(vec && !kept && mappable(x, ldx));
    void *hidden = nullptr, *gathered = nullptr;
    for (int pass = 0; pass < 2; ++pass) {
        Carver c(m->ws);
        s.partial = c.take<float>(ff_partial_floats(m));
        hidden = kept ? kept->hidden : c.take<uint16_t>((size_t)(M * s.fp));
        if (copy)
            gathered = kept ? kept->rows : c.take<uint16_t>((size_t)(M * hp));
        if (kept && !vec && w->activation == ESP_MOE_RELU)
            s.lengths = c.take<float>((size_t)(M + (int64_t)w->E * w->F));
        if (pass == 0 && (st = reserve_space(m, c.used())) != ESP_OK)
            return st;
    }
    if (copy) {
        MOE_CUDA(launch_copy_rows(m, CopyRowsArgs{M, T, ldx, hp, w->H, x, rows, gathered}));
        x = gathered;
        ldx = hp;
        T = M;
        rows = nullptr;
    }
    if (vec) {
        MOE_CUDA(launch_vec(m, s, x, ldx, T, rows, hidden, kept ? kept->pre : nullptr, y, ldy));
        return ESP_OK;
    }
    MOE_CUDA(launch_ff_hidden(m, s, x, ldx, hidden, kept ? kept->pre : nullptr));
    MOE_CUDA(launch_ff_out(m, s, hidden, y, ldy));
    return ESP_OK;
}

esp_status esp_moe_feed_forward_backward(esp_moe *m, const esp_moe_gated *w, int64_t T, int64_t ldx, const void *x,
                                         int64_t M, const int32_t *rows, const int32_t *offsets, const esp_moe_kept *kept,
                                         int64_t lddy, const void *dy, int64_t lddx, void *dx, int32_t dw_dtype,
                                         void *dinner, void *douter)
{
    esp_status st = begin_call(m);
    if (st != ESP_OK)
        return st;
    const bool copied = kept && kept->copied;
    if (!good_rows(w, T, ldx, x, M, rows, offsets) || !kept || (M > 0 && !good_kept(kept, copied)) ||
        (M > 0 && !copied && (rows || !mappable(x, ldx))) || lddy < w->H || lddy >= (int64_t)1 << 39 || (M > 0 && !dy) ||
        !aligned_to(dy, 2) || (dx && (lddx < w->H || lddx >= (int64_t)1 << 39 || !aligned_to(dx, 2))) ||
        (dw_dtype != w->dtype && dw_dtype != ESP_MOE_F32))
        return ESP_ERR_INVALID_ARG;
    const bool f32 = dw_dtype == ESP_MOE_F32;
    if (!aligned_to(dinner, f32 ? 4 : 2) || !aligned_to(douter, f32 ? 4 : 2))
        return ESP_ERR_INVALID_ARG;
    const size_t n = (size_t)w->E * w->F * w->H * (f32 ? 4 : 2);   // bytes of douter
    const auto all_of = [](const void *p, size_t bytes) { return Span{p, 1, (int64_t)bytes, (int64_t)bytes}; };
    if (written_over({rows16(dx, M, lddx, w->H), all_of(dinner, 2 * n), all_of(douter, n)},
                     {rows16(dy, M, lddy, w->H), copied ? rows_of(w, kept, M, true) : rows16(x, T, ldx, w->H), pre_of(w, kept, M),
                      hidden_of(w, kept, M), inner_of(w), outer_of(w)}))
        return ESP_ERR_INVALID_ARG;
    if (M == 0) {
        if (dinner)
            MOE_CUDA(cudaMemsetAsync(dinner, 0, 2 * n, m->stream));
        if (douter)
            MOE_CUDA(cudaMemsetAsync(douter, 0, n, m->stream));
        return ESP_OK;
    }
    FfShape s = shape_of(w, M, offsets);
    const int64_t hp = up64(w->H);
    const bool copy_dy = !mappable(dy, lddy), want_dpre = dx || dinner;
    void *dpre = nullptr, *dy_copy = nullptr, *dpre_tails = nullptr, *x_tails = nullptr, *dy_tails = nullptr,
         *hidden_tails = nullptr;
    const size_t tail_rows = offsets ? (size_t)w->E * kInner : 0;
    for (int pass = 0; pass < 2; ++pass) {
        Carver c(m->ws);
        s.partial = c.take<float>(ff_partial_floats(m));
        if (want_dpre)
            dpre = c.take<uint16_t>((size_t)(2 * M * s.fp));
        if (copy_dy)
            dy_copy = c.take<uint16_t>((size_t)(M * hp));
        if (offsets && dinner) {
            dpre_tails = c.take<uint16_t>(tail_rows * 2 * s.fp);
            x_tails = c.take<uint16_t>(tail_rows * hp);
        }
        if (offsets && douter) {
            dy_tails = c.take<uint16_t>(tail_rows * hp);
            hidden_tails = c.take<uint16_t>(tail_rows * s.fp);
        }
        if (pass == 0 && (st = reserve_space(m, c.used())) != ESP_OK)
            return st;
    }
    if (copy_dy) {
        MOE_CUDA(launch_copy_rows(m, CopyRowsArgs{M, M, lddy, hp, w->H, dy, nullptr, dy_copy}));
        dy = dy_copy;
        lddy = hp;
    }
    if (want_dpre)
        MOE_CUDA(launch_ff_dpre(m, s, dy, lddy, kept->pre, dpre));
    if (dx)
        MOE_CUDA(launch_ff_dx(m, s, dpre, dx, lddx));
    const void *rows_x = copied ? kept->rows : x;
    const int64_t ld_rows = copied ? hp : ldx;
    if (offsets && (dinner || douter)) {
        TailArgs a{};
        a.M = (int32_t)M;
        a.offsets = offsets;
        if (dinner) {
            a.part[a.parts++] = TailArgs::Part{dpre, dpre_tails, 2 * s.fp, 2 * s.fp, (int32_t)(s.fp + w->F)};
            a.part[a.parts++] = TailArgs::Part{rows_x, x_tails, ld_rows, hp, w->H};
        }
        if (douter) {
            a.part[a.parts++] = TailArgs::Part{dy, dy_tails, lddy, hp, w->H};
            a.part[a.parts++] = TailArgs::Part{kept->hidden, hidden_tails, s.fp, s.fp, w->F};
        }
        MOE_CUDA(launch_tails(m, a, w->E));
    }
    if (dinner || douter)
        MOE_CUDA(launch_ff_weights(m, s, FfWeightArgs{dpre, rows_x, dy, kept->hidden, ld_rows, lddy, dpre_tails, x_tails, dy_tails,
                                                      hidden_tails, offsets != nullptr, f32, dinner, douter}));
    return ESP_OK;
}

}  // extern "C"
