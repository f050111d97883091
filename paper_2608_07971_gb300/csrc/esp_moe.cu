// C entry points of the price-routed expert layer (include/esp_moe.h): checks of the arguments, work
// space, and the launches of each call.

#include <algorithm>
#include <cmath>
#include <new>

#include "esp_moe_impl.h"
#include "esp_moe_load.cuh"

using namespace esp_moe_impl;

namespace {

constexpr int64_t kMaxRows = 0x7fffff00;   // row counts fit int32 with a tile to spare
constexpr int64_t kMaxTiles = 1 << 29;

esp_status fail(esp_moe *m)
{
    cudaGetLastError();
    m->poisoned = true;
    return ESP_ERR_CUDA;
}

#define MOE_CUDA(call)              \
    do {                            \
        if ((call) != cudaSuccess)  \
            return fail(m);         \
    } while (0)

bool capturing(cudaStream_t s)
{
    cudaStreamCaptureStatus status = cudaStreamCaptureStatusNone;
    if (cudaStreamIsCapturing(s, &status) != cudaSuccess) {
        cudaGetLastError();
        return true;   // the legacy stream while another stream is being captured
    }
    return status != cudaStreamCaptureStatusNone;
}

// A wait that ran out in work done so far, reported once.
esp_status timed_out(esp_moe *m)
{
    if (!*m->err)
        return ESP_OK;
    m->poisoned = true;
    return ESP_ERR_TIMEOUT;
}

// The handle, its device current.
esp_status check(esp_moe *m)
{
    if (!m)
        return ESP_ERR_INVALID_ARG;
    if (m->poisoned)
        return ESP_ERR_STATE;
    const esp_status st = timed_out(m);
    if (st != ESP_OK)
        return st;
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || (dev != m->device && cudaSetDevice(m->device) != cudaSuccess))
        return fail(m);
    return ESP_OK;
}

// Orders what comes next on the handle's stream, which is not being captured, after all of the handle's earlier work
// that was not captured: it shares the work space. A stream whose capture began after such work, and still runs,
// cannot be waited for.
esp_status join_earlier(esp_moe *m)
{
    if (m->has_direct && m->direct != m->stream) {
        if (!m->marked) {
            if (capturing(m->direct))
                return ESP_ERR_STATE;
            MOE_CUDA(cudaEventRecord(m->handoff, m->direct));
            m->marked = true;
        }
        MOE_CUDA(cudaStreamWaitEvent(m->stream, m->handoff, 0));
    }
    m->direct = m->stream;
    m->has_direct = true;
    m->marked = false;
    return ESP_OK;
}

// Common head of every call that queues work: its place among the earlier ones, no launches yet.
esp_status begin(esp_moe *m)
{
    const esp_status st = check(m);
    if (st != ESP_OK)
        return st;
    m->launches = 0;
    // on the stream that took the last direct work there is nothing to join, captured or not
    if (m->has_direct && m->direct == m->stream && !m->marked)
        return ESP_OK;
    return capturing(m->stream) ? ESP_OK : join_earlier(m);
}

// While one lives, its thread's allocations are neither forbidden by a capture, of this stream or another, nor end it.
class BesideCaptures {
public:
    BesideCaptures() { cudaThreadExchangeStreamCaptureMode(&mode_); }
    ~BesideCaptures() { cudaThreadExchangeStreamCaptureMode(&mode_); }
    BesideCaptures(const BesideCaptures &) = delete;
    BesideCaptures &operator=(const BesideCaptures &) = delete;

private:
    cudaStreamCaptureMode mode_ = cudaStreamCaptureModeRelaxed;
};

// At least `bytes` of work space. A larger block replaces the old one, which is freed once the queued work is done
// with it, or kept as long as the handle: where a captured graph names it, or where the stream is being captured
// and cannot be waited for.
esp_status reserve(esp_moe *m, size_t bytes)
{
    if (bytes == 0)
        return ESP_OK;
    const bool in_capture = capturing(m->stream);
    if (bytes <= m->ws_bytes) {
        m->ws_captured = m->ws_captured || in_capture;
        return ESP_OK;
    }
    const BesideCaptures beside;
    if (m->ws) {
        if (m->ws_captured || in_capture) {
            esp_moe::Kept *k = new (std::nothrow) esp_moe::Kept{m->ws, m->kept};
            if (!k)
                return ESP_ERR_OOM;
            m->kept = k;
        } else {
            MOE_CUDA(cudaStreamSynchronize(m->stream));
            MOE_CUDA(cudaFree(m->ws));
        }
        m->ws = nullptr;
        m->ws_bytes = 0;
    }
    void *p = nullptr;
    if (cudaMalloc(&p, bytes) != cudaSuccess) {
        cudaGetLastError();
        return ESP_ERR_OOM;
    }
    m->ws = static_cast<unsigned char *>(p);
    m->ws_bytes = bytes;
    m->ws_captured = in_capture;
    return ESP_OK;
}

size_t element_size(int32_t dtype)
{
    return dtype == ESP_MOE_F32 ? 4 : 2;
}

bool good_dtype(int32_t dtype)
{
    return dtype == ESP_MOE_F32 || dtype == ESP_MOE_BF16 || dtype == ESP_MOE_F16;
}

bool aligned_to(const void *p, size_t bytes)
{
    return reinterpret_cast<uintptr_t>(p) % bytes == 0;
}

bool good_gate(const esp_moe_gate *g)
{
    return g && (g->kind == ESP_MOE_SOFTMAX || g->kind == ESP_MOE_SIGMOID) && std::isfinite(g->scale);
}

Gate to_gate(const esp_moe_gate *g)
{
    return Gate{g->kind == ESP_MOE_SIGMOID ? 1 : 0, g->renorm ? 1 : 0, g->scale};
}

bool good_choice(int64_t T, int32_t E, int32_t k)
{
    return E >= 1 && E <= ESP_MOE_MAX_EXPERTS && k >= 1 && k <= std::min(E, ESP_MOE_MAX_CHOICES) && T >= 0 &&
           T <= kMaxRows / k;
}

bool good_weight(const esp_moe_weight *w)
{
    return w && w->E >= 1 && w->E <= ESP_MOE_MAX_EXPERTS && w->N >= 1 && w->K >= 1 && w->N <= (1 << 22) &&
           w->K <= (1 << 22) && (int64_t)w->E * w->N <= kMaxRows && (int64_t)w->E * w->K <= kMaxRows &&
           w->q && w->scale && w->ld >= w->K && w->ld % 16 == 0 && aligned_to(w->q, 16) &&
           (!w->qt || (w->ldt >= w->N && w->ldt % 16 == 0 && aligned_to(w->qt, 16)));
}

bool good_product(int64_t T, int64_t M, const int32_t *rows, const esp_moe_weight *w, const int32_t *offsets)
{
    if (!good_weight(w) || T < 0 || M < 0 || T > kMaxRows || M > kMaxRows || (!rows && M != T) ||
        (!offsets && w->E != 1))
        return false;
    // the kernels number their tiles in int32
    const int64_t nb = ceil_div(w->N, kBlock), kb = ceil_div(w->K, kBlock);
    return (M / kBlock + w->E) * std::max(nb, kb) <= kMaxTiles && w->E * nb * kb <= kMaxTiles;
}

int64_t round_up(int64_t v, int64_t to)
{
    return ceil_div(v, to) * to;
}

}  // namespace

extern "C" {

esp_status esp_moe_create(esp_moe **out, int device, void *cuda_stream)
{
    if (!out)
        return ESP_ERR_INVALID_ARG;
    *out = nullptr;
    int n = 0;
    if (cudaGetDeviceCount(&n) != cudaSuccess || n == 0) {
        cudaGetLastError();
        return ESP_ERR_UNSUPPORTED;
    }
    if (device < 0 && cudaGetDevice(&device) != cudaSuccess)
        return ESP_ERR_CUDA;
    if (device >= n)
        return ESP_ERR_INVALID_ARG;
    int major = 0, minor = 0, sms = 0;
    if (cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, device) != cudaSuccess ||
        cudaDeviceGetAttribute(&minor, cudaDevAttrComputeCapabilityMinor, device) != cudaSuccess ||
        cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device) != cudaSuccess)
        return ESP_ERR_CUDA;
    if (major != 10 || minor != 3)
        return ESP_ERR_UNSUPPORTED;
    if (cudaSetDevice(device) != cudaSuccess)
        return ESP_ERR_CUDA;
    esp_moe *m = new (std::nothrow) esp_moe();
    if (!m)
        return ESP_ERR_OOM;
    m->device = device;
    m->stream = static_cast<cudaStream_t>(cuda_stream);
    m->sm_count = sms;
    const BesideCaptures beside;
    void *words = nullptr, *err = nullptr, *d_err = nullptr;
    const size_t bytes = kTickets * sizeof(unsigned int);
    if (cudaMalloc(&words, bytes) != cudaSuccess || cudaMemset(words, 0, bytes) != cudaSuccess ||
        cudaHostAlloc(&err, sizeof(unsigned int), cudaHostAllocMapped) != cudaSuccess ||
        cudaHostGetDevicePointer(&d_err, err, 0) != cudaSuccess ||
        cudaEventCreateWithFlags(&m->handoff, cudaEventDisableTiming) != cudaSuccess) {
        cudaGetLastError();
        if (words)
            cudaFree(words);
        if (err)
            cudaFreeHost(err);
        delete m;
        return ESP_ERR_CUDA;
    }
    m->err = static_cast<volatile unsigned int *>(err);
    *m->err = 0;
    m->d_err = static_cast<unsigned int *>(d_err);
    m->d_ticket = static_cast<unsigned int *>(words);
    *out = m;
    return ESP_OK;
}

esp_status esp_moe_set_stream(esp_moe *m, void *cuda_stream)
{
    esp_status st = check(m);
    if (st != ESP_OK)
        return st;
    const cudaStream_t next = static_cast<cudaStream_t>(cuda_stream), left = m->stream;
    if (next == left)
        return ESP_OK;
    // an event cannot order a stream that is being captured after one that is not, or the other way round
    if (m->has_direct && m->direct == left && !m->marked && !capturing(left)) {
        MOE_CUDA(cudaEventRecord(m->handoff, left));
        m->marked = true;
    }
    m->stream = next;
    if (!capturing(next) && (st = join_earlier(m)) != ESP_OK)
        m->stream = left;
    return st;
}

esp_status esp_moe_route(esp_moe *m, const esp_moe_gate *gate, int32_t dtype, int64_t T, int32_t E, int32_t k,
                         int64_t ld, const void *logits, const float *prices, const uint8_t *valid, int32_t *idx,
                         float *weight, int64_t *counts, int32_t *rows, int32_t *pos, int32_t *offsets)
{
    esp_status st = begin(m);
    if (st != ESP_OK)
        return st;
    if (!good_gate(gate) || !good_dtype(dtype) || !good_choice(T, E, k) || ld < E || !counts ||
        (T > 0 && (!logits || !idx || !weight)))
        return ESP_ERR_INVALID_ARG;
    const bool plan = rows || pos || offsets;
    if (plan && (!offsets || (T > 0 && (!rows || !pos))))
        return ESP_ERR_INVALID_ARG;
    if (!aligned_to(logits, element_size(dtype)))
        return ESP_ERR_INVALID_ARG;
    RouteArgs a{to_gate(gate), T, ld, E, k, logits, prices, valid, idx, weight, counts, rows, pos, offsets, nullptr, false};
    const size_t ints = route_hist_ints(T, E, k);
    if ((st = reserve(m, ints * sizeof(int32_t))) != ESP_OK)
        return st;
    a.hist = reinterpret_cast<int32_t *>(m->ws);
    MOE_CUDA(launch_route(m, dtype, a));
    return ESP_OK;
}

esp_status esp_moe_balance(esp_moe *m, const esp_moe_gate *gate, int32_t dtype, int64_t T, int32_t E, int32_t k,
                           int64_t ld, const void *logits, const int32_t *idx, int32_t B, const int32_t *seq_offsets,
                           float *loss, int64_t *counts, float *share, int64_t *tokens)
{
    esp_status st = begin(m);
    if (st != ESP_OK)
        return st;
    if (!good_gate(gate) || !good_dtype(dtype) || !good_choice(T, E, k) || ld < E || B < 1 ||
        B > ESP_MOE_MAX_SEQUENCES || (!seq_offsets && B != 1) || !loss || !counts || !share || !tokens ||
        (T > 0 && (!logits || !idx)) || !aligned_to(logits, element_size(dtype)))
        return ESP_ERR_INVALID_ARG;
    BalanceArgs a{};
    a.gate = to_gate(gate);
    a.T = T;
    a.ld = ld;
    a.E = E;
    a.k = k;
    a.B = B;
    a.logits = logits;
    a.idx = idx;
    a.seq = seq_offsets;
    a.loss = loss;
    a.counts = counts;
    a.share = share;
    a.tokens = tokens;
    a.ticket = m->d_ticket;
    const size_t slots = (size_t)balance_slots(T, B);
    for (int pass = 0; pass < 2; ++pass) {
        Carver c(m->ws);
        a.part_share = c.take<float>(slots * E);
        a.part_count = c.take<int32_t>(slots * E);
        a.part_lse = c.take<float>(slots);
        a.part_tokens = c.take<int32_t>(slots);
        a.seq_loss = c.take<float>(3 * (size_t)B);
        if (pass == 0 && (st = reserve(m, c.used())) != ESP_OK)
            return st;
    }
    MOE_CUDA(launch_balance(m, dtype, a));
    return ESP_OK;
}

esp_status esp_moe_route_backward(esp_moe *m, const esp_moe_gate *gate, int32_t dtype, int64_t T, int32_t E, int32_t k,
                                  int64_t ld, const void *logits, const int32_t *idx, const float *dweight, int32_t B,
                                  const int32_t *seq_offsets, const int64_t *counts, const int64_t *tokens,
                                  const float *dloss, int64_t ld_out, void *dlogits)
{
    const esp_status st = begin(m);
    if (st != ESP_OK)
        return st;
    if (!good_gate(gate) || !good_dtype(dtype) || !good_choice(T, E, k) || ld < E || ld_out < E ||
        (T > 0 && (!logits || !idx || !dlogits)) || !aligned_to(logits, element_size(dtype)) ||
        !aligned_to(dlogits, element_size(dtype)))
        return ESP_ERR_INVALID_ARG;
    if (dloss && (B < 1 || B > ESP_MOE_MAX_SEQUENCES || (!seq_offsets && B != 1) || !counts || !tokens))
        return ESP_ERR_INVALID_ARG;
    RouteBackwardArgs a{to_gate(gate), T,       ld,          ld_out, E,      k,      dloss ? B : 0,
                        logits,        idx,     dweight,     seq_offsets,              counts, tokens, dloss,
                        dlogits};
    MOE_CUDA(launch_route_backward(m, dtype, a));
    return ESP_OK;
}

esp_status esp_moe_step_prices(esp_moe *m, int32_t E, const int64_t *counts, double eta, double slack, float *prices)
{
    const esp_status st = begin(m);
    if (st != ESP_OK)
        return st;
    if (E < 1 || E > ESP_MOE_MAX_EXPERTS || !counts || !prices || !(eta > 0.0) || !std::isfinite(eta) ||
        !(slack > 0.0) || !std::isfinite(slack))
        return ESP_ERR_INVALID_ARG;
    MOE_CUDA(launch_step_prices(m, E, counts, eta, slack, prices));
    return ESP_OK;
}

esp_status esp_moe_quantize_weight(esp_moe *m, int32_t dtype, const void *w, int64_t ldw, const esp_moe_weight *out)
{
    const esp_status st = begin(m);
    if (st != ESP_OK)
        return st;
    if (!good_dtype(dtype) || !w || !good_weight(out) || ldw < out->K || !aligned_to(w, element_size(dtype)))
        return ESP_ERR_INVALID_ARG;
    MOE_CUDA(launch_quant_weight(m, dtype, w, ldw, *out));
    return ESP_OK;
}

esp_status esp_moe_linear(esp_moe *m, int32_t dtype, int64_t T, int64_t ldx, const void *x, int64_t M,
                          const int32_t *rows, const esp_moe_weight *w, const int32_t *offsets, int64_t ldy, void *y)
{
    esp_status st = begin(m);
    if (st != ESP_OK)
        return st;
    if (!good_dtype(dtype) || !good_product(T, M, rows, w, offsets) || ldx < w->K || ldy < w->N ||
        (M > 0 && (!y || (T > 0 && !x))) || !aligned_to(x, element_size(dtype)) || !aligned_to(y, element_size(dtype)))
        return ESP_ERR_INVALID_ARG;
    if (M == 0)
        return ESP_OK;
    const int64_t kb = ceil_div(w->K, kBlock), nb = ceil_div(w->N, kBlock);
    const bool pick = rows && pick_after_rounding(M, T, w->K);
    // picked after rounding: the T rows once, and one more that is zero
    QuantRowsArgs q{pick ? T + 1 : M, T, ldx, round_up(w->K, 16), round_up(kb, 4), w->K, x, pick ? nullptr : rows,
                    nullptr, nullptr};
    PickRowsArgs r{M, T, q.ldq, q.lds, rows, nullptr, nullptr, nullptr, nullptr};
    float *partial = nullptr;
    for (int pass = 0; pass < 2; ++pass) {
        Carver c(m->ws);
        q.q = c.take<uint8_t>((size_t)(q.M * q.ldq));
        q.scale = c.take<float>((size_t)(q.M * q.lds));
        r.q = pick ? c.take<uint8_t>((size_t)(M * q.ldq)) : q.q;
        r.scale = pick ? c.take<float>((size_t)(M * q.lds)) : q.scale;
        partial = c.take<float>(gemm_partial_floats(m));
        if (pass == 0 && (st = reserve(m, c.used())) != ESP_OK)
            return st;
    }
    MOE_CUDA(launch_quant_rows(m, dtype, q));
    if (pick) {
        r.from_q = q.q;
        r.from_scale = q.scale;
        MOE_CUDA(launch_pick_rows(m, r));
    }
    const GemmRowsArgs g{M, q.ldq, q.lds, w->ld, ldy, w->E, w->N, w->K, r.q, w->q, r.scale, w->scale,
                         nb * kb, kb, 1, offsets, y, partial};
    MOE_CUDA(launch_gemm_rows(m, dtype, g));
    return ESP_OK;
}

esp_status esp_moe_linear_backward(esp_moe *m, int32_t dtype, int64_t T, int64_t ldx, const void *x, int64_t M,
                                   const int32_t *rows, const esp_moe_weight *w, const int32_t *offsets, int64_t lddy,
                                   const void *dy, int64_t lddx, void *dx, int64_t lddw, float *dw)
{
    esp_status st = begin(m);
    if (st != ESP_OK)
        return st;
    if (!good_dtype(dtype) || !good_product(T, M, rows, w, offsets) || lddy < w->N ||
        (M > 0 && !dy) || !aligned_to(dy, element_size(dtype)) || (dx && (!w->qt || lddx < w->K)) ||
        !aligned_to(dx, element_size(dtype)) || !aligned_to(dw, 4) || (dw && (lddw < w->K || ldx < w->K)) ||
        (dw && M > 0 && T > 0 && !x) || !aligned_to(x, element_size(dtype)))
        return ESP_ERR_INVALID_ARG;
    const int64_t kb = ceil_div(w->K, kBlock), nb = ceil_div(w->N, kBlock);
    const int64_t positions = (M / kBlock + w->E) * kBlock;   // every expert's rows rounded up to a block
    if (dw && positions > kMaxRows)
        return ESP_ERR_INVALID_ARG;
    const bool want_dx = dx && M > 0;
    QuantRowsArgs q{M, M, lddy, round_up(w->N, 16), round_up(nb, 4), w->N, dy, nullptr, nullptr, nullptr};
    QuantColsArgs cy{M, M, lddy, positions, round_up(w->N, 4), w->N, w->E, dy, nullptr, offsets, nullptr, nullptr,
                     nullptr, nullptr, 0, 0};
    QuantColsArgs cx{M, T, ldx, positions, round_up(w->K, 4), w->K, w->E, x, rows, offsets, nullptr, nullptr,
                     nullptr, nullptr, 0, 0};
    float *partial = nullptr;
    for (int pass = 0; pass < 2; ++pass) {
        Carver c(m->ws);
        partial = c.take<float>(gemm_partial_floats(m));
        if (want_dx) {
            q.q = c.take<uint8_t>((size_t)(M * q.ldq));
            q.scale = c.take<float>((size_t)(M * q.lds));
        }
        if (dw) {
            cy.q = c.take<uint8_t>((size_t)(w->N * cy.ldq));
            cy.scale = c.take<float>((size_t)(positions / kBlock * cy.lds));
            cx.q = c.take<uint8_t>((size_t)(w->K * cx.ldq));
            cx.scale = c.take<float>((size_t)(positions / kBlock * cx.lds));
        }
        if (pass == 0 && (st = reserve(m, c.used())) != ESP_OK)
            return st;
    }
    if (want_dx && dw) {   // both roundings of dy from one read
        cy.row_q = q.q;
        cy.row_scale = q.scale;
        cy.row_ldq = q.ldq;
        cy.row_lds = q.lds;
    }
    if (dw)
        MOE_CUDA(launch_quant_cols(m, dtype, cy));
    if (want_dx) {
        if (!dw)
            MOE_CUDA(launch_quant_rows(m, dtype, q));
        const GemmRowsArgs g{M, q.ldq, q.lds, w->ldt, lddx, w->E, w->K, w->N, q.q, w->qt, q.scale, w->scale,
                             nb * kb, 1, kb, offsets, dx, partial};
        MOE_CUDA(launch_gemm_rows(m, dtype, g));
    }
    if (dw) {
        MOE_CUDA(launch_quant_cols(m, dtype, cx));
        const GemmColsArgs g{M, cy.ldq, cx.ldq, cy.lds, cx.lds, lddw, w->E, w->N, w->K, cy.q, cx.q, cy.scale, cx.scale,
                             offsets, dw, partial};
        MOE_CUDA(launch_gemm_cols(m, g));
    }
    return ESP_OK;
}

esp_status esp_moe_combine(esp_moe *m, int32_t dtype, int64_t T, int32_t k, int32_t H, int64_t M, int64_t ldy,
                           const void *y, const int32_t *pos, const float *weight, int64_t ldo, void *out)
{
    const esp_status st = begin(m);
    if (st != ESP_OK)
        return st;
    if (!good_dtype(dtype) || k < 1 || k > ESP_MOE_MAX_CHOICES || T < 0 || T > kMaxRows / k || H < 1 || M < 0 ||
        M > kMaxRows || ldy < H || ldo < H || (T > 0 && (!pos || !out || (M > 0 && !y))) ||
        !aligned_to(y, element_size(dtype)) || !aligned_to(out, element_size(dtype)))
        return ESP_ERR_INVALID_ARG;
    CombineArgs a{};
    a.T = T;
    a.M = M;
    a.k = k;
    a.H = H;
    a.ldy = ldy;
    a.ldo = ldo;
    a.y = y;
    a.pos = pos;
    a.weight = weight;
    a.out = out;
    MOE_CUDA(launch_combine(m, dtype, a));
    return ESP_OK;
}

esp_status esp_moe_combine_backward(esp_moe *m, int32_t dtype, int64_t T, int32_t k, int32_t H, int64_t M, int64_t lddo,
                                    const void *dout, int64_t ldy, const void *y, const int32_t *pos,
                                    const float *weight, int64_t lddy, void *dy, float *dweight)
{
    const esp_status st = begin(m);
    if (st != ESP_OK)
        return st;
    if (!good_dtype(dtype) || k < 1 || k > ESP_MOE_MAX_CHOICES || T < 0 || T > kMaxRows / k || H < 1 || M < 0 ||
        M > kMaxRows || lddo < H || (T > 0 && (!pos || !dout)) || (dweight && (ldy < H || (T > 0 && M > 0 && !y))) ||
        (dy && lddy < H) || !aligned_to(y, element_size(dtype)) || !aligned_to(dout, element_size(dtype)) ||
        !aligned_to(dy, element_size(dtype)))
        return ESP_ERR_INVALID_ARG;
    CombineArgs a{};
    a.T = T;
    a.M = M;
    a.k = k;
    a.H = H;
    a.ldy = ldy;
    a.lddo = lddo;
    a.lddy = lddy;
    a.y = y;
    a.pos = pos;
    a.weight = weight;
    a.dout = dout;
    a.dy = dy;
    a.dweight = dweight;
    MOE_CUDA(launch_combine_backward(m, dtype, a));
    return ESP_OK;
}

esp_status esp_moe_synchronize(esp_moe *m)
{
    esp_status st = check(m);
    if (st != ESP_OK)
        return st;
    if (capturing(m->stream))
        return ESP_ERR_STATE;
    if ((st = join_earlier(m)) != ESP_OK)
        return st;
    MOE_CUDA(cudaStreamSynchronize(m->stream));
    return timed_out(m);
}

esp_status esp_moe_last_launch_count(esp_moe *m, int64_t *out)
{
    if (!m || !out)
        return ESP_ERR_INVALID_ARG;
    *out = m->launches;
    return ESP_OK;
}

esp_status esp_moe_debug_set_wait_limit(esp_moe *m, uint32_t limit_ms)
{
    const esp_status st = check(m);
    if (st != ESP_OK)
        return st;
    m->wait_ms = limit_ms == 0 ? kMoeWaitMs : limit_ms;
    return ESP_OK;
}

esp_status esp_moe_debug_hold_load(esp_moe *m)
{
    const esp_status st = check(m);
    if (st != ESP_OK)
        return st;
    m->hold_load = true;
    return ESP_OK;
}

void esp_moe_destroy(esp_moe *m)
{
    if (!m)
        return;
    cudaSetDevice(m->device);
    const BesideCaptures beside;
    if (m->ws)
        cudaFree(m->ws);
    while (m->kept) {
        esp_moe::Kept *k = m->kept;
        m->kept = k->next;
        cudaFree(k->p);
        delete k;
    }
    cudaFree(m->d_ticket);
    cudaFreeHost(const_cast<unsigned int *>(m->err));
    if (m->handoff)
        cudaEventDestroy(m->handoff);
    cudaGetLastError();
    delete m;
}

}  // extern "C"
