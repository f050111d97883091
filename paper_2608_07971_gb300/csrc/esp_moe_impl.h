// Handle and launchers of the price-routed expert layer (include/esp_moe.h).
#pragma once

#include <cstddef>
#include <cstdint>

#include <cuda_runtime.h>

#include "esp_moe.h"

constexpr uint32_t kMoeWaitMs = 4000;   // a bounded wait's limit

struct esp_moe {
    int device = 0;
    cudaStream_t stream = nullptr;
    // the stream that took the last work that is not captured (null as a stream means the legacy one: has_direct),
    // and the event that orders others after it (recorded there since, where marked is set)
    cudaStream_t direct = nullptr;
    bool has_direct = false, marked = false;
    cudaEvent_t handoff = nullptr;
    int sm_count = 0;
    bool poisoned = false;
    int64_t launches = 0;
    unsigned char *ws = nullptr;     // work space of the call in flight (later calls run after it)
    size_t ws_bytes = 0;
    bool ws_captured = false;        // a captured call uses it: its graph names the block as long as it lives
    struct Kept {                    // outgrown blocks that graphs name, freed with the handle
        void *p;
        Kept *next;
    } *kept = nullptr;
    // error word (timeouts of the product kernels) in host memory, so that every call can look at it, and its address
    // on the device
    volatile unsigned int *err = nullptr;
    unsigned int *d_err = nullptr;
    unsigned int *d_ticket = nullptr;   // arrival counters, zero between launches
    int max_pairs = 0;               // CTA pairs of the product kernel that run at once (0: not asked yet)
    // failure-detection hooks (esp_moe.h): limit of a bounded wait, and the next
    // product launch leaving out one load
    uint32_t wait_ms = kMoeWaitMs;
    bool hold_load = false;
};

namespace esp_moe_impl {

constexpr int kBlock = ESP_MOE_BLOCK;
constexpr int kTickets = 1 + 256;   // the losses', and one per tile of a split product (fewer tiles than SMs)

// Carves the handle's work space into 256-byte aligned parts.
class Carver {
public:
    explicit Carver(unsigned char *base) : base_(base) {}
    template <typename T>
    T *take(size_t count)
    {
        T *p = reinterpret_cast<T *>(base_ + used_);
        used_ += (count * sizeof(T) + 255) & ~static_cast<size_t>(255);
        return p;
    }
    size_t used() const { return used_; }

private:
    unsigned char *base_;
    size_t used_ = 0;
};

inline int64_t ceil_div(int64_t a, int64_t b)
{
    return (a + b - 1) / b;
}

struct Gate {
    int32_t sigmoid, renorm;
    float scale;
};

// ---- esp_moe_route.cu
struct RouteArgs {
    Gate gate;
    int64_t T, ld;
    int32_t E, k;
    const void *logits;
    const float *prices;
    const uint8_t *valid;
    int32_t *idx;
    float *weight;
    int64_t *counts;
    int32_t *rows, *pos, *offsets;
    int32_t *hist;        // work space: route_hist_ints
    bool hist16;          // its numbers have 16 bits (set by the launcher)
};
size_t route_hist_ints(int64_t T, int32_t E, int32_t k);
cudaError_t launch_route(esp_moe *m, int32_t dtype, const RouteArgs &a);

struct BalanceArgs {
    Gate gate;
    int64_t T, ld;
    int32_t E, k, B;
    const void *logits;
    const int32_t *idx;
    const int32_t *seq;
    float *loss;
    int64_t *counts;
    float *share;
    int64_t *tokens;
    // work space, one slot for each (chunk of tokens, sequence) pair that meets
    float *part_share;    // slots x E
    int32_t *part_count;  // slots x E
    float *part_lse;      // slots
    int32_t *part_tokens; // slots
    float *seq_loss;      // B x 3: balance loss, sum of squares, tokens
    unsigned int *ticket;
};
int64_t balance_slots(int64_t T, int32_t B);
cudaError_t launch_balance(esp_moe *m, int32_t dtype, const BalanceArgs &a);

struct RouteBackwardArgs {
    Gate gate;
    int64_t T, ld, ld_out;
    int32_t E, k, B;
    const void *logits;
    const int32_t *idx;
    const float *dweight;
    const int32_t *seq;
    const int64_t *counts, *tokens;
    const float *dloss;
    void *dlogits;
};
cudaError_t launch_route_backward(esp_moe *m, int32_t dtype, const RouteBackwardArgs &a);
cudaError_t launch_step_prices(esp_moe *m, int32_t E, const int64_t *counts, double eta, double slack, float *prices);

// ---- esp_moe_combine.cu
struct CombineArgs {
    int64_t T, M;
    int32_t k, H;
    int64_t ldy, ldo, lddo, lddy;
    const void *y;
    const int32_t *pos;
    const float *weight;
    void *out;            // combine
    const void *dout;     // backward
    void *dy;
    float *dweight;
};
cudaError_t launch_combine(esp_moe *m, int32_t dtype, const CombineArgs &a);
cudaError_t launch_combine_backward(esp_moe *m, int32_t dtype, const CombineArgs &a);

// ---- esp_fp8.cu
// Rows as codes (M x ldq bytes) and scales (M x lds fp32, one for each 128 of a row).
struct QuantRowsArgs {
    int64_t M, T, ldx, ldq, lds;
    int32_t K;
    const void *x;
    const int32_t *rows;
    uint8_t *q;
    float *scale;
};
cudaError_t launch_quant_rows(esp_moe *m, int32_t dtype, const QuantRowsArgs &a);
// Rows of codes and scales picked from T + 1 (the last one zero): row i from rows[i], or from row T for an
// index outside [0, T).
struct PickRowsArgs {
    int64_t M, T, ldq, lds;
    const int32_t *rows;
    const uint8_t *from_q;
    const float *from_scale;
    uint8_t *q;
    float *scale;
};
cudaError_t launch_pick_rows(esp_moe *m, const PickRowsArgs &a);
// Whether M gathered rows of T with K elements are rounded once and then copied, instead of rounding each row:
// from two rows of each and 2^24 elements on (65536 rows of 2048 from 8192, the whole product: 580 us, 593
// with every row rounded; smaller ones would pay a third launch for less).
inline bool pick_after_rounding(int64_t M, int64_t T, int64_t K)
{
    return M >= 2 * T && M * K >= (int64_t)1 << 24;
}

// Columns as codes: expert e's rows i (source row rows[offsets[e] + i]) become positions base(e) + i of
// column c's run q[c * ldq + ...], base(e) = the sum of the earlier experts' row counts, each rounded up
// to 128, padded with zero codes; scale[(position / 128) * lds + c].
struct QuantColsArgs {
    int64_t M, T, ldx, ldq, lds;
    int32_t K, E;
    const void *x;
    const int32_t *rows;
    const int32_t *offsets;
    uint8_t *q;
    float *scale;
    uint8_t *row_q;
    float *row_scale;
    int64_t row_ldq, row_lds;
};
cudaError_t launch_quant_cols(esp_moe *m, int32_t dtype, const QuantColsArgs &a);
cudaError_t launch_quant_weight(esp_moe *m, int32_t dtype, const void *w, int64_t ldw, const esp_moe_weight &o);

// ---- esp_fp8_gemm.cu
// Grouped rows (forward and row gradient): out[i][n] for expert e's rows i, from A codes (M x lda), row
// scales (M x lds), B codes (expert e's rows at B + e * rows_b * ldb), block scales at scale_b + e * sb_e +
// (n / 128) * sb_n + kb * sb_k.
struct GemmRowsArgs {
    int64_t M, lda, lds, ldb, ldo;
    int32_t E, N, K;
    const uint8_t *A, *B;
    const float *scale_a, *scale_b;
    int64_t sb_e, sb_n, sb_k;
    const int32_t *offsets;
    void *out;
    float *partial;   // work space: gemm_partial_floats
};
cudaError_t launch_gemm_rows(esp_moe *m, int32_t dtype, const GemmRowsArgs &a);

// Grouped inner axis (weight gradient): out[e][n][k] fp32, from column codes of both operands
// (QuantColsArgs) with the experts' runs of positions.
struct GemmColsArgs {
    int64_t M, lda, ldb, lds_a, lds_b, ldo;
    int32_t E, N, K;
    const uint8_t *A, *B;   // A: N runs, B: K runs
    const float *scale_a, *scale_b;
    const int32_t *offsets;
    float *out;
    float *partial;
};
// Work space of a product whose tiles' inner axes are split over CTAs.
size_t gemm_partial_floats(const esp_moe *m);
cudaError_t launch_gemm_cols(esp_moe *m, const GemmColsArgs &a);

}  // namespace esp_moe_impl
