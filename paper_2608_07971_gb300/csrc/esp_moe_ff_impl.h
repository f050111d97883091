// Launchers of the gated feed-forward blocks (include/esp_moe.h: esp_moe_feed_forward and its gradients).
#pragma once

#include "esp_moe_impl.h"

namespace esp_moe_impl {

constexpr int kInner = 64;   // elements of the inner axis in one 128-byte row of a shared-memory tile

// Rows of 16-bit elements copied to where tensor maps can read them: row i from x[rows[i]] (rows NULL: x[i]), zeros for
// an index outside [0, T).
struct CopyRowsArgs {
    int64_t M, T, ldx, ldo;
    int32_t H;
    const void *x;
    const int32_t *rows;
    void *out;
};
cudaError_t launch_copy_rows(esp_moe *m, const CopyRowsArgs &a);

// The blocks' shapes, weights (esp_moe_gated) and rows.
struct FfShape {
    int32_t dtype, act, E, F, H;
    int64_t M;
    const int32_t *offsets;
    const void *inner, *outer;
    int64_t ld_inner, ld_outer;
    int64_t hp;               // of the rows of x and dy in the tails: H rounded up to 64
    float *partial;           // work space: ff_partial_floats
    int64_t fp;               // elements of a row of a half of `pre` and `dpre`, and of `hidden`: F rounded up to 64
    float *lengths;           // work space of hidden rows that are kept for relu's slope: M + E F
};

// ---- esp_ff_vec.cu
// Whether a forward pass is for the CUDA cores: one dense block, a few rows.
bool use_vec(int64_t M, int32_t E, int32_t F, int32_t H);
// Both products of such a pass: hidden (M x fp), pre where it is given, y. Rows are gathered here.
cudaError_t launch_vec(esp_moe *m, const FfShape &s, const void *x, int64_t ldx, int64_t T, const int32_t *rows, void *hidden,
                       void *pre, void *y, int64_t ldy);

// ---- esp_ff_gemm.cu
// Work space of a product whose tiles' inner axes are split over CTAs.
size_t ff_partial_floats(const esp_moe *m);
// hidden (M x fp) = act(gate) * up; pre (M x 2 x fp fp32: gate, up) is written too where it is given (relu: two launches).
cudaError_t launch_ff_hidden(esp_moe *m, const FfShape &s, const void *x, int64_t ldx, void *hidden, void *pre);
// y (M x H) = hidden O^T.
cudaError_t launch_ff_out(esp_moe *m, const FfShape &s, const void *hidden, void *y, int64_t ldy);
// dpre (M x 2 x fp) from dh = dy O and pre.
cudaError_t launch_ff_dpre(esp_moe *m, const FfShape &s, const void *dy, int64_t lddy, const void *pre, void *dpre);
// dx (M x H) = dpre [G; U].
cudaError_t launch_ff_dx(esp_moe *m, const FfShape &s, const void *dpre, void *dx, int64_t lddx);
// The last rows of each expert that do not fill a block of 64, copied to 64 rows of their own (row 64 e on), zeros behind
// them. Needed where rows of another expert, or of none, may follow in memory.
struct TailArgs {
    struct Part {
        const void *x;      // rows of 16-bit elements, a multiple of 16 bytes apart
        void *out;          // 64 E rows of ld_out
        int64_t ldx, ld_out;
        int32_t width;
    } part[4];
    int32_t parts, M;
    const int32_t *offsets;
};
cudaError_t launch_tails(esp_moe *m, const TailArgs &a, int32_t E);
// dinner (E x 2 F x H) = dpre^T x and douter (E x H x F) = dy^T hidden, either NULL, in one launch; in 32 bits or the rows'
// type. Without tails rows end with M.
struct FfWeightArgs {
    const void *dpre, *x, *dy, *hidden;
    int64_t ldx, lddy;
    const void *dpre_tails, *x_tails, *dy_tails, *hidden_tails;
    bool tails, f32;
    void *dinner, *douter;
};
cudaError_t launch_ff_weights(esp_moe *m, const FfShape &s, const FfWeightArgs &a);

}  // namespace esp_moe_impl
