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
    float *partial;           // work space: few_partial_floats
    int chunk;                // rows of a tile (few_chunk), 0: tiles of many rows
    int64_t fp;               // elements of a row of a half of `pre` and `dpre`, and of `hidden`: F rounded up to 8
};

// ---- esp_ff_few.cu
int few_ctas(const esp_moe *m);
size_t few_partial_floats(const esp_moe *m, int chunk);
// kind, w, x, params: esp_ff.cuh's Kind, tensor maps of the weights and of the rows, FfParams.
cudaError_t launch_few(esp_moe *m, const FfShape &s, int kind, int chunk, const void *w, const void *x, const void *params);

// ---- esp_ff_gemm.cu
// Rows of a tile of a product over these rows: 0 (pairs of CTAs, 256 rows), or 16 to 128 (esp_ff_few.cu).
int few_chunk(const esp_moe *m, int64_t M, int32_t E);
// hidden (M x fp) = act(gate) * up; pre (M x 2 x fp fp32: gate, up) is written too where it is given.
cudaError_t launch_ff_hidden(esp_moe *m, const FfShape &s, const void *x, int64_t ldx, void *hidden, void *pre);
// y (M x H) = hidden O^T.
cudaError_t launch_ff_out(esp_moe *m, const FfShape &s, const void *hidden, void *y, int64_t ldy);
// dpre (M x 2 x fp) from dh = dy O and pre.
cudaError_t launch_ff_dpre(esp_moe *m, const FfShape &s, const void *dy, int64_t lddy, const void *pre, void *dpre);
// dx (M x H) = dpre [G; U].
cudaError_t launch_ff_dx(esp_moe *m, const FfShape &s, const void *dpre, void *dx, int64_t lddx);
// dinner (E x 2 F x H) = dpre^T x, douter (E x H x F) = dy^T hidden, in 32 bits or the rows' type.
cudaError_t launch_ff_dinner(esp_moe *m, const FfShape &s, const void *dpre, const void *x, int64_t ldx, void *dinner,
                             bool f32);
cudaError_t launch_ff_douter(esp_moe *m, const FfShape &s, const void *dy, int64_t lddy, const void *hidden, void *douter,
                             bool f32);

}  // namespace esp_moe_impl
