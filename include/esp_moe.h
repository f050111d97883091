/*
 * esp_moe.h - C ABI of the price-routed expert layer on one GB300 (sm_103a): the allocation problem of
 * esp.h inside a model. Tokens take experts as jobs take configurations: each token the k experts of
 * greatest value (logit) minus shadow price, the demands summed per expert as integers, the prices
 * stepped by excess demand (Eq. price_update of the paper); the chosen experts' products then run on
 * the tensor cores in 8-bit floating point.
 *
 *   esp_moe_route            choice at prices, gate weights, demand per expert, rows sorted by expert
 *   esp_moe_balance          balance and logit losses of a routing, per sequence
 *   esp_moe_route_backward   gradient of the logits from the gate weights, the losses, or both
 *   esp_moe_step_prices      one price update from the demand
 *   esp_moe_quantize_weight  weights as 8-bit codes with one scale per block of 128 x 128
 *   esp_moe_linear           rows (gathered by expert) times those weights
 *   esp_moe_linear_backward  gradients of the rows and of the weights
 *   esp_moe_combine          the experts' rows, weighted and summed back into their tokens
 *   esp_moe_combine_backward gradients of the rows and of the gate weights
 *
 * Conventions are those of esp.h: every function returns an esp_status and no exception crosses the
 * boundary; every data pointer here is a CUDA device pointer on the handle's device, owned by the
 * caller; a handle is used by one host thread at a time and all its work runs on its stream, queued
 * without waiting. Work space belongs to the handle and grows when a call needs more than any
 * earlier one (ESP_ERR_OOM if there is none; growing waits for the handle's stream, except in a
 * call that is being captured into a CUDA graph). Work space that captured calls use lives as long
 * as the handle, also where later calls outgrow it: a graph may be replayed until the handle is
 * destroyed. Logits, rows and weights are fp32, bf16 or fp16 (esp_moe_dtype) with any alignment of
 * their elements' size; a leading dimension ("ld") counts elements between rows and is at least the
 * row's length. Sums, softmax statistics and products accumulate in fp32; results in a 16-bit type
 * are rounded once. Zero tokens or rows do nothing beyond writing empty counts, offsets, losses and
 * gradients. Results are the same from run to run (no floating-point atomics).
 */
#ifndef ESP_MOE_H
#define ESP_MOE_H

#include <stdint.h>

#include "esp.h"

#ifdef __cplusplus
extern "C" {
#endif

#define ESP_MOE_MAX_EXPERTS 1024
#define ESP_MOE_MAX_CHOICES 32
#define ESP_MOE_MAX_SEQUENCES 65536
#define ESP_MOE_BLOCK 128 /* elements that share a scale along a row, and rows along a weight's column */

typedef struct esp_moe esp_moe;

typedef enum { ESP_MOE_F32 = 0, ESP_MOE_BF16 = 1, ESP_MOE_F16 = 2 } esp_moe_dtype;
typedef enum { ESP_MOE_SOFTMAX = 0, ESP_MOE_SIGMOID = 1 } esp_moe_gate_kind;

/* Gate weight of a chosen expert, from the logits z of its token:
 *   renorm != 0: scale * softmax over the chosen experts of a, a = z (SOFTMAX) or log sigmoid(z)
 *                (SIGMOID: the sigmoids divided by their sum);
 *   renorm == 0: scale * softmax(z) over all experts, or scale * sigmoid(z). */
typedef struct {
    int32_t kind;   /* esp_moe_gate_kind */
    int32_t renorm;
    float scale;    /* finite */
} esp_moe_gate;

/* 8-bit weights of E experts, each N x K (row-major, y = x W^T): codes are e4m3, element (e, n, k) at
 * q[(e * N + n) * ld + k] stands for code * scale[(e * ceil(N/128) + n / 128) * ceil(K/128) + k / 128].
 * qt holds the transposed codes, element (e, k, n) at qt[(e * K + k) * ldt + n]; it is needed by
 * esp_moe_linear_backward for the rows' gradient and may be NULL otherwise. q and qt are 16-byte
 * aligned, ld and ldt multiples of 16; bytes between a row's end and the next row are not read. */
typedef struct {
    int32_t E, N, K;
    int64_t ld, ldt;
    uint8_t *q;
    uint8_t *qt;
    float *scale;
} esp_moe_weight;

/* Creates a handle on `device` (-1: the current device) whose work runs on `cuda_stream` (NULL: the
 * legacy default stream). Errors: ESP_ERR_INVALID_ARG, ESP_ERR_UNSUPPORTED (no GPU, or not sm_103),
 * ESP_ERR_OOM, ESP_ERR_CUDA. */
esp_status esp_moe_create(esp_moe **out, int device, void *cuda_stream);

/* Later calls run on `cuda_stream`, after what the handle queued on the streams before (the one it
 * leaves must still exist). Captured calls have no part in that order: the program orders a graph's
 * launches, and the branches inside one, with the handle's other work, as they share its work space.
 * Errors: ESP_ERR_STATE, with the handle and its stream as they were, where the order cannot be had: the
 * stream it leaves is being captured and took the handle's work before its capture began (a call on a
 * stream whose own capture has ended is refused likewise while that one's runs). */
esp_status esp_moe_set_stream(esp_moe *m, void *cuda_stream);

/* Routes T tokens over E experts (logits T x E). An expert can be chosen if profit = logit - price
 * (one fp32 subtraction; prices NULL: 0) is neither NaN nor -inf. Each token with valid[t] != 0
 * (valid NULL: all) takes the k experts of greatest profit in descending order, ties to the lower
 * index; missing choices have idx -1 and weight 0. A gate reads a +inf logit as the largest finite
 * value and a NaN as -inf.
 *   idx     T x k int32            weight  T x k fp32
 *   counts  E int64: tokens that took each expert
 *   rows, pos, offsets: NULL all three, or the plan of the rows sorted by expert, within an expert by
 *   token: offsets (E + 1, int32) are the experts' first rows, rows (T * k, int32) the token of each
 *   row (-1 past offsets[E]), pos (T x k, int32) the row of each choice (-1 where idx is).
 * Errors: ESP_ERR_INVALID_ARG (1 <= E <= 1024, 1 <= k <= min(32, E), 0 <= T, T * k < 2^31). */
esp_status esp_moe_route(esp_moe *m, const esp_moe_gate *gate, int32_t dtype, int64_t T, int32_t E, int32_t k,
                         int64_t ld, const void *logits, const float *prices, const uint8_t *valid, int32_t *idx,
                         float *weight, int64_t *counts, int32_t *rows, int32_t *pos, int32_t *offsets);

/* Losses of a routing over B sequences (seq_offsets: B + 1 int32, ascending, sequence b holds the
 * tokens [seq_offsets[b], seq_offsets[b + 1]); NULL: one sequence of all T tokens, B = 1). Tokens with
 * idx[t][0] < 0 do not count. With r = softmax(a) over all experts (a as in esp_moe_gate), n_b the
 * counted tokens of sequence b and B' the sequences with n_b > 0:
 *   counts  B x E int64: choices of each expert     tokens  B int64: n_b
 *   share   B x E fp32: mean of r
 *   loss    2 fp32: loss[0] = 1/B' sum_b E sum_e counts / (k n_b) * share,
 *           loss[1] = mean over counted tokens of (log sum_e exp z_e)^2; both 0 without tokens. */
esp_status esp_moe_balance(esp_moe *m, const esp_moe_gate *gate, int32_t dtype, int64_t T, int32_t E, int32_t k,
                           int64_t ld, const void *logits, const int32_t *idx, int32_t B, const int32_t *seq_offsets,
                           float *loss, int64_t *counts, float *share, int64_t *tokens);

/* Gradient of the logits (T x E with leading dimension ld_out, written in full, in the logits' type):
 *   dweight  T x k fp32 or NULL: gradient of the gate weights of esp_moe_route;
 *   dloss    2 fp32 or NULL: gradients of esp_moe_balance's losses, with its counts and tokens for the
 *            same B and seq_offsets (the choice itself and the counts are constants).
 * Both given: the sum. Tokens with idx[t][0] < 0 have gradient 0. */
esp_status esp_moe_route_backward(esp_moe *m, const esp_moe_gate *gate, int32_t dtype, int64_t T, int32_t E, int32_t k,
                                  int64_t ld, const void *logits, const int32_t *idx, const float *dweight, int32_t B,
                                  const int32_t *seq_offsets, const int64_t *counts, const int64_t *tokens,
                                  const float *dloss, int64_t ld_out, void *dlogits);

/* prices[e] = max(0, prices[e] + eta * (counts[e] - C) / C), C = slack * sum(counts) / E: Eq. price_update
 * in capacity fractions (ESP_PRICE_NORMALIZED) for experts of equal capacity, in fp64, rounded to fp32.
 * Without counted tokens the prices stay. Errors: ESP_ERR_INVALID_ARG (eta, slack > 0 and finite). */
esp_status esp_moe_step_prices(esp_moe *m, int32_t E, const int64_t *counts, double eta, double slack, float *prices);

/* Codes and scales of w (E x N x K, rows ldw apart, experts N rows apart) into `out` (its E, N, K, ld,
 * ldt and buffers given). For each block: a = max(max |x|, 2^-100), scale = a / 448, code =
 * e4m3(x * (448 / a)), each step rounded to nearest in fp32; a block holding a value that is not
 * finite has scale NaN. */
esp_status esp_moe_quantize_weight(esp_moe *m, int32_t dtype, const void *w, int64_t ldw, const esp_moe_weight *out);

/* y[i] = x[rows[i]] W_e^T for the rows i in [offsets[e], offsets[e + 1]) of expert e; rows NULL: x[i],
 * and then M = T. offsets (E + 1 int32, ascending, at most M) may be NULL for E = 1: all M rows. The
 * rows of x are rounded to e4m3 codes with one scale for each 128 of a row (as esp_moe_quantize_weight
 * does); the products of a block are summed in fp32, then scaled and added. x (T x K) and y (M x N)
 * have type dtype; rows outside every expert are not written; a row index outside [0, T) reads zeros.
 * Offsets that do not ascend leave the rows of y undefined, and touch nothing else.
 * Errors: ESP_ERR_INVALID_ARG (M, T <= 2^31 - 256, at most 2^29 blocks of 128 x 128 in y, the weights or
 * their gradients, 16-byte rules of esp_moe_weight). */
esp_status esp_moe_linear(esp_moe *m, int32_t dtype, int64_t T, int64_t ldx, const void *x, int64_t M,
                          const int32_t *rows, const esp_moe_weight *w, const int32_t *offsets, int64_t ldy, void *y);

/* Gradients of esp_moe_linear at dy (M x N): dx (M x K in dtype, or NULL) = Q(dy) W_e for each row of an
 * expert, with dy rounded in blocks of 128 along a row; dw (E x N x K fp32, rows lddw apart, or NULL) =
 * sum over expert e's rows of Q'(dy) Q'(x), both rounded in blocks of 128 consecutive rows of the
 * expert. An expert without rows has dw 0. Gradients of a gathered token's rows are separate rows of dx
 * (esp_moe_combine with weights NULL sums them). */
esp_status esp_moe_linear_backward(esp_moe *m, int32_t dtype, int64_t T, int64_t ldx, const void *x, int64_t M,
                                   const int32_t *rows, const esp_moe_weight *w, const int32_t *offsets, int64_t lddy,
                                   const void *dy, int64_t lddx, void *dx, int64_t lddw, float *dw);

/* out[t] = sum_j weight[t][j] * y[pos[t][j]] over the choices with pos in [0, M) (weight NULL: 1), for T
 * tokens and rows of H elements: y M x H, out T x H in dtype. */
esp_status esp_moe_combine(esp_moe *m, int32_t dtype, int64_t T, int32_t k, int32_t H, int64_t M, int64_t ldy,
                           const void *y, const int32_t *pos, const float *weight, int64_t ldo, void *out);

/* Gradients of esp_moe_combine at dout (T x H): dy[pos[t][j]] = weight[t][j] * dout[t] (rows that no pos
 * names are not written; a row named twice holds one of its gradients), dweight[t][j] =
 * <dout[t], y[pos[t][j]]> (0 where there is no row). dy or dweight may be NULL; y is read for dweight. */
esp_status esp_moe_combine_backward(esp_moe *m, int32_t dtype, int64_t T, int32_t k, int32_t H, int64_t M, int64_t lddo,
                                    const void *dout, int64_t ldy, const void *y, const int32_t *pos,
                                    const float *weight, int64_t lddy, void *dy, float *dweight);

/* Waits for the handle's work on all streams (not for graphs that the program launches: it waits
 * for those itself first) and reports a device-side failure of the queued work: ESP_ERR_TIMEOUT
 * when a bounded wait of a product kernel gave up (its results are then undefined and the handle
 * refuses further work with ESP_ERR_STATE; any other call that finds such a failure reports it
 * instead), ESP_ERR_CUDA on a CUDA error, ESP_ERR_STATE while the handle's stream is being captured
 * (the handle stays usable). */
esp_status esp_moe_synchronize(esp_moe *m);

/* Kernel launches of the handle's last call. */
esp_status esp_moe_last_launch_count(esp_moe *m, int64_t *out);

/* Failure detection without a GPU fault (tests): the waits of later products give up after about
 * limit_ms milliseconds (0: the default, about 4 s), and the next product launch leaves out one load, so
 * that its waits run out and esp_moe_synchronize reports ESP_ERR_TIMEOUT. */
esp_status esp_moe_debug_set_wait_limit(esp_moe *m, uint32_t limit_ms);
esp_status esp_moe_debug_hold_load(esp_moe *m);

void esp_moe_destroy(esp_moe *m);

#ifdef __cplusplus
}
#endif

#endif /* ESP_MOE_H */
