/*
 * sparse_block.h -- C ABI of the transformer-block operators over kept rows (same library as sparse_conv.h).
 *
 * A row is a token (or a position of a feature map) with all its channels; a mask keeps some rows and drops the others, as it
 * does in the masked convolutions.  The operators are those of the feed-forward half of a block:
 *
 *   sparse_rows_*   the kept rows of a token mask: ascending row list and the slot of every row in it
 *   sparse_norm_*   norm behind a block, its gate, the residual sum and the norm before the next block in one pass; gradients
 *   sparse_ffn_*    gated feed-forward block y = (act(x Wg') * (x Wu')) Wd'; gradients
 *   sparse_q4_*     products with weights in 4 bits with a scale and a zero point per group, for serving a few rows at a time
 *
 * Conventions (those of sparse_conv.h)
 *   - a mask byte != 0 keeps the row; a dropped row of a dense output holds +0.0 in every channel;
 *   - tensors are contiguous, row by row; *_dev is device memory of the caller, aligned to 16 bytes; the library allocates none;
 *   - sums, norm statistics and gradients of parameters are accumulated in float; every result is rounded once to its type, and
 *     so are the operands of the feed-forward block's second products (hidden rows, and the gradients of g and u);
 *   - results do not depend on the order in which workgroups run: the same call gives the same bits;
 *   - status codes; argument checks come before the first HIP call; *_run and *_backward only enqueue work on hip_stream;
 *   - outputs must not overlap inputs, except where noted;
 *   - no rows (or a mask that keeps none) is a valid call: gradients of parameters are then zero.
 */
#ifndef SPARSE_BLOCK_H_
#define SPARSE_BLOCK_H_

#include "sparse_conv.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- kept rows of a mask ---------------------------------------------------------------------------------------------------
 * sparse_rows_plan builds the list in the caller's workspace and synchronises the stream once (the count is needed on the host).
 * sparse_rows_set_mask does the same again for a new mask of as many rows; if it fails, the set keeps no row from then on.
 * rows <= 2^31 - 1; 0 is allowed. */
typedef struct sc_rows sc_rows;

sc_status sparse_rows_workspace_bytes(int64_t rows, size_t* bytes);
sc_status sparse_rows_plan(const uint8_t* mask_dev, int64_t rows, void* workspace_dev, size_t workspace_bytes, void* hip_stream,
                           sc_rows** out);
sc_status sparse_rows_set_mask(sc_rows* set, const uint8_t* mask_dev, void* hip_stream);
/* row_idx_dev: int32[kept], ascending; slot_dev: int32[rows], position in row_idx or -1.  Any of the outputs may be NULL. */
sc_status sparse_rows_info(const sc_rows* set, int64_t* rows, int64_t* kept, const int32_t** row_idx_dev, const int32_t** slot_dev);
void sparse_rows_destroy(sc_rows* set);

/* ---- norms around a block, gate and residual ---------------------------------------------------------------------------------
 *   n     = post(f) * w_post + b_post
 *   x_new = residual_scale * x + branch_scale * gate[row / rows_per_gate] * n      (rows of f_rows; else residual_scale * x)
 *   h     = pre(x_new) * w_pre + b_pre                                             (rows of h_rows)
 * post and pre are RMS norms v / sqrt(mean(v^2) + eps), layer norms, or nothing.  Weights and biases are float[d], may be NULL.
 * f holds the kept rows of f_rows as a [kept x d] matrix, h those of h_rows; NULL stands for all rows.  f may be NULL (no branch:
 * x_new = residual_scale * x), gate may be NULL (1).  x_new or h may be NULL where it is not wanted; x_new may be x itself.
 * pre(x_new) sees the sum in float, before x_new is rounded.  gate has ceil(rows / rows_per_gate) rows of d; rows_per_gate = 0
 * stands for "one row for all".
 * stats_dev: float[rows][4], mean and 1/spread of f's row and of x_new's row; written by run where it is not NULL (a mean is 0
 * for an RMS norm), read by backward. */
typedef enum { SC_NORM_NONE = 0, SC_NORM_RMS = 1, SC_NORM_LAYER = 2 } sc_norm_kind;

typedef struct {
  int32_t d;             /* channels, 1 .. 8192 */
  int32_t dtype;         /* sc_dtype of x, f, gate, x_new, h and of their gradients */
  int32_t post, pre;     /* sc_norm_kind */
  float eps;             /* >= 0 */
  float residual_scale, branch_scale;
  int32_t rows_per_gate; /* >= 0 */
} sc_norm_desc;

sc_status sparse_norm_run(const sc_norm_desc* desc, int64_t rows, const void* x_dev, const void* f_dev, const sc_rows* f_rows,
                          const void* gate_dev, const float* w_post_dev, const float* b_post_dev, const float* w_pre_dev,
                          const float* b_pre_dev, void* x_new_dev, void* h_dev, const sc_rows* h_rows, float* stats_dev,
                          void* hip_stream);

/* Gradients of the above.  dx_new: gradient that reaches x_new from elsewhere (NULL: none); dh: gradient of h (NULL: h was not
 * used).  x, f, gate and the parameters are those of the run, stats its statistics.  Gradients that are not wanted are NULL;
 * df and the post parameters' need f, dgate needs gate, the pre parameters' need dh.  Gradients of parameters are float[d], that
 * of the gate has the gate's shape and type.  dx may be dx_new itself. */
sc_status sparse_norm_workspace_bytes(const sc_norm_desc* desc, int64_t rows, size_t* bytes);
sc_status sparse_norm_backward(const sc_norm_desc* desc, int64_t rows, const void* x_dev, const void* f_dev, const sc_rows* f_rows,
                               const void* gate_dev, const float* w_post_dev, const float* b_post_dev, const float* w_pre_dev,
                               const float* stats_dev, const void* dx_new_dev, const void* dh_dev, const sc_rows* h_rows,
                               void* dx_dev, void* df_dev, void* dgate_dev, float* dw_post_dev, float* db_post_dev,
                               float* dw_pre_dev, float* db_pre_dev, void* workspace_dev, size_t workspace_bytes,
                               void* hip_stream);

/* ---- gated feed-forward block --------------------------------------------------------------------------------------------------
 *   g = x Wg', u = x Wu', hidden = act(g) * u, y = hidden Wd'       over the kept rows
 * w_gate and w_up are [d_hidden x d_in], w_down is [d_out x d_hidden], all of the descriptor's type and used where they lie.
 * rows (sc_rows, may be NULL: all `m` rows are kept) says which rows of x count; m is the number of rows of the mask.  With
 * x_rows = SC_ROWS_DENSE x (and dx) is [m x d_in], with SC_ROWS_COMPACT [kept x d_in]; y_rows says the same of y (and dy).
 * Dropped rows of a dense x or dy are not looked at, whatever they hold.
 * saved_dev: [3][kept][d_hidden] of the descriptor's type for the backward pass, as sparse_ffn_run leaves it: g and u in floats, or in
 * 24 bits each of 16-bit types.  NULL in inference.
 * Sizes need not be multiples of anything; rows of whole 16-byte groups are the fast path, others are copied into the
 * workspace first, in a run with more than 64 kept rows and in every backward pass.
 * SC_F16: hidden rows and gradients of g and u beyond 65 504 are infinite, although y and dx need not be (their row is lost then, and
 * no other).
 * Floats of up to 8 kept rows in a run are multiplied as they are.  Those of more than 64, and of every backward pass, are multiplied in
 * three 16-bit parts, others in either way: a float's precision, but a factor loses what of it lies below 2^-126, and an infinity
 * gives NaN. */
typedef enum { SC_ACT_SILU = 0, SC_ACT_GELU = 1, SC_ACT_GELU_TANH = 2 } sc_activation;

typedef struct {
  int32_t d_in, d_hidden, d_out;
  int32_t dtype;         /* sc_dtype */
  int32_t activation;    /* sc_activation */
} sc_ffn_desc;

/* Bytes for calls with up to `kept` kept rows.  training = 0: sparse_ffn_run without saved_dev; 1: run with it, and backward. */
sc_status sparse_ffn_workspace_bytes(const sc_ffn_desc* desc, int64_t kept, int32_t training, size_t* bytes);
sc_status sparse_ffn_run(const sc_ffn_desc* desc, int64_t m, const sc_rows* rows, const void* x_dev, int32_t x_rows,
                         const void* w_gate_dev, const void* w_up_dev, const void* w_down_dev, void* y_dev, int32_t y_rows,
                         void* saved_dev, void* workspace_dev, size_t workspace_bytes, void* hip_stream);
/* dx has the format of x, dy that of y.  dx or all three weight gradients may be NULL. */
sc_status sparse_ffn_backward(const sc_ffn_desc* desc, int64_t m, const sc_rows* rows, const void* x_dev, int32_t x_rows,
                              const void* w_gate_dev, const void* w_up_dev, const void* w_down_dev, const void* saved_dev,
                              const void* dy_dev, int32_t y_rows, void* dx_dev, void* dw_gate_dev, void* dw_up_dev,
                              void* dw_down_dev, void* workspace_dev, size_t workspace_bytes, void* hip_stream);

/* ---- products with 4-bit weights -------------------------------------------------------------------------------------------------
 *   y[r][n] = sum_k x[r][k] * (code[n][k] - zero[n][k / group]) * scale[n][k / group]
 * codes are [n][ceil(k / 2)] bytes, the even column in the low half; scales and zeros are [n][ceil(k / group)] of the
 * descriptor's type (zeros may be NULL: 8).  The plan lays the weights out once in the caller's workspace, from which every run
 * reads them; codes, scales and zeros are not needed afterwards.  sparse_q4_plan_gated lays out two matrices of one shape,
 * whose run gives act(x Gate') * (x Up'), rounded once (SC_F16: beyond 65 504 to an infinity).  Planning only enqueues work.
 * Up to 65 535 * 64 rows; made for few.  x is finite (a row that is not is lost, and no other), and in SC_BF16 below 2^110 in size: sums of x times up to 143 (SC_F16: 1 039) are formed in float on the way. */
typedef struct {
  int32_t k, n;          /* columns contracted, outputs */
  int32_t group;         /* 32, 64 or 128 columns share a scale */
  int32_t dtype;         /* SC_F16 or SC_BF16: x, y, scales and zeros */
} sc_q4_desc;

typedef struct sc_q4 sc_q4;

sc_status sparse_q4_workspace_bytes(const sc_q4_desc* desc, int32_t gated, size_t* bytes);
sc_status sparse_q4_plan(const sc_q4_desc* desc, const uint8_t* codes_dev, const void* scales_dev, const void* zeros_dev,
                         void* workspace_dev, size_t workspace_bytes, void* hip_stream, sc_q4** out);
sc_status sparse_q4_plan_gated(const sc_q4_desc* desc, int32_t activation, const uint8_t* gate_codes_dev,
                               const void* gate_scales_dev, const void* gate_zeros_dev, const uint8_t* up_codes_dev,
                               const void* up_scales_dev, const void* up_zeros_dev, void* workspace_dev, size_t workspace_bytes,
                               void* hip_stream, sc_q4** out);
sc_status sparse_q4_run(const sc_q4* plan, int64_t rows, const void* x_dev, void* y_dev, void* hip_stream);
void sparse_q4_destroy(sc_q4* plan);

#ifdef __cplusplus
}
#endif

#endif /* SPARSE_BLOCK_H_ */
