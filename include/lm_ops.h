/*
 * lm_ops -- operators of language models around the integer cells, for AMD
 * MI355X (gfx950), in liblstm_int.so: what a layer runs before, behind and
 * instead of a recurrent cell when a model is served in low precision.
 *
 *   rms_norm    root-mean-square norm with the residual's addition, into int8
 *               codes with a scale of each row or at a fixed scale and zero
 *               point (the codes lstm_int_forward, gru_int_forward and
 *               sru_int_forward read), and in floating point
 *   w4_linear   products with 4-bit weights and a scale per group of inputs,
 *               on int8 activations: those of rms_norm, or a cell's output
 *   delta_rule  the gated delta rule, a recurrent cell whose state is a matrix
 *               per head: whole sequences and single steps
 *
 * Error codes are those of lstm_int.h.  Every function returns 0 or a negative
 * code, and no exception crosses this boundary.  `device` is the HIP device
 * that the pointers belong to; the calling thread's current device is left as
 * it was.  The online calls allocate nothing, never synchronize the host and
 * launch kernels only, so that a caller may capture them in a HIP graph once one
 * such call has run outside a capture; a call that returns an error has enqueued
 * nothing that writes beyond its workspace.  Calls share no memory but what the
 * caller passes, so calls with different outputs (and workspaces) may overlap.
 * Unless it says "may be", an output overlaps no other argument.
 * There are no gradients: the library runs trained models.
 */
#ifndef LM_OPS_H
#define LM_OPS_H

#include <stddef.h>
#include <stdint.h>

#include "lstm_int.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Types of floating point tensors */
#define LM_F32 0
#define LM_F16 1
#define LM_BF16 2

/*
 * Root-mean-square norm of `rows` rows of `cols` columns, in groups of
 * D = cols / groups columns each (groups = 1: over the row; groups = the
 * number of heads: over each head's columns):
 *   r = x + residual                              (x alone without a residual)
 *   n = r / sqrt(mean_group(r^2) + eps) * weight [* gate * sigma(gate)]
 * and of n, for codes != NULL,
 *   scale = 0:  s = max_row |n| / 127 into scales (float32 [rows]), codes
 *               floor(n / s + 1/2); a row of zeros has s = 0 and codes 0
 *   scale > 0:  codes clamp(floor(n / scale + 1/2) + zero_point, -128, 127),
 *               lstm_int_quantize_input's rule; `scales` is not used
 * Evaluated in double precision: a code never depends on a rounding before it.
 * A row with a NaN or an infinity in r, or in n, has NaN as its scale and code
 * 0 throughout; at a fixed scale every NaN of n has code 0.
 *   x, residual, gate  DEVICE, of type dtype, rows x_stride, residual_stride
 *                      and gate_stride elements apart; any alignment of rows;
 *                      residual and gate may be NULL
 *   weight             DEVICE float32 [D], shared by the groups
 *   codes              DEVICE int8 [rows, cols], dense; may be NULL
 *   y                  DEVICE dtype [rows, cols], dense: n, rounded; may be NULL
 *   new_residual       DEVICE dtype, rows new_residual_stride apart: r, rounded;
 *                      may be NULL (the sum need not be kept); may be x or
 *                      residual itself, at its own stride
 * LSTM_INT_E_INVALID_ARG: a negative extent, cols no multiple of groups, a
 * stride below cols with rows > 1, an unknown dtype, x or weight NULL, neither codes nor
 * y, codes with scale = 0 and no scales, new_residual without a residual, a
 * zero point beyond -128..127.  LSTM_INT_E_BAD_RANGE: eps not positive and
 * finite, scale negative, NaN or infinite.  LSTM_INT_E_UNSUPPORTED: cols
 * beyond 32768; with groups > 1, cols beyond 8192 or D outside 8..2048; rows
 * beyond 2^31 - 1.  rows = 0 or cols = 0 is a no-op.
 */
typedef struct {
  int64_t rows;
  int32_t cols, groups;
  int32_t dtype;
  int32_t zero_point;
  double eps;
  double scale;
  int64_t x_stride, residual_stride, gate_stride, new_residual_stride;
} rms_norm_args;
int rms_norm_forward(int32_t device, const rms_norm_args *args, const void *x, const void *residual,
                     const void *gate, const float *weight, int8_t *codes, float *scales, void *y,
                     void *new_residual, void *hip_stream);

/*
 * Products with 4-bit weights:
 *   y[m, n] = a[m] sum_g s[n, g] sum_{k in group g} (x[m, k] - zero_point) w[n, k] + bias[n]
 * w: codes -8..7; s: a float32 scale for each output and group of group_size
 * consecutive inputs (the last group of K inputs may be shorter); x: int8.  The
 * sum over a group is an exact integer, also with a zero point; groups are
 * added in float32, in an order that depends on the sizes alone.
 */
typedef struct w4_linear_model w4_linear_model;

/* Every pointer is HOST memory, caller-owned, and may be freed once
 * w4_linear_prepare returns.  Either W, or codes and scales. */
typedef struct {
  int32_t inputs, outputs; /* K, N */
  int32_t group_size;      /* 32, 64 or 128 */
  const float *W;          /* [N, K]; quantized here: s = max_group |W| / 7, codes
                              round(W / s), halves away from zero */
  const int8_t *codes;     /* [N, K], -8..7 */
  const float *scales;     /* [N, ceil(K / group_size)] */
  const float *bias;       /* [N]; may be NULL */
} w4_linear_params;

/* Offline phase: lays the weights out for the kernels and uploads them to
 * `device` (-1: a host-only model, for w4_linear_get_quant).
 * LSTM_INT_E_INVALID_ARG: a missing or surplus tensor, a code out of range, K or
 * N < 1, another group size.  LSTM_INT_E_BAD_RANGE: NaN or infinity among the
 * weights, scales or biases.  LSTM_INT_E_UNSUPPORTED: K beyond 2^17, N beyond 2^24. */
int w4_linear_prepare(const w4_linear_params *params, int32_t device, w4_linear_model **out);

/* Host views, valid until the model is destroyed. */
typedef struct {
  int32_t inputs, outputs, group_size, groups;
  const int8_t *codes;  /* [N, K] */
  const float *scales;  /* [N, groups] */
} w4_linear_quant;
int w4_linear_get_quant(const w4_linear_model *model, w4_linear_quant *out);

/*
 *   x           DEVICE int8, `rows` rows of K codes, x_stride elements apart,
 *               any alignment
 *   row_scales  DEVICE float32 [rows]: a[m]; NULL: a[m] = scale for every row
 *   zero_point  -128..127 (0 for activations that have none)
 *   y           DEVICE dtype, rows y_stride elements apart; columns N and
 *               beyond of a row are left as they are
 * A row that has NaN or an infinity as its scale gives what the formula gives.
 * LSTM_INT_E_INVALID_ARG: NULL, rows < 0, a stride below the row's length with
 * rows > 1, a zero point out of range, an unknown dtype.  LSTM_INT_E_DEVICE: a
 * host-only model.  LSTM_INT_E_UNSUPPORTED: rows beyond 2^24, and more than
 * one launch holds (rows x N beyond some 2^36).  rows = 0 is a no-op.
 */
int w4_linear_forward(const w4_linear_model *model, const int8_t *x, int64_t x_stride, int64_t rows,
                      const float *row_scales, float scale, int32_t zero_point, void *y,
                      int64_t y_stride, int32_t dtype, void *hip_stream);
void w4_linear_destroy(w4_linear_model *model);

/*
 * The gated delta rule.  Per value head a state S [key_dim, value_dim]; per step
 *   S <- e^g S;  u = beta (v - S' k);  S <- S + k u';  y = scale S' q
 * (' is the transpose; g the log of the decay, beta the rate of writing).  Key
 * head h serves the value heads h * value_heads / key_heads and the ones behind
 * it.  normalize = 1: k and q are first divided by sqrt(sum of squares + 1e-6).
 * Sums and the state are float32.  Calls of 12 steps and more run 32 steps at a
 * time on the matrix cores, with float32 operands in two scaled parts of fp16:
 * 22 bits of each element, and of one far below the largest 2^-39 of that
 * largest, of a column of the state 2^-30 and of a key 2^-27.  The largest is
 * over a key or query, over a state's column (one value column, all key
 * columns) and, for the values, over a column's 32 steps, so that a value 2^17
 * times as large as its neighbours costs their outputs bits, those of earlier
 * steps among them.  Shorter calls run step by step in float32.  What overflows
 * float32 gives infinities and NaN: sums of squares of k and q, with normalize
 * too (elements beyond 2^60), S' k and S' q before the decay, and results.
 *   q, k    DEVICE dtype [T, B, key_heads, key_dim]
 *   v, y    DEVICE dtype [T, B, value_heads, value_dim]
 *   g, beta DEVICE float32 [T, B, value_heads]
 *           each with strides, in elements, of step, batch row and head, that
 *           may be anything for the inputs (a slice of a projection's output);
 *           the last dimension of q, k, v, y is dense.
 *           g = -infinity clears the state (of finite numbers); a sum of g over
 *           32 steps stays below 80 (a decay has none above 0).
 *   lengths DEVICE int32 [B]: row b has min(max(lengths[b], 0), T) steps; inputs
 *           behind them are not used and outputs there left as they are;
 *           NULL: every row has T
 *   state, new_state  DEVICE float32 [B, value_heads, key_dim, value_dim], dense: the state
 *           before step 0 (NULL: zeros) and after a row's last step (NULL: not
 *           kept); may be the same
 *   workspace DEVICE, >= delta_rule_workspace_bytes, 256-byte aligned (may be
 *           NULL if that is 0)
 * A NaN or an infinity at one step can reach the outputs of its row and head at
 * the steps before it within the same 32; nothing reaches another row or head.
 * T = 0 copies the state; B = 0 is a no-op.
 * LSTM_INT_E_INVALID_ARG: NULL, a negative extent, value_heads no multiple of
 * key_heads, an unknown dtype, a normalize other than 0 and 1, a stride of y
 * below value_dim (either way) in a dimension of more than one.
 * LSTM_INT_E_BAD_RANGE: a scale that is not finite.
 * LSTM_INT_E_UNSUPPORTED: key_dim or value_dim beyond 256; B * value_heads
 * beyond 2^20; T beyond 2^24.  LSTM_INT_E_WORKSPACE.
 */
typedef struct {
  int32_t steps, batch, key_heads, value_heads, key_dim, value_dim;
  int32_t dtype;
  int32_t normalize;
  double scale;
  int64_t q_stride[3], k_stride[3], v_stride[3], y_stride[3], g_stride[3], beta_stride[3];
} delta_rule_args;
size_t delta_rule_workspace_bytes(const delta_rule_args *args);
int delta_rule_forward(int32_t device, const delta_rule_args *args, const void *q, const void *k,
                       const void *v, const float *g, const float *beta, const int32_t *lengths,
                       const float *state, float *new_state, void *y, void *workspace,
                       size_t workspace_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif
