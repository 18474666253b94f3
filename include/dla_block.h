/*
 * dla_block.h -- C ABI of libdla for the parts of a model of the layer's base form that lie
 * around the recurrence, for training and for serving: the short causal convolution in
 * front of it, the norm with gate, residual sum and next norm behind it, the gated
 * feed-forward block, and the log probabilities of tokens that a loss or an answer is made
 * of.
 *
 * The conventions of dla.h and dla_train.h hold: plain pointers and sizes, every array
 * DEVICE memory owned by the caller, nothing allocated or kept, all work enqueued on
 * `stream`, argument errors returned before anything is enqueued.  Workspaces are 256-byte
 * aligned, hold nothing between calls, and must not be used by another call until the
 * stream has passed the one they were given to.  Every result is the same from call to
 * call: no sum's order depends on timing.  Outputs do not overlap inputs, or each other,
 * but where a call says that they may be the same array: the same address with the same
 * strides (the calls do not check it; the Python binding does).  Arrays need the alignment
 * of their type only; rows that start at multiples of 16 bytes are faster.
 */
#ifndef DLA_BLOCK_H
#define DLA_BLOCK_H

#include "dla_train.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * A causal convolution over the last W tokens, channel by channel, and the SiLU:
 *   z[b][t][c] = bias[c] + sum_{j < W} weight[c][j] x[b][t - (W - 1) + j][c]
 *   y = silu ? z / (1 + exp(-z)) : z
 * where x[b][-i], i = 1 .. W - 1, is state[b][W - 1 - i], the inputs before the call (zero
 * where no state is given).
 *
 * starts: NULL, or bytes [B][T], contiguous: where one is not zero a document starts, and
 * neither that token nor a later one sees an input before it, the state's among them.
 * lengths: NULL, or int32 [B]: sequence b ends after min(max(lengths[b], 0), T) tokens.
 * Nothing is read behind its end (whatever memory holds there, NaN included); outputs and
 * gradients there are zero.
 * The last state is what the next token would see: the W - 1 inputs before the sequence's
 * end, zero where a document started after them; it goes on from the given state where the
 * sequence is shorter.
 *
 * B, T, C >= 0 sequences, tokens and channels, T and C at most 2^30; W 2, 3 or 4.  dtype:
 * type of x, y, states and the gradients of these; weight_dtype (of weight and bias): that
 * type or DLA_F32.  Sums are float32 and rounded once when stored.  weight [C][W], bias [C] and
 * states [B][W - 1][C] are contiguous.  silu: 0 or 1.
 */
typedef struct {
  int32_t B, T, C, W;
  int32_t dtype, weight_dtype; /* dla_dtype */
  int32_t silu;
  const int32_t* lengths;
  const uint8_t* starts;
} dla_conv_desc;

/* Element (b, t, c) at data + b stride_b + t stride_t + c, strides in elements, not negative.
 * Inputs may repeat rows; output rows do not overlap. */
typedef struct {
  void* data;
  int64_t stride_b, stride_t;
} dla_conv_rows;

/* bias, state, state_out may be NULL; state_out may be state's array. */
dla_status dla_short_conv(const dla_conv_desc* desc, const dla_conv_rows* x, const void* weight,
                          const void* bias, const void* state, const dla_conv_rows* y,
                          void* state_out, void* stream);

/* Workspace of the backward pass (for dweight and dbias), in bytes. */
dla_status dla_short_conv_workspace_size(const dla_conv_desc* desc, size_t* bytes);

/* The backward pass, from the forward pass's inputs and the gradients of its outputs: dy, and
 * dstate_out or NULL for zero.  Writes dx, dweight float32 [C][W] and, where not NULL, dbias
 * float32 [C] and dstate, the gradient of the given state (not dstate_out's array). */
dla_status dla_short_conv_backward(const dla_conv_desc* desc, const dla_conv_rows* x,
                                   const void* weight, const void* bias, const void* state,
                                   const dla_conv_rows* dy, const void* dstate_out,
                                   const dla_conv_rows* dx, float* dweight, float* dbias,
                                   void* dstate, void* workspace, size_t workspace_bytes,
                                   void* stream);

/*
 * The norm behind a block with its gate, the scaled residual sum, and the norm before the
 * next block.  Per row, and in it per group of D values:
 *   r = 1 / sqrt(mean(x^2) + eps),  n = r x weight,  b = n gate / (1 + exp(-gate))
 *   h = residual + scale b
 *   r' = 1 / sqrt(mean(h^2) + eps),  y = r' h next_weight
 * gate NULL: b = n.  residual NULL: zero.  next_weight NULL: no r' and no y; otherwise
 * groups = 1.  Everything is computed in float32, y from the unrounded h, and rounded once
 * when it is stored.
 *
 * 0 <= rows <= 2^31 - 4, 1 <= groups <= 65535, 1 <= D <= 16384, groups D <= 2^26.  dtype: type
 * of x, gate, residual, h, y and their gradients; weight_dtype: that type or DLA_F32.  weight is
 * [D], shared by the groups, or with weight_per_group [groups][D]; next_weight [D].
 * eps >= 0, scale finite; as in dla_rms_norm r and r' are right for any finite rows, and zero
 * where the mean plus eps is below 2^-252.
 */
typedef struct {
  int64_t rows;
  int32_t groups, D;
  int32_t dtype, weight_dtype; /* dla_dtype */
  int32_t weight_per_group;
  float eps, scale;
} dla_gated_norm_desc;

/* Element (n, g, i) at data + n stride + g stride_g + i, strides in elements, not negative.
 * Inputs may repeat rows; output rows and groups do not overlap. */
typedef struct {
  void* data;
  int64_t stride, stride_g;
} dla_group_rows;

/* rstd [rows][groups] and y_rstd [rows] float32: r and r' for the backward pass, or NULL.  h may
 * be x's or the residual's array. */
dla_status dla_gated_norm(const dla_gated_norm_desc* desc, const dla_group_rows* x,
                          const dla_group_rows* gate, const dla_group_rows* residual,
                          const void* weight, const void* next_weight, const dla_group_rows* h,
                          const dla_group_rows* y, float* rstd, float* y_rstd, void* stream);

/* Workspace of the backward pass (for dweight and dnext_weight), in bytes. */
dla_status dla_gated_norm_workspace_size(const dla_gated_norm_desc* desc, size_t* bytes);

/* The backward pass, from the forward pass's inputs, its rstd and y_rstd, and the gradients dh of
 * h (NULL for zero) and dy of y (with next_weight; NULL for zero).  Writes dx and, where not
 * NULL, dgate, dresidual (the whole gradient of h), dweight float32 (as weight) and dnext_weight
 * float32 [D].  dx, dgate and dresidual may be the arrays of inputs of their shape, one each. */
dla_status dla_gated_norm_backward(const dla_gated_norm_desc* desc, const dla_group_rows* x,
                                   const dla_group_rows* gate, const dla_group_rows* residual,
                                   const void* weight, const void* next_weight, const float* rstd,
                                   const float* y_rstd, const dla_group_rows* dh,
                                   const dla_group_rows* dy, const dla_group_rows* dx,
                                   const dla_group_rows* dgate, const dla_group_rows* dresidual,
                                   float* dweight, float* dnext_weight, void* workspace,
                                   size_t workspace_bytes, void* stream);

/*
 * Log probabilities of rows of V logits l:
 *   lse = log sum_i exp(l_i),  log p_i = l_i - lse
 *   logprob = log p_token,  entropy = -sum_i p_i log p_i
 * and the `top` largest log p_i with their indices, largest first, of equal logits the lowest
 * index first (-0 equals +0).
 *
 * A logit of -inf has probability zero.  A negative token asks for nothing: its logprob is
 * zero and has no gradient.  A token of V or more is an error that the call cannot report: its
 * logprob and its row's gradient are NaN.  A row of -inf alone has lse and log probabilities
 * -inf, entropy zero and gradient zero.  A row with a NaN or +inf has NaN results; its indices
 * are below V and otherwise not defined.
 *
 * 0 <= rows <= 2^31 - 1, 1 <= V <= 2^30, 0 <= top <= 64, top <= V; each row contiguous, rows
 * `stride` (at least 0, of dlogits at least V) elements apart.  dtype: type of the logits and
 * their gradient.  Everything is computed in float32; differences from the largest logit are
 * taken before they are summed, and its own term is kept out of the sum, so that log
 * probabilities and entropies near zero keep their digits.
 */
typedef struct {
  int64_t rows;
  int32_t V, top;
  int32_t dtype; /* dla_dtype */
} dla_logprobs_desc;

/* tokens: int64 [rows], or NULL with logprob NULL.  logprob, lse, entropy: float32 [rows] or
 * NULL.  top_ids int64 and top_logprobs float32 [rows][top]; NULL where top is 0.  Workspace
 * where rows are few and long (they are then worked on in parts). */
dla_status dla_token_logprobs_workspace_size(const dla_logprobs_desc* desc, size_t* bytes);
dla_status dla_token_logprobs(const dla_logprobs_desc* desc, const dla_norm_rows* logits,
                              const int64_t* tokens, float* logprob, float* lse, float* entropy,
                              int64_t* top_ids, float* top_logprobs, void* workspace,
                              size_t workspace_bytes, void* stream);

/* The gradient of the logits from those of logprob, entropy and lse, float32 [rows] (NULL for
 * zero), and the forward pass's lse, logprob (with dlogprob) and entropy (with dentropy):
 *   dl_i = dlogprob ([i = token] - p_i) - dentropy p_i (log p_i + entropy) + dlse p_i
 * p_i is exp(l_i - lse), off by |lse| 2^-24 of itself for lse's rounding.  dlogits may be the
 * logits' array. */
dla_status dla_token_logprobs_backward(const dla_logprobs_desc* desc, const dla_norm_rows* logits,
                                       const int64_t* tokens, const float* logprob,
                                       const float* lse, const float* entropy,
                                       const float* dlogprob, const float* dentropy,
                                       const float* dlse, const dla_norm_rows* dlogits,
                                       void* stream);

/*
 * The gated feed-forward block:
 *   g = x w_gate^T,  u = x w_up^T,  y = u g / (1 + exp(-g))
 * x [rows][D], w_gate and w_up [F][D] and y [rows][F] of dtype, g and u [rows][F] float32, each a
 * set of rows `stride` elements apart (at least the row's length; inputs may repeat rows),
 * contiguous in themselves.
 *
 * 0 <= rows <= 2^30, 1 <= D, F <= 65536.  Sums are float32.  Of bfloat16 inputs every
 * product is exact; y is formed from unrounded g and u.  float32 inputs are taken as sums of
 * three bfloat16 terms, the largest first, and products of terms below 2^-24 of the whole are
 * left out: results are float32's to about 2^-22 of the sum of the products' magnitudes.  Of
 * float32, magnitudes from 2^-100 to 2^126 are taken to that precision.  Terms do not hold an
 * infinity (its first is one, and times another's zero term NaN): what it reaches is infinite or
 * NaN, which of the two is not defined, and so with what is larger than 2^126.  A forward pass of
 * up to 64 rows multiplies float32 values themselves, without these limits: there an infinity
 * gives what float32's own sums give.
 */
typedef struct {
  int64_t rows;
  int32_t D, F;
  int32_t dtype; /* dla_dtype */
} dla_ff_desc;

/* Workspace of a forward (backward = 0) or backward pass, in bytes.  aligned: whether x and the
 * weights start at multiples of 16 bytes, as do their rows, these at most 2^21 elements apart and
 * both weights' equally far.  (Of bfloat16 such arrays with D, and for the backward pass F, a
 * multiple of 8 are read in place; others, and float32, are first copied to the workspace.)  A call
 * of up to 64 rows forward needs none. */
dla_status dla_gated_ff_workspace_size(const dla_ff_desc* desc, int32_t backward, int32_t aligned,
                                       size_t* bytes);

/* g, u: where the parts that the backward pass needs go, or both NULL.  (Rounded to bfloat16 they
 * would add as much to the gradients' errors as dg's and du's rounding does.) */
dla_status dla_gated_ff(const dla_ff_desc* desc, const dla_norm_rows* x,
                        const dla_norm_rows* w_gate, const dla_norm_rows* w_up,
                        const dla_norm_rows* y, const dla_norm_rows* g, const dla_norm_rows* u,
                        void* workspace, size_t workspace_bytes, void* stream);

/* The backward pass, from dy and the forward pass's g and u.  With
 *   dg = dy u (s + g s (1 - s)),  du = dy g s,  s = 1 / (1 + exp(-g)),
 * formed in float32 and rounded once to dtype:
 *   dx = dg w_gate + du w_up,  dw_gate = dg^T x,  dw_up = du^T x,
 * sums in float32, each rounded once to dtype.  (Of bfloat16, errors of dg's and du's rounding reach
 * the gradients as large as those of their own.)  dx, dw_gate and dw_up may be NULL: not wanted. */
dla_status dla_gated_ff_backward(const dla_ff_desc* desc, const dla_norm_rows* x,
                                 const dla_norm_rows* w_gate, const dla_norm_rows* w_up,
                                 const dla_norm_rows* g, const dla_norm_rows* u,
                                 const dla_norm_rows* dy, const dla_norm_rows* dx,
                                 const dla_norm_rows* dw_gate, const dla_norm_rows* dw_up,
                                 void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* DLA_BLOCK_H */
