/*
 * dla_train.h -- C ABI of libdla for training the layer's base model, and for
 * serving it: the single-state recurrence of gated linear attention (arXiv
 * 2606.10650, Sec. 2.1) with its backward pass, the root-mean-square norm of the
 * residual stream, and AdamW.
 *
 * The conventions of dla.h hold: plain pointers and sizes, every array DEVICE
 * memory owned by the caller, nothing allocated or kept, all work enqueued on
 * `stream`, argument errors returned before anything is enqueued.  Workspaces
 * are 256-byte aligned, hold nothing between calls, and must not be used by
 * another call until the stream has passed the one they were given to.  Every
 * result is the same from call to call: no sum's order depends on timing.
 */
#ifndef DLA_TRAIN_H
#define DLA_TRAIN_H

#include "dla.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Rows of d values, one per sequence, head and token, the d values contiguous:
 * element (b, h, t, i) at data + b stride_b + h stride_h + t stride_t + i, in
 * elements.  [B][H][T][d] arrays, [B][T][H][d] ones and slices of a wider
 * projection's output are all rows.  Token rows start at multiples of 16 bytes:
 * data and every stride whose dimension is larger than 1.  Gates are rows of
 * d = 1 and need no alignment beyond their type's.  0 <= stride_t < 2^26.  Inputs may
 * repeat rows (strides of zero); output rows do not overlap (each stride, of
 * dimensions larger than 1, is at least what d and the smaller strides span), nor
 * any input.
 */
typedef struct {
  void* data;
  int64_t stride_b, stride_h, stride_t;
} dla_rows;

/*
 * The recurrence.  Per sequence and head, from the state S_0 (zero where none is
 * given):
 *   S_t = exp(g_t) S_{t-1} + k_t v_t^T        (d_k x d_v)
 *   o_t = scale S_t^T q_t
 * It is dla_prefill with C = 1 and lambda = scale, as an operator of its own that
 * can be differentiated: with no scores, decisions or cache around it.
 *
 * B, T >= 0 sequences and tokens, T <= 2^30; H heads, which share Hk <= H key heads (H
 * a multiple of Hk): head h has the queries and keys of head h / (H / Hk).  B H is at
 * most 65535, in a forward call of up to 6 tokens 2^21 - 1.  d_k,
 * d_v in {64, 128}.  dtype: type of q, k, v, out and of all gradients but the
 * states', which like the states, and like the gates, are float32.  States are
 * [B][H][d_k][d_v], contiguous, 16-byte aligned.
 * lengths: NULL, or int32 [B]: sequence b ends after min(max(lengths[b], 0), T)
 * tokens.  Nothing is read behind its end (whatever memory holds there, NaN
 * included), outputs and gradients there are zero, and the last state is the one
 * at the end.
 * Gates are log decays, g <= 0.  A gate below -87.33655 (a decay smaller than the
 * smallest normal float32), -inf among them, counts as a decay of zero: it starts a
 * new sequence in the same row, and its own gradient is zero.  The state must be
 * finite there.
 * Sums and states are float32.  Of bfloat16 inputs, the products of two inputs are
 * exact; scores, and what is added to the states, keep 16 bits, so that the states
 * hold float32's precision to about 2^-17; the state that out and dv read is rounded
 * once to bfloat16.  dg adds up what the scores and both states give, in float64, and
 * is rounded to the inputs' type.  Of k, v, scale q and scale dout, magnitudes up to 2^110
 * are taken; they are scaled by up to 2^16 on the way.
 * An infinity or NaN in a token reaches every later output of its head, those behind a
 * gate that cuts among them, and may reach those of up to 31 tokens before it (not in
 * forward calls of up to 6 tokens, which go one by one).
 */
typedef struct {
  int32_t B, H, Hk, T, d_k, d_v;
  int32_t dtype; /* dla_dtype */
  float scale;
  const int32_t* lengths;
} dla_recurrence_desc;

/* Workspace of a forward (backward = 0) or backward pass, in bytes; 0 where none is
 * needed.  Long sequences of few heads are worked on in segments, whose states it
 * holds; a backward pass also keeps a few numbers per token and, where heads share
 * keys, each head's part of dq and dk. */
dla_status dla_recurrence_workspace_size(const dla_recurrence_desc* desc, int32_t backward,
                                         size_t* bytes);

/* out: [B][H][T] rows of d_v.  state: S_0 or NULL.  state_out: the last state or
 * NULL; it may be the same array as state.  T = 0 copies state (or zero) to it.  One
 * or a few tokens (a decode step) go through a kernel that streams the state once. */
dla_status dla_recurrence_forward(const dla_recurrence_desc* desc, const dla_rows* q,
                                  const dla_rows* k, const dla_rows* v, const dla_rows* log_gate,
                                  const float* state, const dla_rows* out, float* state_out,
                                  void* workspace, size_t workspace_bytes, void* stream);

/* The backward pass, from the forward pass's inputs (nothing else is kept) and the
 * gradients of its outputs: dout, rows of d_v, and dstate_out [B][H][d_k][d_v], or
 * NULL for zero.  Writes dq, dk (Hk heads, summed over the heads that share them), dv,
 * dg (rows of one value in the inputs' type) and, where dstate is not NULL, the
 * gradient of S_0 (which may be dstate_out's array). */
dla_status dla_recurrence_backward(const dla_recurrence_desc* desc, const dla_rows* q,
                                   const dla_rows* k, const dla_rows* v, const dla_rows* log_gate,
                                   const float* state, const dla_rows* dout,
                                   const float* dstate_out, const dla_rows* dq, const dla_rows* dk,
                                   const dla_rows* dv, const dla_rows* dg, float* dstate,
                                   void* workspace, size_t workspace_bytes, void* stream);

/*
 * Root-mean-square norm of a residual stream.  Per row of D values:
 *   h = x + residual,  r = 1 / sqrt(mean(h^2) + eps),  y = r h weight
 * 0 <= rows <= 2^31 - 4 rows, 1 <= D <= 16384, each array's rows `stride` elements apart (at
 * least D) and contiguous in themselves, at any alignment of their type.  dtype: type
 * of x, residual, h, y and their gradients; weight_dtype: that type or DLA_F32.
 * Everything is computed in float32 from the unrounded sum x + residual and rounded
 * once when it is stored.  eps >= 0; r is right for any finite x + residual in float32,
 * and zero for a row of which mean(h^2) + eps is below 2^-252 (eps = 0 and a row of zeros
 * or of numbers below the normal ones): y is then zero, and h's only gradient is its own.
 */
typedef struct {
  int64_t rows;
  int32_t D;
  int32_t dtype, weight_dtype; /* dla_dtype */
  float eps;
} dla_norm_desc;

typedef struct {
  void* data;
  int64_t stride;
} dla_norm_rows;

/* residual: NULL for zero.  h: where x + residual goes (it may be x's or the
 * residual's array), or NULL.  rstd: [rows] float32, r of each row for the backward
 * pass, or NULL. */
dla_status dla_rms_norm(const dla_norm_desc* desc, const dla_norm_rows* x,
                        const dla_norm_rows* residual, const void* weight, const dla_norm_rows* h,
                        const dla_norm_rows* y, float* rstd, void* stream);

/* The same with y in 8-bit floating point (4 exponent and 3 mantissa bits, largest
 * value 448, no infinity) and a float32 scale per row: y_scale = max |y| / 448, the
 * codes are y (448 / max |y|) rounded to nearest even.  A row whose max |y| is below 448 times
 * the smallest normal float32 (5.3e-36) has scale and codes zero; a row with an infinity
 * or NaN has NaN codes. */
dla_status dla_rms_norm_fp8(const dla_norm_desc* desc, const dla_norm_rows* x,
                            const dla_norm_rows* residual, const void* weight,
                            const dla_norm_rows* h, const dla_norm_rows* y, float* y_scale,
                            void* stream);

/* Workspace of the backward pass (for dweight), in bytes. */
dla_status dla_rms_norm_workspace_size(const dla_norm_desc* desc, size_t* bytes);

/* Backward pass from dy, the forward pass's h and rstd, and dres, the gradient that
 * reaches h itself (NULL for zero): dx, which is also the residual's gradient, and
 * dweight [D] float32 (NULL: not wanted; the workspace is then not needed).  dx may be
 * dy's or dres's array. */
dla_status dla_rms_norm_backward(const dla_norm_desc* desc, const dla_norm_rows* dy,
                                 const dla_norm_rows* h, const void* weight, const float* rstd,
                                 const dla_norm_rows* dres, const dla_norm_rows* dx, float* dweight,
                                 void* workspace, size_t workspace_bytes, void* stream);

/*
 * One AdamW step over n tensors at once, in place:
 *   g = grad_scale grad
 *   m = beta1 m + (1 - beta1) g,  v = beta2 v + (1 - beta2) g^2
 *   p = p (1 - lr weight_decay) - lr m / (1 - beta1^step) / (sqrt(v / (1 - beta2^step)) + eps)
 * in float32.  p is master where that is given (param is then its rounded copy and
 * only written), else param.  No alignment is needed beyond the types'; 16-byte aligned
 * tensors are faster.  A tensor has 0 to 2^36 - 4096 elements.  Tensors must not overlap.
 *
 * state_format DLA_F32: m, v are float32 [n].  DLA_STATE_FP8: m and v are 8-bit codes
 * [n] of m and of sqrt(v), in the floating point format of dla_rms_norm_fp8, times
 * m_scale, v_scale, float32 [ceil(n / 256)], one per 256 elements in order.  p is updated
 * with the float32 m and v of the step, before they are rounded.  Codes follow from the
 * inputs bit by bit, by these float32 operations, each rounded, beta and 1 - beta (formed in
 * double) rounded to float32:
 *   g = grad_scale grad
 *   m = beta1 (code m_scale) + (1 - beta1) g
 *   v = beta2 (code v_scale)^2 + ((1 - beta2) g) g,  r = sqrt(v)
 * and for x either of m and r, with top the largest |x| of its 256:
 *   scale = top (1 / 448),  y = x ((1 / top) 448)
 * (top at most 1e-30: scale and codes are zero).  seed 0: the code is y, at most 448 in
 * magnitude, rounded to nearest even.  Another seed rounds up or down with the probability
 * that makes the mean right, as a v that moves by a thousandth a step would otherwise stay
 * at its code: with d = max(2^(floor(log2 |y|) - 3), 2^-9) the codes' spacing at y,
 *   |code| = min(floor(|y| / d + u) d, 448)
 * where u is h >> 16 for m and h & 65535 for r, over 65536, and of the element's index in
 * its tensor, the tensor's number in the call and the seed, modulo 2^32,
 *   h = (index + 0x9E3779B9 (number + 1)) ^ seed
 *   h = h 0x2545F491,  h = h ^ (h >> 16),  h = h 0x9E3779B1,  h = h ^ (h >> 15).
 * An r above zero has a code of at least 2^-9.  Give each step a seed of its own.
 *
 * grad_scale: NULL for 1, or one float32 on the device (a clipping or loss-scale factor);
 * where it is infinite or NaN the step changes nothing.
 */
#define DLA_STATE_FP8 2

typedef struct {
  void* param;       /* param_dtype */
  float* master;     /* or NULL */
  const void* grad;  /* grad_dtype */
  void* m;
  void* v;
  float* m_scale;    /* 8-bit states only */
  float* v_scale;
  int64_t n;
  float weight_decay;
} dla_adamw_tensor;

typedef struct {
  double lr, beta1, beta2, eps;
  int64_t step; /* 1 for the first */
  int32_t param_dtype, grad_dtype; /* dla_dtype */
  int32_t state_format;            /* DLA_F32 or DLA_STATE_FP8 */
  uint32_t seed;
  const float* grad_scale;
} dla_adamw_params;

/* tensors: HOST array of n descriptions, read before the call returns. */
dla_status dla_adamw_step(const dla_adamw_tensor* tensors, int32_t n,
                          const dla_adamw_params* params, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* DLA_TRAIN_H */
