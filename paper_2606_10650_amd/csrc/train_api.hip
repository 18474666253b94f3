// Host side of dla_train.h: argument checks, workspaces and the launches of each call.
#include <math.h>
#include <string.h>

#include "adamw.h"
#include "dla_train.h"
#include "recurrence.h"
#include "rms_norm.h"

namespace dla {
dla_status remember(dla_status s);   // api.hip: the calling thread's last status
}

using namespace dla;

namespace {

// Tokens up to which a call goes token by token, streaming the state once, in place of a
// chunk.  128 x 128, bfloat16, 6 tokens so and 8 in a chunk: 2048 heads 53 and 50 us, 256 12
// and 11, 32 9 and 11 (two launches).  float32, whose chunks take twice as long, 12 tokens so
// and 16 in a chunk: 79 and 103, 18 and 17, 10 and 14.
constexpr int kStepTokens = 6, kStepTokensF32 = 12;
int step_tokens(int dtype) { return dtype == DLA_BF16 ? kStepTokens : kStepTokensF32; }

struct Plan {
  bool step;
  int nseg, seg_len;
};

// Segments of a pass: with fewer heads than the chip holds workgroups, sequences are cut
// so that all of them work, at the price of a pass over keys and values (backward also over
// queries and output gradients) for the segments' states.  As many as the chip then holds
// at once, about 512 workgroups, half as many again for each of d_k and d_v that is 64; not
// where that makes but two or three, which costs what it gives.  2048 bfloat16 tokens,
// forward and backward, us by segments, the rule's in brackets:
//   128 x 128   96 heads 1: 481, 4: 358, [5: 336], 6: 406   192 heads [1: 487], 2: 645
//   128 x 64    96 1: 433, 5: 256, [8: 250], 10: 283   192 1: 442, [4: 442], 5: 475
//               300 [1: 666], 2: 725
//   64 x 128    96 1: 471, 5: 254, [8: 262], 10: 296   192 1: 483, [4: 450], 5: 485
//               300 [1: 723], 2: 726, 3: 698
//   64 x 64     96 1: 401, 5: 179, 8: 163, [10: 174]   192 1: 401, 4: 281, [5: 281], 8: 315
//               300 1: 483, [3: 417], 4: 450
// A segment has at least 4 chunks, 2 of float32, whose chunks take longer (15 heads x
// 1531 tokens: 148 us, 158 with 4, 245 with 8).
Plan plan_of(const dla_recurrence_desc& d, bool backward) {
  Plan p{!backward && d.T <= step_tokens(d.dtype), 1, kRecChunk};
  if (d.B == 0 || d.T == 0) return p;   // nothing to plan
  const int heads = d.B * d.H, chunks = (d.T + kRecChunk - 1) / kRecChunk;
  const int narrow = (d.d_k == 64) + (d.d_v == 64);
  const int most = chunks / (d.dtype == DLA_BF16 ? 4 : 2);
  int n = (512 + 256 * narrow) / heads;
  if (n < (narrow == 2 ? 3 : 4)) n = 1;
  if (n > 64) n = 64;
  if (n > most) n = most > 0 ? most : 1;
  // float32: at most 1024 tokens, so that dg's sums keep float32's precision
  if (backward && d.dtype == DLA_F32 && n < (d.T + 1023) / 1024) n = (d.T + 1023) / 1024;
  const int per = (chunks + n - 1) / n;
  p.seg_len = per * kRecChunk;
  p.nseg = (chunks + per - 1) / per;
  return p;
}

struct Space {
  size_t decays, seg_state, seg_adj, seg_decay, qdot, kdot, end_dot, anchor, dq_part, dk_part, total;
};

Space space_of(const dla_recurrence_desc& d, const Plan& p, bool backward) {
  Space s;
  memset(&s, 0, sizeof(s));
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t x = at;
    at = round_up(at + bytes, 256);
    return x;
  };
  const size_t heads = (size_t)d.B * d.H, D = (size_t)d.d_k * d.d_v, tokens = heads * d.T;
  if (p.step || d.T == 0 || heads == 0) return s;
  s.decays = take(heads * rec_padded(d.T) * 16);
  if (p.nseg > 1) {
    s.seg_state = take(heads * p.nseg * D * 4);
    if (backward) s.seg_adj = take(heads * p.nseg * D * 4);
    s.seg_decay = take(heads * p.nseg * 4);
  }
  if (backward) {
    s.qdot = take(tokens * 4);
    s.kdot = take(tokens * 4);
    s.end_dot = take(heads * 4);
    if (p.nseg > 1) s.anchor = take(heads * p.nseg * (D / 256) * 8);
    if (d.Hk != d.H) {
      s.dq_part = take(tokens * d.d_k * 4);
      s.dk_part = take(tokens * d.d_k * 4);
    }
  }
  s.total = at;
  return s;
}

// Heads of a call: chunk kernels have them in a grid dimension of 65535; the step kernel has
// not, and what a launch takes of its up to 1024 threads a head.
constexpr int kHeads = 65535, kStepHeads = (1 << 21) - 1;
static_assert((int64_t)kStepHeads * 1024 < ((int64_t)1 << 32), "fewer than 2^32 threads");

dla_status check(const dla_recurrence_desc* d, bool backward) {
  if (!d) return DLA_ERR_INVALID_ARG;
  if (d->B < 0 || d->T < 0 || d->H < 1 || d->Hk < 1 || d->H % d->Hk) return DLA_ERR_INVALID_ARG;
  if (d->dtype != DLA_F32 && d->dtype != DLA_BF16) return DLA_ERR_INVALID_ARG;
  if ((d->d_k != 64 && d->d_k != 128) || (d->d_v != 64 && d->d_v != 128)) return DLA_ERR_UNSUPPORTED;
  if ((int64_t)d->B * d->H > (!backward && d->T <= kStepTokens ? kStepHeads : kHeads))
    return DLA_ERR_UNSUPPORTED;
  // a token's number with a chunk added stays an int32
  if (d->T > (1 << 30)) return DLA_ERR_UNSUPPORTED;
  return DLA_OK;
}

// Rows of `width` values of a call's tensor: there, aligned to 16 bytes (rows of one value:
// to their type), with a token stride that 32 rows of it keep within 32 bits; an output's
// also apart from each other, each stride no smaller than what the smaller ones span.
bool rows_ok(const dla_rows* r, const dla_recurrence_desc& d, int heads, int width, int elem, bool output) {
  if (!r || !r->data) return false;
  const int align = width > 1 ? 16 : elem;
  if ((uintptr_t)r->data % align) return false;
  const int64_t st[3] = {r->stride_b, r->stride_h, r->stride_t};
  const int n[3] = {d.B, heads, d.T};
  int64_t span = width;
  bool seen[3] = {false, false, false};
  for (int k = 0; k < 3; ++k) {
    int i = -1;   // the smallest stride left
    for (int j = 0; j < 3; ++j)
      if (!seen[j] && n[j] > 1 && (i < 0 || st[j] < st[i])) i = j;
    if (i < 0) break;
    seen[i] = true;
    if ((st[i] * elem) % align || (output && st[i] < span)) return false;
    span += st[i] * (n[i] - 1);
  }
  return d.T <= 1 || (r->stride_t >= 0 && r->stride_t < ((int64_t)1 << 26));
}

bool state_ok(const void* p) { return ((uintptr_t)p & 15u) == 0; }

RecArgs args_of(const dla_recurrence_desc& d, const Plan& p, const dla_rows* gate, const Space& s, char* ws) {
  RecArgs a;
  a.B = d.B;
  a.H = d.H;
  a.Hk = d.Hk;
  a.T = d.T;
  a.dk = d.d_k;
  a.dv = d.d_v;
  a.scale = d.scale;
  a.lengths = d.lengths;
  a.gate = rows_of(gate, 1);
  a.nseg = p.nseg;
  a.seg_len = p.seg_len;
  a.seg_state = (float*)(ws + s.seg_state);
  a.seg_adj = (float*)(ws + s.seg_adj);
  a.seg_decay = (float*)(ws + s.seg_decay);
  a.decays = (float2*)(ws + s.decays);
  return a;
}

__global__ void fill_kernel(float* p, int64_t n, const float* from) {
  const int64_t step = (int64_t)gridDim.x * 256;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += step) p[i] = from ? from[i] : 0.f;
}

hipError_t copy_state(const dla_recurrence_desc& d, const float* from, float* to, hipStream_t st) {
  const int64_t n = (int64_t)d.B * d.H * d.d_k * d.d_v;
  if (!to || to == from || n == 0) return hipSuccess;
  const int64_t groups = (n + 255) / 256;
  hipLaunchKernelGGL(fill_kernel, dim3(groups < 65536 ? (unsigned)groups : 65536u), dim3(256), 0, st, to, n, from);
  return hipGetLastError();
}

bool is_dtype(int t) { return t == DLA_F32 || t == DLA_BF16; }

dla_status check(const dla_norm_desc* d) {
  if (!d || d->rows < 0 || d->D < 1 || !is_dtype(d->dtype)) return DLA_ERR_INVALID_ARG;
  if (d->weight_dtype != d->dtype && d->weight_dtype != DLA_F32) return DLA_ERR_INVALID_ARG;
  if (!(d->eps >= 0.f)) return DLA_ERR_INVALID_ARG;
  if (d->D > 16384 || d->rows > ((int64_t)1 << 31) - 4) return DLA_ERR_UNSUPPORTED;
  return DLA_OK;
}

bool rows_ok(const dla_norm_rows* r, const dla_norm_desc& d, int elem) {
  return r && r->data && !((uintptr_t)r->data % elem) && (d.rows <= 1 || r->stride >= d.D);
}

NormRows norm_rows(const dla_norm_rows* r) {
  NormRows x;
  if (r) {
    x.p = r->data;
    x.st = r->stride;
  }
  return x;
}

int norm_pieces(const dla_norm_desc& d) {
  const int per = d.dtype == DLA_BF16 ? 8 : 4;
  return (d.D + per - 1) / per;
}

NormArgs norm_args(const dla_norm_desc& d, const void* weight) {
  NormArgs a;
  a.rows = d.rows;
  a.D = d.D;
  a.eps = d.eps;
  a.w = weight;
  a.w_f32 = d.weight_dtype == DLA_F32;
  a.rstd = a.y_scale = a.dw_part = nullptr;
  a.groups = 0;
  return a;
}

dla_status norm_forward(const dla_norm_desc* desc, const dla_norm_rows* x,
                        const dla_norm_rows* residual, const void* weight, const dla_norm_rows* h,
                        const dla_norm_rows* y, float* rstd, float* y_scale, bool f8, void* stream) {
  const dla_status s = check(desc);
  if (s != DLA_OK) return s;
  const dla_norm_desc& d = *desc;
  const int e = d.dtype == DLA_BF16 ? 2 : 4;
  if (!weight || (uintptr_t)weight % (d.weight_dtype == DLA_BF16 ? 2 : 4)) return DLA_ERR_INVALID_ARG;
  if (d.rows == 0) return DLA_OK;
  if (!rows_ok(x, d, e) || !rows_ok(y, d, f8 ? 1 : e)) return DLA_ERR_INVALID_ARG;
  if ((residual && !rows_ok(residual, d, e)) || (h && !rows_ok(h, d, e))) return DLA_ERR_INVALID_ARG;
  if ((f8 && !y_scale) || ((uintptr_t)rstd | (uintptr_t)y_scale) & 3) return DLA_ERR_INVALID_ARG;
  NormArgs a = norm_args(d, weight);
  a.x = norm_rows(x);
  a.res = norm_rows(residual);
  a.h = norm_rows(h);
  a.y = norm_rows(y);
  a.rstd = rstd;
  a.y_scale = y_scale;
  return launch_norm(a, d.dtype, f8 ? 1 : 0, (hipStream_t)stream) == hipSuccess ? DLA_OK : DLA_ERR_HIP;
}

bool workspace_ok(const void* ws, size_t bytes, size_t need) {
  return need == 0 || (ws && bytes >= need && ((uintptr_t)ws & 255u) == 0);
}

}  // namespace

extern "C" {

dla_status dla_recurrence_workspace_size(const dla_recurrence_desc* desc, int32_t backward,
                                         size_t* bytes) {
  const dla_status s = check(desc, backward != 0);
  if (s != DLA_OK) return remember(s);
  if (!bytes) return remember(DLA_ERR_INVALID_ARG);
  *bytes = space_of(*desc, plan_of(*desc, backward != 0), backward != 0).total;
  return remember(DLA_OK);
}

dla_status dla_recurrence_forward(const dla_recurrence_desc* desc, const dla_rows* q,
                                  const dla_rows* k, const dla_rows* v, const dla_rows* log_gate,
                                  const float* state, const dla_rows* out, float* state_out,
                                  void* workspace, size_t workspace_bytes, void* stream) {
  const dla_status s = check(desc, false);
  if (s != DLA_OK) return remember(s);
  const dla_recurrence_desc& d = *desc;
  const int e = d.dtype == DLA_BF16 ? 2 : 4, G = d.H / d.Hk;
  if (!state_ok(state) || !state_ok(state_out)) return remember(DLA_ERR_INVALID_ARG);
  hipStream_t st = (hipStream_t)stream;
  if (d.B == 0) return remember(DLA_OK);
  if (d.T == 0) return remember(copy_state(d, state, state_out, st) == hipSuccess ? DLA_OK : DLA_ERR_HIP);
  if (!rows_ok(q, d, d.Hk, d.d_k, e, false) || !rows_ok(k, d, d.Hk, d.d_k, e, false) ||
      !rows_ok(v, d, d.H, d.d_v, e, false) || !rows_ok(out, d, d.H, d.d_v, e, true) ||
      !rows_ok(log_gate, d, d.H, 1, 4, false))
    return remember(DLA_ERR_INVALID_ARG);
  const Plan p = plan_of(d, false);
  const Space sp = space_of(d, p, false);
  if (!workspace_ok(workspace, workspace_bytes, sp.total)) return remember(DLA_ERR_WORKSPACE);
  const RecArgs a = args_of(d, p, log_gate, sp, (char*)workspace);
  const Rows qr = rows_of(q, G), kr = rows_of(k, G), vr = rows_of(v, 1), outr = rows_of(out, 1);
  hipError_t r = hipSuccess;
  if (p.step) {
    r = launch_recurrence_step(a, d.dtype, qr, kr, vr, outr, state, state_out, st);
  } else {
    r = launch_recurrence_decays(a, st);
    if (r == hipSuccess && p.nseg > 1) r = launch_recurrence_segments(a, d.dtype, false, kr, vr, state, nullptr, st);
    if (r == hipSuccess) r = launch_recurrence_forward(a, d.dtype, qr, kr, vr, outr, state, state_out, st);
  }
  return remember(r == hipSuccess ? DLA_OK : DLA_ERR_HIP);
}

dla_status dla_recurrence_backward(const dla_recurrence_desc* desc, const dla_rows* q,
                                   const dla_rows* k, const dla_rows* v, const dla_rows* log_gate,
                                   const float* state, const dla_rows* dout,
                                   const float* dstate_out, const dla_rows* dq, const dla_rows* dk,
                                   const dla_rows* dv, const dla_rows* dg, float* dstate,
                                   void* workspace, size_t workspace_bytes, void* stream) {
  const dla_status s = check(desc, true);
  if (s != DLA_OK) return remember(s);
  const dla_recurrence_desc& d = *desc;
  const int e = d.dtype == DLA_BF16 ? 2 : 4, G = d.H / d.Hk;
  if (!state_ok(state) || !state_ok(dstate_out) || !state_ok(dstate)) return remember(DLA_ERR_INVALID_ARG);
  hipStream_t st = (hipStream_t)stream;
  if (d.B == 0) return remember(DLA_OK);
  if (d.T == 0) return remember(copy_state(d, dstate_out, dstate, st) == hipSuccess ? DLA_OK : DLA_ERR_HIP);
  if (!rows_ok(q, d, d.Hk, d.d_k, e, false) || !rows_ok(k, d, d.Hk, d.d_k, e, false) ||
      !rows_ok(v, d, d.H, d.d_v, e, false) || !rows_ok(dout, d, d.H, d.d_v, e, false) ||
      !rows_ok(dq, d, d.Hk, d.d_k, e, true) || !rows_ok(dk, d, d.Hk, d.d_k, e, true) ||
      !rows_ok(dv, d, d.H, d.d_v, e, true) || !rows_ok(log_gate, d, d.H, 1, 4, false) ||
      !rows_ok(dg, d, d.H, 1, e, true))
    return remember(DLA_ERR_INVALID_ARG);
  const Plan p = plan_of(d, true);
  const Space sp = space_of(d, p, true);
  if (!workspace_ok(workspace, workspace_bytes, sp.total)) return remember(DLA_ERR_WORKSPACE);
  char* ws = (char*)workspace;
  const RecArgs a = args_of(d, p, log_gate, sp, ws);
  const Rows qr = rows_of(q, G), kr = rows_of(k, G), vr = rows_of(v, 1), dor = rows_of(dout, 1);
  // heads that share keys leave their parts of dq and dk in float32, summed afterwards
  const bool shared = G > 1;
  Rows dqr = rows_of(dq, 1), dkr = rows_of(dk, 1);
  Rows dqp, dkp;
  if (shared) {
    dqp.p = ws + sp.dq_part;
    dkp.p = ws + sp.dk_part;
    dqp.st = dkp.st = d.d_k;
    dqp.sh = dkp.sh = (int64_t)d.T * d.d_k;
    dqp.sb = dkp.sb = (int64_t)d.H * d.T * d.d_k;
  } else {
    dqp = dqr;
    dkp = dkr;
  }
  float* qdot = (float*)(ws + sp.qdot);
  float* kdot = (float*)(ws + sp.kdot);
  float* end_dot = (float*)(ws + sp.end_dot);
  double* anchor = (double*)(ws + sp.anchor);
  hipError_t r = launch_recurrence_decays(a, st);
  if (r == hipSuccess && p.nseg > 1) {
    r = launch_recurrence_segments(a, d.dtype, false, kr, vr, state, nullptr, st);
    if (r == hipSuccess) r = launch_recurrence_segments(a, d.dtype, true, qr, dor, dstate_out, anchor, st);
  }
  if (r == hipSuccess)
    r = launch_recurrence_dq(a, d.dtype, qr, kr, vr, dor, dqp, shared, state, dstate_out, qdot, end_dot, st);
  if (r == hipSuccess)
    r = launch_recurrence_adjoint(a, d.dtype, qr, kr, vr, dor, dkp, shared, rows_of(dv, 1), dstate_out, dstate, kdot, st);
  if (r == hipSuccess)
    r = launch_recurrence_dgate(a, d.dtype, qdot, kdot, anchor,
                                dstate_out ? end_dot : nullptr, rows_of(dg, 1), st);
  if (shared && r == hipSuccess)
    r = launch_head_sums(a, d.dtype, (const float*)dqp.p, dqr, (const float*)dkp.p, dkr, st);
  return remember(r == hipSuccess ? DLA_OK : DLA_ERR_HIP);
}

dla_status dla_rms_norm(const dla_norm_desc* desc, const dla_norm_rows* x,
                        const dla_norm_rows* residual, const void* weight, const dla_norm_rows* h,
                        const dla_norm_rows* y, float* rstd, void* stream) {
  return remember(norm_forward(desc, x, residual, weight, h, y, rstd, nullptr, false, stream));
}

dla_status dla_rms_norm_fp8(const dla_norm_desc* desc, const dla_norm_rows* x,
                            const dla_norm_rows* residual, const void* weight,
                            const dla_norm_rows* h, const dla_norm_rows* y, float* y_scale,
                            void* stream) {
  return remember(norm_forward(desc, x, residual, weight, h, y, nullptr, y_scale, true, stream));
}

dla_status dla_rms_norm_workspace_size(const dla_norm_desc* desc, size_t* bytes) {
  const dla_status s = check(desc);
  if (s != DLA_OK) return remember(s);
  if (!bytes) return remember(DLA_ERR_INVALID_ARG);
  *bytes = desc->rows ? (size_t)norm_groups(desc->rows, norm_pieces(*desc)) * desc->D * 4 : 0;
  return remember(DLA_OK);
}

dla_status dla_rms_norm_backward(const dla_norm_desc* desc, const dla_norm_rows* dy,
                                 const dla_norm_rows* h, const void* weight, const float* rstd,
                                 const dla_norm_rows* dres, const dla_norm_rows* dx, float* dweight,
                                 void* workspace, size_t workspace_bytes, void* stream) {
  const dla_status s = check(desc);
  if (s != DLA_OK) return remember(s);
  const dla_norm_desc& d = *desc;
  const int e = d.dtype == DLA_BF16 ? 2 : 4;
  hipStream_t st = (hipStream_t)stream;
  if (!weight || (uintptr_t)weight % (d.weight_dtype == DLA_BF16 ? 2 : 4) || ((uintptr_t)dweight & 3))
    return remember(DLA_ERR_INVALID_ARG);
  NormArgs a = norm_args(d, weight);
  if (d.rows) {
    if (!rows_ok(dy, d, e) || !rows_ok(h, d, e) || !rows_ok(dx, d, e) || (dres && !rows_ok(dres, d, e)))
      return remember(DLA_ERR_INVALID_ARG);
    if (!rstd || ((uintptr_t)rstd & 3)) return remember(DLA_ERR_INVALID_ARG);
    a.groups = norm_groups(d.rows, norm_pieces(d));
    a.y = norm_rows(dy);
    a.h = norm_rows(h);
    a.res = norm_rows(dres);
    a.x = norm_rows(dx);
    a.rstd = const_cast<float*>(rstd);
    if (dweight) {
      if (!workspace_ok(workspace, workspace_bytes, (size_t)a.groups * d.D * 4)) return remember(DLA_ERR_WORKSPACE);
      a.dw_part = (float*)workspace;
    }
  }
  hipError_t r = hipSuccess;
  if (d.rows) r = launch_norm(a, d.dtype, 2, st);
  if (r == hipSuccess && dweight) r = launch_norm_dw(a, dweight, st);
  return remember(r == hipSuccess ? DLA_OK : DLA_ERR_HIP);
}

dla_status dla_adamw_step(const dla_adamw_tensor* tensors, int32_t n, const dla_adamw_params* params,
                          void* stream) {
  if (n < 0 || (n > 0 && !tensors) || !params) return remember(DLA_ERR_INVALID_ARG);
  const dla_adamw_params& p = *params;
  if (!is_dtype(p.param_dtype) || !is_dtype(p.grad_dtype)) return remember(DLA_ERR_INVALID_ARG);
  if (p.state_format != DLA_F32 && p.state_format != DLA_STATE_FP8) return remember(DLA_ERR_INVALID_ARG);
  // (written so that a NaN is refused)
  if (p.step < 1 || !(p.beta1 >= 0 && p.beta1 < 1) || !(p.beta2 >= 0 && p.beta2 < 1) || !(p.eps >= 0) ||
      !isfinite(p.eps) || !isfinite(p.lr) || ((uintptr_t)p.grad_scale & 3))
    return remember(DLA_ERR_INVALID_ARG);
  const bool f8 = p.state_format == DLA_STATE_FP8;
  const uintptr_t pm = p.param_dtype == DLA_BF16 ? 1 : 3, gm = p.grad_dtype == DLA_BF16 ? 1 : 3;
  for (int32_t i = 0; i < n; ++i) {
    const dla_adamw_tensor& t = tensors[i];
    if (t.n < 0 || t.n > ((int64_t)1 << 40) || !isfinite(t.weight_decay)) return remember(DLA_ERR_INVALID_ARG);
    if (t.n > kAdamWMost) return remember(DLA_ERR_UNSUPPORTED);
    if (t.n == 0) continue;
    if (!t.param || !t.grad || !t.m || !t.v || (f8 && (!t.m_scale || !t.v_scale)))
      return remember(DLA_ERR_INVALID_ARG);
    const uintptr_t f32 = (uintptr_t)t.master | (f8 ? (uintptr_t)t.m_scale | (uintptr_t)t.v_scale
                                                    : (uintptr_t)t.m | (uintptr_t)t.v);
    if (((uintptr_t)t.param & pm) || ((uintptr_t)t.grad & gm) || (f32 & 3)) return remember(DLA_ERR_INVALID_ARG);
  }
  AdamWScalars s;
  s.beta1 = (float)p.beta1;
  s.rest1 = (float)(1.0 - p.beta1);
  s.beta2 = (float)p.beta2;
  s.rest2 = (float)(1.0 - p.beta2);
  s.lr = (float)p.lr;
  s.step_size = (float)(p.lr / (1.0 - pow(p.beta1, (double)p.step)));
  s.root2 = (float)(1.0 / sqrt(1.0 - pow(p.beta2, (double)p.step)));
  s.eps = (float)p.eps;
  s.seed = p.seed;
  s.grad_scale = p.grad_scale;
  return remember(launch_adamw(tensors, n, s, p.param_dtype, p.grad_dtype, f8, (hipStream_t)stream) == hipSuccess
                      ? DLA_OK : DLA_ERR_HIP);
}

}  // extern "C"
