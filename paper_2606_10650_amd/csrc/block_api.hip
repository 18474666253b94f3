// Host side of dla_block.h: argument checks, workspaces and the launches of each call.
#include <math.h>
#include <string.h>

#include "dla_block.h"
#include "gated_ff.h"
#include "gated_norm.h"
#include "logprobs.h"
#include "short_conv.h"

namespace dla {
dla_status remember(dla_status s);   // api.hip: the calling thread's last status
}

using namespace dla;

namespace {

bool is_dtype(int t) { return t == DLA_F32 || t == DLA_BF16; }
int size_of(int dtype) { return dtype == DLA_BF16 ? 2 : 4; }
bool at(const void* p, int elem) { return ((uintptr_t)p & (uintptr_t)(elem - 1)) == 0; }
dla_status done(hipError_t r) { return remember(r == hipSuccess ? DLA_OK : DLA_ERR_HIP); }

bool workspace_ok(const void* ws, size_t bytes, size_t need) {
  return need == 0 || (ws && bytes >= need && ((uintptr_t)ws & 255u) == 0);
}

// Rows of two strides: not negative, and of an output apart from each other.
bool strides_ok(int64_t s0, int64_t n0, int64_t s1, int64_t n1, int64_t width, bool output) {
  if ((n0 > 1 && s0 < 0) || (n1 > 1 && s1 < 0)) return false;
  if (!output) return true;
  if (n0 > 1 && n1 > 1) {
    const bool outer = s0 >= s1;
    const int64_t in = outer ? s1 : s0, big = outer ? s0 : s1, n = outer ? n1 : n0;
    return in >= width && big >= in * (n - 1) + width;
  }
  return (n0 <= 1 || s0 >= width) && (n1 <= 1 || s1 >= width);
}

// ---------------------------------------------------------------------------
// short convolution
// ---------------------------------------------------------------------------
dla_status check(const dla_conv_desc* d) {
  if (!d || d->B < 0 || d->T < 0 || d->C < 0 || !is_dtype(d->dtype)) return DLA_ERR_INVALID_ARG;
  if (d->weight_dtype != d->dtype && d->weight_dtype != DLA_F32) return DLA_ERR_INVALID_ARG;
  if (d->silu != 0 && d->silu != 1) return DLA_ERR_INVALID_ARG;
  if (d->W < 2 || d->W > 4 || d->T > (1 << 30) || d->C > (1 << 30)) return DLA_ERR_UNSUPPORTED;
  if (!at(d->lengths, 4)) return DLA_ERR_INVALID_ARG;
  return DLA_OK;
}

bool rows_ok(const dla_conv_rows* r, const dla_conv_desc& d, bool output) {
  return r && r->data && at(r->data, size_of(d.dtype)) && strides_ok(r->stride_b, d.B, r->stride_t, d.T, d.C, output);
}

ConvRows rows_of(const dla_conv_rows* r) {
  ConvRows x;
  if (r) {
    x.p = r->data;
    x.sb = r->stride_b;
    x.st = r->stride_t;
  }
  return x;
}

ConvArgs conv_args(const dla_conv_desc& d, bool backward) {
  ConvArgs a;
  memset(&a, 0, sizeof(a));
  a.B = d.B;
  a.T = d.T;
  a.C = d.C;
  a.W = d.W;
  a.w_f32 = d.weight_dtype == DLA_F32;
  a.silu = d.silu;
  a.lengths = d.lengths;
  a.starts = d.starts;
  plan_conv(a, d.dtype, backward);
  return a;
}

size_t conv_part_bytes(const ConvArgs& a) { return (size_t)a.groups * a.C * (a.W + 1) * 4; }

// a launch has fewer than 2^32 threads
bool conv_fits(const ConvArgs& a) { return ((a.pieces + a.lanes - 1) / a.lanes) * a.groups < ((int64_t)1 << 24); }

// ---------------------------------------------------------------------------
// gated norm
// ---------------------------------------------------------------------------
dla_status check(const dla_gated_norm_desc* d) {
  if (!d || d->rows < 0 || d->groups < 1 || d->D < 1 || !is_dtype(d->dtype)) return DLA_ERR_INVALID_ARG;
  if (d->weight_dtype != d->dtype && d->weight_dtype != DLA_F32) return DLA_ERR_INVALID_ARG;
  if (!(d->eps >= 0.f) || !isfinite(d->scale)) return DLA_ERR_INVALID_ARG;
  if (d->weight_per_group != 0 && d->weight_per_group != 1) return DLA_ERR_INVALID_ARG;
  if (d->D > 16384 || d->groups > 65535 || (int64_t)d->groups * d->D > (1 << 26) || d->rows > ((int64_t)1 << 31) - 4)
    return DLA_ERR_UNSUPPORTED;
  return DLA_OK;
}

bool rows_ok(const dla_group_rows* r, const dla_gated_norm_desc& d, bool output) {
  return r && r->data && at(r->data, size_of(d.dtype)) && strides_ok(r->stride, d.rows, r->stride_g, d.groups, d.D, output);
}

GroupRows rows_of(const dla_group_rows* r) {
  GroupRows x;
  if (r) {
    x.p = r->data;
    x.st = r->stride;
    x.sg = r->stride_g;
  }
  return x;
}

GatedNormArgs norm_args(const dla_gated_norm_desc& d, bool backward) {
  GatedNormArgs a;
  memset(&a, 0, sizeof(a));
  a.rows = d.rows;
  a.G = d.groups;
  a.D = d.D;
  a.eps = d.eps;
  a.scale = d.scale;
  a.w_f32 = d.weight_dtype == DLA_F32;
  a.per_group = d.weight_per_group;
  plan_gated_norm(a, d.dtype, backward);
  return a;
}

struct NormSpace {
  size_t dw2, total;
};
NormSpace space_of(const GatedNormArgs& a) {
  NormSpace s{0, 0};
  if (a.rows == 0) return s;
  s.dw2 = round_up((size_t)gated_norm_dw_parts(a) * a.D * (a.per_group ? a.G : 1) * 4, 256);
  s.total = s.dw2 + (a.G == 1 ? round_up((size_t)a.groups * a.gcols * a.D * 4, 256) : 0);
  return s;
}

// ---------------------------------------------------------------------------
// log probabilities
// ---------------------------------------------------------------------------
dla_status check(const dla_logprobs_desc* d) {
  if (!d || d->rows < 0 || d->V < 1 || !is_dtype(d->dtype) || d->top < 0 || d->top > d->V) return DLA_ERR_INVALID_ARG;
  if (d->rows > ((int64_t)1 << 31) - 1 || d->V > (1 << 30) || d->top > 64) return DLA_ERR_UNSUPPORTED;
  return DLA_OK;
}

struct LogprobSpace {
  size_t keys, total;
};
LogprobSpace space_of(const LogprobArgs& a) {
  LogprobSpace s{0, 0};
  if (a.parts <= 1 || a.rows == 0) return s;
  s.keys = round_up((size_t)a.rows * a.parts * 12, 256);
  s.total = s.keys + (size_t)a.rows * a.parts * a.top * 8;
  return s;
}

LogprobArgs logprob_args(const dla_logprobs_desc& d) {
  LogprobArgs a;
  memset(&a, 0, sizeof(a));
  a.rows = d.rows;
  a.V = d.V;
  a.top = d.top;
  a.bf16 = d.dtype == DLA_BF16;
  plan_logprobs(a, d.dtype);
  return a;
}

// ---------------------------------------------------------------------------
// feed-forward
// ---------------------------------------------------------------------------
dla_status check(const dla_ff_desc* d) {
  if (!d || d->rows < 0 || d->D < 1 || d->F < 1 || !is_dtype(d->dtype)) return DLA_ERR_INVALID_ARG;
  if (d->rows > (1 << 30) || d->D > 65536 || d->F > 65536) return DLA_ERR_UNSUPPORTED;
  return DLA_OK;
}

bool rows_ok(const dla_norm_rows* r, int64_t rows, int64_t width, int elem, bool output) {
  return r && r->data && at(r->data, elem) && (rows <= 1 || r->stride >= (output ? width : 0));
}

FfRows ff_rows(const dla_norm_rows* r) {
  FfRows x;
  if (r) {
    x.p = r->data;
    x.st = r->stride;
  }
  return x;
}

// Whether rows are read in place by the products: 16-byte pieces, 32-bit offsets in a tile of 256
// rows.
bool in_place(const dla_norm_rows* r, int64_t rows) {
  return at(r->data, 16) && (rows <= 1 || (r->stride % 8 == 0 && r->stride <= (1 << 21)));
}

struct FfSpace {
  size_t x, wg, wu, parts, sum, total;
  FfPlan y, dx, dw;
};
FfSpace space_of(const dla_ff_desc& d, bool backward, bool direct) {
  FfSpace s;
  memset(&s, 0, sizeof(s));
  const int planes = d.dtype == DLA_BF16 ? 1 : 3;
  if (d.rows == 0) s.dw = plan_ff_gemm(2, 2 * (int64_t)round_up(d.F, 8), d.D, 0, planes == 1 ? 1 : 6);
  if (d.rows == 0 || (!backward && d.rows <= kFfStepRows)) return s;
  size_t used = 0;
  auto take = [&](size_t bytes) {
    const size_t x = used;
    used = round_up(used + bytes, 256);
    return x;
  };
  const size_t Dp = round_up(d.D, 8), Fp = round_up(d.F, 8);
  if (!direct) {
    s.x = take(planes * d.rows * Dp * 2);
    s.wg = take(planes * d.F * Dp * 2);
    s.wu = take(planes * d.F * Dp * 2);
  }
  if (backward) {
    s.parts = take(planes * d.rows * 2 * Fp * 2);
    s.dx = plan_ff_gemm(1, d.rows, d.D, d.F, planes == 1 ? 2 : 12);
    s.dw = plan_ff_gemm(2, 2 * Fp, d.D, d.rows, planes == 1 ? 1 : 6);
    s.sum = take(s.dx.part_bytes > s.dw.part_bytes ? s.dx.part_bytes : s.dw.part_bytes);
  } else {
    s.y = plan_ff_gemm(0, d.rows, d.F, d.D, planes == 1 ? 1 : 6);
    s.sum = take(s.y.part_bytes);
  }
  s.total = used;
  return s;
}

// The pairs of terms that a float32 product is the sum of, the smallest first; of bfloat16 one.
void pairs_of(FfGemm& g, int planes, int sets) {
  static const uint8_t a[6] = {2, 0, 1, 1, 0, 0}, b[6] = {0, 2, 1, 0, 1, 0};
  g.pairs = 0;
  g.ia = g.ib = 0;
  const int n = planes == 1 ? 1 : 6;
  for (int i = 0; i < n; ++i)
    for (int s = 0; s < sets; ++s) {
      g.ia |= (uint64_t)(planes * s + (planes == 1 ? 0 : a[i])) << (4 * g.pairs);
      g.ib |= (uint64_t)(planes * s + (planes == 1 ? 0 : b[i])) << (4 * g.pairs++);
    }
}

// An operand's planes: in place, or to be packed into the workspace.
struct FfPlanes {
  const uint16_t* p = nullptr;
  int64_t ld = 0, plane = 0;
};
FfPlanes planes_of(bool direct, const dla_norm_rows* r, int64_t rows, int cols, char* to, FfPack& pack) {
  FfPlanes o;
  if (direct) {
    o.p = static_cast<const uint16_t*>(r->data);
    o.ld = rows <= 1 ? cols : r->stride;
  } else {
    o.p = reinterpret_cast<const uint16_t*>(to);
    o.ld = (int64_t)round_up(cols, 8);
    o.plane = rows * o.ld;
    pack.rows = rows;
    pack.cols = cols;
    pack.from = ff_rows(r);
    pack.to = reinterpret_cast<uint16_t*>(to);
  }
  return o;
}

}  // namespace

extern "C" {

dla_status dla_short_conv(const dla_conv_desc* desc, const dla_conv_rows* x, const void* weight,
                          const void* bias, const void* state, const dla_conv_rows* y,
                          void* state_out, void* stream) {
  const dla_status s = check(desc);
  if (s != DLA_OK) return remember(s);
  const dla_conv_desc& d = *desc;
  const int e = size_of(d.dtype), we = size_of(d.weight_dtype);
  if (!at(weight, we) || !at(bias, we) || !at(state, e) || !at(state_out, e)) return remember(DLA_ERR_INVALID_ARG);
  if (d.B == 0 || d.C == 0) return remember(DLA_OK);
  if (!weight || (d.T && (!rows_ok(x, d, false) || !rows_ok(y, d, true)))) return remember(DLA_ERR_INVALID_ARG);
  if (d.T == 0 && !state_out) return remember(DLA_OK);
  ConvArgs a = conv_args(d, false);
  if (!conv_fits(a)) return remember(DLA_ERR_UNSUPPORTED);
  a.w = weight;
  a.bias = bias;
  a.state = state;
  a.x = rows_of(x);
  a.y = rows_of(y);
  a.state_out = state_out;
  return done(launch_conv(a, d.dtype, (hipStream_t)stream));
}

dla_status dla_short_conv_workspace_size(const dla_conv_desc* desc, size_t* bytes) {
  const dla_status s = check(desc);
  if (s != DLA_OK) return remember(s);
  if (!bytes) return remember(DLA_ERR_INVALID_ARG);
  *bytes = conv_part_bytes(conv_args(*desc, true));
  return remember(DLA_OK);
}

dla_status dla_short_conv_backward(const dla_conv_desc* desc, const dla_conv_rows* x,
                                   const void* weight, const void* bias, const void* state,
                                   const dla_conv_rows* dy, const void* dstate_out,
                                   const dla_conv_rows* dx, float* dweight, float* dbias,
                                   void* dstate, void* workspace, size_t workspace_bytes,
                                   void* stream) {
  const dla_status s = check(desc);
  if (s != DLA_OK) return remember(s);
  const dla_conv_desc& d = *desc;
  const int e = size_of(d.dtype), we = size_of(d.weight_dtype);
  if (!at(weight, we) || !at(bias, we) || !at(state, e) || !at(dstate_out, e) || !at(dstate, e) || !at(dweight, 4) ||
      !at(dbias, 4) || (dstate && dstate == dstate_out))
    return remember(DLA_ERR_INVALID_ARG);
  if (d.C == 0) return remember(DLA_OK);
  if (!weight || !dweight) return remember(DLA_ERR_INVALID_ARG);
  if (d.B && d.T && (!rows_ok(x, d, false) || !rows_ok(dy, d, false) || !rows_ok(dx, d, true)))
    return remember(DLA_ERR_INVALID_ARG);
  ConvArgs a = conv_args(d, true);
  if (!conv_fits(a)) return remember(DLA_ERR_UNSUPPORTED);
  if (!workspace_ok(workspace, workspace_bytes, conv_part_bytes(a))) return remember(DLA_ERR_WORKSPACE);
  a.w = weight;
  a.bias = bias;
  a.state = state;
  a.x = rows_of(x);
  a.y = rows_of(dy);
  a.dx = rows_of(dx);
  a.dstate_out = dstate_out;
  a.dstate = dstate;
  a.part = (float*)workspace;
  return done(launch_conv_backward(a, d.dtype, dweight, dbias, (hipStream_t)stream));
}

dla_status dla_gated_norm(const dla_gated_norm_desc* desc, const dla_group_rows* x,
                          const dla_group_rows* gate, const dla_group_rows* residual,
                          const void* weight, const void* next_weight, const dla_group_rows* h,
                          const dla_group_rows* y, float* rstd, float* y_rstd, void* stream) {
  const dla_status s = check(desc);
  if (s != DLA_OK) return remember(s);
  const dla_gated_norm_desc& d = *desc;
  const int we = size_of(d.weight_dtype);
  if (!weight || !at(weight, we) || !at(next_weight, we) || !at(rstd, 4) || !at(y_rstd, 4) || (next_weight && d.groups != 1))
    return remember(DLA_ERR_INVALID_ARG);
  if (d.rows == 0) return remember(DLA_OK);
  if (!rows_ok(x, d, false) || !rows_ok(h, d, true) || (gate && !rows_ok(gate, d, false)) ||
      (residual && !rows_ok(residual, d, false)) || (next_weight && !rows_ok(y, d, true)))
    return remember(DLA_ERR_INVALID_ARG);
  GatedNormArgs a = norm_args(d, false);
  a.w = weight;
  a.w2 = next_weight;
  a.x = rows_of(x);
  a.gate = rows_of(gate);
  a.res = rows_of(residual);
  a.h = rows_of(h);
  a.y = rows_of(y);
  a.rstd = rstd;
  a.rstd2 = y_rstd;
  return done(launch_gated_norm(a, d.dtype, false, (hipStream_t)stream));
}

dla_status dla_gated_norm_workspace_size(const dla_gated_norm_desc* desc, size_t* bytes) {
  const dla_status s = check(desc);
  if (s != DLA_OK) return remember(s);
  if (!bytes) return remember(DLA_ERR_INVALID_ARG);
  *bytes = space_of(norm_args(*desc, true)).total;
  return remember(DLA_OK);
}

dla_status dla_gated_norm_backward(const dla_gated_norm_desc* desc, const dla_group_rows* x,
                                   const dla_group_rows* gate, const dla_group_rows* residual,
                                   const void* weight, const void* next_weight, const float* rstd,
                                   const float* y_rstd, const dla_group_rows* dh,
                                   const dla_group_rows* dy, const dla_group_rows* dx,
                                   const dla_group_rows* dgate, const dla_group_rows* dresidual,
                                   float* dweight, float* dnext_weight, void* workspace,
                                   size_t workspace_bytes, void* stream) {
  const dla_status s = check(desc);
  if (s != DLA_OK) return remember(s);
  const dla_gated_norm_desc& d = *desc;
  const int we = size_of(d.weight_dtype);
  if (!weight || !at(weight, we) || !at(next_weight, we) || !at(rstd, 4) || !at(y_rstd, 4) || !at(dweight, 4) ||
      !at(dnext_weight, 4) || (next_weight && d.groups != 1) || (!next_weight && (dy || dnext_weight)) || (dgate && !gate))
    return remember(DLA_ERR_INVALID_ARG);
  GatedNormArgs a = norm_args(d, true);
  if (d.rows) {
    if (!rows_ok(x, d, false) || !rows_ok(dx, d, true) || (gate && !rows_ok(gate, d, false)) ||
        (residual && !rows_ok(residual, d, false)) || (dh && !rows_ok(dh, d, false)) || (dy && !rows_ok(dy, d, false)) ||
        (dgate && !rows_ok(dgate, d, true)) || (dresidual && !rows_ok(dresidual, d, true)))
      return remember(DLA_ERR_INVALID_ARG);
    if (!rstd || (dy && !y_rstd)) return remember(DLA_ERR_INVALID_ARG);
    a.w = weight;
    a.w2 = next_weight;
    a.x = rows_of(x);
    a.gate = rows_of(gate);
    a.res = rows_of(residual);
    a.h = rows_of(dh);
    a.y = rows_of(dy);
    a.rstd = const_cast<float*>(rstd);
    a.rstd2 = const_cast<float*>(y_rstd);
    a.dx = rows_of(dx);
    a.dgate = rows_of(dgate);
    a.dres = rows_of(dresidual);
    plan_gated_norm(a, d.dtype, true);
    const NormSpace sp = space_of(a);
    if (dweight || dnext_weight) {
      if (!workspace_ok(workspace, workspace_bytes, sp.total)) return remember(DLA_ERR_WORKSPACE);
      a.dw_part = dweight ? (float*)workspace : nullptr;
      a.dw2_part = dnext_weight ? (float*)((char*)workspace + sp.dw2) : nullptr;
    }
  }
  hipStream_t st = (hipStream_t)stream;
  hipError_t r = hipSuccess;
  if (d.rows) r = launch_gated_norm(a, d.dtype, true, st);
  if (r == hipSuccess && (dweight || dnext_weight)) r = launch_gated_norm_dw(a, dweight, dnext_weight, st);
  return done(r);
}

dla_status dla_token_logprobs_workspace_size(const dla_logprobs_desc* desc, size_t* bytes) {
  const dla_status s = check(desc);
  if (s != DLA_OK) return remember(s);
  if (!bytes) return remember(DLA_ERR_INVALID_ARG);
  *bytes = space_of(logprob_args(*desc)).total;
  return remember(DLA_OK);
}

dla_status dla_token_logprobs(const dla_logprobs_desc* desc, const dla_norm_rows* logits,
                              const int64_t* tokens, float* logprob, float* lse, float* entropy,
                              int64_t* top_ids, float* top_logprobs, void* workspace,
                              size_t workspace_bytes, void* stream) {
  const dla_status s = check(desc);
  if (s != DLA_OK) return remember(s);
  const dla_logprobs_desc& d = *desc;
  if (!at(tokens, 8) || !at(logprob, 4) || !at(lse, 4) || !at(entropy, 4) || !at(top_ids, 8) || !at(top_logprobs, 4))
    return remember(DLA_ERR_INVALID_ARG);
  if (d.rows == 0) return remember(DLA_OK);
  if (!rows_ok(logits, d.rows, d.V, size_of(d.dtype), false) || (logprob && !tokens) ||
      (d.top && (!top_ids || !top_logprobs)))
    return remember(DLA_ERR_INVALID_ARG);
  LogprobArgs a = logprob_args(d);
  const LogprobSpace sp = space_of(a);
  if (!workspace_ok(workspace, workspace_bytes, sp.total)) return remember(DLA_ERR_WORKSPACE);
  a.part_sums = (float*)workspace;
  a.part_keys = (uint64_t*)((char*)workspace + sp.keys);
  a.l = logits->data;
  a.st = logits->stride;
  a.tokens = tokens;
  a.lp = logprob;
  a.lse = lse;
  a.ent = entropy;
  a.ids = top_ids;
  a.tops = top_logprobs;
  return done(launch_logprobs(a, d.dtype, (hipStream_t)stream));
}

dla_status dla_token_logprobs_backward(const dla_logprobs_desc* desc, const dla_norm_rows* logits,
                                       const int64_t* tokens, const float* logprob,
                                       const float* lse, const float* entropy,
                                       const float* dlogprob, const float* dentropy,
                                       const float* dlse, const dla_norm_rows* dlogits,
                                       void* stream) {
  const dla_status s = check(desc);
  if (s != DLA_OK) return remember(s);
  const dla_logprobs_desc& d = *desc;
  const int e = size_of(d.dtype);
  if (!at(tokens, 8) || !at(logprob, 4) || !at(lse, 4) || !at(entropy, 4) || !at(dlogprob, 4) || !at(dentropy, 4) ||
      !at(dlse, 4))
    return remember(DLA_ERR_INVALID_ARG);
  if (d.rows == 0) return remember(DLA_OK);
  if (!rows_ok(logits, d.rows, d.V, e, false) || !rows_ok(dlogits, d.rows, d.V, e, true) || !lse ||
      (dlogprob && (!tokens || !logprob)) || (dentropy && !entropy))
    return remember(DLA_ERR_INVALID_ARG);
  LogprobArgs a;
  memset(&a, 0, sizeof(a));
  a.rows = d.rows;
  a.V = d.V;
  a.l = logits->data;
  a.st = logits->stride;
  a.tokens = tokens;
  a.lp = const_cast<float*>(logprob);
  a.lse = const_cast<float*>(lse);
  a.ent = const_cast<float*>(entropy);
  a.dlp = dlogprob;
  a.dent = dentropy;
  a.dlse = dlse;
  a.dl = dlogits->data;
  a.dst = dlogits->stride;
  return done(launch_logprobs_backward(a, d.dtype, (hipStream_t)stream));
}

dla_status dla_gated_ff_workspace_size(const dla_ff_desc* desc, int32_t backward, int32_t aligned,
                                       size_t* bytes) {
  const dla_status s = check(desc);
  if (s != DLA_OK) return remember(s);
  if (!bytes) return remember(DLA_ERR_INVALID_ARG);
  const bool direct = aligned && desc->dtype == DLA_BF16 && desc->D % 8 == 0 && (!backward || desc->F % 8 == 0);
  *bytes = space_of(*desc, backward != 0, direct).total;
  return remember(DLA_OK);
}

dla_status dla_gated_ff(const dla_ff_desc* desc, const dla_norm_rows* x,
                        const dla_norm_rows* w_gate, const dla_norm_rows* w_up,
                        const dla_norm_rows* y, const dla_norm_rows* g, const dla_norm_rows* u,
                        void* workspace, size_t workspace_bytes, void* stream) {
  const dla_status s = check(desc);
  if (s != DLA_OK) return remember(s);
  const dla_ff_desc& d = *desc;
  const int e = size_of(d.dtype);
  if (d.rows == 0) return remember(DLA_OK);
  if (!rows_ok(x, d.rows, d.D, e, false) || !rows_ok(w_gate, d.F, d.D, e, false) || !rows_ok(w_up, d.F, d.D, e, false) ||
      !rows_ok(y, d.rows, d.F, e, true) || (g && !rows_ok(g, d.rows, d.F, 4, true)) ||
      (u && !rows_ok(u, d.rows, d.F, 4, true)) || !g != !u)
    return remember(DLA_ERR_INVALID_ARG);
  hipStream_t st = (hipStream_t)stream;
  if (d.rows <= kFfStepRows)
    return done(launch_ff_step(d.rows, d.D, d.F, d.dtype, ff_rows(x), ff_rows(w_gate), ff_rows(w_up), ff_rows(y),
                               ff_rows(g), ff_rows(u), st));
  // both weights have one stride in the products
  const bool direct = d.dtype == DLA_BF16 && d.D % 8 == 0 && in_place(x, d.rows) && in_place(w_gate, d.F) &&
                      in_place(w_up, d.F) && (d.F <= 1 || w_gate->stride == w_up->stride);
  const FfSpace sp = space_of(d, false, direct);
  if (!workspace_ok(workspace, workspace_bytes, sp.total)) return remember(DLA_ERR_WORKSPACE);
  char* ws = (char*)workspace;
  const int planes = d.dtype == DLA_BF16 ? 1 : 3;
  FfPacks packs;
  const FfPlanes px = planes_of(direct, x, d.rows, d.D, ws + sp.x, packs.set[0]);
  const FfPlanes pg = planes_of(direct, w_gate, d.F, d.D, ws + sp.wg, packs.set[1]);
  const FfPlanes pu = planes_of(direct, w_up, d.F, d.D, ws + sp.wu, packs.set[2]);
  const hipError_t r = launch_ff_pack(packs, d.dtype, st);
  if (r != hipSuccess) return done(r);
  FfGemm p;
  memset(&p, 0, sizeof(p));
  p.kind = 0;
  p.out_f32 = d.dtype == DLA_F32;
  p.M = d.rows;
  p.N = d.F;
  p.K = d.D;
  for (int i = 0; i < planes; ++i) {
    p.a[i] = px.p + i * px.plane;
    p.b[i] = pg.p + i * pg.plane;
    p.b2[i] = pu.p + i * pu.plane;
  }
  p.lda = px.ld;
  p.ldb = pg.ld;
  pairs_of(p, planes, 1);
  p.c = ff_rows(y);
  p.g = ff_rows(g);
  p.u = ff_rows(u);
  p.part = (float*)(ws + sp.sum);
  return done(launch_ff_gemm(p, sp.y, st));
}

dla_status dla_gated_ff_backward(const dla_ff_desc* desc, const dla_norm_rows* x,
                                 const dla_norm_rows* w_gate, const dla_norm_rows* w_up,
                                 const dla_norm_rows* g, const dla_norm_rows* u,
                                 const dla_norm_rows* dy, const dla_norm_rows* dx,
                                 const dla_norm_rows* dw_gate, const dla_norm_rows* dw_up,
                                 void* workspace, size_t workspace_bytes, void* stream) {
  const dla_status s = check(desc);
  if (s != DLA_OK) return remember(s);
  const dla_ff_desc& d = *desc;
  const int e = size_of(d.dtype);
  if ((dw_gate && !rows_ok(dw_gate, d.F, d.D, e, true)) || (dw_up && !rows_ok(dw_up, d.F, d.D, e, true)))
    return remember(DLA_ERR_INVALID_ARG);
  if (d.rows && (!rows_ok(x, d.rows, d.D, e, false) || !rows_ok(w_gate, d.F, d.D, e, false) ||
                 !rows_ok(w_up, d.F, d.D, e, false) || !rows_ok(g, d.rows, d.F, 4, false) ||
                 !rows_ok(u, d.rows, d.F, 4, false) || !rows_ok(dy, d.rows, d.F, e, false) ||
                 (dx && !rows_ok(dx, d.rows, d.D, e, true))))
    return remember(DLA_ERR_INVALID_ARG);
  hipStream_t st = (hipStream_t)stream;
  const bool direct = d.rows && d.dtype == DLA_BF16 && d.D % 8 == 0 && d.F % 8 == 0 && in_place(x, d.rows) &&
                      in_place(w_gate, d.F) && in_place(w_up, d.F) && (d.F <= 1 || w_gate->stride == w_up->stride);
  const FfSpace sp = space_of(d, true, direct);
  if (!workspace_ok(workspace, workspace_bytes, sp.total)) return remember(DLA_ERR_WORKSPACE);
  char* ws = (char*)workspace;
  const int planes = d.dtype == DLA_BF16 ? 1 : 3;
  const int64_t Fp = (int64_t)round_up(d.F, 8);
  FfPlanes px, pg, pu;
  uint16_t* parts = (uint16_t*)(ws + sp.parts);
  hipError_t r = hipSuccess;
  if (d.rows) {
    FfPacks packs;
    px = planes_of(direct, x, d.rows, d.D, ws + sp.x, packs.set[0]);
    if (dx) {
      pg = planes_of(direct, w_gate, d.F, d.D, ws + sp.wg, packs.set[1]);
      pu = planes_of(direct, w_up, d.F, d.D, ws + sp.wu, packs.set[2]);
    }
    r = launch_ff_pack(packs, d.dtype, st);
    if (r == hipSuccess) r = launch_ff_parts(d.rows, d.F, d.dtype, ff_rows(g), ff_rows(u), ff_rows(dy), parts, st);
    if (r != hipSuccess) return done(r);
  }
  FfGemm p;
  memset(&p, 0, sizeof(p));
  p.out_f32 = d.dtype == DLA_F32;
  p.lda = 2 * Fp;
  p.part = (float*)(ws + sp.sum);
  const int64_t plane = d.rows * 2 * Fp;
  if (d.rows && dx) {
    p.kind = 1;
    p.M = d.rows;
    p.N = d.D;
    p.K = d.F;
    for (int i = 0; i < planes; ++i) {
      p.a[i] = parts + i * plane;
      p.a[planes + i] = parts + i * plane + Fp;
      p.b[i] = pg.p + i * pg.plane;
      p.b[planes + i] = pu.p + i * pu.plane;
    }
    p.ldb = pg.ld;
    pairs_of(p, planes, 2);
    p.c = ff_rows(dx);
    r = launch_ff_gemm(p, sp.dx, st);
  }
  if (r == hipSuccess && (dw_gate || dw_up)) {
    p.kind = 2;
    p.M = 2 * Fp;
    p.N = d.D;
    p.K = d.rows;
    for (int i = 0; i < planes; ++i) {
      p.a[i] = parts + i * plane;
      p.b[i] = px.p + i * px.plane;
    }
    p.ldb = px.ld;
    pairs_of(p, planes, 1);
    p.c = ff_rows(dw_gate);
    p.c2 = ff_rows(dw_up);
    p.half = Fp;
    p.rows = d.F;
    r = launch_ff_gemm(p, sp.dw, st);
  }
  return done(r);
}

}  // extern "C"
