// C ABI of the norms, the dense layer and the AdamW step: argument checks and the choice of kernel.  Declarations and the meaning of every
// argument are in include/gws.h.
#include <math.h>
#include <string.h>

#include "gws_adamw.h"
#include "gws_bench.h"
#include "gws_check.h"
#include "gws_dense_out.h"
#include "gws_norm.h"

namespace gws {

namespace {

inline Span2 span_f32(const void* p, int64_t n) { return Span2{p, 1, (size_t)n * 4, (size_t)n * 4}; }
inline Span2 span_bytes(const void* p, size_t n) { return Span2{p, 1, n, n}; }

// ---- norms ----
size_t norm_bytes(int64_t M, int64_t C) {
  size_t n = (size_t)norm_bwd_parts((uint64_t)M, (uint64_t)C) * 2 * (size_t)C * sizeof(float);
  n = (n + 15) & ~(size_t)15;
  return n + (norm_is_wide((uint64_t)C) ? (size_t)M * 2 * sizeof(float) : 0);
}

// ---- the dense layer ----
size_t dense_bytes(int64_t M, int64_t F) { return M <= 16 ? 0 : (size_t)((M + 15) / 16) * (size_t)F * sizeof(float); }

// Outputs, kept Z and the bias gradient's workspace of the two backward calls.
int dense_bwd_args(int64_t M, int64_t F, int act, const void* z, int64_t ldz, void* dz, int64_t lddz, void* h, int64_t ldh, float* dbias, void* workspace,
                   size_t workspace_bytes, GemmArgs& g, DenseArgs& d, Buffers& b) {
  if ((z == nullptr && (act != GWS_ACT_NONE || h != nullptr))) return GWS_ERR_NULL;
  if ((z && !ld_ok(ldz, F)) || (dz && !ld_ok(lddz, F)) || (h && !ld_ok(ldh, F))) return GWS_ERR_SHAPE;
  const size_t need = dbias ? dense_bytes(M, F) : 0;
  if (need && !workspace) return GWS_ERR_NULL;
  if (need && workspace_bytes < need) return GWS_ERR_SHAPE;
  if (!aligned(z, 16) || !aligned(dz, 16) || !aligned(h, 16) || !aligned(dbias, 4) || (need && !aligned(workspace, 16))) return GWS_ERR_ALIGN;
  if (act == GWS_ACT_NONE && h == nullptr) z = nullptr;   // what is not used is not read
  b.reads(span16(z, M, F, ldz));
  b.writes(span16(dz, M, F, lddz));
  b.writes(span16(h, M, F, ldh));
  b.writes(span_f32(dbias, F));
  if (need) b.writes(span_bytes(workspace, need));
  g.M = (uint32_t)M; g.N = (uint32_t)F;
  g.y = (uint16_t*)dz; g.ldy = ld_of(dz, lddz);
  d.z = (uint16_t*)z; d.ldz = ld_of(z, ldz);
  d.h = (uint16_t*)h; d.ldh = ld_of(h, ldh);
  d.act = act;
  return GWS_OK;
}
// Runs a backward pass whose tiles are `rows` rows high, and adds its partial sums up.
template <class Launch>
int with_bias_gradient(const GemmArgs& g, DenseArgs& d, uint64_t rows, float* dbias, void* workspace, hipStream_t stream, Launch&& launch) {
  const uint64_t parts = ((uint64_t)g.M + rows - 1) / rows;
  d.part = !dbias ? nullptr : parts == 1 ? dbias : (float*)workspace;
  const int rc = launch();
  if (rc != GWS_OK || !dbias || parts == 1) return rc;
  return launch_sum_partials(d.part, (uint32_t)parts, g.N, g.N, dbias, nullptr, stream);
}

// Whether Y, or dZ and H, of 128 x 128 tiles and larger ones go past the caches: by the call's time together with what reads them next (a graph over two sets of buffers,
// ratios of past to ordinary stores; Y, or dZ and H together, of 64 to 88, 110 to 165, 172 to 352 MB).
// Forward, with the product that follows: 2048 -> 5632 1.00 to 1.07, 1.00 to 1.03, 0.99 (16384 tokens 617, 609 us, 32768 1173, 1163); 1024 -> 4096 1.02 to 1.05, 0.99 to 1.05, 0.97 to
// 1.01; 768 -> 2048 1.00 to 1.05, 0.99 to 1.03, 0.96 to 0.98 (45056 tokens 345, 333).  Nothing kept: 0.99 to 1.04, 0.98 to 1.06, 0.96 to 1.04.
// Backward, with dX and the two weight gradients: D = 2048, F = 5632 1.00 to 1.02, 0.96 to 1.01, 0.99 to 1.03 (8192 tokens 633, 654; on another box 664, 657; 12288 993, 987);
// 1024, 4096 1.00 to 1.02, 1.01 to 1.03, 0.97 to 1.00; 768, 2048 1.06 to 1.10, 1.05 to 1.10, 1.00 to 1.05 (22528 tokens 434, 455): its products wait for what they read.  Without H 2048, 5632
// 1.02 to 1.04, 1.02 to 1.03, 0.98 to 1.02.  The call alone is 2 to 13 % faster past the caches.
bool stored_past(DenseOp op, int64_t M, int64_t N, int64_t K, int matrices) {
  return (uint64_t)M * (uint64_t)N * 2 * matrices >= (uint64_t)172 << 20 && (op == DenseOp::kFwd || K >= 1024);
}
int launch_dense(const GemmArgs& g, const DenseArgs& d, const DensePlan& p, DenseOp op, int w_is_nk, hipStream_t stream) {
  switch (p.form) {
    case GemmForm::kStream: return launch_dense_stream(g, d, op, w_is_nk, p.route.stream, stream);
    case GemmForm::kMiddle: return launch_dense128(g, d, op, w_is_nk, p.route.middle_nj, p.shared, stream);
    case GemmForm::kLarge:
    case GemmForm::kLargeEdge:
    case GemmForm::kNarrow: return launch_dense256(g, d, op, w_is_nk, p.form, stream);
    default: return launch_dense_any(g, d, op, w_is_nk, stream);
  }
}

// ---- AdamW ----
constexpr uint64_t kMaxWorkgroups = 0xFFFFFF;   // of 256 threads: a launch has fewer than 2^32
inline uint64_t norm_wgs(const gws_adamw_tensor& t) {
  return t.rows <= 0 || t.cols <= 0 ? 0 : ((uint64_t)t.rows * (((uint64_t)t.cols + 7) / 8) + kNormGroups - 1) / kNormGroups;
}
// Fours a row: of codes in whole blocks of 32.
inline uint64_t fours(const gws_adamw_tensor& t, bool codes) { return codes ? ((uint64_t)t.cols + 31) / 32 * 8 : ((uint64_t)t.cols + 3) / 4; }
int check_gradient(const gws_adamw_tensor& t) {
  if (!size_ok(t.rows) || !size_ok(t.cols)) return GWS_ERR_SHAPE;
  if (t.rows == 0 || t.cols == 0) return GWS_OK;
  if (!ld_ok(t.ld, t.cols) || norm_wgs(t) > kMaxWorkgroups) return GWS_ERR_SHAPE;
  if (!t.g) return GWS_ERR_NULL;
  return aligned(t.g, 16) ? GWS_OK : GWS_ERR_ALIGN;
}
inline Span2 gradient_span(const gws_adamw_tensor& t) {
  const size_t e = t.g_is_fp32 ? 4 : 2;
  return Span2{t.g, (size_t)t.rows, (size_t)t.cols * e, (size_t)t.ld * e};
}
int check_adamw(const gws_adamw_tensor& t, const float* grad_scale) {
  int rc = check_gradient(t);
  if (rc != GWS_OK || t.rows == 0 || t.cols == 0) return rc;
  const bool codes = t.m8.codes || t.v8.codes;
  if (codes && (t.m || t.v)) return GWS_ERR_FORMAT;
  if (!t.p) return GWS_ERR_NULL;
  if (!isfinite(t.lr_scale) || !isfinite(t.weight_decay)) return GWS_ERR_FORMAT;
  if ((uint64_t)t.rows * fours(t, codes) > kMaxWorkgroups * kAdamwGroups) return GWS_ERR_SHAPE;
  const size_t m = (size_t)t.rows, n = (size_t)t.cols, ld = (size_t)t.ld;
  Span2 out[6], in[2] = {gradient_span(t), span_f32(grad_scale, 1)};
  int outs = 0;
  if (codes) {
    if ((rc = check_act8(t.m8, t.rows, t.cols)) != GWS_OK || (rc = check_act8(t.v8, t.rows, t.cols)) != GWS_OK) return rc;
    if (t.m8.ldc != t.ld || t.v8.ldc != t.ld || t.m8.lds != t.v8.lds) return GWS_ERR_SHAPE;
    for (const gws_act8* s : {&t.m8, &t.v8}) {
      out[outs++] = Span2{s->codes, m, n, ld};
      out[outs++] = Span2{s->xscale, m, (n + 31) / 32, (size_t)s->lds};
    }
  } else {
    if (!t.m || !t.v) return GWS_ERR_NULL;
    if (!aligned(t.m, 16) || !aligned(t.v, 16)) return GWS_ERR_ALIGN;
    out[outs++] = Span2{t.m, m, n * 4, ld * 4};
    out[outs++] = Span2{t.v, m, n * 4, ld * 4};
  }
  if (!aligned(t.p, 16) || !aligned(t.w, 16)) return GWS_ERR_ALIGN;
  out[outs++] = Span2{t.p, m, n * 4, ld * 4};
  if (t.w) out[outs++] = Span2{t.w, m, n * 2, ld * 2};
  // whole ranges first: a model has hundreds of tensors, and matrices that lie between each other's rows are rare
  Range r[8];
  for (int i = 0; i < outs; ++i) r[i] = range_of(out[i]);
  r[outs] = range_of(in[0]);
  r[outs + 1] = range_of(in[1]);
  for (int i = 0; i < outs; ++i)
    for (int j = i + 1; j < outs + 2; ++j)
      if (!ranges_apart(r[i], r[j]) && !apart(out[i], j < outs ? out[j] : in[j - outs])) return GWS_ERR_ALIAS;
  return GWS_OK;
}

// Tensors in launches of as many as a list holds: add(descriptor, its workgroups), and finish() for the rest.
template <class List, class Launch>
struct Launches {
  List list;
  int held = 0;
  uint64_t wgs = 0;
  Launch launch;   // (list, workgroups)
  explicit Launches(Launch l) : launch(l) {}
  template <class Desc>
  int add(const Desc& d, uint64_t wc) {
    if (held == List::kMax || wgs + wc > kMaxWorkgroups) {
      const int rc = finish();
      if (rc != GWS_OK) return rc;
    }
    list.begin[held] = (uint32_t)wgs;
    list.t[held++] = d;
    wgs += wc;
    return GWS_OK;
  }
  int finish() {
    if (held == 0) return GWS_OK;
    for (int i = held; i < List::kMax; ++i) list.begin[i] = 0x7FFFFFFFu;
    const int rc = launch(list, (uint32_t)wgs);
    held = 0;
    wgs = 0;
    return rc;
  }
};
inline bool few_groups(uint64_t groups) { return groups + 0x100000 < ((uint64_t)1 << 32); }   // those past the end of the last workgroup too

// Buffers that a call has been given before: the starts of what it writes, as bits of a table, and only where a bit is set a look at the tensors so far.
class GivenBefore {
  uint64_t bits_[2048];
  bool set(const void* p) {
    const uint64_t h = ((uint64_t)(uintptr_t)p * 0x9E3779B97F4A7C15ull) >> 47;   // 17 bits
    const bool was = (bits_[h >> 6] >> (h & 63) & 1) != 0;
    bits_[h >> 6] |= (uint64_t)1 << (h & 63);
    return was;
  }
  struct Written {
    const void* at[6];
    explicit Written(const gws_adamw_tensor& t)
        : at{t.p, t.w, t.m8.codes ? t.m8.codes : t.m, t.v8.codes ? t.v8.codes : t.v, t.m8.codes ? t.m8.xscale : nullptr, t.v8.codes ? t.v8.xscale : nullptr} {}
  };

 public:
  GivenBefore() { memset(bits_, 0, sizeof bits_); }
  bool any(const gws_adamw_tensor* t, int i) {
    const gws_adamw_tensor& n = t[i];
    if (n.rows == 0 || n.cols == 0) return false;
    const Written mine(n);
    bool seen = false;
    for (const void* p : mine.at) seen |= p != nullptr && set(p);
    if (!seen) return false;
    for (int j = 0; j < i; ++j) {
      const gws_adamw_tensor& o = t[j];
      if (o.rows == 0 || o.cols == 0) continue;
      const Written theirs(o);
      for (const void* p : mine.at)
        for (const void* q : theirs.at)
          if (p != nullptr && p == q) return true;
    }
    return false;
  }
};

}  // namespace

// Tiles of 128 x 128, two workgroups a compute unit, in us: one's way out runs under the other's loop, where in the forms with one workgroup (and one wavefront a
// SIMD) it stands alone.  Rounds are of two tiles a compute unit; a last one of up to half is one tile each; many tiles go out of step.  Fitted to 151 sizes of 257
// to 1734 tiles, GELU with Z kept and the backward pass with H and the bias gradient, 5 % off in the root mean square.
static double shared_us(double M, double N, double K, DenseOp op) {
  const bool back = op == DenseOp::kBwd;
  const double cus = compute_units() > 0 ? compute_units() : 256, x = ceil(M / 128.0) * ceil(N / 128.0) / (2 * cus), nk = ceil(K / 64.0);
  const double rounds = ceil(x), last = x - (rounds - 1), both = fmax(0.0, 2 * last - 1), alone = fmin(1.0, 2 * last);
  const double start = back ? 8.2 : 5.6, full = back ? 9.3 + 0.85 * nk : 4.2 + 0.84 * nk;
  const double one = back ? 6.1 + nk * (0.41 + 0.27 * alone) : 2.1 + nk * (0.61 + 0.045 * alone);
  const double in_rounds = start + (rounds - 1 + both) * full + (1 - both) * one;
  return rounds <= 2 ? in_rounds : fmin(in_rounds, start + (x + 0.25) * (back ? 23.8 + 0.81 * nk : 14.6 + 0.80 * nk));
}
// What the way out adds to the plain product's estimate: a part a round (of `tn` columns a tile).
static double with_way_out(const GemmArgs& g, double us, double tm, double tn, double fixed, double a_round) {
  const double cus = compute_units() > 0 ? compute_units() : 256;
  return us + fixed + a_round * ceil(ceil(g.M / tm) * ceil(g.N / tn) / cus);
}

// The kernel that the plain product of these sizes takes, or two workgroups a compute unit where that is faster.  us of the plain product's kernel and of two, GELU,
// Z kept: 798 x 672 -> 5632 19.8, 16.2; 1118 x 352 -> 4864 17.5, 13.1; 1545 x 1728 -> 2848 29.6, 26.0; 5469 x 5632 -> 800 104, 70; 4911 x 896 -> 5632 65.5, 62.4;
// 7474 x 2304 -> 1504 54, 65; 8192 x 2048 -> 5632 160, 190; backward 5299 x 896 -> 1536 35.4, 28.1; 2381 x 288 -> 2528 25.7, 20.0; 3281 x 5632 -> 4320 135, 162.  Over 182
// drawn sizes of more than 200 tiles the choice is 1.02 of the fastest form (without two workgroups 1.10).
// Leading dimensions of outputs that the kernels' 32-bit lane offsets do not reach: the kernel for any sizes.
DensePlan plan_dense(const GemmArgs& g, const DenseArgs& d, DenseOp op, int w_is_nk) {
  DensePlan p;
  p.shared = false;
  p.form = gemm_form(g, w_is_nk, 0, p.route);
  const bool back = op == DenseOp::kBwd;
  double us = 0.0;
  switch (p.form) {
    case GemmForm::kStream: us = p.route.stream.us + (back ? 3.0 : 1.5); break;
    case GemmForm::kMiddle: us = with_way_out(g, p.route.middle_us, 128, 32 * p.route.middle_nj, back ? 0.9 : -1.8, back ? 6.1 : 4.0); break;
    case GemmForm::kLarge:
    case GemmForm::kLargeEdge: us = with_way_out(g, p.route.large_us, 256, 256, back ? -0.7 : -2.4, back ? 16.0 : 8.5); break;
    case GemmForm::kNarrow: us = with_way_out(g, p.route.narrow_us, 256, 192, back ? -2.6 : -4.7, back ? 16.0 : 10.3); break;
    default: break;
  }
  const double tiles = ceil(g.M / 128.0) * ceil(g.N / 128.0), cus = compute_units() > 0 ? compute_units() : 256;
  if (gemm128_applicable(g) && tiles > cus && shared_us(g.M, g.N, g.K, op) < 0.97 * us) {
    p.form = GemmForm::kMiddle;
    p.shared = true;
  }
  if (g.ldy >= kMaxLdOut || d.ldr >= kMaxLdOut || d.ldz >= kMaxLdOut || d.ldh >= kMaxLdOut) p.form = GemmForm::kAnyShape;
  switch (p.form) {
    case GemmForm::kStream: p.rows = (uint32_t)p.route.stream.bm; break;
    case GemmForm::kMiddle: p.rows = 64; break;
    case GemmForm::kLarge:
    case GemmForm::kLargeEdge:
    case GemmForm::kNarrow: p.rows = 128; break;
    default: p.rows = kDenseAnyRows;
  }
  return p;
}

}  // namespace gws

using namespace gws;

extern "C" {

int gws_norm_fwd(const void* x, int64_t M, int64_t C, int64_t ldx, int kind, const float* gamma, const float* beta, float eps, void* y, int64_t ldy,
                 float* mean, float* rstd, void* stream) {
  if (!size_ok(M) || !size_ok(C) || C == 0) return GWS_ERR_SHAPE;
  if (kind != GWS_NORM_LAYER && kind != GWS_NORM_RMS) return GWS_ERR_FORMAT;
  if (!(eps > 0.0f) || !isfinite(eps)) return GWS_ERR_FORMAT;
  if (M == 0) return GWS_OK;
  if (!ld_ok(ldx, C) || !ld_ok(ldy, C)) return GWS_ERR_SHAPE;
  if (!x || !y) return GWS_ERR_NULL;
  if (kind == GWS_NORM_LAYER ? (mean == nullptr) != (rstd == nullptr) : mean != nullptr) return GWS_ERR_NULL;
  if (!aligned(x, 16) || !aligned(y, 16) || !aligned(gamma, 4) || !aligned(beta, 4) || !aligned(mean, 4) || !aligned(rstd, 4)) return GWS_ERR_ALIGN;
  Buffers b;
  b.reads(span_f32(gamma, C));
  b.reads(span_f32(beta, C));
  b.writes(span_f32(mean, M));
  b.writes(span_f32(rstd, M));
  const Span2 in = span16(x, M, C, ldx), out = span16(y, M, C, ldy);
  if (!same_place(in, out)) b.reads(in);
  b.writes(out);
  if (!b.apart_all(false) || !apart(in, span_f32(mean, M)) || !apart(in, span_f32(rstd, M))) return GWS_ERR_ALIAS;
  NormArgs a;
  memset(&a, 0, sizeof a);
  a.x = (const uint16_t*)x; a.y = (uint16_t*)y;
  a.gamma = gamma; a.beta = beta; a.mean = mean; a.rstd = rstd;
  a.M = (uint32_t)M; a.C = (uint32_t)C; a.ldx = (uint32_t)ldx; a.ldy = (uint32_t)ldy;
  a.eps = eps;
  return launch_norm_fwd(a, kind == GWS_NORM_RMS, (hipStream_t)stream);
}

size_t gws_norm_bwd_workspace_bytes(int64_t M, int64_t C) {
  return !size_ok(M) || !size_ok(C) || M == 0 || C == 0 ? 0 : norm_bytes(M, C);
}

int gws_norm_bwd(const void* dy, int64_t lddy, const void* x, int64_t M, int64_t C, int64_t ldx, int kind, const float* gamma, const float* mean,
                 const float* rstd, const void* residual, int64_t ldr, void* dx, int64_t lddx, float* dgamma, float* dbeta, void* workspace,
                 size_t workspace_bytes, void* stream) {
  if (!size_ok(M) || !size_ok(C) || C == 0) return GWS_ERR_SHAPE;
  if (kind != GWS_NORM_LAYER && kind != GWS_NORM_RMS) return GWS_ERR_FORMAT;
  if (!aligned(dgamma, 4) || !aligned(dbeta, 4)) return GWS_ERR_ALIGN;
  if (!apart(span_f32(dgamma, C), span_f32(dbeta, C))) return GWS_ERR_ALIAS;
  if (M == 0) {
    int rc = dgamma ? launch_zero(dgamma, (uint64_t)C, (hipStream_t)stream) : GWS_OK;
    if (rc == GWS_OK && dbeta) rc = launch_zero(dbeta, (uint64_t)C, (hipStream_t)stream);
    return rc;
  }
  if (!ld_ok(ldx, C) || !ld_ok(lddy, C) || !ld_ok(lddx, C) || (residual && !ld_ok(ldr, C))) return GWS_ERR_SHAPE;
  if (!dy || !x || !dx || !rstd || (kind == GWS_NORM_LAYER && !mean)) return GWS_ERR_NULL;
  if (!aligned(x, 16) || !aligned(dy, 16) || !aligned(dx, 16) || !aligned(residual, 16) || !aligned(gamma, 4) || !aligned(mean, 4) || !aligned(rstd, 4))
    return GWS_ERR_ALIGN;
  const bool needed = dgamma || dbeta || norm_is_wide((uint64_t)C);
  const size_t need = needed ? norm_bytes(M, C) : 0;
  if (needed && !workspace) return GWS_ERR_NULL;
  if (needed && !aligned(workspace, 16)) return GWS_ERR_ALIGN;
  if (needed && workspace_bytes < need) return GWS_ERR_SHAPE;
  Buffers b, v;   // dX, which may lie on a matrix; and everything else
  const Span2 out = span16(dx, M, C, lddx);
  b.writes(out);
  for (const Span2& m : {span16(x, M, C, ldx), span16(dy, M, C, lddy), span16(residual, M, C, ldr)}) {
    b.reads(m);
    v.reads(m);
  }
  for (const Span2& m : {span_f32(gamma, C), span_f32(kind == GWS_NORM_LAYER ? mean : nullptr, M), span_f32(rstd, M)}) {
    v.reads(m);
    if (!apart(out, m)) return GWS_ERR_ALIAS;
  }
  for (const Span2& m : {span_f32(dgamma, C), span_f32(dbeta, C), span_bytes(needed ? workspace : nullptr, need)}) {
    v.writes(m);
    if (!apart(out, m)) return GWS_ERR_ALIAS;
  }
  if (!b.apart_all(true) || !v.apart_all(false)) return GWS_ERR_ALIAS;
  NormArgs a;
  memset(&a, 0, sizeof a);
  a.x = (const uint16_t*)x; a.dy = (const uint16_t*)dy; a.r = (const uint16_t*)residual; a.y = (uint16_t*)dx;
  a.gamma = gamma; a.mean = (float*)mean; a.rstd = (float*)rstd;
  a.M = (uint32_t)M; a.C = (uint32_t)C;
  a.ldx = (uint32_t)ldx; a.lddy = (uint32_t)lddy; a.ldr = (uint32_t)ldr; a.ldy = (uint32_t)lddx;
  a.want_gamma = dgamma != nullptr;
  a.want_beta = dbeta != nullptr;
  a.part = (float*)workspace;
  if (norm_is_wide((uint64_t)C)) a.rows = (float*)((char*)workspace + (need - (size_t)M * 2 * sizeof(float)));
  return launch_norm_bwd(a, kind == GWS_NORM_RMS, dgamma, dbeta, (hipStream_t)stream);
}

int gws_dense_fwd(const void* x, int64_t M, int64_t K, int64_t ldx, const void* w, int64_t N, int64_t ldw, int w_is_nk, void* y, int64_t ldy,
                  const gws_epilogue* e, void* stream) {
  if (!size_ok(M) || !size_ok(K) || !size_ok(N)) return GWS_ERR_SHAPE;
  if (!e) return GWS_ERR_NULL;
  if (!known_dense_act(e->act)) return GWS_ERR_FORMAT;
  if (M == 0 || N == 0) return GWS_OK;
  if (K == 0 || ((K | N) & 31) != 0) return GWS_ERR_SHAPE;
  if (!ld_ok(ldx, K) || !ld_ok(ldw, w_is_nk ? K : N) || !ld_ok(ldy, N)) return GWS_ERR_SHAPE;
  if ((e->residual && !ld_ok(e->ldr, N)) || (e->z && !ld_ok(e->ldz, N))) return GWS_ERR_SHAPE;
  if (!x || !w || !y) return GWS_ERR_NULL;
  if (!aligned(x, 16) || !aligned(w, 16) || !aligned(y, 16) || !aligned(e->residual, 16) || !aligned(e->z, 16) || !aligned(e->bias, 4)) return GWS_ERR_ALIGN;
  Buffers b;
  b.reads(span16(x, M, K, ldx));
  b.reads(w_is_nk ? span16(w, N, K, ldw) : span16(w, K, N, ldw));
  b.reads(span_f32(e->bias, N));
  const Span2 r = span16(e->residual, M, N, e->ldr), out = span16(y, M, N, ldy), z = span16(e->z, M, N, e->ldz);
  if (!same_place(r, out)) b.reads(r);
  b.writes(out);
  b.writes(z);
  if (!b.apart_all(false) || !apart(r, z)) return GWS_ERR_ALIAS;
  GemmArgs g;
  memset(&g, 0, sizeof g);
  g.x = (const uint16_t*)x; g.w = (const uint16_t*)w; g.y = (uint16_t*)y;
  g.M = (uint32_t)M; g.N = (uint32_t)N; g.K = (uint32_t)K;
  g.ldx = (uint32_t)ldx; g.ldw = (uint32_t)ldw; g.ldy = (uint32_t)ldy;
  if (!e->bias && !e->residual && !e->z && e->act == GWS_ACT_NONE) return launch_gemm(g, w_is_nk, 0, GWS_FMT_BF16, (hipStream_t)stream);
  DenseArgs d;
  memset(&d, 0, sizeof d);
  d.bias = e->bias;
  d.act = e->act;
  d.r = (const uint16_t*)e->residual; d.ldr = ld_of(e->residual, e->ldr);
  d.z = (uint16_t*)e->z; d.ldz = ld_of(e->z, e->ldz);
  d.past_caches = stored_past(DenseOp::kFwd, M, N, K, 1);
  return launch_dense(g, d, plan_dense(g, d, DenseOp::kFwd, w_is_nk), DenseOp::kFwd, w_is_nk, (hipStream_t)stream);
}

size_t gws_dense_bwd_workspace_bytes(int64_t M, int64_t F) { return !size_ok(M) || !size_ok(F) ? 0 : dense_bytes(M, F); }

int gws_dense_bwd(const void* dy, int64_t M, int64_t D, int64_t lddy, const void* wd, int64_t F, int64_t ldw, int w_is_nk, int act, const void* z,
                  int64_t ldz, void* dz, int64_t lddz, void* h, int64_t ldh, float* dbias, void* workspace, size_t workspace_bytes, void* stream) {
  if (!size_ok(M) || !size_ok(D) || !size_ok(F)) return GWS_ERR_SHAPE;
  if (!known_dense_act(act)) return GWS_ERR_FORMAT;
  if (F == 0) return GWS_OK;
  if (M == 0) return !dbias ? GWS_OK : !aligned(dbias, 4) ? GWS_ERR_ALIGN : launch_zero(dbias, (uint64_t)F, (hipStream_t)stream);
  if (D == 0 || ((D | F) & 31) != 0) return GWS_ERR_SHAPE;
  if (!ld_ok(lddy, D) || !ld_ok(ldw, w_is_nk ? F : D)) return GWS_ERR_SHAPE;
  if (!dy || !wd || !dz) return GWS_ERR_NULL;
  if (!aligned(dy, 16) || !aligned(wd, 16)) return GWS_ERR_ALIGN;
  GemmArgs g;
  DenseArgs d;
  memset(&g, 0, sizeof g);
  memset(&d, 0, sizeof d);
  Buffers own, in;   // outputs on Z at the very same place, and on nothing else
  int rc = dense_bwd_args(M, F, act, z, ldz, dz, lddz, h, ldh, dbias, workspace, workspace_bytes, g, d, own);
  if (rc != GWS_OK) return rc;
  in.reads(span16(dy, M, D, lddy));
  in.reads(w_is_nk ? span16(wd, D, F, ldw) : span16(wd, F, D, ldw));
  for (int i = 0; i < own.outs; ++i) in.writes(own.out[i]);
  if (!own.apart_all(true) || !in.apart_all(false)) return GWS_ERR_ALIAS;
  g.x = (const uint16_t*)dy; g.w = (const uint16_t*)wd;
  g.K = (uint32_t)D; g.ldx = (uint32_t)lddy; g.ldw = (uint32_t)ldw;
  const int nk = !w_is_nk;   // the product's columns are Wd's rows
  d.past_caches = stored_past(DenseOp::kBwd, M, F, D, h ? 2 : 1);
  const DensePlan p = plan_dense(g, d, DenseOp::kBwd, nk);
  return with_bias_gradient(g, d, p.rows, dbias, workspace, (hipStream_t)stream,
                            [&] { return launch_dense(g, d, p, DenseOp::kBwd, nk, (hipStream_t)stream); });
}

int gws_dense_bwd_h(const void* dh, int64_t M, int64_t F, int64_t lddh, int act, const void* z, int64_t ldz, void* dz, int64_t lddz, void* h,
                    int64_t ldh, float* dbias, void* workspace, size_t workspace_bytes, void* stream) {
  if (!size_ok(M) || !size_ok(F)) return GWS_ERR_SHAPE;
  if (!known_dense_act(act)) return GWS_ERR_FORMAT;
  if (F == 0) return GWS_OK;
  if (M == 0) return !dbias ? GWS_OK : !aligned(dbias, 4) ? GWS_ERR_ALIGN : launch_zero(dbias, (uint64_t)F, (hipStream_t)stream);
  if ((F & 7) != 0 || !ld_ok(lddh, F)) return GWS_ERR_SHAPE;
  if (!dh || (!dz && act != GWS_ACT_NONE)) return GWS_ERR_NULL;
  if (!aligned(dh, 16)) return GWS_ERR_ALIGN;
  GemmArgs g;
  DenseArgs d;
  memset(&g, 0, sizeof g);
  memset(&d, 0, sizeof d);
  Buffers b;
  int rc = dense_bwd_args(M, F, act, z, ldz, dz, lddz, h, ldh, dbias, workspace, workspace_bytes, g, d, b);
  if (rc != GWS_OK) return rc;
  b.reads(span16(dh, M, F, lddh));
  if (!b.apart_all(true)) return GWS_ERR_ALIAS;
  g.x = (const uint16_t*)dh; g.ldx = (uint32_t)lddh;
  return with_bias_gradient(g, d, dense_h_rows(g.M, g.N), dbias, workspace, (hipStream_t)stream, [&] { return launch_dense_bwd_h(g, d, (hipStream_t)stream); });
}

int gws_dense_form(int op, int64_t M, int64_t K, int64_t N, int64_t ldx, int64_t ldw, int w_is_nk) {
  if (op != GWS_DENSE_FWD && op != GWS_DENSE_BWD) return 0;
  if (!size_ok(M) || !size_ok(K) || !size_ok(N) || M == 0 || K == 0 || N == 0 || ((K | N) & 31) != 0) return 0;
  const int nk = op == GWS_DENSE_FWD ? w_is_nk != 0 : w_is_nk == 0;
  if (!ld_ok(ldx, K) || !ld_ok(ldw, nk ? K : N)) return 0;
  GemmArgs g;
  DenseArgs d;
  memset(&g, 0, sizeof g);
  memset(&d, 0, sizeof d);
  g.M = (uint32_t)M; g.N = (uint32_t)N; g.K = (uint32_t)K;
  g.ldx = (uint32_t)ldx; g.ldw = (uint32_t)ldw; g.ldy = (uint32_t)N;
  const DensePlan p = plan_dense(g, d, op == GWS_DENSE_FWD ? DenseOp::kFwd : DenseOp::kBwd, nk);
  return p.shared && p.form == GemmForm::kMiddle ? GWS_DENSE_SHARED : (int)p.form;
}

int gws_adamw(const gws_adamw_tensor* t, int n, const gws_adamw_settings* s, void* stream) {
  if (n < 0) return GWS_ERR_SHAPE;
  if (!s) return GWS_ERR_NULL;
  if (!isfinite(s->lr) || !isfinite(s->eps) || !((float)s->eps > 0.0f) || !(s->beta1 >= 0.0 && s->beta1 < 1.0) || !(s->beta2 >= 0.0 && s->beta2 < 1.0) || s->step == 0)
    return GWS_ERR_FORMAT;
  if (!aligned(s->grad_scale, 4)) return GWS_ERR_ALIGN;
  if (n == 0) return GWS_OK;
  if (!t) return GWS_ERR_NULL;
  GivenBefore before;
  for (int i = 0; i < n; ++i) {
    const int rc = check_adamw(t[i], s->grad_scale);
    if (rc != GWS_OK) return rc;
    if (before.any(t, i)) return GWS_ERR_ALIAS;
  }
  const double c1 = 1.0 - pow(s->beta1, (double)s->step), c2 = 1.0 - pow(s->beta2, (double)s->step);
  const AdamwStep a = {(float)s->beta1, (float)(1.0 - s->beta1), (float)s->beta2, (float)(1.0 - s->beta2), (float)(1.0 / sqrt(c2)), (float)s->eps,
                       (uint32_t)s->step, (uint32_t)(s->step >> 32), s->grad_scale};
  auto runs_launch = [&](const AdamwRuns& l, uint32_t wgs) { return launch_adamw_runs(l, a, wgs, (hipStream_t)stream); };
  auto matrices_launch = [&](const AdamwMatrices& l, uint32_t wgs) {
    bool with = false, without = false;
    for (int i = 0; i < AdamwMatrices::kMax && l.begin[i] != 0x7FFFFFFFu; ++i) (l.t[i].form & kCodes ? with : without) = true;
    return launch_adamw_matrices(l, a, wgs, !with ? 0 : without ? 1 : 2, (hipStream_t)stream);
  };
  Launches<AdamwRuns, decltype(runs_launch)> runs(runs_launch);
  Launches<AdamwMatrices, decltype(matrices_launch)> matrices(matrices_launch);
  for (int i = 0; i < n; ++i) {
    const gws_adamw_tensor& o = t[i];
    if (o.rows == 0 || o.cols == 0) continue;
    const double lr = s->lr * o.lr_scale;
    const float keep = (float)(1.0 - lr * o.weight_decay), rate = (float)(lr / c1);
    int rc;
    if (!o.m8.codes && (o.rows == 1 || o.cols == o.ld)) {
      const uint64_t elements = (uint64_t)o.rows * (uint64_t)o.cols;
      rc = runs.add(AdamwRun{o.p, (uint16_t*)o.w, o.g, o.m, o.v, elements | (o.g_is_fp32 ? kRunGradFp32 : 0), keep, rate}, (elements + 4 * kAdamwGroups - 1) / (4 * kAdamwGroups));
    } else {
      const bool codes = o.m8.codes != nullptr;
      const uint32_t per_row = (uint32_t)fours(o, codes);
      const uint64_t groups = (uint64_t)o.rows * per_row;
      rc = matrices.add(AdamwMatrix{o.p, (uint16_t*)o.w, o.g, codes ? o.m8.codes : o.m, codes ? o.v8.codes : o.v, o.m8.xscale, o.v8.xscale, (uint32_t)o.rows, (uint32_t)o.cols,
                                    (uint32_t)o.ld, (uint32_t)o.m8.lds, keep, rate, (uint32_t)o.seed, (uint32_t)(o.seed >> 32), per_row, reciprocal(per_row),
                                    (o.g_is_fp32 ? kGradFp32 : 0) | (codes ? kCodes : 0) | (few_groups(groups) ? kFewGroups : 0), 0},
                        (groups + kAdamwGroups - 1) / kAdamwGroups);
    }
    if (rc != GWS_OK) return rc;
  }
  const int rc = runs.finish();
  return rc != GWS_OK ? rc : matrices.finish();
}

size_t gws_grad_norm_workspace_bytes(const gws_adamw_tensor* t, int n) {
  uint64_t wgs = 0;
  for (int i = 0; t && i < n; ++i) wgs += norm_wgs(t[i]);
  return (size_t)(wgs * sizeof(double) + 15) & ~(size_t)15;
}

int gws_grad_norm(const gws_adamw_tensor* t, int n, double max_norm, float* out, void* workspace, size_t workspace_bytes, void* stream) {
  if (n < 0) return GWS_ERR_SHAPE;
  if (!out || (n > 0 && !t)) return GWS_ERR_NULL;
  if (!aligned(out, 4)) return GWS_ERR_ALIGN;
  if (!(max_norm <= 0.0) && !isfinite(max_norm)) return GWS_ERR_FORMAT;
  for (int i = 0; i < n; ++i) {
    const int rc = check_gradient(t[i]);
    if (rc != GWS_OK) return rc;
  }
  const size_t need = gws_grad_norm_workspace_bytes(t, n);
  if (need && !workspace) return GWS_ERR_NULL;
  if (need && !aligned(workspace, 16)) return GWS_ERR_ALIGN;
  if (need && workspace_bytes < need) return GWS_ERR_SHAPE;
  const Span2 ws = span_bytes(need ? workspace : nullptr, need), to = span_f32(out, 2);
  if (!apart(ws, to)) return GWS_ERR_ALIAS;
  const Range rw = range_of(ws), ro = range_of(to);
  for (int i = 0; i < n; ++i) {
    if (t[i].rows == 0 || t[i].cols == 0) continue;
    const Range r = range_of(gradient_span(t[i]));
    if ((!ranges_apart(r, rw) && !apart(gradient_span(t[i]), ws)) || (!ranges_apart(r, ro) && !apart(gradient_span(t[i]), to))) return GWS_ERR_ALIAS;
  }
  double* part = (double*)workspace;
  auto launch = [&](const GradList& l, uint32_t wgs) {
    const int r = launch_grad_squares(l, part, wgs, (hipStream_t)stream);
    part += wgs;
    return r;
  };
  Launches<GradList, decltype(launch)> list(launch);
  for (int i = 0; i < n; ++i) {
    if (t[i].rows == 0 || t[i].cols == 0) continue;
    const uint32_t rows = (uint32_t)t[i].rows, cols = (uint32_t)t[i].cols, per_row = (uint32_t)(((uint64_t)cols + 7) / 8);
    const int rc = list.add(GradSquares{t[i].g, rows | (t[i].g_is_fp32 ? kHighBit : 0), cols | (few_groups((uint64_t)rows * per_row) ? kHighBit : 0), (uint32_t)t[i].ld,
                                        reciprocal(per_row)}, norm_wgs(t[i]));
    if (rc != GWS_OK) return rc;
  }
  const int rc = list.finish();
  return rc != GWS_OK ? rc : launch_grad_norm((const double*)workspace, (uint64_t)(part - (double*)workspace), max_norm, out, (hipStream_t)stream);
}

}  // extern "C"
