// C ABI of the gated feed-forward block and of activations kept in 8 bits: argument checks and the choice of kernel.
// Declarations and the meaning of every argument are in include/gws.h.
#include <math.h>
#include <string.h>

#include "gws_bench.h"
#include "gws_check.h"
#include "gws_gated.h"

namespace gws {

namespace {

constexpr int64_t kMaxDim = (int64_t)1 << 31;

inline bool size_ok(int64_t n) { return n >= 0 && n < kMaxDim; }
// A BF16 matrix's leading dimension.
inline bool ld_ok(int64_t ld, int64_t cols) { return ld >= cols && ld < kMaxDim && (ld & 7) == 0; }
inline Span2 span16(const void* p, int64_t rows, int64_t cols, int64_t ld) { return Span2{p, (size_t)rows, (size_t)cols * 2, (size_t)ld * 2}; }
inline bool same_place(const Span2& a, const Span2& b) { return a.p == b.p && a.pitch == b.pitch; }

int check_act8(const gws_act8& a, int64_t M, int64_t C) {
  if (!a.codes || !a.xscale) return GWS_ERR_NULL;
  if (a.ldc < C || a.ldc >= kMaxDim || (a.ldc & 7) != 0 || a.lds < (C + 31) / 32 || a.lds >= kMaxDim) return GWS_ERR_SHAPE;
  return aligned(a.codes, 8) ? GWS_OK : GWS_ERR_ALIGN;
}

// A list of matrices of which some are written.
struct Buffers {
  Span2 in[8], out[8];
  int ins = 0, outs = 0;
  void reads(const Span2& s) { if (s.p) in[ins++] = s; }
  void writes(const Span2& s) { if (s.p) out[outs++] = s; }
  // No output on another one; none on an input, but for the ones at the very same place where `in_place` allows those.
  bool apart_all(bool in_place) const {
    for (int i = 0; i < outs; ++i) {
      for (int j = 0; j < i; ++j)
        if (!apart(out[i], out[j])) return false;
      for (int j = 0; j < ins; ++j)
        if (!apart(out[i], in[j]) && !(in_place && same_place(out[i], in[j]))) return false;
    }
    return true;
  }
};

// G and U as they are kept; `optional`: NULL keeps nothing.
int kept_args(const gws_gated_saved* s, int64_t M, int64_t F, bool optional, Kept& form, KeptArgs& k) {
  memset(&k, 0, sizeof k);
  form = Kept::kNone;
  if (!s) return optional ? GWS_OK : GWS_ERR_NULL;
  if (s->g || s->u) {
    if (!s->g || !s->u) return GWS_ERR_NULL;
    if (s->g8.codes || s->g8.xscale || s->u8.codes || s->u8.xscale) return GWS_ERR_FORMAT;   // one form or the other
    if (!ld_ok(s->ldg, F) || !ld_ok(s->ldu, F)) return GWS_ERR_SHAPE;
    if (!aligned(s->g, 16) || !aligned(s->u, 16)) return GWS_ERR_ALIGN;
    k = KeptArgs{(uint8_t*)s->g, (uint8_t*)s->u, nullptr, nullptr, (uint32_t)s->ldg, (uint32_t)s->ldu, 0, 0};
    form = Kept::kBf16;
    return GWS_OK;
  }
  int rc = check_act8(s->g8, M, F);
  if (rc == GWS_OK) rc = check_act8(s->u8, M, F);
  if (rc != GWS_OK) return rc;
  k = KeptArgs{(uint8_t*)s->g8.codes, (uint8_t*)s->u8.codes, s->g8.xscale, s->u8.xscale,
               (uint32_t)s->g8.ldc, (uint32_t)s->u8.ldc, (uint32_t)s->g8.lds, (uint32_t)s->u8.lds};
  form = Kept::kE4m3;
  return GWS_OK;
}
void kept_buffers(const KeptArgs& k, Kept form, int64_t M, int64_t F, bool written, Buffers& b) {
  const size_t e = form == Kept::kBf16 ? 2 : 1, m = (size_t)M, w = (size_t)F * e, blocks = (size_t)(F / 32);
  const Span2 all[4] = {{k.g, m, w, k.ldg * e}, {k.u, m, w, k.ldu * e}, {k.gs, m, blocks, k.lsg}, {k.us, m, blocks, k.lsu}};
  for (const Span2& s : all) {
    if (written) b.writes(s);
    else b.reads(s);
  }
}

// The kernel by the sizes: the fastest by estimates in us, each a launch and, per round of workgroups (one per compute unit), what a tile takes
// beside its K-steps, the gate and the kept values among it, and the K-steps of 64, which take longer the more compute units are at work (busy).
// Measured and estimated, in 256 x 256 tiles and in 128 x 128:
//   forward, nothing kept: 1021 x 768 -> 2048 20.7, 20.3 and 9.9, 10.2; 256 x 2048 -> 5632 39.4, 37.7 and 17.3, 17.7; 2048 x 2048 -> 5632 87, 90
//   and 97, 97; 8192 x 2048 -> 5632 291, 267 and 420, 348
//   backward, BF16 kept: 1021 x 768 -> 2048 39, 41 and 14.5, 16.9; 3000 x 1024 -> 4096 62, 54 and 54, 54; 8192 x 2048 -> 5632 213, 223 and 306, 262
//   input gradient: 5000 x 2 x 1280 -> 640 51, 50 and 21.7, 23.7; 2048 x 2 x 5632 -> 2048 192, 207 and 100, 99; 8192 x 2 x 5632 -> 2048 263, 262
enum class GatedForm { kAny = GWS_GATED_ANY, kStream = GWS_GATED_STREAM, kMiddle = GWS_GATED_MIDDLE, kLarge = GWS_GATED_LARGE, kShared = GWS_GATED_SHARED };
GatedForm gated_form(const GatedArgs& g, GatedOp op, bool b_oc, Kept kept, GatedStreamPlan& plan) {
  plan = gated_stream_plan(g, op, b_oc, kept);
  const double cus = compute_units() > 0 ? compute_units() : 256, nk = ceil(g.K / 64.0) * (op == GatedOp::kDx ? 2 : 1);
  const bool keeps = op == GatedOp::kFwd && kept != Kept::kNone;
  double large = 1e30, middle = 1e30, shared = 1e30;
  if (gated256_applicable(g)) {
    const double n = ceil(g.M / 256.0) * ceil(g.N / (op == GatedOp::kFwd ? 128.0 : 256.0)), busy = n / (ceil(n / cus) * cus);
    const double beside = op == GatedOp::kBwd ? 20.0 + 9.0 * busy : keeps ? 12.0 : 6.5;
    const double step = op == GatedOp::kDx ? 1.03 + 0.42 * busy : 0.875 + 0.3 * busy;
    large = 2.5 + ceil(n / cus) * (beside + nk * step);
  }
  if (gated128_applicable(g)) {
    const double n = ceil(g.M / 128.0) * ceil(g.N / (op == GatedOp::kFwd ? 64.0 : 128.0)), busy = n / (ceil(n / cus) * cus);
    const double beside = op == GatedOp::kBwd ? 8.0 + 2.5 * busy : keeps ? 5.6 : 2.6;
    const double step = op == GatedOp::kDx ? 0.35 + 0.18 * busy * busy : 0.34 + 0.07 * busy;
    middle = 2.7 + ceil(n / cus) * (beside + nk * step);
    if (n > cus && op != GatedOp::kDx) {   // two workgroups a compute unit
      const double both = n / (ceil(n / (2 * cus)) * 2 * cus), way_out = op == GatedOp::kBwd ? 3.0 + 13.0 * both : keeps ? 6.5 : 3.0;
      shared = 2.7 + ceil(n / (2 * cus)) * (way_out + nk * (0.5 + 0.3 * both));
    }
  }
  const double best = fmin(large, fmin(middle, shared));
  if (plan.p > 0 && plan.us < best) return GatedForm::kStream;
  if (best > 1e29) return GatedForm::kAny;
  return best == large ? GatedForm::kLarge : best == shared ? GatedForm::kShared : GatedForm::kMiddle;
}

int launch_gated(const GatedArgs& g, GatedOp op, bool b_oc, Kept kept, hipStream_t stream) {
  GatedStreamPlan plan;
  switch (gated_form(g, op, b_oc, kept, plan)) {
    case GatedForm::kStream: return launch_gated_stream(g, op, b_oc, kept, plan, stream);
    case GatedForm::kMiddle: return launch_gated128(g, op, b_oc, kept, false, stream);
    case GatedForm::kShared: return launch_gated128(g, op, b_oc, kept, true, stream);
    case GatedForm::kLarge: return launch_gated256(g, op, b_oc, kept, stream);
    default: return launch_gated_any(g, op, b_oc, kept, stream);
  }
}

}  // namespace
}  // namespace gws

using namespace gws;

extern "C" {

int gws_act8_encode(const void* x, int64_t M, int64_t C, int64_t ldx, const gws_act8* o, void* stream) {
  if (!size_ok(M) || !size_ok(C)) return GWS_ERR_SHAPE;
  if (M == 0 || C == 0) return GWS_OK;
  if (!x || !o) return GWS_ERR_NULL;
  if (!ld_ok(ldx, C)) return GWS_ERR_SHAPE;
  const int rc = check_act8(*o, M, C);
  if (rc != GWS_OK) return rc;
  if (!aligned(x, 16)) return GWS_ERR_ALIGN;
  Buffers b;
  b.reads(span16(x, M, C, ldx));
  b.writes(Span2{o->codes, (size_t)M, (size_t)C, (size_t)o->ldc});
  b.writes(Span2{o->xscale, (size_t)M, (size_t)((C + 31) / 32), (size_t)o->lds});
  if (!b.apart_all(false)) return GWS_ERR_ALIAS;
  return launch_act8(true, x, (uint64_t)M, (uint64_t)C, (uint64_t)ldx, *o, (hipStream_t)stream);
}

int gws_act8_decode(const gws_act8* a, int64_t M, int64_t C, void* x, int64_t ldx, void* stream) {
  if (!size_ok(M) || !size_ok(C)) return GWS_ERR_SHAPE;
  if (M == 0 || C == 0) return GWS_OK;
  if (!x || !a) return GWS_ERR_NULL;
  if (!ld_ok(ldx, C)) return GWS_ERR_SHAPE;
  const int rc = check_act8(*a, M, C);
  if (rc != GWS_OK) return rc;
  if (!aligned(x, 16)) return GWS_ERR_ALIGN;
  Buffers b;
  b.writes(span16(x, M, C, ldx));
  b.reads(Span2{a->codes, (size_t)M, (size_t)C, (size_t)a->ldc});
  b.reads(Span2{a->xscale, (size_t)M, (size_t)((C + 31) / 32), (size_t)a->lds});
  if (!b.apart_all(false)) return GWS_ERR_ALIAS;
  return launch_act8(false, x, (uint64_t)M, (uint64_t)C, (uint64_t)ldx, *a, (hipStream_t)stream);
}

int gws_gated_fwd(const void* x, int64_t M, int64_t K, int64_t ldx, const void* wg, const void* wu, int64_t F, int64_t ldw,
                  int w_is_nk, int act, void* h, int64_t ldh, const gws_gated_saved* saved, void* stream) {
  if (!size_ok(M) || !size_ok(K) || !size_ok(F)) return GWS_ERR_SHAPE;
  GatedArgs g;
  memset(&g, 0, sizeof g);
  if (!known_act(act)) return GWS_ERR_FORMAT;
  g.act = act;
  if (M == 0 || F == 0) return GWS_OK;
  if (K == 0 || ((K | F) & 31) != 0) return GWS_ERR_SHAPE;
  if (!ld_ok(ldx, K) || !ld_ok(ldw, w_is_nk ? K : F) || !ld_ok(ldh, F)) return GWS_ERR_SHAPE;
  if (!x || !wg || !wu || !h) return GWS_ERR_NULL;
  if (!aligned(x, 16) || !aligned(wg, 16) || !aligned(wu, 16) || !aligned(h, 16)) return GWS_ERR_ALIGN;
  Kept form;
  const int rc = kept_args(saved, M, F, true, form, g.kept);
  if (rc != GWS_OK) return rc;
  Buffers b;
  b.reads(span16(x, M, K, ldx));
  b.reads(w_is_nk ? span16(wg, F, K, ldw) : span16(wg, K, F, ldw));
  b.reads(w_is_nk ? span16(wu, F, K, ldw) : span16(wu, K, F, ldw));
  b.writes(span16(h, M, F, ldh));
  kept_buffers(g.kept, form, M, F, true, b);
  if (!b.apart_all(false)) return GWS_ERR_ALIAS;
  g.a = (const uint16_t*)x; g.b = (const uint16_t*)wg; g.b2 = (const uint16_t*)wu;
  g.M = (uint32_t)M; g.N = (uint32_t)F; g.K = (uint32_t)K;
  g.lda = (uint32_t)ldx; g.ldb = (uint32_t)ldw;
  g.h = (uint16_t*)h; g.ldh = (uint32_t)ldh;
  g.stream_h = (uint64_t)M * (uint64_t)F * 2 >= (uint64_t)64 << 20;
  return launch_gated(g, GatedOp::kFwd, !w_is_nk, form, (hipStream_t)stream);
}

// What the two forms of the gate's backward pass share: outputs and kept values.
static int bwd_args(int64_t M, int64_t F, const gws_gated_saved* saved, void* dg, void* du, int64_t ldd, void* h, int64_t ldh,
                    Kept& form, GatedArgs& g, Buffers& b) {
  if (!dg || !du) return GWS_ERR_NULL;
  if (!ld_ok(ldd, F) || (h && !ld_ok(ldh, F))) return GWS_ERR_SHAPE;
  if (!aligned(dg, 16) || !aligned(du, 16) || !aligned(h, 16)) return GWS_ERR_ALIGN;
  const int rc = kept_args(saved, M, F, false, form, g.kept);
  if (rc != GWS_OK) return rc;
  g.M = (uint32_t)M; g.N = (uint32_t)F;
  g.dg = (uint16_t*)dg; g.du = (uint16_t*)du; g.h = (uint16_t*)h;
  g.ldd = (uint32_t)ldd; g.ldh = (uint32_t)ldh;
  b.writes(span16(dg, M, F, ldd));
  b.writes(span16(du, M, F, ldd));
  b.writes(span16(h, M, F, ldh));
  return GWS_OK;
}

int gws_gated_bwd(const void* dy, int64_t M, int64_t D, int64_t lddy, const void* wd, int64_t F, int64_t ldw, int w_is_nk, int act,
                  const gws_gated_saved* saved, void* dg, void* du, int64_t ldd, void* h, int64_t ldh, void* stream) {
  if (!size_ok(M) || !size_ok(D) || !size_ok(F)) return GWS_ERR_SHAPE;
  GatedArgs g;
  memset(&g, 0, sizeof g);
  if (!known_act(act)) return GWS_ERR_FORMAT;
  g.act = act;
  if (M == 0 || F == 0) return GWS_OK;
  if (D == 0 || ((D | F) & 31) != 0) return GWS_ERR_SHAPE;
  if (!ld_ok(lddy, D) || !ld_ok(ldw, w_is_nk ? F : D)) return GWS_ERR_SHAPE;
  if (!dy || !wd) return GWS_ERR_NULL;
  if (!aligned(dy, 16) || !aligned(wd, 16)) return GWS_ERR_ALIGN;
  Kept form;
  Buffers b, k;
  const int rc = bwd_args(M, F, saved, dg, du, ldd, h, ldh, form, g, b);
  if (rc != GWS_OK) return rc;
  // a workgroup reads the kept values where it writes the gradients: those may lie at the very same place, the operands not
  k = b;
  kept_buffers(g.kept, form, M, F, false, k);
  b.reads(span16(dy, M, D, lddy));
  b.reads(w_is_nk ? span16(wd, D, F, ldw) : span16(wd, F, D, ldw));
  if (!k.apart_all(form == Kept::kBf16) || !b.apart_all(false)) return GWS_ERR_ALIAS;
  g.a = (const uint16_t*)dy; g.b = (const uint16_t*)wd;
  g.K = (uint32_t)D;
  g.lda = (uint32_t)lddy; g.ldb = (uint32_t)ldw;
  return launch_gated(g, GatedOp::kBwd, w_is_nk != 0, form, (hipStream_t)stream);   // contraction over D: [D x F] lies across it
}

int gws_gated_bwd_h(const void* dh, int64_t M, int64_t F, int64_t lddh, int act, const gws_gated_saved* saved, void* dg, void* du,
                    int64_t ldd, void* h, int64_t ldh, void* stream) {
  if (!size_ok(M) || !size_ok(F)) return GWS_ERR_SHAPE;
  GatedArgs g;
  memset(&g, 0, sizeof g);
  if (!known_act(act)) return GWS_ERR_FORMAT;
  g.act = act;
  if (M == 0 || F == 0) return GWS_OK;
  if ((F & 31) != 0 || !ld_ok(lddh, F)) return GWS_ERR_SHAPE;
  if (!dh) return GWS_ERR_NULL;
  if (!aligned(dh, 16)) return GWS_ERR_ALIGN;
  Kept form;
  Buffers b;
  const int rc = bwd_args(M, F, saved, dg, du, ldd, h, ldh, form, g, b);
  if (rc != GWS_OK) return rc;
  Buffers k = b;
  kept_buffers(g.kept, form, M, F, false, k);
  b.reads(span16(dh, M, F, lddh));
  if (!k.apart_all(form == Kept::kBf16) || !b.apart_all(true)) return GWS_ERR_ALIAS;   // element by element: in place
  g.a = (const uint16_t*)dh;
  g.lda = (uint32_t)lddh;
  return launch_gated_bwd_h(g, form, (hipStream_t)stream);
}

int gws_gated_bwd_x(const void* dg, const void* du, int64_t M, int64_t F, int64_t ldd, const void* wg, const void* wu, int64_t K,
                    int64_t ldw, int w_is_nk, void* dx, int64_t ldx, void* stream) {
  if (!size_ok(M) || !size_ok(K) || !size_ok(F)) return GWS_ERR_SHAPE;
  if (M == 0 || K == 0) return GWS_OK;
  if (F == 0 || ((K | F) & 31) != 0) return GWS_ERR_SHAPE;
  if (!ld_ok(ldd, F) || !ld_ok(ldw, w_is_nk ? K : F) || !ld_ok(ldx, K)) return GWS_ERR_SHAPE;
  if (!dg || !du || !wg || !wu || !dx) return GWS_ERR_NULL;
  if (!aligned(dg, 16) || !aligned(du, 16) || !aligned(wg, 16) || !aligned(wu, 16) || !aligned(dx, 16)) return GWS_ERR_ALIGN;
  Buffers b;
  b.reads(span16(dg, M, F, ldd));
  b.reads(span16(du, M, F, ldd));
  b.reads(w_is_nk ? span16(wg, F, K, ldw) : span16(wg, K, F, ldw));
  b.reads(w_is_nk ? span16(wu, F, K, ldw) : span16(wu, K, F, ldw));
  b.writes(span16(dx, M, K, ldx));
  if (!b.apart_all(false)) return GWS_ERR_ALIAS;
  GatedArgs g;
  memset(&g, 0, sizeof g);
  g.a = (const uint16_t*)dg; g.a2 = (const uint16_t*)du; g.b = (const uint16_t*)wg; g.b2 = (const uint16_t*)wu;
  g.M = (uint32_t)M; g.N = (uint32_t)K; g.K = (uint32_t)F;
  g.lda = (uint32_t)ldd; g.ldb = (uint32_t)ldw;
  g.h = (uint16_t*)dx; g.ldh = (uint32_t)ldx;
  return launch_gated(g, GatedOp::kDx, w_is_nk != 0, Kept::kNone, (hipStream_t)stream);   // contraction over F: [F x K] lies across it
}

int gws_gated_form(int op, int64_t M, int64_t K, int64_t F, int64_t lda, int64_t ldw, int w_is_nk, int kept) {
  if (op < 0 || op > 2 || kept < 0 || kept > 2 || (op == GWS_GATED_BWD && kept == 0) || M <= 0 || K <= 0 || F <= 0 || ((K | F) & 31) != 0 ||
      !size_ok(M) || !size_ok(K) || !size_ok(F) || !ld_ok(lda, op == GWS_GATED_BWD_X ? F : K) ||
      !ld_ok(ldw, op == GWS_GATED_BWD ? (w_is_nk ? F : K) : (w_is_nk ? K : F))) return 0;
  GatedArgs g;
  memset(&g, 0, sizeof g);
  g.M = (uint32_t)M;
  g.N = (uint32_t)(op == GWS_GATED_BWD_X ? K : F);
  g.K = (uint32_t)(op == GWS_GATED_BWD_X ? F : K);
  g.lda = (uint32_t)lda;
  g.ldb = (uint32_t)ldw;
  GatedStreamPlan plan;
  const GatedOp o = op == GWS_GATED_FWD ? GatedOp::kFwd : op == GWS_GATED_BWD ? GatedOp::kBwd : GatedOp::kDx;
  const GatedForm form = gated_form(g, o, op == GWS_GATED_FWD ? !w_is_nk : w_is_nk != 0, o == GatedOp::kDx ? Kept::kNone : (Kept)kept, plan);
  return (int)form | (form == GatedForm::kStream ? plan.mt << 16 | plan.nt << 8 : 0);
}

}  // extern "C"
