// C ABI of the gated feed-forward block and of activations kept in 8 bits: argument checks and the choice of kernel.
// Declarations and the meaning of every argument are in include/gws.h.
#include <math.h>
#include <string.h>

#include "gws_bench.h"
#include "gws_check.h"
#include "gws_gated.h"

namespace gws {

namespace {

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

// The kernel by the sizes: the fastest by estimates in us, each a launch and, per round of workgroups, what a tile takes beside its K-steps,
// the gate and the kept values among it, and the K-steps of 64, which take longer the more compute units are at work (busy).  Of 100 drawn
// sizes of more than 256 tiles of 128 x 128 the choice takes at worst 1.09 of the fastest single launch's time, in the mean, two launches
// included, 0.99; of 40 backward passes with D under 1024 1.12 and 1.02, of 24 forward passes with H of 64 to 172 MB 1.04 and 0.99.  Measured with the sums in 256 x 256 tiles, in 128 x 128, and in those two workgroups a compute unit:
//   forward, nothing kept: 1021 x 768 -> 2048 20.6, 10.0, 11.7; 2048 x 2048 -> 5632 87, 99, 84; 8192 x 2048 -> 5632 289, 424, 359
//   forward, 8 bits kept: 8192 x 2048 -> 5632 320, 478, 402; BF16 kept: 4096 x 768 -> 2048 31.2, 36.4, 31.4
//   backward, BF16 kept: 1021 x 768 -> 2048 35.5, 16.2, 17.7 (8 x 4 of the streaming kernel: 13.1); 3000 x 1024 -> 4096 51, 57, 55
//   backward, 8 bits kept: 4096 x 768 -> 2048 38.8, 35.0, 27.8; 8192 x 2048 -> 5632 201, 261, 227
//   input gradient (no third form): 5000 x 2 x 1280 -> 640 51, 22.7; 2048 x 2 x 5632 -> 2048 197, 102; 8192 x 2 x 5632 -> 2048 266, 387
enum class GatedForm { kAny = GWS_GATED_ANY, kStream = GWS_GATED_STREAM, kMiddle = GWS_GATED_MIDDLE, kLarge = GWS_GATED_LARGE, kShared = GWS_GATED_SHARED };
struct GatedPlan {
  GatedForm form;
  GatedStreamPlan stream;
  double us;
};
// The tiles of a form: rows and columns of one, and how many are at work together.
struct Tiles {
  uint32_t rows, cols;
  double together;
};
double units() { return compute_units() > 0 ? compute_units() : 256; }
Tiles tiles_of(GatedForm form, GatedOp op) {
  const uint32_t half = op == GatedOp::kFwd ? 2 : 1;   // of a pair of weights the tile has half of its columns of each
  return form == GatedForm::kLarge ? Tiles{256, 256 / half, units()} : Tiles{128, 128 / half, units() * (form == GatedForm::kShared ? 2.0 : 1.0)};
}
double form_us(const GatedArgs& g, GatedOp op, Kept kept, GatedForm form) {
  if (form == GatedForm::kLarge ? !gated256_applicable(g) : !gated128_applicable(g)) return 1e30;
  const Tiles t = tiles_of(form, op);
  // n tiles in rounds, of which the last may leave compute units idle
  const double n = ceil(g.M / (double)t.rows) * ceil(g.N / (double)t.cols), rounds = ceil(n / t.together), busy = n / (rounds * t.together);
  const double nk = ceil(g.K / 64.0) * (op == GatedOp::kDx ? 2 : 1);
  const bool keeps = op == GatedOp::kFwd && kept != Kept::kNone, back = op == GatedOp::kBwd, two = op == GatedOp::kDx;
  if (form == GatedForm::kLarge) return 2.5 + rounds * ((back ? 22.0 + 13.0 * busy : keeps ? 12.0 : 6.5) + nk * (two ? 1.03 + 0.42 * busy : 0.875 + 0.3 * busy));
  const double off_lines = (g.lda & 63) != 0 ? 1.1 : 1.0;   // rows of 128-byte pieces on two lines each
  auto round_us = [&](double f) {   // of 128 x 128 tiles, f of the compute units with one each
    return (back ? 8.0 + 2.5 * f : keeps ? 5.6 : 2.6) + nk * (two ? (0.35 + 0.18 * f * f) * off_lines : 0.34 + 0.07 * f);
  };
  const double last = n / t.together - (rounds - 1);
  if (form == GatedForm::kMiddle) return 2.7 + (rounds - 1) * round_us(1.0) + round_us(last);
  if (two || n <= units()) return 1e30;   // a compute unit has one workgroup, or the form is not built
  // Many tiles go out of step: a compute unit takes the next one while its other goes on.  A few go in rounds, of which a last one of up to half
  // is one tile a compute unit, faster alone.
  if (rounds > (back ? 1 : 3)) return 2.7 + (n / t.together + 0.25) * (back ? 11.5 + nk * 0.88 : (keeps ? 3.5 : 0.3) + nk * 0.95);
  const double full = back ? 16.0 + nk * 0.94 : keeps ? 2.9 + nk * 0.98 : 1.5 + nk * 0.95, both = fmax(0.0, 2 * last - 1);
  return 2.7 + (rounds - 1 + both) * full + (1 - both) * round_us(fmin(1.0, 2 * last));
}
GatedPlan plan_whole(const GatedArgs& g, GatedOp op, bool b_oc, Kept kept) {
  GatedPlan best = {GatedForm::kAny, gated_stream_plan(g, op, b_oc, kept), 1e30};
  if (best.stream.p > 0) best = {GatedForm::kStream, best.stream, best.stream.us};
  for (GatedForm form : {GatedForm::kLarge, GatedForm::kMiddle, GatedForm::kShared}) {
    const double us = form_us(g, op, kept, form);
    if (us < best.us) best = {form, best.stream, us};
  }
  return best;
}

// Whether the results of a call are stored past the caches: by its time together with what reads them next, not by its own, which ordinary stores
// mostly lengthen.
// Forward: H of 172 MB and more.  2048 -> 5632, G and U kept in 8 bits, ordinary and past the caches, us: 8192 tokens (H of 88 MB) alone 324, 307, with
// the product that follows 457, 462; 12288 (132 MB) 474, 467 and 708, 719; 15360 (165 MB) 593, 578 and 856, 865; 16384 (176 MB) 617, 600 and 898, 886;
// 32768 (352 MB) 1221, 1207 and 1777, 1759.  Nothing kept: 8192 298, 282 and 429, 433; 15360 537, 532 and 805, 808; 32768 1110, 1104 and 1665, 1661.
// Backward: dG, dU and H where the products that read them are bound by the matrix cores, D of 1024 and more.  The whole pass (this call, Wd's weight
// gradient, dX, the two other weight gradients; kept in 8 bits), ordinary and past the caches, us: 2048 tokens, D 768, F 2048 82.8, 90.8; 4096 125, 137;
// 8192 254, 262; 4096, 768, 2304 154, 157; 2048, 1024, 4096 152, 150; 8192, 1024, 4096 465, 458; 1024, 2048, 5632 205, 199; 2048, 2048, 5632 320, 314;
// 8192, 2048, 5632 958, 960.  (D = 768 alone: 2048 tokens 19.5, 18.3, 4096 28.6, 27.8.)
bool stored_past_caches(GatedOp op, int64_t M, int64_t N, int64_t K) {
  return op == GatedOp::kFwd ? (uint64_t)M * (uint64_t)N * 2 >= (uint64_t)172 << 20 : op == GatedOp::kBwd && K >= 1024;
}

// Rows [m0, m0 + M) and columns [n0, n0 + N) of a call's result; n0 a multiple of 32.
GatedArgs part_of(GatedArgs g, GatedOp op, bool b_oc, Kept kept, uint32_t m0, uint32_t M, uint32_t n0, uint32_t N) {
  const size_t m = m0, n = n0, e = kept == Kept::kBf16 ? 2 : 1;
  g.M = M;
  g.N = N;
  g.a += m * g.lda;
  if (g.a2) g.a2 += m * g.lda;
  g.b += b_oc ? n : n * g.ldb;
  if (g.b2) g.b2 += b_oc ? n : n * g.ldb;
  if (g.h) g.h += m * g.ldh + n;
  if (op == GatedOp::kBwd) {
    g.dg += m * g.ldd + n;
    g.du += m * g.ldd + n;
  }
  if (kept != Kept::kNone) {
    g.kept.g += (m * g.kept.ldg + n) * e;
    g.kept.u += (m * g.kept.ldu + n) * e;
  }
  if (kept == Kept::kE4m3) {
    g.kept.gs += m * g.kept.lsg + n / 32;
    g.kept.us += m * g.kept.lsu + n / 32;
  }
  return g;
}

// One launch, or two: where a form's tiles leave a round of compute units partly empty, its whole rounds' columns or rows by that form and the
// rest by whatever is the fastest for it, where the estimates say that this is worth a second launch.  Of 180 drawn sizes that take two, they
// are 0.89 of the fastest single launch in the mean, at worst 1.03.  The best single launch and the two, us: forward 2217 x 1152 -> 3808 45.5, 38.7, with
// BF16 kept 1796 x 1184 -> 4416 58.3, 44.3; backward 4621 x 1664 -> 3520 91, 74, with 8 bits kept 5271 x 1664 -> 3104 95, 87; input gradient
// 2866 x 2 x 2176 -> 1728 65, 52, 8088 x 2 x 2368 -> 544 71, 61.
struct GatedSplit {
  GatedPlan first, rest;
  uint32_t rows, cols;   // of the first part; 0, 0: one launch
  double us;
};
GatedSplit plan_gated(const GatedArgs& g, GatedOp op, bool b_oc, Kept kept) {
  const GatedPlan whole = plan_whole(g, op, b_oc, kept);
  GatedSplit best = {whole, whole, 0, 0, 0.98 * whole.us};
  if (whole.form == GatedForm::kAny || whole.form == GatedForm::kStream) return best;
  for (GatedForm form : {GatedForm::kLarge, GatedForm::kMiddle, GatedForm::kShared}) {
    const Tiles t = tiles_of(form, op);
    const uint64_t mt = ((uint64_t)g.M + t.rows - 1) / t.rows, nt = ((uint64_t)g.N + t.cols - 1) / t.cols;
    const uint64_t fit = (uint64_t)(floor((double)(mt * nt) / t.together) * t.together);   // tiles of whole rounds
    const uint64_t cols = fit / mt * t.cols, rows = fit / nt * t.rows;
    for (int by_rows = 0; by_rows < 2; ++by_rows) {
      if (by_rows ? rows == 0 || rows >= g.M : cols == 0 || cols >= g.N) continue;
      const uint32_t m = by_rows ? (uint32_t)rows : g.M, n = by_rows ? g.N : (uint32_t)cols;
      const GatedArgs first = part_of(g, op, b_oc, kept, 0, m, 0, n);
      const GatedArgs rest = part_of(g, op, b_oc, kept, by_rows ? m : 0, by_rows ? g.M - m : g.M, by_rows ? 0 : n, by_rows ? g.N : g.N - n);
      const double us = form_us(first, op, kept, form);
      const GatedPlan after = plan_whole(rest, op, b_oc, kept);
      const double both = us + after.us + 4.0;   // the second launch's start and a second end of work
      if (both < best.us) best = {{form, whole.stream, us}, after, by_rows ? m : 0, by_rows ? 0 : n, both};
    }
  }
  return best;
}

int launch_form(const GatedArgs& g, GatedOp op, bool b_oc, Kept kept, const GatedPlan& plan, hipStream_t stream) {
  switch (plan.form) {
    case GatedForm::kStream: return launch_gated_stream(g, op, b_oc, kept, plan.stream, stream);
    case GatedForm::kMiddle: return launch_gated128(g, op, b_oc, kept, false, stream);
    case GatedForm::kShared: return launch_gated128(g, op, b_oc, kept, true, stream);
    case GatedForm::kLarge: return launch_gated256(g, op, b_oc, kept, stream);
    default: return launch_gated_any(g, op, b_oc, kept, stream);
  }
}

int launch_gated(const GatedArgs& g, GatedOp op, bool b_oc, Kept kept, hipStream_t stream) {
  const GatedSplit p = plan_gated(g, op, b_oc, kept);
  if (p.rows + p.cols == 0) return launch_form(g, op, b_oc, kept, p.first, stream);
  const uint32_t m = p.rows ? p.rows : g.M, n = p.cols ? p.cols : g.N;
  const int rc = launch_form(part_of(g, op, b_oc, kept, 0, m, 0, n), op, b_oc, kept, p.first, stream);
  if (rc != GWS_OK) return rc;
  return launch_form(part_of(g, op, b_oc, kept, p.rows, g.M - p.rows, p.cols, g.N - p.cols), op, b_oc, kept, p.rest, stream);
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
  g.past_caches = stored_past_caches(GatedOp::kFwd, M, F, K);
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
  g.ldd = (uint32_t)ldd; g.ldh = ld_of(h, ldh);
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
  g.past_caches = stored_past_caches(GatedOp::kBwd, M, F, D);
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
  const GatedOp o = op == GWS_GATED_FWD ? GatedOp::kFwd : op == GWS_GATED_BWD ? GatedOp::kBwd : GatedOp::kDx;
  const GatedSplit p = plan_gated(g, o, op == GWS_GATED_FWD ? !w_is_nk : w_is_nk != 0, o == GatedOp::kDx ? Kept::kNone : (Kept)kept);
  return (int)p.first.form | (p.first.form == GatedForm::kStream ? p.first.stream.mt << 16 | p.first.stream.nt << 8 : 0) |
         (p.rows + p.cols ? (int)p.rest.form << 24 | (p.rows ? 1 << 28 : 0) : 0) | (stored_past_caches(o, g.M, g.N, g.K) ? 1 << 29 : 0);
}

}  // extern "C"
