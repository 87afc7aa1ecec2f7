// The entry points of include/spec_step.h: argument checks and launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <new>
#include <vector>

#include "../../include/spec.h"
#include "../../include/spec_step.h"
#include "kernels.h"

using namespace spec;

namespace {

bool aligned(const void *p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) == 0; }
bool is_dtype(int32_t d) { return d == SPEC_DTYPE_FP32 || d == SPEC_DTYPE_BF16; }
uintptr_t size_of(int32_t dtype) { return dtype == SPEC_DTYPE_BF16 ? 2 : 4; }
int done(hipError_t e) { return e == hipSuccess ? SPEC_OK : SPEC_EHIP; }
constexpr int64_t kMostStride = (int64_t)1 << 40;
bool stride_ok(int64_t ld, int64_t least, int64_t rows) { return ld >= 0 && ld <= kMostStride && (rows <= 1 || ld >= least); }

// ---- embedding
constexpr int kMaxCols = 1 << 20, kMaxVocab = 1 << 24, kMaxRows = 1 << 24, kMaxGradRows = 1 << 20;
bool table_ok(int32_t vocab, int32_t d) { return vocab >= 1 && vocab <= kMaxVocab && d >= 1 && d <= kMaxCols; }

// ---- norms of heads: what both directions check of the plan, the parts' rotary side and the weights
bool plan_ok(const spec_rotary_plan *plan, int32_t n_parts, int32_t hd, int32_t rows, const int32_t *pos, float eps) {
  if (!plan || n_parts < 1 || n_parts > 3 || rows < 1 || rows > (1 << 24) || hd < 1 || hd > SPEC_ROPE_MAX_DIM || !aligned(pos, 4)) return false;
  if (plan->rot < 0 || plan->rot > hd || plan->rot % 2 || (plan->layout != SPEC_ROPE_HALF && plan->layout != SPEC_ROPE_INTERLEAVED)) return false;
  return eps >= 0.f && std::isfinite(eps);
}
bool part_ok(const spec_rotary_part &p, int32_t hd, int32_t rows) {
  if (!p.x || !p.out || !is_dtype(p.dtype) || !is_dtype(p.out_dtype) || p.heads < 1 || p.heads > 1024) return false;
  if (!aligned(p.x, size_of(p.dtype)) || !aligned(p.out, size_of(p.out_dtype))) return false;
  if (!stride_ok(p.hsx, hd, p.heads) || !stride_ok(p.hso, hd, p.heads) || !stride_ok(p.ldx, hd, rows) || !stride_ok(p.ldo, hd, rows)) return false;
  return p.x != p.out || (p.dtype == p.out_dtype && (rows == 1 || p.ldx == p.ldo) && (p.heads == 1 || p.hsx == p.hso));
}
bool weight_ok(const void *w, int32_t w_dtype, float offset) {
  return !w || (is_dtype(w_dtype) && aligned(w, size_of(w_dtype)) && std::isfinite(offset));
}
HeadnormArgs headnorm_args(const spec_rotary_plan *plan, int32_t n_parts, int32_t hd, int32_t rows, const int32_t *pos, int32_t pos0, float eps) {
  HeadnormArgs a{};
  a.n_parts = n_parts; a.hd = hd; a.rows = rows; a.rot = plan->rot; a.interleaved = plan->layout == SPEC_ROPE_INTERLEAVED;
  a.pos = pos; a.pos0 = pos0; a.mscale = plan->mscale; a.eps = eps;
  for (int j = 0; j < plan->rot / 2; j++) a.turns[j] = plan->freq[j] / 6.283185307179586476925286766559;
  return a;
}
RotaryPart rotary_part(const spec_rotary_part &p) { return RotaryPart{p.x, p.out, p.ldx, p.hsx, p.ldo, p.hso, p.heads, p.dtype, p.out_dtype, p.turn != 0}; }

// ---- feed-forward block
bool ffn_sizes_ok(int32_t rows, int32_t d, int32_t f) {
  const int most = 1 << 20;
  if (rows < 1 || rows > most || d < 8 || d > most || d % 8 || f < 8 || f > most || f % 8) return false;
  const int64_t area = (int64_t)1 << 36;
  return (int64_t)rows * d <= area && (int64_t)rows * f <= area && (int64_t)d * f <= area;
}
bool ffn_matrix_ok(const void *p, int64_t ld, int64_t rows, int64_t cols) {   // rows so far apart that 256 of them fit 31 bits
  return p && aligned(p, 16) && ld >= 0 && ld <= (1 << 21) && (rows == 1 || (ld >= cols && ld % 8 == 0));
}
int64_t row_step(int64_t ld, int32_t rows, int32_t cols) { return rows == 1 ? cols : ld; }   // one row's stride may be anything; the kernels place rows that are not there by it

// ---- clipping
bool grad_ok(const spec_grad_part &p, bool clip) {
  if (p.n < 0 || p.n > kMostStride || !is_dtype(p.dtype)) return false;
  if (p.n == 0) return true;
  if (!p.g || !aligned(p.g, size_of(p.dtype))) return false;
  return !clip || (p.out && is_dtype(p.out_dtype) && aligned(p.out, size_of(p.out_dtype)) && (p.out != p.g || p.dtype == p.out_dtype));
}

// Whether the bytes at p and those at q meet
bool meet(const void *p, uint64_t bytes, const void *q, uint64_t more) { return (uintptr_t)p < (uintptr_t)q + more && (uintptr_t)q < (uintptr_t)p + bytes; }
bool grad_meets(const spec_grad_part &p, const void *q, uint64_t bytes, bool clip) {   // the gradient, or its output (clip), with the sums or the norm
  return p.n > 0 && q && (meet(p.g, (uint64_t)p.n * size_of(p.dtype), q, bytes) || (clip && meet(p.out, (uint64_t)p.n * size_of(p.out_dtype), q, bytes)));
}
constexpr uint64_t kSumsBytes = SPEC_GRAD_SUMS * sizeof(double);

// The tensors, as many as a launch takes at a time.  launch(args) is called once at least.
template <typename Launch> int for_each_launch(int32_t n_parts, const spec_grad_part *parts, GradArgs &a, Launch launch) {
  int at = 0;
  do {
    a.n = a.chunks = 0;
    for (; at < n_parts && a.n < kGradTensors; at++) {
      const spec_grad_part &p = parts[at];
      if (p.n == 0) continue;
      const int64_t chunks = grad_chunks(p.g, p.n, p.dtype);
      if (a.chunks + chunks > (1 << 30)) break;
      a.t[a.n] = GradTensor{p.g, p.out, p.n | (p.dtype == SPEC_DTYPE_BF16 ? kGradBf16 : 0) | (p.out_dtype == SPEC_DTYPE_BF16 ? kGradToBf16 : 0)};
      a.begin[a.n++] = a.chunks;
      a.chunks += (int)chunks;
    }
    const hipError_t e = launch(a);
    if (e != hipSuccess) return SPEC_EHIP;
    a.first = 0;
    a.norm = nullptr;
  } while (at < n_parts);
  return SPEC_OK;
}

// Whether what is written overlaps anything else that is: the outputs by address, each against its neighbour, then every input against the outputs (but its own, in place).
bool apart(int32_t n_parts, const spec_grad_part *parts) {
  struct Range { uintptr_t lo, hi; };
  std::vector<Range> outs;
  for (int n = 0; n < n_parts; n++)
    if (parts[n].n > 0) outs.push_back(Range{(uintptr_t)parts[n].out, (uintptr_t)parts[n].out + (uintptr_t)parts[n].n * size_of(parts[n].out_dtype)});
  std::sort(outs.begin(), outs.end(), [](const Range &x, const Range &y) { return x.lo < y.lo; });
  for (size_t i = 1; i < outs.size(); i++)
    if (outs[i].lo < outs[i - 1].hi) return false;
  for (int n = 0; n < n_parts; n++) {
    const spec_grad_part &p = parts[n];
    if (p.n == 0 || p.g == p.out) continue;
    const uintptr_t lo = (uintptr_t)p.g, hi = lo + (uintptr_t)p.n * size_of(p.dtype);
    const auto next = std::lower_bound(outs.begin(), outs.end(), lo, [](const Range &x, uintptr_t v) { return x.lo < v; });
    if ((next != outs.end() && next->lo < hi) || (next != outs.begin() && (next - 1)->hi > lo)) return false;
  }
  return true;
}

}  // namespace

extern "C" {

int spec_k_embed(int32_t dtype, const void *table, int64_t ldt, int32_t vocab, int32_t d, const int32_t *tok, int32_t rows, float scale,
                 int32_t out_dtype, void *out, int64_t ldo, void *stream) {
  if (!is_dtype(dtype) || !is_dtype(out_dtype) || !table || !tok || !out || !table_ok(vocab, d) || rows < 1 || rows > kMaxRows) return SPEC_EINVAL;
  if (!stride_ok(ldt, d, vocab) || !stride_ok(ldo, d, rows) || !aligned(table, size_of(dtype)) || !aligned(out, size_of(out_dtype)) || !aligned(tok, 4))
    return SPEC_EINVAL;
  if (out == table || out == tok) return SPEC_EINVAL;
  return done(launch_embed(dtype, table, ldt, vocab, d, tok, rows, scale, out_dtype, out, ldo, (hipStream_t)stream));
}

uint64_t spec_k_embed_grad_scratch_bytes(int32_t rows, int32_t vocab, int32_t d) {
  if (!table_ok(vocab, d) || rows < 1 || rows > kMaxGradRows) return 0;
  return embed_grad_scratch_bytes(rows, vocab, d);
}

int spec_k_embed_grad(int32_t dtype, const void *dy, int64_t ldy, const int32_t *tok, int32_t rows, int32_t d, int32_t vocab, float scale,
                      int32_t accumulate, int32_t out_dtype, void *dtable, int64_t ldt, void *scratch, uint64_t scratch_bytes, void *stream) {
  if (!is_dtype(dtype) || !is_dtype(out_dtype) || !dy || !tok || !dtable || !scratch || !table_ok(vocab, d) || rows < 1 || rows > kMaxGradRows) return SPEC_EINVAL;
  if (!stride_ok(ldy, d, rows) || !stride_ok(ldt, d, vocab) || !aligned(dy, size_of(dtype)) || !aligned(dtable, size_of(out_dtype)) || !aligned(tok, 4))
    return SPEC_EINVAL;
  if (!aligned(scratch, 256) || scratch_bytes < embed_grad_scratch_bytes(rows, vocab, d)) return SPEC_EINVAL;
  if (dtable == dy || dtable == tok || dtable == scratch || scratch == dy || scratch == tok) return SPEC_EINVAL;
  EmbedGradArgs a{};
  a.dy = dy; a.ldy = ldy; a.dtype = dtype; a.tok = tok; a.rows = rows; a.d = d; a.vocab = vocab; a.accumulate = accumulate != 0; a.scale = scale;
  a.dtable = dtable; a.ldt = ldt; a.out_dtype = out_dtype;
  return done(launch_embed_grad(a, scratch, (hipStream_t)stream));
}

int spec_k_headnorm_rotary(const spec_rotary_plan *plan, int32_t n_parts, const spec_headnorm_part *parts, int32_t hd, int32_t rows, const int32_t *pos,
                           int32_t pos0, float eps, void *stream) {
  if (!parts || !plan_ok(plan, n_parts, hd, rows, pos, eps)) return SPEC_EINVAL;
  HeadnormArgs a = headnorm_args(plan, n_parts, hd, rows, pos, pos0, eps);
  for (int n = 0; n < n_parts; n++) {
    const spec_headnorm_part &q = parts[n];
    if (!part_ok(q.p, hd, rows) || !weight_ok(q.w, q.w_dtype, q.offset) || q.p.out == q.w) return SPEC_EINVAL;
    for (int o = 0; o < n; o++)
      if (q.p.out == parts[o].p.out || q.p.out == parts[o].p.x || q.p.x == parts[o].p.out || q.p.out == parts[o].w || q.w == parts[o].p.out) return SPEC_EINVAL;
    a.part[n].p = rotary_part(q.p);
    a.part[n].w = q.w; a.part[n].w_dtype = q.w_dtype; a.part[n].offset = q.offset;
  }
  return done(launch_headnorm(a, (hipStream_t)stream));
}

uint64_t spec_k_headnorm_rotary_grad_scratch_bytes(int32_t n_parts, int32_t hd) {
  if (n_parts < 1 || n_parts > 3 || hd < 1 || hd > SPEC_ROPE_MAX_DIM) return 0;
  return ((uint64_t)n_parts * headnorm_grad_groups() * hd * sizeof(float) + 255) / 256 * 256;
}

int spec_k_headnorm_rotary_grad(const spec_rotary_plan *plan, int32_t n_parts, const spec_headnorm_grad_part *parts, int32_t hd, int32_t rows,
                                const int32_t *pos, int32_t pos0, float eps, void *scratch, uint64_t scratch_bytes, void *stream) {
  if (!parts || !plan_ok(plan, n_parts, hd, rows, pos, eps)) return SPEC_EINVAL;
  HeadnormArgs a = headnorm_args(plan, n_parts, hd, rows, pos, pos0, eps);
  bool sums = false;
  for (int n = 0; n < n_parts; n++) {
    const spec_headnorm_grad_part &q = parts[n];
    if (!part_ok(q.p, hd, rows) || !weight_ok(q.w, q.w_dtype, q.offset) || (q.dw && (!q.w || !aligned(q.dw, 4)))) return SPEC_EINVAL;
    if (q.w && (!q.x || !is_dtype(q.x_dtype) || !aligned(q.x, size_of(q.x_dtype)) || !stride_ok(q.ld, hd, rows) || !stride_ok(q.hs, hd, q.p.heads))) return SPEC_EINVAL;
    sums = sums || q.dw;
    // what is written, against everything else
    for (int o = 0; o < n_parts; o++) {
      const spec_headnorm_grad_part &r = parts[o];
      if (q.p.out == r.x || q.p.out == r.w || (o != n && (q.p.out == r.p.out || q.p.out == r.p.x))) return SPEC_EINVAL;
      if (q.dw && (q.dw == r.x || q.dw == r.w || q.dw == r.p.x || q.dw == r.p.out || (o != n && q.dw == r.dw))) return SPEC_EINVAL;
    }
    if (scratch && (q.p.out == scratch || q.p.x == scratch || q.x == scratch || q.w == scratch || q.dw == scratch)) return SPEC_EINVAL;
    a.part[n].p = rotary_part(q.p);
    a.part[n].w = q.w; a.part[n].w_dtype = q.w_dtype; a.part[n].offset = q.offset;
    a.part[n].x = q.x; a.part[n].ld = q.ld; a.part[n].hs = q.hs; a.part[n].x_dtype = q.x_dtype; a.part[n].dw = q.dw;
  }
  if (sums && (!scratch || !aligned(scratch, 256) || scratch_bytes < spec_k_headnorm_rotary_grad_scratch_bytes(n_parts, hd))) return SPEC_EINVAL;
  a.scratch = (float *)scratch;
  return done(launch_headnorm_grad(a, (hipStream_t)stream));
}

int spec_k_ffn_gated(const void *x, int64_t ldx, int32_t rows, int32_t d, const void *w_gate, const void *w_up, int64_t ldw, int32_t f, int32_t act,
                     void *h, int64_t ldh, void *stream) {
  static_assert(SPEC_ACT_SILU == kActSilu && SPEC_ACT_GELU == kActGelu && SPEC_ACT_GELU_TANH == kActGeluTanh, "header and kernel agree on the activations");
  if (!ffn_sizes_ok(rows, d, f) || act < SPEC_ACT_SILU || act > SPEC_ACT_GELU_TANH) return SPEC_EINVAL;
  if (!ffn_matrix_ok(x, ldx, rows, d) || !ffn_matrix_ok(w_gate, ldw, f, d) || !ffn_matrix_ok(w_up, ldw, f, d) || !ffn_matrix_ok(h, ldh, rows, f)) return SPEC_EINVAL;
  if (h == x || h == w_gate || h == w_up) return SPEC_EINVAL;
  FfnCall c{};
  c.x = x; c.ldx = row_step(ldx, rows, d); c.wg = w_gate; c.wu = w_up; c.ldw = ldw; c.rows = rows; c.d = d; c.f = f; c.act = act; c.h = h; c.ldh = row_step(ldh, rows, f);
  return done(launch_ffn(c, (hipStream_t)stream));
}

uint64_t spec_k_ffn_gated_grad_scratch_bytes(int32_t rows, int32_t d, int32_t f) {
  return ffn_sizes_ok(rows, d, f) ? ffn_grad_scratch_bytes(rows, d, f) : 0;
}

int spec_k_ffn_gated_grad(const void *x, int64_t ldx, int32_t rows, int32_t d, const void *w_gate, const void *w_up, int64_t ldw, int32_t f, int32_t act,
                          const void *dh, int64_t lddh, void *dx, int64_t lddx, void *dw_gate, void *dw_up, int64_t lddw, void *scratch,
                          uint64_t scratch_bytes, void *stream) {
  if (!ffn_sizes_ok(rows, d, f) || act < SPEC_ACT_SILU || act > SPEC_ACT_GELU_TANH) return SPEC_EINVAL;
  if (!ffn_matrix_ok(x, ldx, rows, d) || !ffn_matrix_ok(w_gate, ldw, f, d) || !ffn_matrix_ok(w_up, ldw, f, d) || !ffn_matrix_ok(dh, lddh, rows, f)) return SPEC_EINVAL;
  if ((dx && !ffn_matrix_ok(dx, lddx, rows, d)) || !dw_gate != !dw_up) return SPEC_EINVAL;
  if (dw_gate && (!ffn_matrix_ok(dw_gate, lddw, f, d) || !ffn_matrix_ok(dw_up, lddw, f, d))) return SPEC_EINVAL;
  if (!scratch || !aligned(scratch, 256) || scratch_bytes < ffn_grad_scratch_bytes(rows, d, f)) return SPEC_EINVAL;
  const void *in[4] = {x, w_gate, w_up, dh}, *out[4] = {dx, dw_gate, dw_up, scratch};
  for (int o = 0; o < 4; o++) {
    for (int i = 0; i < 4; i++)
      if (out[o] == in[i] || (out[o] && i < o && out[o] == out[i])) return SPEC_EINVAL;
  }
  FfnCall c{};
  c.x = x; c.ldx = row_step(ldx, rows, d); c.wg = w_gate; c.wu = w_up; c.ldw = ldw; c.rows = rows; c.d = d; c.f = f; c.act = act; c.h = const_cast<void *>(dh); c.ldh = row_step(lddh, rows, f);
  c.dx = dx; c.lddx = row_step(lddx, rows, d); c.dwg = dw_gate; c.dwu = dw_up; c.lddw = lddw;
  return done(launch_ffn_grad(c, scratch, (hipStream_t)stream));
}

int spec_k_ffn_gated_plan(int32_t rows, int32_t d, int32_t f, int32_t *forward, int32_t *again, int32_t *dx, int32_t *dx_ranges, int32_t *dw, int32_t *dw_ranges,
                          int32_t *together) {
  if (!ffn_sizes_ok(rows, d, f) || !forward || !again || !dx || !dx_ranges || !dw || !dw_ranges || !together) return SPEC_EINVAL;
  const FfnPlans p = ffn_plans(rows, d, f);
  *forward = p.forward; *again = p.again; *dx = p.dx; *dx_ranges = p.dx_ranges; *dw = p.dw; *dw_ranges = p.dw_ranges; *together = p.together;
  return SPEC_OK;
}

int spec_k_grad_sums(int32_t n_parts, const spec_grad_part *parts, double *sums, void *stream) {
  static_assert(SPEC_GRAD_SUMS == kGradSums, "header and kernel agree on the sums");
  if (n_parts < 0 || (n_parts > 0 && !parts) || !sums || !aligned(sums, 8)) return SPEC_EINVAL;
  for (int n = 0; n < n_parts; n++)
    if (!grad_ok(parts[n], false) || grad_meets(parts[n], sums, kSumsBytes, false)) return SPEC_EINVAL;
  GradArgs a{};
  a.sums = sums; a.first = 1;
  return for_each_launch(n_parts, parts, a, [&](const GradArgs &b) { return launch_grad_sums(b, (hipStream_t)stream); });
}

int spec_k_grad_clip(int32_t n_parts, const spec_grad_part *parts, const double *sums, double max_norm, float *norm, void *stream) {
  if (n_parts < 0 || (n_parts > 0 && !parts) || !sums || !aligned(sums, 8) || !aligned(norm, 4)) return SPEC_EINVAL;
  if (norm && meet(norm, sizeof(float), sums, kSumsBytes)) return SPEC_EINVAL;
  if (!(max_norm >= 0.0) || !std::isfinite(max_norm)) return SPEC_EINVAL;
  for (int n = 0; n < n_parts; n++) {
    const spec_grad_part &p = parts[n];
    if (!grad_ok(p, true) || grad_meets(p, sums, kSumsBytes, true) || grad_meets(p, norm, sizeof(float), true)) return SPEC_EINVAL;
  }
  try {
    if (!apart(n_parts, parts)) return SPEC_EINVAL;
  } catch (const std::bad_alloc &) { return SPEC_EINVAL; }    // (of the host's memory; nothing was launched)
  GradArgs a{};
  a.sums = const_cast<double *>(sums); a.max_norm = max_norm; a.norm = norm;
  return for_each_launch(n_parts, parts, a, [&](const GradArgs &b) { return launch_grad_clip(b, (hipStream_t)stream); });
}

}  // extern "C"
