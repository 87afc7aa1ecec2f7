// The entry points of include/spec_layer8.h: argument checks and launches.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "../../include/spec.h"
#include "../../include/spec_layer8.h"
#include "fp8.h"
#include "kernels.h"

using namespace spec;

namespace {

bool aligned(const void *p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) == 0; }
bool is_dtype(int32_t d) { return d == SPEC_DTYPE_FP32 || d == SPEC_DTYPE_BF16; }
uintptr_t size_of(int32_t dtype) { return dtype == SPEC_DTYPE_BF16 ? 2 : 4; }
int done(hipError_t e) { return e == hipSuccess ? SPEC_OK : SPEC_EHIP; }

constexpr int kMaxM8 = 1 << 20, kMaxIn8 = 1 << 20, kMaxRows8 = 1 << 24;
bool matrix_ok(int32_t rows, int32_t in) { return rows >= 1 && rows <= kMaxRows8 && in >= 1 && in <= kMaxIn8; }

constexpr int kMaxKvHeads = 128;
bool heads_ok(int32_t hkv, int32_t hd) { return (hd == 64 || hd == 128) && hkv >= 1 && hkv <= kMaxKvHeads; }
bool attention_ok(int32_t rows, int32_t hq, int32_t hkv, int32_t hd, int32_t n_blocks, int32_t win_rows) {
  if (!heads_ok(hkv, hd) || hq < hkv || hq % hkv || rows < 1 || rows > (1 << 20) || n_blocks < 0 || n_blocks > (1 << 24) || win_rows < 1 || win_rows > (1 << 24)) return false;
  const int g = hq / hkv;
  return g == 1 || g == 2 || g == 4 || g == 8;
}

}  // namespace

extern "C" {

uint64_t spec_packed8_bytes(int32_t rows, int32_t in) {
  if (!matrix_ok(rows, in)) return 0;
  return (packed8_bytes(packed8(rows, in)) + 255) / 256 * 256;
}

int spec_pack_weight8(int32_t dtype, const void *src, int32_t rows, int32_t in, void *dst, void *stream) {
  if (!is_dtype(dtype) || !src || !dst || !matrix_ok(rows, in) || !aligned(src, size_of(dtype)) || !aligned(dst, 256)) return SPEC_EINVAL;
  return done(launch_pack_weight8(dtype, src, rows, in, dst, (hipStream_t)stream));
}

uint64_t spec_k_gemm8_scratch_bytes(int32_t m, int32_t in, int32_t rows) {
  if (m < 1 || m > kMaxM8 || !matrix_ok(rows, in)) return 0;
  return (gemm8_scratch_bytes(m, in, rows) + 255) / 256 * 256;
}

int spec_k_gemm8(int32_t dtype, const void *x, int32_t ldx, int32_t m, int32_t in, const void *w8, int32_t rows, int32_t out_dtype, void *y,
                 int32_t ldy, void *scratch, uint64_t scratch_bytes, void *stream) {
  const uint64_t need = spec_k_gemm8_scratch_bytes(m, in, rows);
  if (!is_dtype(dtype) || !is_dtype(out_dtype) || !x || !w8 || !y || m < 1 || m > kMaxM8 || !matrix_ok(rows, in) || ldx < in || ldy < rows) return SPEC_EINVAL;
  if (need > 0 && (!scratch || scratch_bytes < need)) return SPEC_EINVAL;
  if (!aligned(x, size_of(dtype)) || !aligned(y, size_of(out_dtype)) || !aligned(w8, 256) || !aligned(scratch, 256)) return SPEC_EINVAL;
  if (y == x || y == w8 || y == scratch) return SPEC_EINVAL;
  Gemm8Args a{};
  a.x = x; a.ldx = ldx; a.w8 = (const unsigned char *)w8; a.m = m; a.in = in; a.rows = rows; a.y = y; a.ldy = ldy;
  return done(launch_gemm8(dtype, out_dtype, a, scratch, (hipStream_t)stream));
}

uint64_t spec_kv8_bytes(int32_t n_blocks, int32_t hkv, int32_t hd) {
  if (!heads_ok(hkv, hd) || n_blocks < 1 || n_blocks > (1 << 24)) return 0;
  return (uint64_t)n_blocks * kv8_block_bytes(hkv, hd);
}

static bool kv8_ok(const void *k, const void *v, int64_t ld, int32_t n_blocks, int32_t hkv, int32_t hd, const void *cache8, int32_t first_block) {
  return k && v && cache8 && heads_ok(hkv, hd) && ld >= (int64_t)hkv * hd && ld <= (1 << 24) && n_blocks >= 0 && first_block >= 0 &&
         (int64_t)first_block + n_blocks <= (1 << 24) && aligned(k, 2) && aligned(v, 2) && aligned(cache8, 256);
}

int spec_k_kv8_store(const void *k, const void *v, int64_t ld, int32_t n_blocks, int32_t hkv, int32_t hd, void *cache8, int32_t first_block,
                     void *stream) {
  static_assert(SPEC_KV8_BLOCK == kKv8Block, "header and kernel agree on the block");
  if (!kv8_ok(k, v, ld, n_blocks, hkv, hd, cache8, first_block)) return SPEC_EINVAL;
  return done(launch_kv8_store(k, v, ld, n_blocks, hkv, hd, cache8, first_block, (hipStream_t)stream));
}

int spec_k_kv8_load(const void *cache8, int32_t first_block, int32_t n_blocks, int32_t hkv, int32_t hd, void *k, void *v, int64_t ld, void *stream) {
  if (!kv8_ok(k, v, ld, n_blocks, hkv, hd, cache8, first_block) || k == v) return SPEC_EINVAL;
  return done(launch_kv8_load(cache8, first_block, n_blocks, hkv, hd, k, v, ld, (hipStream_t)stream));
}

uint64_t spec_k_attention8_scratch_bytes(int32_t rows, int32_t hq, int32_t hkv, int32_t hd, int32_t n_blocks, int32_t win_rows) {
  if (!attention_ok(rows, hq, hkv, hd, n_blocks, win_rows)) return 0;
  return ((uint64_t)attention8_scratch_floats(rows, hq, hkv, hd, n_blocks, win_rows) * sizeof(float) + 255) / 256 * 256;
}

int spec_k_attention8(const float *q, const void *cache8, int32_t n_blocks, const void *kwin, const void *vwin, int32_t win_rows, int32_t rows,
                      int32_t hq, int32_t hkv, int32_t hd, int32_t base, const int32_t *depth, const int32_t *anc, int32_t max_depth,
                      void *scratch, uint64_t scratch_bytes, void *out, void *stream) {
  if (!q || (!cache8 && n_blocks > 0) || !kwin || !vwin || !depth || !out || !attention_ok(rows, hq, hkv, hd, n_blocks, win_rows)) return SPEC_EINVAL;
  const uint64_t need = spec_k_attention8_scratch_bytes(rows, hq, hkv, hd, n_blocks, win_rows);
  if (need > 0 && (!scratch || scratch_bytes < need)) return SPEC_EINVAL;
  if (max_depth < 0 || (anc && max_depth > kMaxDepth) || base < n_blocks * kKv8Block || (int64_t)base + max_depth >= INT32_MAX) return SPEC_EINVAL;
  if (!aligned(q, 16) || !aligned(kwin, 16) || !aligned(vwin, 16) || !aligned(out, 16) || !aligned(cache8, 256) || !aligned(scratch, 256) ||
      !aligned(depth, 4) || !aligned(anc, 4))
    return SPEC_EINVAL;
  if (out == q || out == cache8 || out == kwin || out == vwin || out == scratch) return SPEC_EINVAL;
  Attn8Args a{};
  a.q = q; a.cache8 = (const unsigned char *)cache8; a.n_blocks = n_blocks; a.kwin = kwin; a.vwin = vwin; a.win_rows = win_rows;
  a.rows = rows; a.hq = hq; a.hkv = hkv; a.hd = hd; a.base = base; a.depth = depth; a.anc = anc; a.max_depth = max_depth;
  a.scale = (float)(1.4426950408889634 / std::sqrt((double)hd)); a.part = (float *)scratch; a.out = out;
  return done(launch_attention8(a, (hipStream_t)stream));
}

int spec_k_attention8_plan(int32_t rows, int32_t hq, int32_t hkv, int32_t hd, int32_t n_blocks, int32_t win_rows, int32_t *waves, int32_t *query_blocks,
                           int32_t *block_parts, int32_t *win_parts) {
  if (!waves || !query_blocks || !block_parts || !win_parts || !attention_ok(rows, hq, hkv, hd, n_blocks, win_rows)) return SPEC_EINVAL;
  attention8_plan(rows, hq, hkv, n_blocks, win_rows, waves, query_blocks, block_parts, win_parts);
  return SPEC_OK;
}

int spec_rotary_init(int32_t rot, int32_t layout, double theta, const spec_rope_scaling *scaling, spec_rotary_plan *plan) {
  static_assert(SPEC_ROPE_MAX_DIM == 2 * kRotaryMaxPlanes, "header and kernel agree on the planes");
  const double kTwoPi = 6.283185307179586476925286766559;
  if (!plan || rot < 0 || rot > SPEC_ROPE_MAX_DIM || rot % 2 || (layout != SPEC_ROPE_HALF && layout != SPEC_ROPE_INTERLEAVED)) return SPEC_EINVAL;
  if (!(theta > 1.0) || !std::isfinite(theta)) return SPEC_EINVAL;
  const int kind = scaling ? scaling->kind : SPEC_ROPE_NONE;
  if (kind < SPEC_ROPE_NONE || kind > SPEC_ROPE_YARN) return SPEC_EINVAL;
  if (kind != SPEC_ROPE_NONE && (!(scaling->factor >= 1.0) || !std::isfinite(scaling->factor))) return SPEC_EINVAL;
  if (kind >= SPEC_ROPE_LLAMA3 && (scaling->trained_len < 1 || !(scaling->low > 0.0) || !(scaling->high > scaling->low) || !std::isfinite(scaling->high)))
    return SPEC_EINVAL;
  spec_rotary_plan p{};
  p.rot = rot; p.layout = layout; p.mscale = 1.0;
  double first = 0.0, last = 0.0;                             // YARN: the ramp
  if (kind == SPEC_ROPE_YARN && rot > 0) {
    auto place = [&](double times) { return rot * std::log(scaling->trained_len / (times * kTwoPi)) / (2.0 * std::log(theta)); };
    first = std::fmax(std::floor(place(scaling->high)), 0.0);
    last = std::fmin(std::ceil(place(scaling->low)), rot - 1.0);
    p.mscale = 0.1 * std::log(scaling->factor) + 1.0;
  }
  for (int j = 0; j < rot / 2; j++) {
    double f = std::pow(theta, -2.0 * j / rot);
    if (kind == SPEC_ROPE_LINEAR) f /= scaling->factor;
    if (kind == SPEC_ROPE_LLAMA3) {
      const double keep = (scaling->trained_len * f / kTwoPi - scaling->low) / (scaling->high - scaling->low);
      const double kept = std::fmin(std::fmax(keep, 0.0), 1.0);
      f = kept * f + (1.0 - kept) * f / scaling->factor;
    }
    if (kind == SPEC_ROPE_YARN) {
      const double far = std::fmin(std::fmax((j - first) / std::fmax(last - first, 0.001), 0.0), 1.0);
      f = (1.0 - far) * f + far * f / scaling->factor;
    }
    p.freq[j] = f;
  }
  *plan = p;
  return SPEC_OK;
}

int spec_k_rotary(const spec_rotary_plan *plan, int32_t n_parts, const spec_rotary_part *parts, int32_t hd, int32_t rows, const int32_t *pos,
                  int32_t pos0, int32_t adjoint, void *stream) {
  if (!plan || !parts || n_parts < 1 || n_parts > 3 || rows < 1 || rows > (1 << 24) || hd < 1 || hd > SPEC_ROPE_MAX_DIM || !aligned(pos, 4)) return SPEC_EINVAL;
  if (plan->rot < 0 || plan->rot > hd || plan->rot % 2 || (plan->layout != SPEC_ROPE_HALF && plan->layout != SPEC_ROPE_INTERLEAVED)) return SPEC_EINVAL;
  RotaryArgs a{};
  for (int n = 0; n < n_parts; n++) {
    const spec_rotary_part &p = parts[n];
    if (!p.x || !p.out || !is_dtype(p.dtype) || !is_dtype(p.out_dtype) || p.heads < 1 || p.heads > 1024) return SPEC_EINVAL;
    if (!aligned(p.x, size_of(p.dtype)) || !aligned(p.out, size_of(p.out_dtype))) return SPEC_EINVAL;
    if (p.heads > 1 && (p.hsx < hd || p.hso < hd)) return SPEC_EINVAL;
    if (rows > 1 && (p.ldx < hd || p.ldo < hd)) return SPEC_EINVAL;
    const int64_t most = (int64_t)1 << 40;
    if (p.ldx < 0 || p.hsx < 0 || p.ldo < 0 || p.hso < 0 || p.ldx > most || p.hsx > most || p.ldo > most || p.hso > most) return SPEC_EINVAL;
    if (p.x == p.out && (p.dtype != p.out_dtype || (rows > 1 && p.ldx != p.ldo) || (p.heads > 1 && p.hsx != p.hso))) return SPEC_EINVAL;
    for (int o = 0; o < n; o++)
      if (p.out == parts[o].out || p.out == parts[o].x || p.x == parts[o].out) return SPEC_EINVAL;
    a.part[n] = RotaryPart{p.x, p.out, p.ldx, p.hsx, p.ldo, p.hso, p.heads, p.dtype, p.out_dtype, p.turn != 0};
  }
  a.n_parts = n_parts; a.hd = hd; a.rows = rows; a.rot = plan->rot; a.interleaved = plan->layout == SPEC_ROPE_INTERLEAVED;
  a.adjoint = adjoint != 0; a.pos = pos; a.pos0 = pos0; a.mscale = plan->mscale;
  for (int j = 0; j < plan->rot / 2; j++) a.turns[j] = plan->freq[j] / 6.283185307179586476925286766559;
  return done(launch_rotary(a, (hipStream_t)stream));
}

}  // extern "C"
