// Attention over a cache of 64-token blocks in 8 bits with a bf16 window behind it, and the cache's store and load (include/spec_layer8.h).
#include <type_traits>

#include "common.h"
#include "fp8.h"
#include "kernels.h"

namespace spec {

namespace {

// Where a block's codes lie.  Scores are taken as S^T = K Q^T and outputs as O^T = V^T P^T with 32 x 32 x 16 products; a wavefront reads 1 KiB at a time, lane
// (c = lane % 32, g = lane / 32) 16 bytes, which are its operands of two products:
//   keys  : piece (32 keys, 32 dims): key c, dims 16 g + 0 .. 15,
//   values: piece (32 keys, 32 dims): dim c, keys 4 g + {0..3, 8..11, 16..19, 24..27}: the keys whose weights the lane holds after the scores.
template <int HD> __device__ __forceinline__ int key_at(int t, int d) {   // token t, dim d
  return (t >> 5) * 32 * HD + (d >> 5) * 1024 + (((d >> 4) & 1) * 32 + (t & 31)) * 16 + (d & 15);
}
template <int HD> __device__ __forceinline__ int value_at(int t, int d) {
  return (t >> 5) * 32 * HD + (d >> 5) * 1024 + (((t >> 2) & 1) * 32 + (d & 31)) * 16 + ((t >> 3) & 3) * 4 + (t & 3);
}

__device__ __forceinline__ float code_to_f32(unsigned char c) { return __builtin_amdgcn_cvt_f32_fp8((int)c, 0); }

// A workgroup puts one head's keys or values of a block into 8 bits.
template <int HD>
__global__ __launch_bounds__(256) void kv8_store_kernel(const bf16_t *k, const bf16_t *v, int64_t ld, int hkv, unsigned char *cache8, int first_block) {
  __shared__ __attribute__((aligned(16))) unsigned char codes[kKv8Block * HD];
  __shared__ float sh[16];
  const int h = blockIdx.x >> 1, values = blockIdx.x & 1, blk = blockIdx.y;
  const bf16_t *src = (values ? v : k) + (int64_t)blk * kKv8Block * ld + (int64_t)h * HD;
  constexpr int kEach = kKv8Block * HD / 256;                 // consecutive values of a thread
  const int t = threadIdx.x * kEach / HD, d0 = threadIdx.x * kEach % HD;
  float x[kEach], amax = 0.f;
#pragma unroll
  for (int i = 0; i < kEach; i++) {
    x[i] = to_f32(src[t * ld + d0 + i]);
    amax = fmaxf(amax, finite_abs(x[i]));
  }
  const int e = exponent8(block_max(amax, sh));
  const float down = pow2(-e);
#pragma unroll
  for (int i = 0; i < kEach; i += 4) {
    const uint32_t c = codes4(x[i] * down, x[i + 1] * down, x[i + 2] * down, x[i + 3] * down);
#pragma unroll
    for (int j = 0; j < 4; j++) codes[values ? value_at<HD>(t, d0 + i + j) : key_at<HD>(t, d0 + i + j)] = (unsigned char)(c >> (8 * j));
  }
  __syncthreads();
  unsigned char *block = cache8 + (size_t)(first_block + blk) * kv8_block_bytes(hkv, HD);
  u32x4_t *dst = (u32x4_t *)(block + (size_t)(2 * h + values) * kKv8Block * HD);
  for (int i = threadIdx.x; i < kKv8Block * HD / 16; i += 256) dst[i] = ((const u32x4_t *)codes)[i];
  if (threadIdx.x == 0) block[(size_t)hkv * 2 * kKv8Block * HD + 2 * h + values] = (unsigned char)(e + 127);
}

template <int HD>
__global__ __launch_bounds__(256) void kv8_load_kernel(const unsigned char *cache8, int first_block, int hkv, bf16_t *k, bf16_t *v, int64_t ld) {
  const int h = blockIdx.x >> 1, values = blockIdx.x & 1, blk = blockIdx.y;
  const unsigned char *block = cache8 + (size_t)(first_block + blk) * kv8_block_bytes(hkv, HD);
  const unsigned char *src = block + (size_t)(2 * h + values) * kKv8Block * HD;
  const float up = pow2((int)block[(size_t)hkv * 2 * kKv8Block * HD + 2 * h + values] - 127);
  bf16_t *dst = (values ? v : k) + (int64_t)blk * kKv8Block * ld + (int64_t)h * HD;
  for (int i = threadIdx.x; i < kKv8Block * HD; i += 256) {
    const int t = i / HD, d = i % HD;
    dst[t * ld + d] = from_f32<bf16_t>(code_to_f32(src[values ? value_at<HD>(t, d) : key_at<HD>(t, d)]) * up);
  }
}

// ---- attention --------------------------------------------------------------------
// The queries of a kv head are numbered row * G + head in group; a wavefront owns 32 of them as the columns of its products: lane (c = lane % 32, g = lane / 32)
// holds query c, of a 32-key tile's scores the keys 8 i + 4 g + 0 .. 3 (i < 4), of the outputs the same dims of every 32.
//
// In the blocks the products are fp16: codes are exact there, a query row is divided by the power of two of its largest value and rounded once (2^-11), and
// a weight is cut once.  Weights are 2^(score - reference): the reference is put kRefLift under the largest score and moves when it lags kRefLag more, so that the largest weight is
// 2^12 to 2^15 and weights keep fp16's full precision (2^-14 on) down to 2^-26 of it; smaller ones are cut to multiples of 2^-36 of it (2^-24).  (A lift of 7 and a lag of 8 moved the reference less
// often, in the same time, and took up to 2^-6 of weights 2^-25 of the largest, as of keys behind an attention sink.)  A block's exponents go into the scores' factor and into the weights (relative
// to the largest of the blocks so far, which the outputs are in units of); nothing is done per value for them.
constexpr float kRefLift = 12.f, kRefLag = 3.f;
// Weights go to fp16 by the conversion that cuts off, two at a time (rounding to nearest takes three instructions): they are made 2^-12 too large first, which
// centres the error (at most 2^-10 either way, in the mean none), and their sum is corrected for it.
constexpr float kCutLift = 0.00035223863f;                    // log2(1 + 2^-12)
constexpr float kCutSum = 1.f / (1.f + 1.f / 4096.f);

typedef __attribute__((ext_vector_type(8))) _Float16 f16x8_t;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_t;
typedef __attribute__((ext_vector_type(16))) float f32x16_t;
__device__ __forceinline__ f32x16_t mul_f16(const u32x4_t &a, const u32x4_t &b, f32x16_t c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8_t, a), __builtin_bit_cast(f16x8_t, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x16_t mul_bf16(const u32x4_t &a, const u32x4_t &b, f32x16_t c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}
__device__ __forceinline__ uint32_t cut_f16x2(float lo, float hi) { return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(lo, hi)); }
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
  typedef __attribute__((ext_vector_type(2))) float f2_t;
  typedef __attribute__((ext_vector_type(2))) _Float16 h2_t;
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f2_t{lo, hi}, h2_t));   // to nearest even
}
// Sixteen codes as the fp16 operands of two products
__device__ __forceinline__ void widen(const u32x4_t &w, u32x4_t &first, u32x4_t &second) {
  first = u32x4_t{f16_of_codes<false>(w.x, 1.f), f16_of_codes<true>(w.x, 1.f), f16_of_codes<false>(w.y, 1.f), f16_of_codes<true>(w.y, 1.f)};
  second = u32x4_t{f16_of_codes<false>(w.z, 1.f), f16_of_codes<true>(w.z, 1.f), f16_of_codes<false>(w.w, 1.f), f16_of_codes<true>(w.w, 1.f)};
}

// The work of a launch.  waves: of 32 queries each in a workgroup; 0: few queries.  Parts 0 .. block_parts - 1 are ranges of the cache's blocks, the others ranges of win_part
// rows of the window, or, with win_parts 0, the last range of blocks goes on into the whole window; of eight wavefronts it has as many blocks fewer as the rows that a
// block of queries sees cost (win_cost: per query block, win_base: for the first, in 1/16 of a block).
struct Plan8 { int waves, query_blocks, block_parts, win_parts, win_part, win_base, win_cost; };
__host__ __device__ inline int range_at(int n, int parts, int i) { return (int)((int64_t)n * i / parts); }
__device__ __forceinline__ int joined_range_at(const Plan8 &p, int n, int qb, int i) {
  if (i == p.block_parts) return n;
  const int64_t all = 16 * (int64_t)n + p.win_base + (int64_t)p.win_cost * qb;
  return (int)min(all * i / p.block_parts / 16, (int64_t)n);
}

// Running softmax of 32 queries (this lane's)
template <int HD> struct Running {
  f32x16_t o[HD / 32];
  float m = -INFINITY, l = 0.f;                               // reference of the weights (lifted: m + kRefLift is the scores'), sum of this lane's weights
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int db = 0; db < HD / 32; db++)
#pragma unroll
      for (int i = 0; i < 16; i++) o[db][i] = 0.f;
  }
  __device__ __forceinline__ void turn_by(float t) {
#pragma unroll
    for (int db = 0; db < HD / 32; db++) o[db] *= t;
    l *= t;
  }
  // top: the largest score of this query's new keys
  __device__ __forceinline__ void raise(float top) {
    const bool move = top - kRefLift > m + kRefLag;            // (also the first keys; NaN moves nothing)
    if (__builtin_amdgcn_ballot_w64(move) == 0) return;
    const float m_new = move ? top - kRefLift : m;
    turn_by(move ? exp2_(m - m_new) : 1.f);
    m = m_new;
  }
};

template <int HD> struct Query8 {
  u32x4_t f[HD / 16];
  float scale;                                                // of the scores, without a block's exponent
};
// Query `index` of the kv head (clamped by the caller); lane's dims: those of the keys' pieces, 32 u + 16 g + 0 .. 15
template <int HD> __device__ __forceinline__ Query8<HD> load_query8(const float *q, int g, float scale) {
  float x[HD / 2], amax = 0.f;
#pragma unroll
  for (int u = 0; u < HD / 32; u++) {
    float v[16];
    load16(q + 32 * u + 16 * g, v);
#pragma unroll
    for (int i = 0; i < 16; i++) { x[16 * u + i] = v[i]; amax = fmaxf(amax, finite_abs(v[i])); }
  }
  amax = max_halves(amax);
  const int e = min(max((int)(__float_as_uint(amax) >> 23) - 127, -126), 126);
  const float down = pow2(-e);
  Query8<HD> r;
#pragma unroll
  for (int s = 0; s < HD / 16; s++)
#pragma unroll
    for (int i = 0; i < 4; i++) r.f[s][i] = pack_f16x2(x[8 * s + 2 * i] * down, x[8 * s + 2 * i + 1] * down);
  r.scale = scale * pow2(e);
  return r;
}

// The weights of 64 keys of a block for 32 queries, out of their scores; exps: the block's exponents + 127 of keys and values; top_exp: the largest value exponent so
// far, r.o is in units of 2^top_exp.  p: those of 16 keys each, in fp16.
template <int HD>
__device__ __forceinline__ void weigh(Running<HD> &r, float q_scale, uint32_t exps, int &top_exp, f32x16_t (&s)[2], u32x4_t (&p)[4]) {
  const int ek = (int)(exps & 0xFF) - 127, ev = (int)((exps >> 8) & 0xFF) - 127;
  if (ev > top_exp) {
    const float t = exp2_((float)(top_exp - ev));
#pragma unroll
    for (int db = 0; db < HD / 32; db++) r.o[db] *= t;
    top_exp = ev;
  }
  const float f = q_scale * pow2(ek);
  float top = s[0][0];
#pragma unroll
  for (int kt = 0; kt < 2; kt++)
#pragma unroll
    for (int i = 0; i < 16; i++) top = __builtin_elementwise_maximum(top, s[kt][i]);   // (v_maximum3: no quieting ahead of it; with a NaN among them the query's result is NaN, whatever the reference)
  r.raise(max_halves(top) * f);
  const int under = max(ev - top_exp, -60);                   // (from about -40 on the weights are nothing in fp16, but their sum still has to hold)
  const float minus = (float)under + kCutLift - r.m;          // (the reference of a query whose scores are all NaN stays -inf: its weights are NaN)
  float sum = 0.f;
#pragma unroll
  for (int h = 0; h < 4; h++)
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      const float x = exp2_(fmaf(s[h >> 1][8 * (h & 1) + i], f, minus)), y = exp2_(fmaf(s[h >> 1][8 * (h & 1) + i + 1], f, minus));
      sum += x + y;
      p[h][i / 2] = cut_f16x2(x, y);
    }
  r.l = fmaf(sum, pow2(-under), r.l);
}

// 64 keys of a block for 32 queries.  keys(kt, s), values(kt, db, a): the fp16 operands (s: 16 dims, a: 16 keys)
template <int HD, typename K, typename V>
__device__ __forceinline__ void block_step(Running<HD> &r, const Query8<HD> &q, uint32_t exps, int &top_exp, K keys, V values) {
  f32x16_t s[2];
#pragma unroll
  for (int kt = 0; kt < 2; kt++) {
#pragma unroll
    for (int i = 0; i < 16; i++) s[kt][i] = 0.f;
#pragma unroll
    for (int t = 0; t < HD / 16; t++) s[kt] = mul_f16(keys(kt, t), q.f[t], s[kt]);
  }
  u32x4_t p[4];
  weigh<HD>(r, q.scale, exps, top_exp, s, p);
#pragma unroll
  for (int h = 0; h < 4; h++)
#pragma unroll
    for (int db = 0; db < HD / 32; db++) r.o[db] = mul_f16(values(h >> 1, db, h & 1), p[h], r.o[db]);
}

// ---- the window: 32 of its rows at a time for a wavefront's 32 queries ----
// Queries and weights go through the bf16 products as two terms each (value and what its rounding left).  Values that are not finite are taken out of the products, where they
// would reach every query, and added by hand to those that see them.
template <int HD> struct QueryWin { u32x4_t hi[HD / 16], lo[HD / 16]; };
template <int HD> __device__ __forceinline__ QueryWin<HD> load_query_win(const float *q, int g) {
  QueryWin<HD> r;
#pragma unroll
  for (int s = 0; s < HD / 16; s++) {
    const f32x4_t a = *(const f32x4_t *)(q + 16 * s + 8 * g), b = *(const f32x4_t *)(q + 16 * s + 8 * g + 4);
    const float x[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const uint32_t h = pack_bf16x2(x[2 * i], x[2 * i + 1]);
      r.hi[s][i] = h;
      r.lo[s][i] = pack_bf16x2(x[2 * i] - __uint_as_float(h << 16), x[2 * i + 1] - __uint_as_float(h & 0xFFFF0000u));
    }
  }
  return r;
}
// What a query sees of the window: rows below `first`, and its path: rows path[0 .. deep] (anc; -1: outside), or first .. first + deep
struct Sight { int deep, last, whole, path[kAncStride]; };    // last: the highest row it sees; whole: the rows below this one it sees all, once each
__device__ __forceinline__ Sight sight_of(const Attn8Args &a, int row, bool any) {
  Sight s;
  const int first = a.base - a.n_blocks * kKv8Block;
  const int deep = a.depth[row];
  if (a.anc)
#pragma unroll
    for (int d = 0; d < kAncStride; d++) s.path[d] = a.anc[(size_t)row * kAncStride + d];   // (all at once: one trip to memory)
  s.deep = any ? min(deep, a.max_depth) : -1;
  s.last = s.deep < 0 ? -1 : a.anc ? first - 1 : (int)min((int64_t)first + s.deep, (int64_t)a.win_rows - 1);
  s.whole = a.anc ? first : s.last + 1;
  if (a.anc)
#pragma unroll
    for (int d = 0; d < kAncStride; d++) {
      const int64_t r = (int64_t)first + s.path[d];
      s.path[d] = d <= s.deep && r >= 0 && r < a.win_rows ? (int)r : -1;
      s.last = max(s.last, s.path[d]);
      if (s.path[d] >= 0) s.whole = min(s.whole, s.path[d]);
    }
  s.last = min(s.last, a.win_rows - 1);
  s.whole = s.deep < 0 ? 0x7FFFFFFF : min(s.whole, a.win_rows);   // (a query that is none takes any weights)
  return s;
}
__device__ __forceinline__ int wave_max_i(int x) { return __builtin_amdgcn_readfirstlane(wave_reduce(x, [](int a, int b) { return max(a, b); })); }

// A 16-byte piece of a value row without what is not finite in it; whether there was any
__device__ __forceinline__ bool finite_piece(u32x4_t &v) {
  uint32_t over = 0;                                          // bit 15 of a half: its magnitude is 0x7F80 or more
#pragma unroll
  for (int j = 0; j < 4; j++) over |= (v[j] & 0x7FFF7FFFu) + 0x00800080u;
  if ((over & 0x80008000u) == 0) return false;
#pragma unroll
  for (int j = 0; j < 4; j++) {
    const bool lo = (v[j] & 0x7F80u) == 0x7F80u, hi = (v[j] & 0x7F800000u) == 0x7F800000u;
    v[j] &= (lo ? 0xFFFF0000u : 0xFFFFFFFFu) & (hi ? 0xFFFFu : 0xFFFFFFFFu);
  }
  return true;
}

// Rows w0 .. w0 + 31.  key(t): the operands of 16 dims; v_lds: the value rows (those not finite as zeros; odd: the rows that held such), w0's at row v_row of it; count:
// 1 KiB of this wavefront.
template <int HD, typename K>
__device__ __forceinline__ void window_step(const Attn8Args &a, Running<HD> &r, const QueryWin<HD> &q, int kvh, const Sight &see, bool whole, int w0, K key, const unsigned char *v_lds,
                                            int v_row, uint32_t odd, uint32_t *count) {
  const int lane = threadIdx.x & 63, c = lane & 31, g = lane >> 5;
  f32x16_t s;
#pragma unroll
  for (int i = 0; i < 16; i++) s[i] = 0.f;
#pragma unroll
  for (int t = 0; t < HD / 16; t++) {
    const u32x4_t k = key(t);
    s = mul_bf16(k, q.hi[t], s);
    s = mul_bf16(k, q.lo[t], s);
  }
  uint32_t seen = 0xFFFFFFFFu;                                // bit w: the query sees row w0 + w
  bool counts = false;                                        // one of the queries sees a row more than once
  float top = -INFINITY;                                      // of the scores; NaN if one is
  if (whole) {
#pragma unroll
    for (int i = 0; i < 16; i++) { s[i] *= a.scale; top = __builtin_elementwise_maximum(top, s[i]); }
  } else {
    const int below = min(!a.anc ? see.last + 1 : see.deep < 0 ? 0 : a.base - a.n_blocks * kKv8Block, a.win_rows) - w0;   // rows that every position up to the query's brings
    seen = below >= 32 ? 0xFFFFFFFFu : below <= 0 ? 0u : (1u << below) - 1;
    if (a.anc) {
      uint32_t again = 0;
#pragma unroll
      for (int d = 0; d < kAncStride; d++) {
        const uint32_t w = (uint32_t)(see.path[d] - w0), bit = w < 32u ? 1u << w : 0u;   // (-1 - w0: far beyond)
        again |= seen & bit;
        seen |= bit;
      }
      counts = __builtin_amdgcn_ballot_w64(again != 0) != 0;
    }
    const uint32_t own = seen >> (4 * g);
#pragma unroll
    for (int i = 0; i < 16; i++) {
      s[i] = (own >> (8 * (i >> 2) + (i & 3))) & 1 ? s[i] * a.scale : -INFINITY;
      top = __builtin_elementwise_maximum(top, s[i]);
    }
  }
  if (__builtin_amdgcn_ballot_w64(top != top)) {              // (never, as a rule)
    // Where a score is an infinity (by a key's or a query's, or beyond fp32), the products with what the query's rounding left may make NaN of it: such a score is that of the first terms.
    f32x16_t first;
#pragma unroll
    for (int i = 0; i < 16; i++) first[i] = 0.f;
#pragma unroll
    for (int t = 0; t < HD / 16; t++) {
      first = mul_bf16(key(t), q.hi[t], first);
      __builtin_amdgcn_sched_barrier(0);                      // (one key in registers at a time)
    }
    top = -INFINITY;
#pragma unroll
    for (int i = 0; i < 16; i++) {
      s[i] = s[i] == s[i] ? s[i] : first[i] * a.scale;
      top = fmaxf(top, s[i]);
    }
  }
  r.raise(max_halves(top));
  const float m = r.m == -INFINITY ? 0.f : r.m;
#pragma unroll
  for (int i = 0; i < 16; i++) s[i] = exp2_(s[i] - m);
  if (counts) {                                               // (paths that hold a row twice: no tree's)
    wave_fence();                                             // (the counts before have been read)
    uint32_t *mine = count + c * 8;
    *(u32x4_t *)(mine + 4 * g) = u32x4_t{0, 0, 0, 0};
    wave_fence();
    if (g == 0)
#pragma unroll
      for (int d = 0; d < kAncStride; d++) {
        const uint32_t w = (uint32_t)(see.path[d] - w0);
        if (w < 32u) __hip_atomic_fetch_add(mine + (w >> 2), 1u << (8 * (w & 3)), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WAVEFRONT);
      }
    wave_fence();
    const int first = see.deep < 0 ? 0 : a.base - a.n_blocks * kKv8Block;
#pragma unroll
    for (int i = 0; i < 16; i++) {
      const uint32_t times = ((mine[2 * (i >> 2) + g] >> (8 * (i & 3))) & 0xFF) + (w0 + 8 * (i >> 2) + 4 * g + (i & 3) < first ? 1 : 0);
      if (times > 1) s[i] *= (float)times;
    }
  }
#pragma unroll
  for (int i = 0; i < 16; i++) r.l += s[i];
#pragma unroll
  for (int h = 0; h < 2; h++) {
    u32x4_t hi, lo;
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const float x = s[8 * h + 2 * i], y = s[8 * h + 2 * i + 1];
      hi[i] = pack_bf16x2(x, y);
      lo[i] = pack_bf16x2(x - __uint_as_float(hi[i] << 16), y - __uint_as_float(hi[i] & 0xFFFF0000u));
    }
#pragma unroll
    for (int db = 0; db < HD / 32; db++) {
      const u32x4_t v = value_fragment<HD>(v_lds, value_lane<HD>(lane), db, v_row + 16 * h);
      r.o[db] = mul_bf16(v, hi, r.o[db]);
      r.o[db] = mul_bf16(v, lo, r.o[db]);
    }
  }
  while (odd) {                                               // (never, as a rule)
    const int w = __builtin_ctz(odd);
    odd &= odd - 1;
    const uint16_t *vr = (const uint16_t *)a.vwin + (size_t)min(w0 + w, a.win_rows - 1) * ((size_t)a.hkv * HD) + (size_t)kvh * HD;
    float p = 0.f;
#pragma unroll
    for (int i = 0; i < 16; i++)
      if (i == ((w >> 3) << 2 | (w & 3))) p = s[i];
    p = __shfl(p, ((w >> 2) & 1) * 32 + c);
#pragma unroll
    for (int db = 0; db < HD / 32; db++)
#pragma unroll
      for (int i = 0; i < 16; i++) {
        const uint32_t b = vr[db * 32 + 8 * (i >> 2) + 4 * g + (i & 3)];
        if (((seen >> w) & 1) && (b & 0x7F80u) == 0x7F80u) r.o[db][i] = fmaf(p, bf16_bits_to_f32(b), r.o[db][i]);
      }
  }
}

// Rows from w up to `stop` for WAVES wavefronts of 32 queries each: 64 rows at a time in the LDS (two buffers), keys in the order of the operands.
template <int HD, int WAVES> struct WindowLds {
  static constexpr int kKeys = 128 * HD, kBuffer = 2 * kKeys, kCounts = 2 * kBuffer, kOdd = kCounts + WAVES * 1024, kLast = kOdd + 24, total = kLast + WAVES * 4;
};
template <int HD, int WAVES>
__device__ __forceinline__ void window_together(const Attn8Args &a, Running<HD> &r, const float *qp, int row, bool real, int kvh, int w, int stop, unsigned char *lds) {
  using L = WindowLds<HD, WAVES>;
  constexpr int kPieces = HD / 8, kEach = 64 * kPieces / (WAVES * 64);   // 16-byte pieces of a row; of the keys (and the values) per thread
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 5;
  const size_t ld = (size_t)a.hkv * HD;
  const uint16_t *kw = (const uint16_t *)a.kwin + (size_t)kvh * HD, *vw = (const uint16_t *)a.vwin + (size_t)kvh * HD;
  uint32_t *odd = (uint32_t *)(lds + L::kOdd);                // [3][2]: of a tile's halves, the rows with values that are not finite
  int *lasts = (int *)(lds + L::kLast);
  u32x4_t key[kEach], val[kEach];
  auto fetch = [&](int w0) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kEach; i++) {
      const int at = i * WAVES * 64 + tid;
      const size_t from = (size_t)min(w0 + at / kPieces, a.win_rows - 1) * ld + at % kPieces * 8;
      key[i] = *(const u32x4_t *)(kw + from);
      val[i] = *(const u32x4_t *)(vw + from);
    }
  };
  auto put = [&](int tile) __attribute__((always_inline)) {
    unsigned char *buf = lds + (tile & 1) * L::kBuffer;
#pragma unroll
    for (int i = 0; i < kEach; i++) {
      const int at = i * WAVES * 64 + tid, wr = at / kPieces, piece = at % kPieces;
      *(u32x4_t *)(buf + (wr >> 5) * 64 * HD + (piece >> 1) * 1024 + ((piece & 1) * 32 + (wr & 31)) * 16) = key[i];
      if (finite_piece(val[i])) __hip_atomic_fetch_or(odd + tile % 3 * 2 + (wr >> 5), 1u << (wr & 31), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
      *(u32x4_t *)(buf + L::kKeys + value_piece<HD>(wr, piece)) = val[i];
    }
    if (tid < 2) odd[(tile + 1) % 3 * 2 + tid] = 0;           // (last read two tiles ago)
  };
  fetch(w);
  const Sight see = sight_of(a, row, real);
  const QueryWin<HD> q = load_query_win<HD>(qp, g);
  const int own_last = wave_max_i(see.last), whole = -wave_max_i(-see.whole);
  if (lane == 0) lasts[wave] = own_last;
  if (tid < 2) odd[tid] = 0;
  __syncthreads();
  int last = lasts[0];
#pragma unroll
  for (int i = 1; i < WAVES; i++) last = max(last, lasts[i]);
  last = min(__builtin_amdgcn_readfirstlane(last), stop - 1);
  if (w > last) return;
  put(0);
  for (int tile = 0; w <= last; tile++, w += 64) {
    __syncthreads();
    if (w + 64 <= last) fetch(w + 64);
    const unsigned char *buf = lds + (tile & 1) * L::kBuffer;
#pragma unroll 1
    for (int h = 0; h < 2; h++) {
      const int w0 = w + 32 * h;
      if (w0 > own_last || w0 >= stop) break;
      window_step<HD>(a, r, q, kvh, see, w0 + 32 <= whole, w0, [&](int t) { return *(const u32x4_t *)(buf + h * 64 * HD + t * 1024 + lane * 16); }, buf + L::kKeys, 32 * h,
                      __builtin_amdgcn_readfirstlane((int)odd[tile % 3 * 2 + h]), (uint32_t *)(lds + L::kCounts) + wave * 256);
    }
    if (w + 64 <= last) put(tile + 1);
  }
}

// The same for a wavefront alone: rows w .. w + 31, then `by` further on, straight into its registers; v_lds: 64 * HD + 1024 bytes of its own
template <int HD>
__device__ __forceinline__ void window_alone(const Attn8Args &a, Running<HD> &r, const float *qp, int row, bool real, int kvh, int w, int by, int stop, unsigned char *v_lds) {
  const int lane = threadIdx.x & 63, c = lane & 31, g = lane >> 5;
  const size_t ld = (size_t)a.hkv * HD;
  constexpr int kPieces = HD / 8;
  u32x4_t key[HD / 16], val[HD / 16];
  auto fetch = [&](int w0) __attribute__((always_inline)) {
    const uint16_t *kr = (const uint16_t *)a.kwin + (size_t)min(w0 + c, a.win_rows - 1) * ld + (size_t)kvh * HD + 8 * g;
#pragma unroll
    for (int i = 0; i < HD / 16; i++) key[i] = *(const u32x4_t *)(kr + 16 * i);
#pragma unroll
    for (int i = 0; i < HD / 16; i++) {
      const int at = i * 64 + lane;
      val[i] = *(const u32x4_t *)((const uint16_t *)a.vwin + (size_t)min(w0 + at / kPieces, a.win_rows - 1) * ld + (size_t)kvh * HD + at % kPieces * 8);
    }
  };
  fetch(w);                                                   // (the queries, paths and rows in one trip to memory)
  const Sight see = sight_of(a, row, real);
  const QueryWin<HD> q = load_query_win<HD>(qp, g);
  const int last = min(wave_max_i(see.last), stop - 1), whole = -wave_max_i(-see.whole);
  for (; w <= last; w += by) {
    wave_fence();                                             // (the tile before has been read)
    uint32_t odd = 0;
#pragma unroll
    for (int i = 0; i < HD / 16; i++) {
      const int at = i * 64 + lane;
      uint64_t mask = __builtin_amdgcn_ballot_w64(finite_piece(val[i]));
      *(u32x4_t *)(v_lds + value_piece<HD>(at / kPieces, at % kPieces)) = val[i];
      while (mask) {
        odd |= 1u << ((i * 64 + __builtin_ctzll(mask)) / kPieces);
        mask &= mask - 1;
      }
    }
    wave_fence();
    window_step<HD>(a, r, q, kvh, see, w + 32 <= whole, w, [&](int t) { return key[t]; }, v_lds, 0, odd, (uint32_t *)(v_lds + 64 * HD));
    if (w + by <= last) fetch(w + by);
  }
}

// A part of the scratch: references and sums of all queries, padded to 16 bytes, then their outputs (every output 16 bytes aligned, whatever the number of queries)
__host__ __device__ inline size_t part_stats(size_t queries) { return 2 * ((queries + 1) / 2 * 2); }
__host__ __device__ inline size_t part_floats(size_t queries, int hd) { return part_stats(queries) + queries * hd; }
// A part's result of this lane's query: reference, sum and outputs, or, if the launch has one part, the query's result
template <int HD>
__device__ __forceinline__ void put_dims(const Attn8Args &a, size_t query, int part, int parts, int db, int g, const f32x16_t &o, float m, float l) {
  if (parts == 1) {
    const float inv = l == 0.f ? 0.f : 1.f / l;
    uint16_t *out = (uint16_t *)a.out + query * HD + db * 32 + 4 * g;
#pragma unroll
    for (int i = 0; i < 4; i++)
      *(u32x2_t *)(out + 8 * i) = u32x2_t{pack_bf16x2(o[4 * i] * inv, o[4 * i + 1] * inv), pack_bf16x2(o[4 * i + 2] * inv, o[4 * i + 3] * inv)};
    return;
  }
  const size_t queries = (size_t)a.rows * a.hq;
  float *p = a.part + part * part_floats(queries, HD);
  float *po = p + part_stats(queries) + query * HD + db * 32 + 4 * g;
#pragma unroll
  for (int i = 0; i < 4; i++) *(f32x4_t *)(po + 8 * i) = f32x4_t{o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]};
  if (db == 0 && g == 0) ((float2 *)p)[query] = make_float2(m, l);
}
__device__ __forceinline__ float sum_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Which kv head, part and block of queries a workgroup has.  A unit is a part of a kv head; ids 8 apart run on one XCD, which gets consecutive units (the query blocks of a part read the same
// keys) as evenly as they go; in launches of several rounds over the compute units whose units do not go into 8, single query blocks in turn.  The last query block, which sees most of the
// window, comes first (us the other way round: 4000 rows on 8 kv heads behind 16 blocks 309 -> 385, 3000 behind 64 352 -> 434).
struct Place8 { int kvh, part, qb; };
__device__ __forceinline__ bool place_of(const Plan8 &p, int hkv, Place8 &at) {
  const int parts = p.block_parts + p.win_parts, units = hkv * parts, all = units * p.query_blocks, each = (all + 7) / 8;
  int id = (int)blockIdx.x;
  if (units % 8 == 0 || all <= 256) {
    if (id / 8 >= each) return false;
    id = id % 8 * each + id / 8;
  }
  if (id >= all) return false;
  const int unit = id / p.query_blocks;
  at.qb = p.query_blocks - 1 - id % p.query_blocks;
  at.kvh = unit / parts; at.part = unit % parts;
  return true;
}

// Many queries: WAVES wavefronts of 32 queries each walk the part's keys together.  A block's codes are widened once, on their way into the LDS (two buffers; the
// next block's are in registers meanwhile), in the order in which the products read them.
// Eight wavefronts take 1.84 us a block: 256 workgroups together 1.17 PFLOP/s.  Without reads from the LDS 1.75, without the weights' arithmetic 1.53, without both 1.36 (1.58
// PFLOP/s: at the clock of 1.5 GHz that the products alone leave the chip), without the products 1.23.
// Tried, with the same time: two teams of four wavefronts that take turns at the matrix instructions and at the weights, a barrier between; the next block's scores among the
// instructions of this one's weights; slower: four wavefronts of 64 queries, scores of the
// next tile beside the weights of this one (2.4: the sums of 64 queries lie in the accumulation registers, and every read of one is an instruction).
// Registers: two wavefronts may take 512 each (us, and with 256, of which 85 would lie in memory: 300 queries on 4 kv heads behind 20 blocks 25.4, 32.1, 64 on 32 of 64 behind 256 blocks 30.2, 32.2,
// 60 on 32 behind 64 blocks 24.5, 23.6, but 104 on 8 behind 64 blocks 20.6, 18.3). Four do better with 256, of which 11 of heads of 128 lie in memory (480 queries on 2 behind 300 blocks 29.9, with 512 34.0; 240 on 8
// behind 128 blocks 29.1, 33.9; 60 on 32 behind 8 blocks 14.3, 15.7).
template <int HD, int WAVES>
__global__ __launch_bounds__(WAVES * 64, WAVES == 2 ? 1 : 2) void attention8_wide_kernel(Attn8Args a, Plan8 plan) {
  constexpr int kCodes = 2 * kKv8Block * HD, kUnits = kCodes / 16, kThreads = WAVES * 64, kEach = kUnits / kThreads;   // of 16 codes, per thread
  static_assert(kEach * kThreads == kUnits, "whole units");
  extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];   // 2 x 2 kCodes, or WindowLds
  Place8 at;
  if (!place_of(plan, a.hkv, at)) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 31, g = lane >> 5;
  const int G = a.hq / a.hkv, index = (at.qb * WAVES + wave) * 32 + c, parts = plan.block_parts + plan.win_parts;
  const bool real = index < a.rows * G;
  const bool any = index - c < a.rows * G;                    // this wavefront has queries (else it only loads and widens)
  const int row = real ? index / G : a.rows - 1;
  const size_t query = (size_t)row * a.hq + at.kvh * G + (real ? index % G : 0);
  const float *qp = a.q + query * HD;
  Running<HD> r;
  r.clear();
  const int b0 = at.part < plan.block_parts ? joined_range_at(plan, a.n_blocks, at.qb, at.part) : 0;
  const int b1 = at.part < plan.block_parts ? joined_range_at(plan, a.n_blocks, at.qb, at.part + 1) : 0;
  if (b0 < b1) {
    const size_t block_bytes = kv8_block_bytes(a.hkv, HD);
    const unsigned char *base = a.cache8 + (size_t)at.kvh * kCodes + tid * 16;
    const unsigned char *exps = a.cache8 + (size_t)a.hkv * kCodes + 2 * at.kvh;
    const Query8<HD> q = load_query8<HD>(qp, g, a.scale);
    u32x4_t next[kEach];
    uint32_t next_exps;
    auto fetch = [&](int b) {
      const unsigned char *p = base + (size_t)b * block_bytes;
#pragma unroll
      for (int i = 0; i < kEach; i++) next[i] = *(const u32x4_t *)(p + i * kThreads * 16);
      next_exps = *(const uint16_t *)(exps + (size_t)b * block_bytes);
    };
    auto put = [&](unsigned char *buf) {
#pragma unroll
      for (int i = 0; i < kEach; i++) {
        u32x4_t x, y;
        widen(next[i], x, y);
        unsigned char *p = buf + ((i * kThreads + tid) >> 6) * 2048 + lane * 16;
        *(u32x4_t *)p = x;
        *(u32x4_t *)(p + 1024) = y;
      }
    };
    int top_exp = -127;
    fetch(b0);
    put(lds);
    uint32_t now_exps = __builtin_amdgcn_readfirstlane(next_exps);
    __syncthreads();
    auto walk = [&](auto with_queries) __attribute__((always_inline)) {
      for (int b = b0; b < b1; b++) {
        const unsigned char *buf = lds + ((b - b0) & 1) * 2 * kCodes + lane * 16;
        if (b + 1 < b1) fetch(b + 1);
        if constexpr (decltype(with_queries)::value)
          block_step<HD>(r, q, now_exps, top_exp,
                         [&](int kt, int s) { return *(const u32x4_t *)(buf + (kt * (HD / 16) + s) * 1024); },
                         [&](int kt, int db, int h) { return *(const u32x4_t *)(buf + kCodes + (kt * (HD / 16) + 2 * db + h) * 1024); });
        if (b + 1 < b1) {
          put(lds + ((b + 1 - b0) & 1) * 2 * kCodes);
          now_exps = __builtin_amdgcn_readfirstlane(next_exps);
        }
        __syncthreads();
      }
    };
    if (any) walk(std::true_type{});
    else walk(std::false_type{});                             // (as many barriers, which count wavefronts)
    r.l *= kCutSum;
    const float up = exp2_((float)top_exp);
#pragma unroll
    for (int db = 0; db < HD / 32; db++) r.o[db] *= up;
  }
  if (plan.win_parts ? at.part >= plan.block_parts : at.part == plan.block_parts - 1) {   // (behind a loop over blocks: its last barrier frees the LDS)
    const int w_begin = plan.win_parts ? (at.part - plan.block_parts) * plan.win_part : 0;
    window_together<HD, WAVES>(a, r, qp, row, real, at.kvh, w_begin, plan.win_parts ? min(w_begin + plan.win_part, a.win_rows) : a.win_rows, lds);
  }
  const float l = sum_halves(r.l);
  if (!real || (parts == 1 && a.depth[row] < 0)) return;
#pragma unroll
  for (int db = 0; db < HD / 32; db++) put_dims<HD>(a, query, at.part, parts, db, g, r.o[db], r.m, l);
}

// Up to 32 queries: the four wavefronts share the part's keys, a block (or 32 rows of the window) each in turn, straight into registers, and are merged in the LDS.
constexpr int kFewWaves = 4;
template <int HD>
__global__ __launch_bounds__(kFewWaves * 64) void attention8_few_kernel(Attn8Args a, Plan8 plan) {
  constexpr int kCodes = 2 * kKv8Block * HD, kPieces = kCodes / 1024;
  extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];   // outputs of each wavefront (or its value rows and counts), then references and sums
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 31, g = lane >> 5;
  const int parts = plan.block_parts + plan.win_parts, kvh = blockIdx.x / parts, part = blockIdx.x % parts;
  const int G = a.hq / a.hkv;
  const bool real = c < a.rows * G;
  const int row = real ? c / G : a.rows - 1;
  const size_t query = (size_t)row * a.hq + kvh * G + (real ? c % G : 0);
  const float *qp = a.q + query * HD;
  Running<HD> r;
  r.clear();
  if (part < plan.block_parts) {
    const int b0 = range_at(a.n_blocks, plan.block_parts, part) + wave, b1 = range_at(a.n_blocks, plan.block_parts, part + 1);
    const size_t block_bytes = kv8_block_bytes(a.hkv, HD);
    const unsigned char *base = a.cache8 + (size_t)kvh * kCodes + lane * 16;
    const unsigned char *exps = a.cache8 + (size_t)a.hkv * kCodes + 2 * kvh;
    u32x4_t next[kPieces], now[kPieces];
    uint32_t next_exps = 0;
    auto fetch = [&](int b) {
      const unsigned char *p = base + (size_t)b * block_bytes;
#pragma unroll
      for (int i = 0; i < kPieces; i++) next[i] = *(const u32x4_t *)(p + i * 1024);
      next_exps = *(const uint16_t *)(exps + (size_t)b * block_bytes);
    };
    if (b0 < b1) fetch(b0);
    const Query8<HD> q = load_query8<HD>(qp, g, a.scale);
    int top_exp = -127;
    for (int b = b0; b < b1; b += kFewWaves) {
#pragma unroll
      for (int i = 0; i < kPieces; i++) now[i] = next[i];
      const uint32_t now_exps = __builtin_amdgcn_readfirstlane(next_exps);
      if (b + kFewWaves < b1) fetch(b + kFewWaves);
      auto half = [&](const u32x4_t &w, int h) {
        u32x4_t x, y;
        widen(w, x, y);
        return h ? y : x;
      };
      block_step<HD>(r, q, now_exps, top_exp, [&](int kt, int s) { return half(now[kt * (HD / 32) + s / 2], s & 1); },
                     [&](int kt, int db, int h) { return half(now[kPieces / 2 + kt * (HD / 32) + db], h); });
    }
    r.l *= kCutSum;
    const float up = exp2_((float)top_exp);
#pragma unroll
    for (int db = 0; db < HD / 32; db++) r.o[db] *= up;
  }
  if (part >= plan.block_parts || plan.win_parts == 0) {
    const int w_begin = plan.win_parts ? (part - plan.block_parts) * plan.win_part : 0, w_stop = plan.win_parts ? min(w_begin + plan.win_part, a.win_rows) : a.win_rows;
    window_alone<HD>(a, r, qp, row, real, kvh, w_begin + 32 * wave, 32 * kFewWaves, w_stop, lds + wave * (64 * HD + 1024));
    __syncthreads();                                          // the value rows make place for the outputs
  }
  float *outs = (float *)lds;                                 // [wave][db][16][64]
  float2 *stats = (float2 *)(lds + kFewWaves * HD * 128);     // [wave][32]
#pragma unroll
  for (int db = 0; db < HD / 32; db++)
#pragma unroll
    for (int i = 0; i < 16; i++) outs[((wave * (HD / 32) + db) * 16 + i) * 64 + lane] = r.o[db][i];
  const float own_l = sum_halves(r.l);
  if (g == 0) stats[wave * 32 + c] = make_float2(r.m, own_l);
  __syncthreads();
  if (wave >= HD / 32 || !real || (parts == 1 && a.depth[row] < 0)) return;
  RowMerge all;                                               // this wavefront joins the dims 32 wave .. + 31
  f32x16_t o;
#pragma unroll
  for (int i = 0; i < 16; i++) o[i] = 0.f;
#pragma unroll
  for (int w = 0; w < kFewWaves; w++) {
    const float2 s = stats[w * 32 + c];
    if (s.y == 0.f) continue;                                 // saw nothing
    float weight;
    const float turn = all.step(s.x, s.y, weight);
#pragma unroll
    for (int i = 0; i < 16; i++) o[i] = fmaf(outs[((w * (HD / 32) + wave) * 16 + i) * 64 + lane], weight, o[i] * turn);
  }
  put_dims<HD>(a, query, part, parts, wave, g, o, all.m, all.l);
}

// The parts of a query put together: HD / 4 threads take a query's dims, GROUPS of them every GROUPS-th part each (up to eight on their way at a time), then the
// groups' sums in ascending order.
template <int HD, int GROUPS>
__global__ __launch_bounds__(256) void attention8_merge_kernel(Attn8Args a, int parts) {
  constexpr int kThreads = HD / 4, kQueries = 256 / (kThreads * GROUPS);
  static_assert(kQueries >= 1, "threads");
  __shared__ f32x4_t sums[GROUPS > 1 ? 256 : 1];
  __shared__ float2 stats[GROUPS > 1 ? kQueries * GROUPS : 1];
  const int in_query = threadIdx.x % (kThreads * GROUPS), slot = threadIdx.x / (kThreads * GROUPS), group = in_query / kThreads, d = in_query % kThreads * 4;
  const size_t all_queries = (size_t)a.rows * a.hq, query = ((size_t)blockIdx.y * gridDim.x + blockIdx.x) * kQueries + slot, at = query < all_queries ? query : all_queries - 1;
  RowMerge all;
  f32x4_t o{0.f, 0.f, 0.f, 0.f};
  const size_t part_size = part_floats(all_queries, HD), stats_size = part_stats(all_queries);
  for (int i0 = group; i0 < parts; i0 += 8 * GROUPS) {
    float2 s[8];
    f32x4_t x[8];
#pragma unroll
    for (int j = 0; j < 8; j++) {
      const float *p = a.part + min(i0 + j * GROUPS, parts - 1) * part_size;
      s[j] = ((const float2 *)p)[at];
      x[j] = *(const f32x4_t *)(p + stats_size + at * HD + d);
    }
#pragma unroll
    for (int j = 0; j < 8; j++) {
      if (i0 + j * GROUPS >= parts || s[j].y == 0.f) continue;   // (it saw nothing: its outputs may be anything)
      float weight;
      const float turn = all.step(s[j].x, s[j].y, weight);
#pragma unroll
      for (int e = 0; e < 4; e++) o[e] = fmaf(x[j][e], weight, o[e] * turn);
    }
  }
  if constexpr (GROUPS > 1) {
    sums[threadIdx.x] = o;
    if (d == 0) stats[slot * GROUPS + group] = make_float2(all.m, all.l);
    __syncthreads();
    if (group > 0) return;
    all = RowMerge{};
    o = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < GROUPS; j++) {
      const float2 s = stats[slot * GROUPS + j];
      if (s.y == 0.f) continue;
      float weight;
      const float turn = all.step(s.x, s.y, weight);
      const f32x4_t x = sums[threadIdx.x + j * kThreads];
#pragma unroll
      for (int e = 0; e < 4; e++) o[e] = fmaf(x[e], weight, o[e] * turn);
    }
  }
  if (query >= all_queries || a.depth[query / a.hq] < 0) return;
  const float inv = all.l == 0.f ? 0.f : 1.f / all.l;
  *(u32x2_t *)((uint16_t *)a.out + query * HD + d) = u32x2_t{pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv)};
}

Plan8 plan8(int rows, int hq, int hkv, int n_blocks, int win_rows) {
  Plan8 p{};
  const int G = hq / hkv;
  const int64_t queries = (int64_t)rows * G;
  // Wavefronts by the work, in tiles of 32 queries over 64 keys.  Up to 64 queries: four, of which those without queries only load and widen, where there is little work, two, for more workgroups, where
  // there is much.  More queries: eight, which share the widening, where there is much work, two where there is little in few tiles, else four.  us with 2, 4, 8: 60 queries on 32 kv heads, 8 blocks 16.0, 14.2, 15.5, 128 blocks 32, 35, 35;
  // 240 on 8, 8 blocks 15.2, 17.0, 19.2, 128 blocks 30, 26, 34, 512 blocks 74, 58, 54; 1200 on 8, 8 blocks 31, 27, 30, 128 blocks 221, 160, 67.
  const int64_t tiles = (queries + 31) / 32, wide = hkv * tiles, work = wide * (n_blocks + win_rows / 32);
  p.waves = queries <= 32 ? 0 : tiles <= 2 ? (work <= 4096 ? 4 : 2) : work >= (wide >= 96 ? 6144 : 20480) ? 8 : wide <= 64 && work <= 2304 ? 2 : 4;
  const int of = p.waves ? 32 * p.waves : 32;
  p.query_blocks = (int)((queries + of - 1) / of);
  const int64_t units = (int64_t)hkv * p.query_blocks;
  // rows of the window per part: the step of a workgroup where the blocks are hardly more than one each, too (us with 32 against 64: 50 queries on 8 kv heads of 64, 512 keys 9.6, 10.7;
  // 60 on 32, 512 keys 14.4, 14.8, but 16384 keys 48.5, 46.8); long windows come in tiles of 64
  p.win_part = win_rows > 256 || p.waves == 8 ? 256 : p.waves && units * n_blocks <= 256 ? 32 : 64;
  while ((win_rows + p.win_part - 1) / p.win_part > 8) p.win_part *= 2;
  p.win_parts = (win_rows + p.win_part - 1) / p.win_part;
  const int64_t most = p.waves ? n_blocks : (n_blocks + kFewWaves - 1) / kFewWaves;
  // Short: one part, no second launch and no scratch.  us on the card alone, against two launches: a row on 8 kv heads behind 4 blocks 11.3, 10.9 (head_dim 64: 7.9, 8.5), but 8 blocks, two a
  // wavefront, 12.6, 11.0; a call's host time is 9.3 against 13
  if (p.waves == 0 && n_blocks > 0 && n_blocks <= kFewWaves && win_rows <= 32 * kFewWaves) {
    p.block_parts = 1;
    p.win_parts = 0;
    return p;
  }
  if (p.waves == 8 && n_blocks > 0) {
    // A window costs 2.5 blocks, and 2.25 for 64 rows.  Joined to the last range of blocks, if that is not more than the range's share of all (us with this, and with 1.5 for 64 rows alone:
    // 1024 rows on 8 kv heads behind 128 blocks 167, 176, behind 32 blocks and 100 rows 83, 91; a tree of 60 rows behind 512 blocks 79, 83), else as many parts as it has shares.
    const int parts = (int)(units >= 256 ? 1 : 256 / units);
    const int64_t win_cost = 40 + (int64_t)win_rows * 36 / 64, all = 16 * (int64_t)n_blocks + win_cost;
    if (parts > 1 && win_cost * parts > all) {
      const int shares = (int)((win_cost * parts + all / 2) / all), of_window = shares < 1 ? 1 : shares < parts ? shares : parts - 1;
      p.win_part = ((win_rows + of_window - 1) / of_window + 63) / 64 * 64;
      p.win_parts = (win_rows + p.win_part - 1) / p.win_part;
      p.block_parts = parts - of_window < n_blocks ? parts - of_window : n_blocks;
      return p;
    }
    p.win_parts = 0;
    p.block_parts = parts < n_blocks ? parts : n_blocks;
    // rows of the window that the first query block sees, if they are a chain, and how many more each further one does
    const int each = of / G < 1 ? 1 : of / G, recent = win_rows > rows ? win_rows - rows : 0;
    p.win_base = 40 + (recent + each) * 36 / 64;
    p.win_cost = each * 36 / 64;
    return p;
  }
  // One workgroup a unit; two of two wavefronts where each would have eight blocks or more (us: 60 queries on 32 kv heads, 512 keys 15.7 against 18.1 with 512 workgroups, 4096 29 against 25,
  // 16384 79 against 48; one query on 8, 16384 keys 15 against 22; 104 on 8, 32768 42 against 52)
  const int64_t parts = (p.waves == 2 && units * n_blocks >= 2048 ? 512 : 256) / units - p.win_parts;
  p.block_parts = n_blocks == 0 ? 0 : (int)(parts < 1 ? 1 : parts > most ? most : parts);
  return p;
}

template <int HD, int WAVES> hipError_t launch_wide(const Attn8Args &a, const Plan8 &p, unsigned grid, hipStream_t st) {
  constexpr int kLds = WindowLds<HD, WAVES>::total;
  static_assert(kLds >= 512 * HD, "keys and values fit");
  static bool allowed[64] = {};
  const hipError_t e = allow_lds((const void *)attention8_wide_kernel<HD, WAVES>, kLds, allowed);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((attention8_wide_kernel<HD, WAVES>), dim3(grid), dim3(WAVES * 64), kLds, st, a, p);
  return hipGetLastError();
}

template <int HD, int GROUPS> hipError_t launch_merge(const Attn8Args &a, int parts, hipStream_t st) {
  constexpr int kEach = 1024 / (HD * GROUPS);                 // queries of a workgroup
  const int64_t groups = ((int64_t)a.rows * a.hq + kEach - 1) / kEach, deep = (groups + (1 << 23) - 1) >> 23;   // (a grid's dimension holds less than 2^32 threads; at most 2^7 deep)
  hipLaunchKernelGGL((attention8_merge_kernel<HD, GROUPS>), dim3((unsigned)((groups + deep - 1) / deep), (unsigned)deep), dim3(256), 0, st, a, parts);
  return hipGetLastError();
}

template <int HD> hipError_t launch_hd(const Attn8Args &a, hipStream_t st) {
  const Plan8 p = plan8(a.rows, a.hq, a.hkv, a.n_blocks, a.win_rows);
  const int parts = p.block_parts + p.win_parts;
  const int64_t units = (int64_t)a.hkv * parts, grid = (units * p.query_blocks + 7) / 8 * 8;
  if (grid * 512 >> 32) return hipErrorInvalidValue;          // (beyond any memory: the limit of a grid's threads)
  hipError_t e;
  if (p.waves == 0) {
    constexpr int kLds = kFewWaves * (HD * 128 + 256);
    static_assert(kLds >= kFewWaves * (64 * HD + 1024), "value rows and counts fit");
    static bool allowed[64] = {};
    if ((e = allow_lds((const void *)attention8_few_kernel<HD>, kLds, allowed)) != hipSuccess) return e;
    hipLaunchKernelGGL(attention8_few_kernel<HD>, dim3((unsigned)units), dim3(kFewWaves * 64), kLds, st, a, p);
    e = hipGetLastError();
  } else if (p.waves == 2) e = launch_wide<HD, 2>(a, p, (unsigned)grid, st);
  else if (p.waves == 4) e = launch_wide<HD, 4>(a, p, (unsigned)grid, st);
  else e = launch_wide<HD, 8>(a, p, (unsigned)grid, st);
  if (e != hipSuccess || parts == 1) return e;
  // groups that share a query's parts, us for 1, 2, 4, 8 of them (both launches): 8 parts of 1920 queries 14.4, 16.1, 16.2, 17.9; 17 of 32 13.8, 12.7, 11.8, 12.1; 32 of 832 26.7,
  // 24.9, 24.9, 25.1; 128 of 480 53, 42, 38, 37; 256 of 64 61, 39, 29, 24
  if (parts <= 8) return launch_merge<HD, 1>(a, parts, st);
  if (parts <= 16) return launch_merge<HD, 2>(a, parts, st);
  return parts <= 32 ? launch_merge<HD, 4>(a, parts, st) : launch_merge<HD, 8>(a, parts, st);
}

}  // namespace

hipError_t launch_kv8_store(const void *k, const void *v, int64_t ld, int n_blocks, int hkv, int hd, void *cache8, int first_block, hipStream_t st) {
  for (int b = 0; b < n_blocks; b += 65535) {                 // (the grid's second dimension)
    const int n = n_blocks - b < 65535 ? n_blocks - b : 65535;
    const bf16_t *ks = (const bf16_t *)k + (int64_t)b * kKv8Block * ld, *vs = (const bf16_t *)v + (int64_t)b * kKv8Block * ld;
    if (hd == 128) hipLaunchKernelGGL(kv8_store_kernel<128>, dim3(2 * hkv, n), dim3(256), 0, st, ks, vs, ld, hkv, (unsigned char *)cache8, first_block + b);
    else hipLaunchKernelGGL(kv8_store_kernel<64>, dim3(2 * hkv, n), dim3(256), 0, st, ks, vs, ld, hkv, (unsigned char *)cache8, first_block + b);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_kv8_load(const void *cache8, int first_block, int n_blocks, int hkv, int hd, void *k, void *v, int64_t ld, hipStream_t st) {
  for (int b = 0; b < n_blocks; b += 65535) {
    const int n = n_blocks - b < 65535 ? n_blocks - b : 65535;
    bf16_t *ks = (bf16_t *)k + (int64_t)b * kKv8Block * ld, *vs = (bf16_t *)v + (int64_t)b * kKv8Block * ld;
    if (hd == 128) hipLaunchKernelGGL(kv8_load_kernel<128>, dim3(2 * hkv, n), dim3(256), 0, st, (const unsigned char *)cache8, first_block + b, hkv, ks, vs, ld);
    else hipLaunchKernelGGL(kv8_load_kernel<64>, dim3(2 * hkv, n), dim3(256), 0, st, (const unsigned char *)cache8, first_block + b, hkv, ks, vs, ld);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

size_t attention8_scratch_floats(int rows, int hq, int hkv, int hd, int n_blocks, int win_rows) {
  const Plan8 p = plan8(rows, hq, hkv, n_blocks, win_rows);
  const int parts = p.block_parts + p.win_parts;
  return parts == 1 ? 0 : parts * part_floats((size_t)rows * hq, hd);
}

void attention8_plan(int rows, int hq, int hkv, int n_blocks, int win_rows, int *waves, int *query_blocks, int *block_parts, int *win_parts) {
  const Plan8 p = plan8(rows, hq, hkv, n_blocks, win_rows);
  *waves = p.waves; *query_blocks = p.query_blocks; *block_parts = p.block_parts; *win_parts = p.win_parts;
}

hipError_t launch_attention8(const Attn8Args &a, hipStream_t st) { return a.hd == 128 ? launch_hd<128>(a, st) : launch_hd<64>(a, st); }

}  // namespace spec
