// The gated half of a feed-forward block, h = act(x Wg^T) * (x Wu^T), and its gradients (include/spec_step.h).
//
// Products of matrices as they lie in memory (weights change with every step of a training run, so that nothing is packed ahead): out[m][n] = sum over k of A(m, k) B(n, k),
// either side with k along its rows (x, the weights of the forward products) or with k across them (both sides of the weights' gradients, the weights of dx).
//   forward    : m = rows of x, n = columns of h; a workgroup's n are gate and up rows of the same columns, so that a lane holds both sums of an element of h
//   dg and du  : the same sums again, then dg = dh u act'(g), du = dh act(g), rounded to bf16 for the products that follow
//   dx         : dg Wg + du Wu, k = the columns of dg and then those of du
//   dWg, dWu   : dg^T x, du^T x, k = rows of x
// Bound: the matrix cores from some hundreds of rows on; below, the weights' way from memory.
#include "common.h"
#include "kernels.h"

namespace spec {

namespace {

typedef __attribute__((ext_vector_type(16))) float f32x16_t;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_t;
typedef __attribute__((address_space(3))) void lds_void;

// ---- activations: act(g) = g p(g), and act'(g)
struct Act { float p, slope; };
template <bool SLOPE> __device__ __forceinline__ Act activation(int act, float g) {
  Act r{0.f, 0.f};
  if (act == kActGelu) {                                      // p: the normal distribution's, through erfc, which keeps its tail
    r.p = 0.5f * erfcf(g * -0.70710678118654752f);
    if constexpr (SLOPE) r.slope = fmaf(g * 0.39894228040143268f, __builtin_amdgcn_exp2f(g * g * -0.72134752044448170f), r.p);
    return r;
  }
  // p = 1 / (1 + e^-z), z = g or twice the argument of the tanh
  const float z = act == kActSilu ? g : 1.5957691216057308f * fmaf(0.044715f * g, g * g, g);
  r.p = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * -1.4426950408889634f));
  if constexpr (SLOPE) {
    const float dz = act == kActSilu ? 1.0f : fmaf(0.21406881920f * g, g, 1.5957691216057308f);
    r.slope = fmaf(g * dz, r.p * (1.0f - r.p), r.p);
  }
  return r;
}

// ---- tiles -----------------------------------------------------------------------------------------
// Stages of 64 k in the LDS, copied there straight from memory, 16 bytes a lane and 1 KB a wavefront's instruction.
// K along the rows (MAJOR = false): a row's 128 bytes, their eight pieces permuted by row / 2 so that sixteen rows' reads of one piece touch all banks.  K across
// (MAJOR = true): per k the tile's columns, their chunks of 32 permuted by k so that the four k of a transposing read touch all banks.
constexpr int kStageK = 64;
template <int TW_, int TB_, int WQ_, int WB_> struct Tile {
  static constexpr int TW = TW_, TB = TB_, WQ = WQ_, WB = WB_;
  static constexpr int kWaves = TW * WQ, kThreads = kWaves * 64, kM = TW * TB * 32, kN = WQ * WB * 32;
  static constexpr int kMBytes = kM * 128, kNBytes = kN * 128;       // of a stage
  static constexpr int kMLoads = kM / 8 / kWaves, kNLoads = kN / 8 / kWaves;   // copies of a wavefront
};

__device__ __forceinline__ void wg_barrier() {                 // (without a wait for the copies under way)
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// One side of a tile: LOADS copies of this wavefront per stage
template <int LOADS, bool MAJOR, int COLS> struct Side {
  const char *base;                                           // of the segment, at the tile's first row (column, if MAJOR)
  uint32_t off[LOADS];                                        // of a lane, in the first stage
  int k[LOADS];                                               // of a lane within a stage
  int64_t step;                                               // bytes from one stage to the next
  // rows: how many there are from the tile's first on; ld in elements
  __device__ __forceinline__ void place(int q0, int lane, int rows, int64_t ld) {
#pragma unroll
    for (int i = 0; i < LOADS; i++) {
      const int q = q0 + i;
      if constexpr (!MAJOR) {
        const int r = q * 8 + (lane >> 3), piece = (lane & 7) ^ ((r >> 1) & 7);
        off[i] = (uint32_t)min(r, rows - 1) * (uint32_t)(2 * ld) + piece * 16;
        k[i] = piece * 8;
      } else {
        constexpr int kSlots = COLS / 8;
        const int kr = q * (64 / kSlots) + lane / kSlots, slot = lane % kSlots, col = ((slot >> 2) ^ (kr & 3)) * 32 + (slot & 3) * 8;
        off[i] = (uint32_t)kr * (uint32_t)(2 * ld) + (uint32_t)(col < rows ? col : 0) * 2;
        k[i] = kr;
      }
    }
    step = MAJOR ? (int64_t)kStageK * ld * 2 : kStageK * 2;
  }
  // stage s of the segment, of which `left` k are there from its first on
  __device__ __forceinline__ void copy(int s, int left, int64_t ld, unsigned char *to, int i0, int i1) const {
    const __amdgpu_buffer_rsrc_t src = __builtin_amdgcn_make_buffer_rsrc((void *)(base + s * step), 0, 0x7FFFFFFF, 0x00027000);
#pragma unroll
    for (int i = 0; i < LOADS; i++) {
      if (i < i0 || i >= i1) continue;
      uint32_t o = off[i];
      if (left < kStageK && k[i] >= left) o -= MAJOR ? (uint32_t)k[i] * (uint32_t)(2 * ld) : (uint32_t)k[i] * 2;   // past the end: the stage's first k, cleared when it is here
      __builtin_amdgcn_raw_ptr_buffer_load_lds(src, (lds_void *)(to + i * 1024), 16, (int)o, 0, 0, 0);
    }
  }
  __device__ __forceinline__ void clear(int left, unsigned char *mine, int lane) const {   // mine: this wavefront's share of the stage
#pragma unroll
    for (int i = 0; i < LOADS; i++)
      if (k[i] >= left) *(u32x4_t *)(mine + i * 1024 + lane * 16) = u32x4_t{0u, 0u, 0u, 0u};
  }
};
// Fragments of a block of 32 rows (columns): lane (c, g) has row c at k = 16 j + 8 g + 0 .. 7
template <bool MAJOR, int COLS> __device__ __forceinline__ int frag_lane(int lane, int block) {
  const int c = lane & 31, g = lane >> 5;
  if constexpr (!MAJOR) return (block * 32 + c) * 128 + ((g ^ ((c >> 1) & 7)) * 16);
  const int kr = 8 * g + ((lane & 15) >> 2);
  return kr * COLS * 2 + ((block ^ (kr & 3)) * 64) + ((lane >> 4) & 1) * 32 + (lane & 3) * 8;
}
template <bool MAJOR, int COLS> __device__ __forceinline__ u32x4_t frag(const unsigned char *p, int at, int t, int j) {   // block t of those that `at` begins with
  if constexpr (!MAJOR) return *(const u32x4_t *)(p + (at ^ (j * 32)) + t * 4096);
  const unsigned char *q = p + (at ^ (t * 64)) + j * 16 * COLS * 2;
  const u32x2_t a = read_columns(q), b = read_columns(q + 4 * COLS * 2);
  return u32x4_t{a.x, a.y, b.x, b.y};
}

// Two bf16 pairs of the lanes (c, 0) and (c, 1), four values each of the columns 8 b + 4 g and 8 (b + 1) + 4 g, to eight consecutive columns a lane: 8 (b + g) ..
__device__ __forceinline__ u32x4_t gather8(uint32_t a0, uint32_t a1, uint32_t b0, uint32_t b1) {
  const auto x = __builtin_amdgcn_permlane32_swap(a0, b0, false, false), y = __builtin_amdgcn_permlane32_swap(a1, b1, false, false);
  return u32x4_t{x[0], y[0], x[1], y[1]};
}

enum { kToH = 0, kToDgu = 1, kToOut = 2, kToParts = 3 };

// One tile and range of stages.  SEGS: segments of k (two: dx).
template <class L, bool MM, bool NM, int TO>
__device__ __forceinline__ void tile_body(const FfnArgs &a, int half, int m0, int n0, int s0, int s1, float *part, unsigned char *ms0, unsigned char *ms1, unsigned char *ns0,
                                          unsigned char *ns1, unsigned char *ns2) {
  constexpr int ML = L::kMLoads, NL = L::kNLoads, TB = L::TB, WB = L::WB;
  constexpr bool kGated = TO == kToH || TO == kToDgu;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 31, g = lane >> 5, th = wave % L::TW, wq = wave / L::TW;
  const int seg_stages = (a.k + kStageK - 1) / kStageK;       // of a segment
  Side<ML, MM, L::kM> ms;
  Side<NL, NM, L::kN> ns;
  const int64_t ldm = a.ldm, ldn = a.ldn;
  ms.place(wave * ML, lane, a.m - m0, ldm);
  if constexpr (kGated) {                                     // blocks of 32: gate, up, gate, .. of the same columns; a wavefront's copies are of one of them
    static_assert(NL == 4 || NL == 2, "a wavefront copies a block, or half of one");
    const int q0 = wave * NL, block = q0 / 4;
    ns.place(q0 - block * 4, lane, a.n - n0 - block / 2 * 32 > 0 ? a.n - n0 - block / 2 * 32 : 1, ldn);
    const int first = min(n0 + block / 2 * 32, a.n - 1);
    ns.base = (const char *)(block & 1 ? a.n_src[1] : a.n_src[0]) + (int64_t)first * ldn * 2;
  } else {
    ns.place(wave * NL, lane, a.n - n0, ldn);
  }
  auto m_base = [&](int seg) { return (const char *)(MM ? (half ? a.m_src[1] : a.m_src[0]) : (seg ? a.m_src[1] : a.m_src[0])) + (MM ? (int64_t)m0 * 2 : (int64_t)m0 * ldm * 2); };
  auto n_base = [&](int seg) { return (const char *)(seg ? a.n_src[1] : a.n_src[0]) + (NM ? (int64_t)n0 * 2 : (int64_t)n0 * ldn * 2); };
  ms.base = m_base(0);
  if constexpr (!kGated) ns.base = n_base(0);

  struct At { int s, left; bool second; };                    // a stage within its segment
  auto at_of = [&](int s) {
    s = min(s, s1 - 1);                                       // past the end: the last stage again (never read)
    At r;
    r.second = s >= seg_stages;
    r.s = r.second ? s - seg_stages : s;
    r.left = a.k - r.s * kStageK;
    return r;
  };
  auto load_n = [&](unsigned char *buf, int s, int i0, int i1) __attribute__((always_inline)) {
    const At at = at_of(s);
    if constexpr (!kGated) { if (a.segs == 2) ns.base = n_base(at.second); }
    ns.copy(at.s, at.left, ldn, buf + wave * NL * 1024, i0, i1);
  };
  auto load_m = [&](unsigned char *buf, int s) __attribute__((always_inline)) {
    const At at = at_of(s);
    if (a.segs == 2) ms.base = m_base(at.second);
    ms.copy(at.s, at.left, ldm, buf + wave * ML * 1024, 0, ML);
  };
  auto clear_end = [&](unsigned char *mb, unsigned char *nb, int s) __attribute__((always_inline)) {   // what was copied for k past the end
    const At at = at_of(s);
    if (at.left >= kStageK) return;
    ms.clear(at.left, mb + wave * ML * 1024, lane);
    ns.clear(at.left, nb + wave * NL * 1024, lane);
    __builtin_amdgcn_s_waitcnt(0xC07F);                       // lgkmcnt(0)
  };

  f32x16_t acc[WB][TB];
#pragma unroll
  for (int b = 0; b < WB; b++)
#pragma unroll
    for (int t = 0; t < TB; t++)
#pragma unroll
      for (int v = 0; v < 16; v++) acc[b][t][v] = 0.f;
  const int mat = frag_lane<MM, L::kM>(lane, th * TB), nat = frag_lane<NM, L::kN>(lane, wq * WB);
  struct Frag { u32x4_t m[TB], n[WB]; };
  auto read = [&](Frag &f, const unsigned char *mb, const unsigned char *nb, int j) __attribute__((always_inline)) {
#pragma unroll
    for (int b = 0; b < WB; b++) f.n[b] = frag<NM, L::kN>(nb, nat, b, j);
#pragma unroll
    for (int t = 0; t < TB; t++) f.m[t] = frag<MM, L::kM>(mb, mat, t, j);
  };
  auto mul = [&](const Frag &f) __attribute__((always_inline)) {
#pragma unroll
    for (int b = 0; b < WB; b++)
#pragma unroll
      for (int t = 0; t < TB; t++)
        acc[b][t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, f.n[b]), __builtin_bit_cast(bf16x8_t, f.m[t]), acc[b][t], 0, 0, 0);
  };
  Frag f[2];
  constexpr int kReads = TB * (MM ? 2 : 1) + WB * (NM ? 2 : 1);
  auto spread = [&]() __attribute__((always_inline)) {        // the next step's reads behind the first products, the copies behind the others
#pragma unroll
    for (int i = 0; i < TB * WB; i++) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);      // a matrix instruction
      __builtin_amdgcn_sched_group_barrier(0x100, (kReads + TB * WB - 1) / (TB * WB), 0);
      if (i >= 2) __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  auto stage = [&](unsigned char *mc, unsigned char *nc, unsigned char *mn, unsigned char *nn, unsigned char *np, int s) __attribute__((always_inline)) {
    // on entry f[0] = the fragments of step 0
#pragma unroll
    for (int j = 0; j < 3; j++) {
      read(f[(j + 1) & 1], mc, nc, j + 1);
      if (j == 0) load_n(np, s + 2, 0, NL / 2);
      if (j == 1) load_n(np, s + 2, NL / 2, NL);
      mul(f[j & 1]);
      spread();
    }
    // every fragment of this stage is in registers, and this wavefront's share of the next one has arrived (only the copies of the n side
    // of the stage after it may still be under way)
    __builtin_amdgcn_s_waitcnt(0x0070 | NL);                  // vmcnt(NL) lgkmcnt(0)
    clear_end(mn, nn, s + 1);
    wg_barrier();
    read(f[0], mn, nn, 0);
    load_m(mc, s + 2);
    mul(f[1]);
    spread();
  };
  load_n(ns0, s0, 0, NL);
  load_m(ms0, s0);
  load_n(ns1, s0 + 1, 0, NL);
  load_m(ms1, s0 + 1);
  __builtin_amdgcn_s_waitcnt(0x0F70 | (ML + NL));             // the first stage is here
  clear_end(ms0, ns0, s0);
  wg_barrier();
  read(f[0], ms0, ns0, 0);
  int s = s0;
  for (; s + 6 <= s1; s += 6) {
    stage(ms0, ns0, ms1, ns1, ns2, s);
    stage(ms1, ns1, ms0, ns2, ns0, s + 1);
    stage(ms0, ns2, ms1, ns0, ns1, s + 2);
    stage(ms1, ns0, ms0, ns1, ns2, s + 3);
    stage(ms0, ns1, ms1, ns2, ns0, s + 4);
    stage(ms1, ns2, ms0, ns0, ns1, s + 5);
  }
  if (s < s1) stage(ms0, ns0, ms1, ns1, ns2, s);
  if (s + 1 < s1) stage(ms1, ns1, ms0, ns2, ns0, s + 1);
  if (s + 2 < s1) stage(ms0, ns2, ms1, ns0, ns1, s + 2);
  if (s + 3 < s1) stage(ms1, ns0, ms0, ns1, ns2, s + 3);
  if (s + 4 < s1) stage(ms0, ns1, ms1, ns2, ns0, s + 4);
  __builtin_amdgcn_s_waitcnt(0x0F70);                         // no copy into the LDS outlives the workgroup

  // lane (c, g) holds row c of a block of m at the columns 8 (v / 4) + 4 g + v % 4 of a block of n
#pragma unroll
  for (int t = 0; t < TB; t++) {
    const int m = m0 + (th * TB + t) * 32 + c;
    const bool there = m < a.m;
    if constexpr (kGated) {
      static_assert(!kGated || WB == 2, "gate and up");
      const int n1 = n0 + wq * 32;
#pragma unroll
      for (int q = 0; q < 2; q++) {                           // columns 16 q ..
        uint32_t first[4], second[4];                         // h, or dg; du
#pragma unroll
        for (int e = 0; e < 2; e++) {
          const int b = 2 * q + e, n = n1 + 8 * b + 4 * g;
          float dh[4] = {0.f, 0.f, 0.f, 0.f};
          if constexpr (TO == kToDgu) {
            if (there && n < a.n) {
              const u32x2_t d = *(const u32x2_t *)((const bf16_t *)a.dh + (int64_t)m * a.lddh + n);
              dh[0] = __uint_as_float(d.x << 16); dh[1] = __uint_as_float(d.x & 0xFFFF0000u);
              dh[2] = __uint_as_float(d.y << 16); dh[3] = __uint_as_float(d.y & 0xFFFF0000u);
            }
          }
          float x[4], y[4];
#pragma unroll
          for (int v = 0; v < 4; v++) {
            const float gate = acc[0][t][4 * b + v], up = acc[WB - 1][t][4 * b + v];
            const Act r = activation<TO == kToDgu>(a.act, gate);
            if constexpr (TO == kToH) { x[v] = gate * r.p * up; y[v] = 0.f; }
            else { x[v] = dh[v] * up * r.slope; y[v] = dh[v] * (gate * r.p); }
          }
          first[2 * e] = pack_bf16x2(x[0], x[1]); first[2 * e + 1] = pack_bf16x2(x[2], x[3]);
          second[2 * e] = pack_bf16x2(y[0], y[1]); second[2 * e + 1] = pack_bf16x2(y[2], y[3]);
        }
        const u32x4_t h = gather8(first[0], first[1], first[2], first[3]);
        const int n = n1 + 16 * q + 8 * g;
        const bool store = there && n < a.n;
        if (store) *(u32x4_t *)((bf16_t *)a.out[0] + (int64_t)m * a.ldo + n) = h;
        if constexpr (TO == kToDgu) {
          const u32x4_t d = gather8(second[0], second[1], second[2], second[3]);
          if (store) *(u32x4_t *)((bf16_t *)a.out[1] + (int64_t)m * a.ldo + n) = d;
        }
      }
    } else {
#pragma unroll
      for (int w = 0; w < WB; w++) {
        const int n1 = n0 + (wq * WB + w) * 32;
        if constexpr (TO == kToParts) {
#pragma unroll
          for (int b = 0; b < 4; b++) {
            const int n = n1 + 8 * b + 4 * g;
            if (there && n < a.n)
              *(f32x4_t *)(part + (int64_t)m * a.n + n) = f32x4_t{acc[w][t][4 * b], acc[w][t][4 * b + 1], acc[w][t][4 * b + 2], acc[w][t][4 * b + 3]};
          }
        } else {
#pragma unroll
          for (int q = 0; q < 2; q++) {
            const f32x16_t &s_ = acc[w][t];
            const u32x4_t o = gather8(pack_bf16x2(s_[8 * q], s_[8 * q + 1]), pack_bf16x2(s_[8 * q + 2], s_[8 * q + 3]), pack_bf16x2(s_[8 * q + 4], s_[8 * q + 5]),
                                      pack_bf16x2(s_[8 * q + 6], s_[8 * q + 7]));
            const int n = n1 + 16 * q + 8 * g;
            if (there && n < a.n) *(u32x4_t *)((bf16_t *)(half ? a.out[1] : a.out[0]) + (int64_t)m * a.ldo + n) = o;
          }
        }
      }
    }
    __builtin_amdgcn_sched_barrier(0);                        // one block at a time: registers
  }
}

// The tile of a workgroup.  Ids 8 apart run on one XCD: it has the n tiles x, x + 8, .. and walks them four at a time, for each m tile those four.
template <class L, bool MM, bool NM, int TO>
__global__ __launch_bounds__(L::kThreads, L::kThreads == 512 ? 2 : 2) void ffn_tile_kernel(FfnArgs a) {
  __shared__ __attribute__((aligned(1024))) unsigned char ms0[L::kMBytes], ms1[L::kMBytes], ns0[L::kNBytes], ns1[L::kNBytes], ns2[L::kNBytes];
  constexpr int kGroup = 4;
  const int mt = a.m_tiles * a.halves, x = (int)blockIdx.x % 8, j = (int)blockIdx.x / 8;
  const int mine = (a.n_tiles - x + 7) / 8;                   // n tiles of this XCD
  if (j >= mine * mt) return;
  const int group = j / (kGroup * mt), in = j - group * kGroup * mt, wide = min(mine - group * kGroup, kGroup);
  const int nt = (group * kGroup + in % wide) * 8 + x, m = in / wide, half = m / a.m_tiles;
  const int total = a.segs * ((a.k + kStageK - 1) / kStageK), split = blockIdx.y;
  const int s0 = (int)((int64_t)total * split / a.splits), s1 = (int)((int64_t)total * (split + 1) / a.splits);
  float *part = TO == kToParts ? a.part + ((int64_t)split * a.halves + half) * (int64_t)a.m * a.n : nullptr;
  tile_body<L, MM, NM, TO>(a, __builtin_amdgcn_readfirstlane(half), __builtin_amdgcn_readfirstlane((m - half * a.m_tiles) * L::kM),
                           __builtin_amdgcn_readfirstlane(nt * (TO == kToH || TO == kToDgu ? L::kN / 2 : L::kN)), __builtin_amdgcn_readfirstlane(s0),
                           __builtin_amdgcn_readfirstlane(s1), part, ms0, ms1, ns0, ns1, ns2);
}

// The ranges' sums, in ascending order: eight columns a thread
__global__ __launch_bounds__(256) void ffn_join_kernel(const float *part, int splits, int halves, int m, int n, void *out0, void *out1, int64_t ldo) {
  const int per = n / 8;
  const int64_t all = (int64_t)m * per, set = (int64_t)m * n * halves;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all * halves; i += (int64_t)gridDim.x * 256) {
    const int half = i >= all;
    const int64_t at = half ? i - all : i, row = at / per;
    const int col = (int)(at - row * per) * 8;
    const float *p = part + half * (int64_t)m * n + row * n + col;
    f32x4_t a = *(const f32x4_t *)p, b = *(const f32x4_t *)(p + 4);
    for (int s = 1; s < splits; s++) { a += *(const f32x4_t *)(p + s * set); b += *(const f32x4_t *)(p + s * set + 4); }
    *(u32x4_t *)((bf16_t *)(half ? out1 : out0) + row * ldo + col) =
        u32x4_t{pack_bf16x2(a.x, a.y), pack_bf16x2(a.z, a.w), pack_bf16x2(b.x, b.y), pack_bf16x2(b.z, b.w)};
  }
}

// ---- few rows ----------------------------------------------------------------------------------------
// Up to 64 rows: the weights are read once and little is done with them.  A workgroup has 16 columns of h, its four wavefronts a quarter of k each, with a ring
// of stages of their own in the LDS (16 gate and 16 up rows x 64 k, 4 KB): nobody waits for anybody until the quarters meet.  x comes out of the L2, straight
// into registers, as many stages ahead.
constexpr int kFewStage = 4096, kFewRows = 64;
template <int TB>                                             // blocks of 16 rows of x
__global__ __launch_bounds__(256) void ffn_few_kernel(FfnArgs a) {
  __shared__ __attribute__((aligned(1024))) unsigned char r0[4 * kFewStage], r1[4 * kFewStage], r2[4 * kFewStage];   // (arrays of their own: the compiler waits for the copies into what it reads)
  __shared__ float sums[4][TB * 8][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, q = lane >> 4;
  const int n0 = blockIdx.x * 16, stages = (a.k + kStageK - 1) / kStageK;
  const int s0 = stages * wave / 4, s1 = stages * (wave + 1) / 4;
  // copy i (0, 1: gate, 2, 3: up) has rows 8 (i % 2) + lane / 8, whose eight pieces are permuted by row / 2
  uint32_t off[2];
  int k[2];
#pragma unroll
  for (int i = 0; i < 2; i++) {
    k[i] = ((lane & 7) ^ (4 * i + (lane >> 4))) * 8;
    off[i] = (uint32_t)min(8 * i + (lane >> 3), a.n - 1 - n0) * (uint32_t)(2 * a.ldn) + k[i] * 2;
  }
  const char *w0 = (const char *)a.n_src[0] + (int64_t)n0 * a.ldn * 2, *w1 = (const char *)a.n_src[1] + (int64_t)n0 * a.ldn * 2;
  auto copy = [&](unsigned char *ring, int s) __attribute__((always_inline)) {
    s = min(s, s1 - 1);                                       // past the end: the last stage again (never read)
    const int left = a.k - s * kStageK;
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const __amdgpu_buffer_rsrc_t src = __builtin_amdgcn_make_buffer_rsrc((void *)((i < 2 ? w0 : w1) + s * (kStageK * 2)), 0, 0x7FFFFFFF, 0x00027000);
      uint32_t o = off[i & 1];
      if (k[i & 1] >= left) o -= k[i & 1] * 2;                // past k: the stage's first (not used)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(src, (lds_void *)(ring + wave * kFewStage + i * 1024), 16, (int)o, 0, 0, 0);
    }
  };
  const char *xrow[TB];
#pragma unroll
  for (int t = 0; t < TB; t++) xrow[t] = (const char *)a.m_src[0] + (int64_t)min(16 * t + r, a.m - 1) * a.ldm * 2;
  struct X { u32x4_t v[2][TB]; };
  auto load_x = [&](X &x, int s) __attribute__((always_inline)) {
    s = min(s, s1 - 1);
#pragma unroll
    for (int j = 0; j < 2; j++) {
      const int kk = s * kStageK + j * 32 + q * 8;
#pragma unroll
      for (int t = 0; t < TB; t++) x.v[j][t] = *(const u32x4_t *)(xrow[t] + (kk < a.k ? kk : 0) * 2);
    }
  };
  f32x4_t acc[2][TB];
#pragma unroll
  for (int b = 0; b < 2; b++)
#pragma unroll
    for (int t = 0; t < TB; t++) acc[b][t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  const int at = wave * kFewStage + r * 128 + ((q ^ (r >> 1)) * 16);
  auto stage = [&](unsigned char *ring, X &x, int s) __attribute__((always_inline)) {
    __builtin_amdgcn_s_waitcnt(0x0F70 | ((8 + 4 * TB) & 15) | (((8 + 4 * TB) >> 4) << 14));   // this stage's copies and x are here, the next two's may be under way
    u32x4_t w[2][2];
#pragma unroll
    for (int j = 0; j < 2; j++)
#pragma unroll
      for (int b = 0; b < 2; b++) w[j][b] = *(const u32x4_t *)(ring + (at ^ (j * 64)) + b * 2048);
    __builtin_amdgcn_s_waitcnt(0xC07F);                       // lgkmcnt(0): read before the next copy into this stage is asked for
    asm volatile("" ::: "memory");
    if ((s + 1) * kStageK > a.k) {                            // past k: zeros on both sides
      const u32x4_t zero = {0u, 0u, 0u, 0u};
#pragma unroll
      for (int j = 0; j < 2; j++)
        if (s * kStageK + j * 32 + q * 8 >= a.k) {
          w[j][0] = w[j][1] = zero;
#pragma unroll
          for (int t = 0; t < TB; t++) x.v[j][t] = zero;
        }
    }
#pragma unroll
    for (int j = 0; j < 2; j++)
#pragma unroll
      for (int b = 0; b < 2; b++)
#pragma unroll
        for (int t = 0; t < TB; t++)
          acc[b][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, w[j][b]), __builtin_bit_cast(bf16x8_t, x.v[j][t]), acc[b][t], 0, 0, 0);
  };
  if (s0 < s1) {
    X x0, x1, x2;
    load_x(x0, s0); copy(r0, s0);
    load_x(x1, s0 + 1); copy(r1, s0 + 1);
    for (int s = s0; s < s1; s += 3) {
      load_x(x2, s + 2); copy(r2, s + 2);
      stage(r0, x0, s);
      load_x(x0, s + 3); copy(r0, s + 3);
      if (s + 1 < s1) stage(r1, x1, s + 1);
      load_x(x1, s + 4); copy(r1, s + 4);
      if (s + 2 < s1) stage(r2, x2, s + 2);
    }
  }
  __builtin_amdgcn_s_waitcnt(0x0F70);                         // no copy into the LDS outlives the workgroup
  // lane (r, q) holds row r of a block of x at the columns 4 q + v
#pragma unroll
  for (int b = 0; b < 2; b++)
#pragma unroll
    for (int t = 0; t < TB; t++)
#pragma unroll
      for (int v = 0; v < 4; v++) sums[wave][(b * TB + t) * 4 + v][lane] = acc[b][t][v];
  __syncthreads();
  if (wave >= TB) return;
  const int m = wave * 16 + r, n = n0 + 4 * q;
  float h[4];
#pragma unroll
  for (int v = 0; v < 4; v++) {
    float s[2];
#pragma unroll
    for (int b = 0; b < 2; b++) {
      const int e = (b * TB + wave) * 4 + v;
      s[b] = ((sums[0][e][lane] + sums[1][e][lane]) + sums[2][e][lane]) + sums[3][e][lane];
    }
    h[v] = s[0] * activation<false>(a.act, s[0]).p * s[1];
  }
  if (m < a.m && n < a.n) *(u32x2_t *)((bf16_t *)a.out[0] + (int64_t)m * a.ldo + n) = u32x2_t{pack_bf16x2(h[0], h[1]), pack_bf16x2(h[2], h[3])};
}

// ---- launches -----------------------------------------------------------------------------------------

using Big = Tile<2, 4, 4, 2>;                                 // 256 x 256
using Mid = Tile<2, 2, 4, 2>;                                 // 128 x 256
using Small = Tile<2, 2, 2, 2>;                               // 128 x 128

template <class L, bool MM, bool NM, int TO> hipError_t launch_tiles(FfnArgs a, hipStream_t st) {
  constexpr int kCols = TO == kToH || TO == kToDgu ? L::kN / 2 : L::kN;
  a.m_tiles = (a.m + L::kM - 1) / L::kM;
  a.n_tiles = (a.n + kCols - 1) / kCols;
  const int64_t grid = (int64_t)a.m_tiles * a.halves * ((a.n_tiles + 7) / 8) * 8;
  if (grid > 0x7FFFFFFF / L::kThreads) return hipErrorInvalidValue;
  hipLaunchKernelGGL((ffn_tile_kernel<L, MM, NM, TO>), dim3((unsigned)grid, a.splits), dim3(L::kThreads), 0, st, a);
  return hipGetLastError();
}

// Which tile, and into how many ranges k is cut (1: not at all)
struct FfnPlan { int tile, splits; };                         // tile: 0 .. 2, as above
constexpr int kTileM[3] = {256, 128, 128}, kTileN[3] = {256, 256, 128};
FfnPlan ffn_plan(int64_t m, int64_t n, int64_t k, int halves, int segs, bool gated) {
  const int stages = segs * (int)((k + kStageK - 1) / kStageK);
  FfnPlan p{0, 1};
  auto tiles = [&](int t) { const int64_t cols = gated ? kTileN[t] / 2 : kTileN[t]; return ((m + kTileM[t] - 1) / kTileM[t]) * ((n + cols - 1) / cols) * halves; };
  while (p.tile < 2 && tiles(p.tile) < 256) p.tile++;
  if (!gated && tiles(p.tile) < 256) {
    int64_t s = 256 / tiles(p.tile);
    s = s < stages / 4 ? s : stages / 4;
    p.splits = s < 1 ? 1 : s > 32 ? 32 : (int)s;
  }
  return p;
}
template <bool MM, bool NM, int TO> hipError_t launch_planned(const FfnArgs &a, int tile, hipStream_t st) {
  return tile == 0 ? launch_tiles<Big, MM, NM, TO>(a, st) : tile == 1 ? launch_tiles<Mid, MM, NM, TO>(a, st) : launch_tiles<Small, MM, NM, TO>(a, st);
}
// A product into out, through ranges' sums if k is cut
template <bool MM, bool NM> hipError_t launch_product(FfnArgs a, hipStream_t st) {
  const FfnPlan p = ffn_plan(a.m, a.n, a.k, a.halves, a.segs, false);
  a.splits = p.splits;
  if (p.splits == 1) return launch_planned<MM, NM, kToOut>(a, p.tile, st);
  const hipError_t e = launch_planned<MM, NM, kToParts>(a, p.tile, st);
  if (e != hipSuccess) return e;
  const int64_t pieces = (int64_t)a.m * (a.n / 8) * a.halves, groups = (pieces + 255) / 256;
  hipLaunchKernelGGL(ffn_join_kernel, dim3((unsigned)(groups < 4096 ? groups : 4096)), dim3(256), 0, st, a.part, a.splits, a.halves, a.m, a.n, a.out[0], a.out[1], a.ldo);
  return hipGetLastError();
}
uint64_t parts_bytes(int64_t m, int64_t n, int64_t k, int halves, int segs) {
  const FfnPlan p = ffn_plan(m, n, k, halves, segs, false);
  return p.splits == 1 ? 0 : (uint64_t)p.splits * halves * m * n * 4;
}
uint64_t up256(uint64_t b) { return (b + 255) / 256 * 256; }

}  // namespace

// dg and du, and behind them room for the ranges' sums of one product at a time
uint64_t ffn_grad_scratch_bytes(int rows, int d, int f) {
  const uint64_t x = parts_bytes(rows, d, f, 1, 2), w = parts_bytes(f, d, rows, 2, 1);
  return 2 * up256((uint64_t)rows * f * 2) + up256(x > w ? x : w);
}

hipError_t launch_ffn(const FfnCall &c, hipStream_t st) {
  FfnArgs a{};
  a.m = c.rows; a.n = c.f; a.k = c.d; a.segs = a.halves = a.splits = 1; a.act = c.act;
  a.m_src[0] = c.x; a.ldm = c.ldx; a.n_src[0] = c.wg; a.n_src[1] = c.wu; a.ldn = c.ldw; a.out[0] = c.h; a.ldo = c.ldh;
  if (c.rows > kFewRows) return launch_planned<false, false, kToH>(a, ffn_plan(a.m, a.n, a.k, 1, 1, true).tile, st);
  const auto kernel = c.rows <= 16 ? ffn_few_kernel<1> : c.rows <= 32 ? ffn_few_kernel<2> : c.rows <= 48 ? ffn_few_kernel<3> : ffn_few_kernel<4>;
  hipLaunchKernelGGL(kernel, dim3((c.f + 15) / 16), dim3(256), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_ffn_grad(const FfnCall &c, void *scratch, hipStream_t st) {
  const uint64_t each = up256((uint64_t)c.rows * c.f * 2);
  void *dg = scratch, *du = (char *)scratch + each;
  FfnArgs a{};
  a.m = c.rows; a.n = c.f; a.k = c.d; a.segs = a.halves = a.splits = 1; a.act = c.act;
  a.m_src[0] = c.x; a.ldm = c.ldx; a.n_src[0] = c.wg; a.n_src[1] = c.wu; a.ldn = c.ldw;
  a.dh = c.h; a.lddh = c.ldh; a.out[0] = dg; a.out[1] = du; a.ldo = c.f;
  hipError_t e = launch_planned<false, false, kToDgu>(a, ffn_plan(a.m, a.n, a.k, 1, 1, true).tile, st);
  if (e != hipSuccess) return e;
  FfnArgs b{};
  b.part = (float *)((char *)scratch + 2 * each);
  if (c.dx) {
    b.m = c.rows; b.n = c.d; b.k = c.f; b.segs = 2; b.halves = 1;
    b.m_src[0] = dg; b.m_src[1] = du; b.ldm = c.f; b.n_src[0] = c.wg; b.n_src[1] = c.wu; b.ldn = c.ldw; b.out[0] = c.dx; b.ldo = c.lddx;
    if ((e = launch_product<false, true>(b, st)) != hipSuccess) return e;
  }
  if (c.dwg) {
    b.m = c.f; b.n = c.d; b.k = c.rows; b.segs = 1; b.halves = 2;
    b.m_src[0] = dg; b.m_src[1] = du; b.ldm = c.f; b.n_src[0] = b.n_src[1] = c.x; b.ldn = c.ldx; b.out[0] = c.dwg; b.out[1] = c.dwu; b.ldo = c.lddw;
    if ((e = launch_product<true, true>(b, st)) != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace spec
