// The gated half of a feed-forward block, h = act(x Wg^T) * (x Wu^T), and its gradients (include/spec_step.h).
//
// Products of matrices as they lie in memory (weights change with every step of a training run, so that nothing is packed ahead):
// out[m][n] = sum over k of A(m, k) B(n, k), either side with k along its rows (x, the weights of the forward products) or with k
// across them (both sides of the weights' gradients, the weights of dx).
//   forward    : m = rows of x, n = columns of h; a workgroup's n are gate and up rows of the same columns, so that a lane holds both sums of an element of h
//   dg and du  : the same sums again, then dg = dh u act'(g), du = dh act(g), rounded to bf16 for the products that follow (the
//                matrix instruction takes both sides in one type: the gradients are 2.35e-3 of their norm off where their own
//                rounding alone is 1.66e-3; as sums of two bf16 each they would cost 20 instead of 12 rows * d * f operations)
//   dx         : dg Wg + du Wu, k = the columns of dg and then those of du
//   dWg, dWu   : dg^T x, du^T x, k = rows of x
// Bound: the matrix cores, under the power they take, from some hundreds of rows on; below, the weights' way from memory.
// Measured (4096 rows, 4096 x 11008): forward 545 us (1.36 PFLOP/s; matrix cores 74 % busy at the 1.7 GHz that they leave; 607 in
// thirty launches on end, as the clock falls), dg and du 584, dx 630 (58 % at 1.95), dWg and dWu 606 (62 % at 1.97).  With all copies
// out of the L2 1 % less for the forward call and 3 % for the gradients' products; without the wait for the m side's copies the same.
// One row 28.0 us (6.4 TB/s of weights).
#include "common.h"
#include "kernels.h"

namespace spec {

namespace {

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
  constexpr double kTwice = 1.5957691216057308, kCube = 0.044715;   // 2 sqrt(2 / pi), and the share of the cube in the tanh's argument
  const float z = act == kActSilu ? g : (float)kTwice * fmaf((float)kCube * g, g * g, g);
  r.p = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * -1.4426950408889634f));
  if constexpr (SLOPE) {
    const float c = act == kActSilu ? g : fminf(fmaxf(g, -64.0f), 64.0f);   // (far out p (1 - p) is zero, and the cube of g would be infinite)
    const float dz = act == kActSilu ? 1.0f : fmaf((float)(3.0 * kCube * kTwice) * c, c, (float)kTwice);
    r.slope = fmaf(c * dz, r.p * (1.0f - r.p), r.p);
  }
  return r;
}

// ---- tiles -----------------------------------------------------------------------------------------
// Stages of 64 k in the LDS, copied there straight from memory, 16 bytes a lane and 1 KB a wavefront's instruction.
// K along the rows (MAJOR = false): a row's 128 bytes, their eight pieces permuted by row / 2 so that sixteen rows' reads of one piece touch all banks.  K across
// (MAJOR = true): per k the tile's columns, their chunks of 16 permuted by k so that the eight k of half a transposing read touch all banks.
// Products of 16 x 16 x 32: from registers alone they run at 2.00 PFLOP/s on normally distributed data where those of 32 x 32 x 16,
// which move their sums twice as often, run at 1.78 (what limits both is the power).
constexpr int kStageK = 64;
// Loads marked nontemporal: of weights that nobody reads again (one row of 4096 x 11008 32.4 -> 30.1 us, of 8192 x 28672 159 -> 145)
constexpr int kOnce = 2;
template <int TW_, int MB_, int WQ_, int NB_> struct Tile {   // wavefronts and 16-blocks of each along m and n
  static constexpr int TW = TW_, MB = MB_, WQ = WQ_, NB = NB_;
  static constexpr int kWaves = TW * WQ, kThreads = kWaves * 64, kM = TW * MB * 16, kN = WQ * NB * 16;
  static constexpr int kMBytes = kM * 128, kNBytes = kN * 128;       // of a stage
  static constexpr int kMLoads = kM / 8 / kWaves, kNLoads = kN / 8 / kWaves;   // copies of a wavefront
};

__device__ __forceinline__ void wg_barrier() {                 // (without a wait for the copies under way)
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}
// Which 16 columns of a row of k (MAJOR) stand where: chunk ^ chunk_turn(k)
__device__ __forceinline__ int chunk_turn(int k) { return (k & 3) | ((k >> 1) & 4); }

// One side of a tile: LOADS copies of this wavefront per stage.  The buffer ends with the matrix: what lies behind it (rows past the
// last, k past the end in the last row) is not accessed; rows and columns past the tile's are never used, and k past the end is cleared.
template <int LOADS, bool MAJOR, int COLS> struct Side {
  const char *base, *end;                                     // of the segment: the tile's first row (column, if MAJOR), and the matrix's end
  uint32_t off[LOADS];                                        // of a lane
  int64_t step;                                               // bytes from one stage to the next
  // k within a stage of copy q's lane
  static __device__ __forceinline__ int k_of(int q, int lane) {
    if constexpr (MAJOR) return q * (512 / COLS) + lane / (COLS / 8);
    return ((lane & 7) ^ ((q * 4 + (lane >> 4)) & 7)) * 8;
  }
  // copy i is copy q of the tile's rows (columns); ld in elements
  __device__ __forceinline__ void place(int i, int q, int lane, int64_t ld) {
    const int k = k_of(q, lane);
    if constexpr (!MAJOR) {
      off[i] = (uint32_t)(q * 8 + (lane >> 3)) * (uint32_t)(2 * ld) + k * 2;
    } else {
      const int slot = lane % (COLS / 8);
      off[i] = (uint32_t)k * (uint32_t)(2 * ld) + (uint32_t)(((slot >> 1) ^ chunk_turn(k)) * 32 + (slot & 1) * 16);
    }
    step = MAJOR ? (int64_t)kStageK * ld * 2 : kStageK * 2;
  }
  // copies i0 .. of stage s of the segment
  template <int KIND = 0> __device__ __forceinline__ void copy(int s, unsigned char *to, int i0, int i1) const {
#pragma unroll
    for (int i = 0; i < LOADS; i++) {
      if (i < i0 || i >= i1) continue;
      const char *at = base + s * step;
      const int64_t left = end - at;
      const __amdgpu_buffer_rsrc_t src = __builtin_amdgcn_make_buffer_rsrc((void *)at, 0, left < 0x7FFFFFFF ? (int)left : 0x7FFFFFFF, 0x00027000);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(src, (lds_void *)(to + i * 1024), 16, (int)off[i], 0, 0, KIND);
    }
  }
  __device__ __forceinline__ void clear(int left, int q0, unsigned char *mine) const {   // mine: this wavefront's share of the stage, from its copy q0 on
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));                            // (nothing of this is worth registers outside)
#pragma unroll
    for (int i = 0; i < LOADS; i++)
      if (k_of(q0 + i, lane) >= left) *(u32x4_t *)(mine + i * 1024 + lane * 16) = u32x4_t{0u, 0u, 0u, 0u};
  }
};
// Fragments of a block of 16 rows (columns): lane 16 q + r has row r at k = 32 j + 8 q + 0 .. 7
template <bool MAJOR, int COLS> __device__ __forceinline__ int frag_lane(int lane, int block) {
  const int r = lane & 15, q = lane >> 4;
  if constexpr (!MAJOR) return (block * 16 + r) * 128 + ((q ^ (r >> 1)) * 16);
  const int kr = 8 * q + (r >> 2);
  return kr * COLS * 2 + ((block ^ chunk_turn(kr)) * 32) + (r & 3) * 8;
}
template <bool MAJOR, int COLS> __device__ __forceinline__ u32x4_t frag(const unsigned char *p, int at, int t, int j) {   // block t of those that `at` begins with
  if constexpr (!MAJOR) return *(const u32x4_t *)(p + (at ^ (j * 64)) + t * 2048);
  const unsigned char *q = p + (at ^ (t * 32)) + j * 32 * COLS * 2;
  const u32x2_t a = read_columns(q), b = read_columns(q + 4 * COLS * 2);
  return u32x4_t{a.x, a.y, b.x, b.y};
}

// Four bf16 of block a (columns 4 q ..) and of block b in each of the lanes 16 q + r, to eight consecutive columns a lane: those from
// 8 (q / 2) on of block a (q even) or b
__device__ __forceinline__ u32x4_t gather8(uint32_t a0, uint32_t a1, uint32_t b0, uint32_t b1) {
  const auto x = __builtin_amdgcn_permlane16_swap(a0, b0, false, false), y = __builtin_amdgcn_permlane16_swap(a1, b1, false, false);
  return u32x4_t{x[0], y[0], x[1], y[1]};
}
__device__ __forceinline__ u32x4_t gather8(f32x4_t a, f32x4_t b) { return gather8(pack_bf16x2(a.x, a.y), pack_bf16x2(a.z, a.w), pack_bf16x2(b.x, b.y), pack_bf16x2(b.z, b.w)); }

enum { kToH = 0, kToDgu = 1, kToOut = 2, kToParts = 3 };

// A wavefront's sums to where they go: rows from m0 on, columns from n0 on (gated: of h)
template <int MB, int NB, int TO>
__device__ __forceinline__ void finish(const FfnArgs &a, const f32x4_t (&acc)[NB][MB], int m0, int n0, int half, float *part) {
  constexpr bool kGated = TO == kToH || TO == kToDgu;
  const int r = threadIdx.x & 15, q = (threadIdx.x & 63) >> 4;
  // lane 16 q + r holds row r of a block of m at the columns 4 q + 0 .. 3 of a block of n
  u32x2_t dhs[TO == kToDgu ? MB : 1][TO == kToDgu ? NB / 2 : 1];   // (all asked for at once: block by block every block waited for its own)
  if constexpr (TO == kToDgu) {
#pragma unroll
    for (int t = 0; t < MB; t++)
#pragma unroll
      for (int e = 0; e < NB / 2; e++) {
        const int m = m0 + t * 16 + r, n = n0 + 16 * e + 4 * q;
        dhs[t][e] = u32x2_t{0u, 0u};
        if (m < a.m && n < a.n) dhs[t][e] = *(const u32x2_t *)((const bf16_t *)a.dh + (int64_t)m * a.lddh + n);
      }
    __builtin_amdgcn_sched_barrier(0);
  }
#pragma unroll
  for (int t = 0; t < MB; t++) {
    const int m = m0 + t * 16 + r;
    const bool there = m < a.m;
    if constexpr (kGated) {
#pragma unroll
      for (int p = 0; p < NB / 4; p++) {                      // 32 columns: gate sums in the blocks 4 p and 4 p + 1, up sums in the two behind
        const int n1 = n0 + p * 32;
        f32x4_t first[2], second[2];                          // h, or dg; du
#pragma unroll
        for (int e = 0; e < 2; e++) {
          float dh[4] = {0.f, 0.f, 0.f, 0.f};
          if constexpr (TO == kToDgu) {
            const u32x2_t d = dhs[t][2 * p + e];
            dh[0] = __uint_as_float(d.x << 16); dh[1] = __uint_as_float(d.x & 0xFFFF0000u);
            dh[2] = __uint_as_float(d.y << 16); dh[3] = __uint_as_float(d.y & 0xFFFF0000u);
          }
#pragma unroll
          for (int v = 0; v < 4; v++) {
            const float gate = acc[4 * p + e][t][v], up = acc[4 * p + 2 + e][t][v];
            const Act c = activation<TO == kToDgu>(a.act, gate);
            if constexpr (TO == kToH) first[e][v] = gate * c.p * up;
            else { first[e][v] = dh[v] * up * c.slope; second[e][v] = dh[v] * (gate * c.p); }
          }
        }
        const int n = n1 + 16 * (q & 1) + 8 * (q >> 1);
        const bool store = there && n < a.n;
        const u32x4_t h = gather8(first[0], first[1]);
        if (store) *(u32x4_t *)((bf16_t *)a.out[0] + (int64_t)m * a.ldo + n) = h;
        if constexpr (TO == kToDgu) {
          const u32x4_t d = gather8(second[0], second[1]);
          if (store) *(u32x4_t *)((bf16_t *)a.out[1] + (int64_t)m * a.ldo + n) = d;
        }
      }
    } else {
#pragma unroll
      for (int b = 0; b < NB; b += 2) {
        const int n1 = n0 + b * 16;
        if constexpr (TO == kToParts) {
#pragma unroll
          for (int e = 0; e < 2; e++) {
            const int n = n1 + 16 * e + 4 * q;
            if (there && n < a.n) *(f32x4_t *)(part + (int64_t)m * a.n + n) = acc[b + e][t];
          }
        } else {
          const u32x4_t o = gather8(acc[b][t], acc[b + 1][t]);
          const int n = n1 + 16 * (q & 1) + 8 * (q >> 1);
          if (there && n < a.n) *(u32x4_t *)((bf16_t *)(half ? a.out[1] : a.out[0]) + (int64_t)m * a.ldo + n) = o;
        }
      }
    }
    __builtin_amdgcn_sched_barrier(0);                        // one block at a time: registers
  }
}

// One tile and range of stages.
template <class L, bool MM, bool NM, int TO>
__device__ __forceinline__ void tile_body(const FfnArgs &a, int half, int m0, int n0, int s0, int s1, float *part, unsigned char *ms0, unsigned char *ms1, unsigned char *ns0,
                                          unsigned char *ns1, unsigned char *ns2) {
  constexpr int ML = L::kMLoads, NL = L::kNLoads, MB = L::MB, NB = L::NB;
  constexpr bool kGated = TO == kToH || TO == kToDgu;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, q = lane >> 4, th = wave % L::TW, wq = wave / L::TW;
  const int seg_stages = (a.k + kStageK - 1) / kStageK;       // of a segment
  Side<ML, MM, L::kM> ms;
  Side<NL, NM, L::kN> ns;
  const int64_t ldm = a.ldm, ldn = a.ldn;
#pragma unroll
  for (int i = 0; i < ML; i++) ms.place(i, wave * ML + i, lane, ldm);
  // where a matrix of a segment begins for this tile, and where it ends
  auto m_base = [&](int seg) {
    const char *p = (const char *)((MM ? half : seg) ? a.m_src[1] : a.m_src[0]);
    ms.base = p + (MM ? (int64_t)m0 * 2 : (int64_t)m0 * ldm * 2);
    ms.end = p + ((int64_t)((MM ? a.k : a.m) - 1) * ldm + (MM ? a.m : a.k)) * 2;
  };
  auto n_base = [&](int seg) {
    const char *p = (const char *)(seg ? a.n_src[1] : a.n_src[0]);
    ns.base = p + (NM ? (int64_t)n0 * 2 : (int64_t)n0 * ldn * 2);
    ns.end = p + ((int64_t)((NM ? a.k : a.n) - 1) * ldn + (NM ? a.n : a.k)) * 2;
  };
  m_base(0);
  if constexpr (kGated) {                                     // blocks of 32: gate, up, gate, .. of the same columns; a wavefront copies one
    static_assert(NL == 4, "a block");
    const int first = min(n0 + wave / 2 * 32, a.n - 1);
    const char *p = (const char *)(wave & 1 ? a.n_src[1] : a.n_src[0]);
    ns.base = p + (int64_t)first * ldn * 2;
    ns.end = p + ((int64_t)(a.n - 1) * ldn + a.k) * 2;
#pragma unroll
    for (int i = 0; i < NL; i++) ns.place(i, i, lane, ldn);
  } else {
#pragma unroll
    for (int i = 0; i < NL; i++) ns.place(i, wave * NL + i, lane, ldn);
    n_base(0);
  }

  struct At { int s, left; bool second; };                    // a stage within its segment
  auto at_of = [&](int s) {
    s = min(s, s1 - 1);                                       // past the end: the last stage again (never read)
    At p;
    p.second = s >= seg_stages;
    p.s = p.second ? s - seg_stages : s;
    p.left = a.k - p.s * kStageK;
    return p;
  };
  auto load_n = [&](unsigned char *buf, int s, int i0, int i1) __attribute__((always_inline)) {
    const At at = at_of(s);
    if constexpr (!kGated) { if (a.segs == 2) n_base(at.second); }
    ns.copy(at.s, buf + wave * NL * 1024, i0, i1);
  };
  auto load_m = [&](unsigned char *buf, int s, int i0, int i1) __attribute__((always_inline)) {
    const At at = at_of(s);
    if constexpr (!kGated && !MM) { if (a.segs == 2) m_base(at.second); }
    ms.copy(at.s, buf + wave * ML * 1024, i0, i1);
  };
  auto clear_end = [&](unsigned char *mb, unsigned char *nb, int s) __attribute__((always_inline)) {   // what was copied for k past the end
    const At at = at_of(s);
    if (at.left >= kStageK) return;
    ms.clear(at.left, wave * ML, mb + wave * ML * 1024);
    ns.clear(at.left, wave * NL, nb + wave * NL * 1024);
    __builtin_amdgcn_s_waitcnt(0xC07F);                       // lgkmcnt(0)
  };

  f32x4_t acc[NB][MB];
#pragma unroll
  for (int b = 0; b < NB; b++)
#pragma unroll
    for (int t = 0; t < MB; t++) acc[b][t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  const int mat_ = frag_lane<MM, L::kM>(lane, th * MB), nat_ = frag_lane<NM, L::kN>(lane, wq * NB);
  // A step is the products of 32 k, block by block of m.  Behind block t's products block t + 3 (of this step or the next) is read, three blocks
  // ahead of its turn; the next step's blocks of n are read behind the last products of this one.  `last`: the step ends its stage, and what
  // follows is read from the next one, after the barrier that is behind the stage's last read.
  u32x4_t fm[4], fn[2][NB];
  constexpr int kBarrier = MB - 4, kEach = (NB + 1) / 2;
  static_assert(MB % 4 == 0 && MB >= NL, "a ring of four blocks, a copy of the n side behind each");
  auto step = [&](int now, bool last, unsigned char *mc, unsigned char *nc, unsigned char *mn, unsigned char *nn, auto copies, auto turn) __attribute__((always_inline)) {
    int mat = mat_, nat = nat_;
    asm volatile("" : "+v"(mat), "+v"(nat));                  // (else the addresses of all steps are kept in registers at once)
#pragma unroll
    for (int t = 0; t < MB; t++) {
#pragma unroll
      for (int i = 0; i < NB; i++) {
        const int b = t & 1 ? NB - 1 - i : i;                 // (back and forth: one operand less changes, half a percent)
        acc[b][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, fn[now][b]), __builtin_bit_cast(bf16x8_t, fm[t & 3]), acc[b][t], 0, 0, 0);
      }
      if (t + 3 < MB) fm[(t + 3) & 3] = frag<MM, L::kM>(mc, mat, t + 3, last ? 1 : 0);
      if (t == kBarrier) turn();
      if (t > kBarrier) {                                     // the next step's
        const int u = t - kBarrier - 1;
        fm[u & 3] = frag<MM, L::kM>(last ? mn : mc, mat, u, last ? 0 : 1);
#pragma unroll
        for (int b = u * kEach; b < (u + 1) * kEach && b < NB; b++) fn[now ^ 1][b] = frag<NM, L::kN>(last ? nn : nc, nat, b, last ? 0 : 1);
      }
      copies(t);
      if (t & 1) __builtin_amdgcn_sched_barrier(0);           // (at every block the forward products needed two registers too many)
    }
  };
  auto stage = [&](unsigned char *mc, unsigned char *nc, unsigned char *mn, unsigned char *nn, unsigned char *np, int s) __attribute__((always_inline)) {
    step(0, false, mc, nc, mn, nn, [&](int t) __attribute__((always_inline)) { load_n(np, s + 2, min(t, NL), min(t + 1, NL)); },
         []() {});
    step(1, true, mc, nc, mn, nn, [&](int t) __attribute__((always_inline)) {
      constexpr int kHalf = (ML + 1) / 2;
      if (t > kBarrier) load_m(mc, s + 2, min((t - kBarrier - 1) * kHalf, ML), min((t - kBarrier) * kHalf, ML));
    }, [&]() __attribute__((always_inline)) {
      // every fragment of this stage is in registers, and this wavefront's share of the next one has arrived (only the copies of the n side
      // of the stage after it may still be under way)
      __builtin_amdgcn_s_waitcnt(0x0070 | NL);                // vmcnt(NL) lgkmcnt(0)
      clear_end(mn, nn, s + 1);
      wg_barrier();
    });
  };
  load_n(ns0, s0, 0, NL);
  load_m(ms0, s0, 0, ML);
  load_n(ns1, s0 + 1, 0, NL);
  load_m(ms1, s0 + 1, 0, ML);
  static_assert(ML + NL < 64 && NL < 16, "the counts of the waits");
  __builtin_amdgcn_s_waitcnt(0x0F70 | ((ML + NL) & 15) | (((ML + NL) >> 4) << 14));   // the first stage is here
  clear_end(ms0, ns0, s0);
  wg_barrier();
#pragma unroll
  for (int b = 0; b < NB; b++) fn[0][b] = frag<NM, L::kN>(ns0, nat_, b, 0);
#pragma unroll
  for (int t = 0; t < 3; t++) fm[t] = frag<MM, L::kM>(ms0, mat_, t, 0);
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

  finish<MB, NB, TO>(a, acc, m0 + th * MB * 16, n0 + wq * NB * (kGated ? 8 : 16), half, part);
}

// The tile of a workgroup.  Ids 8 apart run on one XCD.  The XCDs share the tiles out in m_parts x 8 / m_parts: XCD x has the m tiles
// x % m_parts, + m_parts, .. and the n tiles x / m_parts, + 8 / m_parts, .., and walks them four n tiles at a time, for each m tile those
// four (32 compute units then read 8 + 4 panels).
constexpr int kGroup = 4, kXcdUnits = 32;
struct TilePlace { int m, n, count; };                        // count: tiles of this XCD
__device__ __forceinline__ TilePlace tile_place(const FfnArgs &a, int id, int j) {
  const int x = id % 8, xm = x % a.m_parts, xn = x / a.m_parts, n_parts = 8 / a.m_parts;
  const int ms = (a.m_tiles * a.halves - xm + a.m_parts - 1) / a.m_parts, ns = (a.n_tiles - xn + n_parts - 1) / n_parts;
  TilePlace p{-1, -1, ms * ns};
  if (j >= p.count) return p;
  const int group = j / (kGroup * ms), in = j - group * kGroup * ms, wide = min(ns - group * kGroup, kGroup);
  p.n = (group * kGroup + in % wide) * n_parts + xn;
  p.m = (in / wide) * a.m_parts + xm;
  return p;
}
template <class L, bool MM, bool NM, int TO>
__device__ __forceinline__ void tile_at(const FfnArgs &a, int mt, int nt, int rows, int split, unsigned char *ms0, unsigned char *ms1, unsigned char *ns0, unsigned char *ns1, unsigned char *ns2) {
  // rows: of the m tile, how far in the body begins
  const int total = a.segs * ((a.k + kStageK - 1) / kStageK), half = mt / a.m_tiles;
  const int s0 = (int)((int64_t)total * split / a.splits), s1 = (int)((int64_t)total * (split + 1) / a.splits);
  float *part = TO == kToParts ? a.part + ((int64_t)split * a.halves + half) * (int64_t)a.m * a.n : nullptr;
  tile_body<L, MM, NM, TO>(a, __builtin_amdgcn_readfirstlane(half), __builtin_amdgcn_readfirstlane((mt - half * a.m_tiles) * a.tile_m + rows),
                           __builtin_amdgcn_readfirstlane(nt * (TO == kToH || TO == kToDgu ? L::kN / 2 : L::kN)), __builtin_amdgcn_readfirstlane(s0),
                           __builtin_amdgcn_readfirstlane(s1), part, ms0, ms1, ns0, ns1, ns2);
}
template <class L, bool MM, bool NM, int TO>
__global__ __launch_bounds__(L::kThreads, 2) void ffn_tile_kernel(FfnArgs a) {
  __shared__ __attribute__((aligned(1024))) unsigned char ms0[L::kMBytes], ms1[L::kMBytes], ns0[L::kNBytes], ns1[L::kNBytes], ns2[L::kNBytes];
  const TilePlace p = tile_place(a, blockIdx.x, (int)blockIdx.x / 8);
  if (p.m >= 0) tile_at<L, MM, NM, TO>(a, p.m, p.n, 0, blockIdx.y, ms0, ms1, ns0, ns1, ns2);
}
using Big = Tile<2, 8, 4, 4>;                                 // 256 x 256
using Mid = Tile<2, 4, 4, 4>;                                 // 128 x 256
using Small = Tile<2, 4, 2, 4>;                               // 128 x 128
// Tiles of 256 x 256, and halves of 128 x 256 for what an XCD's compute units would be half empty with (up to 16 tiles behind the last
// whole round) and for ends of m of up to 128 rows.
__host__ __device__ inline int halved_tiles(int count) { return count % kXcdUnits <= kXcdUnits / 2 ? count % kXcdUnits : 0; }
template <bool MM, bool NM, int TO>
__global__ __launch_bounds__(Big::kThreads, 2) void ffn_mixed_kernel(FfnArgs a) {
  __shared__ __attribute__((aligned(1024))) unsigned char ms0[Big::kMBytes], ms1[Big::kMBytes], ns0[Big::kNBytes], ns1[Big::kNBytes], ns2[Big::kNBytes];
  const int j = (int)blockIdx.x / 8, count = tile_place(a, blockIdx.x, 0x7FFFFFFF).count, whole = count - halved_tiles(count);
  const TilePlace p = tile_place(a, blockIdx.x, j < whole ? j : whole + (j - whole) / 2);
  if (p.m < 0) return;
  const int left = a.m - (p.m % a.m_tiles) * Big::kM, rows = j < whole ? 0 : ((j - whole) & 1) * Mid::kM;   // of the tile; of those, where this workgroup begins
  if (rows >= left) return;
  if (j < whole && left > Mid::kM) tile_at<Big, MM, NM, TO>(a, p.m, p.n, 0, blockIdx.y, ms0, ms1, ns0, ns1, ns2);
  else tile_at<Mid, MM, NM, TO>(a, p.m, p.n, rows, blockIdx.y, ms0, ms1, ns0, ns1, ns2);
}

// dx and the weights' gradients of a small call in one launch, where neither fills the chip for long: the workgroups of dx, range of k
// by range, then those of the others.
struct FfnBoth { FfnArgs dx, dw; int dx_each, dw_each; };     // ..each: workgroups of a range
template <int TX, int TW>
__global__ __launch_bounds__(Small::kThreads, 2) void ffn_both_kernel(FfnBoth b) {
  using L = Small;
  __shared__ __attribute__((aligned(1024))) unsigned char ms0[L::kMBytes], ms1[L::kMBytes], ns0[L::kNBytes], ns1[L::kNBytes], ns2[L::kNBytes];
  const int id = blockIdx.x, first = b.dx_each * b.dx.splits;
  if (id < first) {
    const int split = id / b.dx_each;
    const TilePlace p = tile_place(b.dx, id, (id - split * b.dx_each) / 8);
    if (p.m >= 0) tile_at<L, false, true, TX>(b.dx, p.m, p.n, 0, split, ms0, ms1, ns0, ns1, ns2);
  } else {
    const int split = (id - first) / b.dw_each;
    const TilePlace p = tile_place(b.dw, id, (id - first - split * b.dw_each) / 8);
    if (p.m >= 0) tile_at<L, true, true, TW>(b.dw, p.m, p.n, 0, split, ms0, ms1, ns0, ns1, ns2);
  }
}

// The ranges' sums of one product, or of both of a small call (1024 rows, 512 x 1376: 36.0 us, with a launch each 37.5), in ascending order: eight columns a thread
struct FfnJoin { const float *part; int splits, halves, m, n; void *out[2]; int64_t ldo; };
__global__ __launch_bounds__(256) void ffn_join_kernel(FfnJoin first, FfnJoin second) {
  const int64_t here = (int64_t)first.m * (first.n / 8) * first.halves, all = here + (int64_t)second.m * (second.n / 8) * second.halves;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
    const FfnJoin j = i < here ? first : second;
    const int per = j.n / 8;
    const int64_t each = (int64_t)j.m * per, set = (int64_t)j.m * j.n * j.halves, k = i < here ? i : i - here;
    const int half = k >= each;
    const int64_t at = half ? k - each : k, row = at / per;
    const int col = (int)(at - row * per) * 8;
    const float *p = j.part + half * (int64_t)j.m * j.n + row * j.n + col;
    f32x4_t a = *(const f32x4_t *)p, b = *(const f32x4_t *)(p + 4);
    for (int s = 1; s < j.splits; s++) { a += *(const f32x4_t *)(p + s * set); b += *(const f32x4_t *)(p + s * set + 4); }
    *(u32x4_t *)((bf16_t *)(half ? j.out[1] : j.out[0]) + row * j.ldo + col) =
        u32x4_t{pack_bf16x2(a.x, a.y), pack_bf16x2(a.z, a.w), pack_bf16x2(b.x, b.y), pack_bf16x2(b.z, b.w)};
  }
}

// ---- few rows ----------------------------------------------------------------------------------------
// Up to 16 rows: the weights are read once and little is done with them.  A workgroup has 16 columns of h, its four wavefronts a quarter of k each, with a ring
// of stages of their own in the LDS (16 gate and 16 up rows x 64 k, 4 KB): nobody waits for anybody until the quarters meet.  x comes out of the L2, straight
// into registers, as many stages ahead.
constexpr int kFewStage = 4096, kFewRows = 16;
__global__ __launch_bounds__(256) void ffn_few_kernel(FfnArgs a) {
  // (arrays of their own: the compiler waits for the copies into what it reads)
  __shared__ __attribute__((aligned(1024))) unsigned char r0[4 * kFewStage], r1[4 * kFewStage], r2[4 * kFewStage];
  __shared__ float sums[4][8][64];
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
      __builtin_amdgcn_raw_ptr_buffer_load_lds(src, (lds_void *)(ring + wave * kFewStage + i * 1024), 16, (int)o, 0, 0, kOnce);
    }
  };
  const char *xrow = (const char *)a.m_src[0] + (int64_t)min(r, a.m - 1) * a.ldm * 2;
  struct X { u32x4_t v[2]; };
  auto load_x = [&](X &x, int s) __attribute__((always_inline)) {
    s = min(s, s1 - 1);
#pragma unroll
    for (int j = 0; j < 2; j++) {
      const int kk = s * kStageK + j * 32 + q * 8;
      x.v[j] = *(const u32x4_t *)(xrow + (kk < a.k ? kk : 0) * 2);
    }
  };
  f32x4_t acc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
  const int at = wave * kFewStage + r * 128 + ((q ^ (r >> 1)) * 16);
  auto stage = [&](unsigned char *ring, X &x, int s) __attribute__((always_inline)) {
    __builtin_amdgcn_s_waitcnt(0x0F70 | 12);                 // this stage's copies and x are here, the next two's may be under way
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
        if (s * kStageK + j * 32 + q * 8 >= a.k) w[j][0] = w[j][1] = x.v[j] = zero;
    }
#pragma unroll
    for (int j = 0; j < 2; j++)
#pragma unroll
      for (int b = 0; b < 2; b++)
        acc[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, w[j][b]), __builtin_bit_cast(bf16x8_t, x.v[j]), acc[b], 0, 0, 0);
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
  // lane (r, q) holds row r of x at the columns 4 q + v
#pragma unroll
  for (int b = 0; b < 2; b++)
#pragma unroll
    for (int v = 0; v < 4; v++) sums[wave][b * 4 + v][lane] = acc[b][v];
  __syncthreads();
  if (wave != 0) return;
  const int n = n0 + 4 * q;
  float h[4];
#pragma unroll
  for (int v = 0; v < 4; v++) {
    float s[2];
#pragma unroll
    for (int b = 0; b < 2; b++) {
      const int e = b * 4 + v;
      s[b] = ((sums[0][e][lane] + sums[1][e][lane]) + sums[2][e][lane]) + sums[3][e][lane];
    }
    h[v] = s[0] * activation<false>(a.act, s[0]).p * s[1];
  }
  if (r < a.m && n < a.n) *(u32x2_t *)((bf16_t *)a.out[0] + (int64_t)r * a.ldo + n) = u32x2_t{pack_bf16x2(h[0], h[1]), pack_bf16x2(h[2], h[3])};
}

// ---- some rows ---------------------------------------------------------------------------------------
// 17 to 128 rows: still bound by the weights' way from memory, but x has to come through the LDS too (read by every wavefront for itself
// it took twice the weights' way: 98 us for 60 rows, 4096 x 14336).  A workgroup has all rows and 32 columns of h, so that there are
// workgroups enough to keep the memory busy (tiles of 64 columns: 66 us); four wavefronts with a quarter of the rows each; a ring of
// four (three) stages of 64 k, two workgroups to a compute unit.
template <int MB>                                             // blocks of 16 rows of a wavefront
__global__ __launch_bounds__(256, 2) void ffn_some_kernel(FfnArgs a) {
  constexpr int kRows = MB * 64, NB = 4, ML = MB * 2, NL = 2, kRing = MB == 1 ? 4 : 3, kBytes = (kRows + 64) * 128;
  __shared__ __attribute__((aligned(1024))) unsigned char b0[kBytes], b1[kBytes], b2[kBytes], b3[kRing > 3 ? kBytes : 16];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n0 = blockIdx.x * 32;
  const int stages = (a.k + kStageK - 1) / kStageK;
  Side<ML, false, kRows> ms;
  Side<NL, false, 64> ns;
#pragma unroll
  for (int i = 0; i < ML; i++) ms.place(i, wave * ML + i, lane, a.ldm);
  ms.base = (const char *)a.m_src[0];
  ms.end = ms.base + ((int64_t)(a.m - 1) * a.ldm + a.k) * 2;
#pragma unroll
  for (int i = 0; i < NL; i++) ns.place(i, (wave & 1) * NL + i, lane, a.ldn);   // wavefronts 0 and 1 copy the gate rows, 2 and 3 the up rows
  const char *w = (const char *)(wave >> 1 ? a.n_src[1] : a.n_src[0]);
  ns.base = w + (int64_t)n0 * a.ldn * 2;
  ns.end = w + ((int64_t)(a.n - 1) * a.ldn + a.k) * 2;
  unsigned char *const ring[4] = {b0, b1, b2, b3};
  auto copy = [&](unsigned char *to, int s) __attribute__((always_inline)) {
    s = min(s, stages - 1);                                   // past the end: the last stage again (never read)
    ns.template copy<kOnce>(s, to + kRows * 128 + wave * NL * 1024, 0, NL);
    ms.copy(s, to + wave * ML * 1024, 0, ML);
  };
  f32x4_t acc[NB][MB];
#pragma unroll
  for (int b = 0; b < NB; b++)
#pragma unroll
    for (int t = 0; t < MB; t++) acc[b][t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  const int mat = frag_lane<false, kRows>(lane, wave * MB), nat = kRows * 128 + frag_lane<false, 64>(lane, 0);
  auto stage = [&](unsigned char *now, unsigned char *free, int s) __attribute__((always_inline)) {
    // this wavefront's share of the stage has arrived, its reads of the stage before are in registers
    __builtin_amdgcn_s_waitcnt(0x0070 | ((kRing - 2) * (ML + NL)));
    const int left = a.k - s * kStageK;
    if (left < kStageK) {
      ms.clear(left, wave * ML, now + wave * ML * 1024);
      ns.clear(left, (wave & 1) * NL, now + kRows * 128 + wave * NL * 1024);
      __builtin_amdgcn_s_waitcnt(0xC07F);                     // lgkmcnt(0)
    }
    wg_barrier();
    copy(free, s + kRing - 1);
#pragma unroll
    for (int j = 0; j < 2; j++) {
      u32x4_t fm[MB], fn[NB];
#pragma unroll
      for (int b = 0; b < NB; b++) fn[b] = frag<false, 64>(now, nat, b, j);
#pragma unroll
      for (int t = 0; t < MB; t++) fm[t] = frag<false, kRows>(now, mat, t, j);
#pragma unroll
      for (int b = 0; b < NB; b++)
#pragma unroll
        for (int t = 0; t < MB; t++)
          acc[b][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, fn[b]), __builtin_bit_cast(bf16x8_t, fm[t]), acc[b][t], 0, 0, 0);
    }
  };
  static_assert((kRing - 2) * (ML + NL) < 16, "the count of the wait");
#pragma unroll
  for (int i = 0; i < kRing - 1; i++) copy(ring[i], i);
  for (int s = 0; s < stages; s += kRing) {
    stage(b0, ring[kRing - 1], s);
    if (s + 1 < stages) stage(b1, b0, s + 1);
    if (s + 2 < stages) stage(b2, b1, s + 2);
    if constexpr (kRing > 3) { if (s + 3 < stages) stage(b3, b2, s + 3); }
  }
  __builtin_amdgcn_s_waitcnt(0x0F70);                         // no copy into the LDS outlives the workgroup
  finish<MB, NB, kToH>(a, acc, wave * MB * 16, n0, 0, nullptr);
}

// ---- launches -----------------------------------------------------------------------------------------

// Tiles of the fullest XCD where the m tiles are shared out in m_parts
int64_t fullest(int64_t m_tiles, int64_t n_tiles, int m_parts) { return (m_tiles + m_parts - 1) / m_parts * ((n_tiles + 8 / m_parts - 1) / (8 / m_parts)); }
// In two parts (m) by four (n), if that is no less even than all n tiles' eighths: of a training step at the 7B widths dx and the weights'
// gradients are 2 % sooner than with one by eight and the same with four by two, the forward product is the same with each.
int parts_of_m(int64_t m_tiles, int64_t n_tiles) { return fullest(m_tiles, n_tiles, 2) <= fullest(m_tiles, n_tiles, 1) ? 2 : 1; }

template <class L, int TO> bool set_tiles(FfnArgs &a) {       // false: more tiles than a grid holds
  constexpr int kCols = TO == kToH || TO == kToDgu ? L::kN / 2 : L::kN;
  a.tile_m = L::kM;
  a.m_tiles = (a.m + L::kM - 1) / L::kM;
  a.n_tiles = (a.n + kCols - 1) / kCols;
  a.m_parts = parts_of_m(a.m_tiles * a.halves, a.n_tiles);
  return fullest(a.m_tiles * a.halves, a.n_tiles, a.m_parts) <= 0x7FFFFFFF / L::kThreads / 8 - kXcdUnits;
}
template <class L, bool MM, bool NM, int TO> hipError_t launch_tiles(FfnArgs a, hipStream_t st) {
  if (!set_tiles<L, TO>(a)) return hipErrorInvalidValue;
  const int64_t count = fullest(a.m_tiles * a.halves, a.n_tiles, a.m_parts);
  constexpr bool kMixed = L::kM == 256;
  const dim3 grid((unsigned)(8 * (kMixed ? count + kXcdUnits / 2 : count)), a.splits);   // (an XCD may have fewer tiles and more halves)
  if constexpr (kMixed) hipLaunchKernelGGL((ffn_mixed_kernel<MM, NM, TO>), grid, dim3(L::kThreads), 0, st, a);
  else hipLaunchKernelGGL((ffn_tile_kernel<L, MM, NM, TO>), grid, dim3(L::kThreads), 0, st, a);
  return hipGetLastError();
}

// Which tile, and into how many ranges k is cut (1: not at all): as many as fill the chip once, with halves of the large tile or two
// workgroups of the small one to a compute unit.  Measured (us):
//   dx of 1024 rows, 4096 x 11008 (64 large tiles, 344 stages) in 1, 2, 3, 4, 6 ranges 352, 207, 266, 220, 236, small tiles 277, 215,
//   234, 222, 237; of 512 rows, 4096 x 14336 (32 large tiles) 441, 233, 161, 142, 177, small (128) 346, 186, 162, 142, 156; of 777 rows,
//   1000 x 2728 (16, 56) 91, 54, 42, 36, 31, small 72, 43, 35, 30, 30, in eight 29;
//   forward, large / small: 512 rows of 4096 x 14336 (224 large tiles) 96 / 113, 777 of 1000 x 2728 (88) 19.6 / 20.9, 300 of
//   4096 x 4096 (64) 42.6 / 40.3, 200 of 8192 x 2000 (16) 74 / 62.
struct FfnPlan { int tile, splits; };                         // tile 0: 256 x 256 and halves, 1: 128 x 128
FfnPlan ffn_plan(int64_t m, int64_t n, int64_t k, int halves, int segs, bool gated, bool both = false) {
  auto tiles_m = [&](int t) { const int size = t ? Small::kM : Big::kM; return (m + size - 1) / size * halves; };
  auto tiles_n = [&](int t) { const int size = (t ? Small::kN : Big::kN) / (gated ? 2 : 1); return (n + size - 1) / size; };
  FfnPlan p{tiles_m(0) * tiles_n(0) >= 64 ? 0 : 1, 1};
  if (gated) return p;
  const int64_t m_tiles = tiles_m(p.tile), n_tiles = tiles_n(p.tile), stages = segs * ((k + kStageK - 1) / kStageK);
  const int64_t units = p.tile == 0 ? kXcdUnits / 2 : both ? kXcdUnits * 3 / 4 : 2 * kXcdUnits, most = stages / 4 < 16 ? stages / 4 : 16;
  const int64_t ranges = units / fullest(m_tiles, n_tiles, parts_of_m(m_tiles, n_tiles));
  p.splits = (int)(ranges < most ? ranges : most);
  if (p.splits < 1) p.splits = 1;
  return p;
}
template <bool MM, bool NM, int TO> hipError_t launch_planned(const FfnArgs &a, int tile, hipStream_t st) {
  return tile == 0 ? launch_tiles<Big, MM, NM, TO>(a, st) : launch_tiles<Small, MM, NM, TO>(a, st);
}
FfnJoin join_of(const FfnArgs &a) { return FfnJoin{a.part, a.splits, a.halves, a.splits > 1 ? a.m : 0, a.n, {a.out[0], a.out[1]}, a.ldo}; }   // (no rows if k is not cut)
hipError_t launch_join(const FfnJoin &a, const FfnJoin &b, hipStream_t st) {
  const int64_t pieces = (int64_t)a.m * (a.n / 8) * a.halves + (int64_t)b.m * (b.n / 8) * b.halves, groups = (pieces + 255) / 256;
  hipLaunchKernelGGL(ffn_join_kernel, dim3((unsigned)(groups < 4096 ? groups : 4096)), dim3(256), 0, st, a, b);
  return hipGetLastError();
}
// A product into out, through ranges' sums if k is cut
template <bool MM, bool NM> hipError_t launch_product(FfnArgs a, bool both, hipStream_t st) {
  const FfnPlan p = ffn_plan(a.m, a.n, a.k, a.halves, a.segs, false, both);
  a.splits = p.splits;
  if (p.splits == 1) return launch_planned<MM, NM, kToOut>(a, p.tile, st);
  const hipError_t e = launch_planned<MM, NM, kToParts>(a, p.tile, st);
  return e != hipSuccess ? e : launch_join(join_of(a), FfnJoin{}, st);
}
// dx and the weights' gradients in one launch, if dx takes small tiles and the others are at most two rounds of them (gradients in all,
// one after the other / together: 777 rows, 1000 x 2728 79 / 68 us, 300 of 4096 x 4096 139 / 121, 100 of 1024 x 2752 43 / 36, 4096 of
// 512 x 1376 91 / 89).  Neither has the chip to itself then, and fewer ranges are written and read again: with ranges for 64 / 32 / 24 /
// 16 workgroups an XCD 777 rows of 1000 x 2728 take 67.6, 61.7, 60.7, 68.4 us, 512 of 768 x 2048 51.8, 35.0, 36.1, 39.2, 300 of
// 1024 x 2752 45.0, 43.2, 38.9, 41.8, 4096 of 256 x 688 56.7, 49.4, 44.5, 40.6.  (Calls for one of the two alone keep those ranges, so
// that a sum's order does not depend on what else is asked for.)
bool both_pay(int64_t rows, int64_t d, int64_t f) {
  return ffn_plan(rows, d, f, 1, 2, false).tile == 1 && (f + Small::kM - 1) / Small::kM * 2 * ((d + Small::kN - 1) / Small::kN) <= 1024;
}
hipError_t launch_both(FfnBoth b, hipStream_t st) {
  for (FfnArgs *a : {&b.dx, &b.dw}) {
    a->splits = ffn_plan(a->m, a->n, a->k, a->halves, a->segs, false, true).splits;
    if (!set_tiles<Small, kToOut>(*a)) return hipErrorInvalidValue;
  }
  b.dx_each = (int)(8 * fullest(b.dx.m_tiles, b.dx.n_tiles, b.dx.m_parts));
  b.dw_each = (int)(8 * fullest(b.dw.m_tiles * b.dw.halves, b.dw.n_tiles, b.dw.m_parts));
  const bool x = b.dx.splits > 1, w = b.dw.splits > 1;
  const auto kernel = x ? (w ? ffn_both_kernel<kToParts, kToParts> : ffn_both_kernel<kToParts, kToOut>) : w ? ffn_both_kernel<kToOut, kToParts> : ffn_both_kernel<kToOut, kToOut>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)(b.dx_each * b.dx.splits + b.dw_each * b.dw.splits)), dim3(Small::kThreads), 0, st, b);
  const hipError_t e = hipGetLastError();
  return e != hipSuccess || !(x || w) ? e : launch_join(join_of(b.dx), join_of(b.dw), st);
}
uint64_t parts_bytes(int64_t m, int64_t n, int64_t k, int halves, int segs, bool both) {
  const FfnPlan p = ffn_plan(m, n, k, halves, segs, false, both);
  return p.splits == 1 ? 0 : (uint64_t)p.splits * halves * m * n * 4;
}
uint64_t up256(uint64_t b) { return (b + 255) / 256 * 256; }

}  // namespace

// dg and du, and behind them room for the ranges' sums
uint64_t ffn_grad_scratch_bytes(int rows, int d, int f) {
  const bool both = both_pay(rows, d, f);
  const uint64_t x = parts_bytes(rows, d, f, 1, 2, both), w = parts_bytes(f, d, rows, 2, 1, both);
  return 2 * up256((uint64_t)rows * f * 2) + up256(x) + up256(w);
}

// Which of the three takes a forward call (us; few / some / tiles of 128 x 128): 16 rows of 4096 x 11008 37.8 / 45.6 / 58.2, 24
// 46.5 / 45.8 / 58.6, 60 74 / 48.9 / 61.4, 128 - / 62.2 / 65.8; of 4096 x 14336 16 48.7 / 52.2 / 60.9, 60 98 / 55.0 / 64.0, 128
// - / 66.2 / 68.1; of 1024 x 2752 16 6.1 / 9.7 / 14.1, 60 11.3 / 10.1 / 14.5.  Where the tiles fill the chip by themselves they have
// less of x to read: 8192 x 28672 16 165 / 174 / 177, 32 208 / 177 / 177, 60 304 / 189 / 176, 128 - / 240 / 178.
static bool some_pays(int rows, int f) { return rows <= 32 || (rows <= 128 && (f + 63) / 64 < 256); }
static FfnKernel forward_kernel(int rows, int d, int f) {
  if (rows <= kFewRows) return kFfnFew;
  if (some_pays(rows, f)) return rows <= 64 ? kFfnSome64 : kFfnSome128;
  return ffn_plan(rows, f, d, 1, 1, true).tile == 0 ? kFfnTiles256 : kFfnTiles128;
}

FfnPlans ffn_plans(int rows, int d, int f) {
  const bool both = both_pay(rows, d, f);
  const FfnPlan x = ffn_plan(rows, d, f, 1, 2, false, both), w = ffn_plan(f, d, rows, 2, 1, false, both);
  auto tile = [](int t) { return t == 0 ? kFfnTiles256 : kFfnTiles128; };
  return FfnPlans{forward_kernel(rows, d, f), tile(ffn_plan(rows, f, d, 1, 1, true).tile), tile(x.tile), x.splits, tile(w.tile), w.splits, both};
}

hipError_t launch_ffn(const FfnCall &c, hipStream_t st) {
  FfnArgs a{};
  a.m = c.rows; a.n = c.f; a.k = c.d; a.segs = a.halves = a.splits = 1; a.act = c.act;
  a.m_src[0] = c.x; a.ldm = c.ldx; a.n_src[0] = c.wg; a.n_src[1] = c.wu; a.ldn = c.ldw; a.out[0] = c.h; a.ldo = c.ldh;
  const FfnKernel kernel = forward_kernel(c.rows, c.d, c.f);
  if (kernel == kFfnTiles128 || kernel == kFfnTiles256) return launch_planned<false, false, kToH>(a, kernel == kFfnTiles256 ? 0 : 1, st);
  if (kernel == kFfnFew) hipLaunchKernelGGL(ffn_few_kernel, dim3((c.f + 15) / 16), dim3(256), 0, st, a);
  else hipLaunchKernelGGL((kernel == kFfnSome64 ? ffn_some_kernel<1> : ffn_some_kernel<2>), dim3((c.f + 31) / 32), dim3(256), 0, st, a);
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
  const bool both = both_pay(c.rows, c.d, c.f);
  FfnBoth b{};
  b.dx.part = (float *)((char *)scratch + 2 * each);
  b.dw.part = (float *)((char *)b.dx.part + up256(parts_bytes(c.rows, c.d, c.f, 1, 2, both)));
  b.dx.m = c.rows; b.dx.n = c.d; b.dx.k = c.f; b.dx.segs = 2; b.dx.halves = 1;
  b.dx.m_src[0] = dg; b.dx.m_src[1] = du; b.dx.ldm = c.f; b.dx.n_src[0] = c.wg; b.dx.n_src[1] = c.wu; b.dx.ldn = c.ldw; b.dx.out[0] = c.dx; b.dx.ldo = c.lddx;
  b.dw.m = c.f; b.dw.n = c.d; b.dw.k = c.rows; b.dw.segs = 1; b.dw.halves = 2;
  b.dw.m_src[0] = dg; b.dw.m_src[1] = du; b.dw.ldm = c.f; b.dw.n_src[0] = b.dw.n_src[1] = c.x; b.dw.ldn = c.ldx; b.dw.out[0] = c.dwg; b.dw.out[1] = c.dwu; b.dw.ldo = c.lddw;
  if (c.dx && c.dwg && both) return launch_both(b, st);
  if (c.dx && (e = launch_product<false, true>(b.dx, both, st)) != hipSuccess) return e;
  if (c.dwg && (e = launch_product<true, true>(b.dw, both, st)) != hipSuccess) return e;
  return hipSuccess;
}

}  // namespace spec
