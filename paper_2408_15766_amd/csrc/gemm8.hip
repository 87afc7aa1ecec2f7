// Projections in 8 bits: y = xq . wq^T with e4m3 codes and a power of two per row and 128 k (include/spec_layer8.h; layout in fp8.h).
//
// The exponents go into the scaled matrix instruction (v_mfma_scale_f32_16x16x128_f8f6f4: one operand scale per row and 32 k, here four times the
// same), so that the accumulator holds the sum itself and nothing is done per block.  That instruction lines its 128 products up with the largest and
// drops what lies 2^-14 below it: 1.4e-5 of a sum, fine for bf16 results.  For fp32 results the codes are widened to bf16, which holds
// code * 2^e exactly (the conversion takes the scale), and go through the bf16 instruction: exact products, fp32 sums.
#include "common.h"
#include "fp8.h"
#include "kernels.h"

namespace spec {

namespace {

typedef __attribute__((ext_vector_type(8))) int i32x8_t;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_t;

// ---- into 8 bits ---------------------------------------------------------------
// The exponent of the 128 values that eight neighbouring lanes hold (16 each, all lanes active), and this lane's codes
__device__ __forceinline__ int codes_of_eight_lanes(const float (&v)[16], u32x4_t &c) {
  float amax = 0.f;
#pragma unroll
  for (int i = 0; i < 16; i++) amax = fmaxf(amax, finite_abs(v[i]));
  amax = fmaxf(amax, dpp_f32<0xB1>(amax));
  amax = fmaxf(amax, dpp_f32<0x4E>(amax));
  amax = fmaxf(amax, dpp_f32<0x141>(amax));
  const int e = exponent8(amax);
  const float down = pow2(-e);
#pragma unroll
  for (int i = 0; i < 4; i++) c[i] = codes4(v[4 * i] * down, v[4 * i + 1] * down, v[4 * i + 2] * down, v[4 * i + 3] * down);
  return e;
}

// A wavefront owns 8 rows x 128 k: lane = row * 8 + piece, 16 k each.  Rows beyond `rows` are written as zeros if `pad` (weights: the whole
// buffer is defined), else left out (their products are never stored).
template <typename T, bool VEC>
__global__ __launch_bounds__(256) void quant8_kernel(const T *x, int64_t ldx, int rows, int in, int pad, unsigned char *dst) {
  const Packed8 pk = packed8(rows, in);
  const int lane = threadIdx.x & 63, r8 = lane >> 3, piece = lane & 7;
  const int64_t wave = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 4 + (threadIdx.x >> 6);
  const int64_t rb8 = wave / pk.groups;                       // eight rows
  const int g = (int)(wave - rb8 * pk.groups);
  const int64_t row = rb8 * 8 + r8;
  if (rb8 * 8 >= (int64_t)pk.blocks * 16) return;
  float v[16];
  const int k0 = g * 128 + piece * 16;
#pragma unroll
  for (int i = 0; i < 16; i++) v[i] = 0.f;
  if (row < rows) {
    const T *p = x + row * ldx + k0;
    if (VEC && k0 + 16 <= in) load16(p, v);
    else
      for (int i = 0; i < 16; i++)
        if (k0 + i < in) v[i] = to_f32(p[i]);
  }
  u32x4_t c;
  const int e = codes_of_eight_lanes(v, c);
  if (row >= rows && !pad) return;
  const int64_t b = row >> 4;
  const int r = (int)(row & 15);
  *(u32x4_t *)(dst + ((size_t)b * pk.groups + g) * kTile8 + (piece >> 2) * 1024 + ((piece & 3) * 16 + r) * 16) = c;
  unsigned char *ex = dst + packed8_exps(pk) + ((size_t)b * pk.quads + g / 4) * 64 + r * 4;
  if (piece == 0) ex[g & 3] = (unsigned char)(e + 127);
  if (piece == 1 && pad && g == pk.groups - 1)
    for (int i = (g & 3) + 1; i < 4; i++) ex[i] = 0;
}

template <typename T>
hipError_t quant8(const T *x, int64_t ldx, int rows, int in, int pad, void *dst, hipStream_t st) {
  const Packed8 pk = packed8(rows, in);
  const int64_t waves = (int64_t)pk.blocks * 2 * pk.groups;
  const int64_t groups = (waves + 3) / 4, deep = (groups + (1 << 23) - 1) >> 23;   // (a grid's dimension holds less than 2^32 threads; at most 2^9 deep)
  const dim3 grid((unsigned)((groups + deep - 1) / deep), (unsigned)deep);
  const bool vec = ((uintptr_t)x & 15) == 0 && ldx % (16 / (int)sizeof(T)) == 0;
  if (vec) hipLaunchKernelGGL((quant8_kernel<T, true>), grid, dim3(256), 0, st, x, ldx, rows, in, pad, (unsigned char *)dst);
  else hipLaunchKernelGGL((quant8_kernel<T, false>), grid, dim3(256), 0, st, x, ldx, rows, in, pad, (unsigned char *)dst);
  return hipGetLastError();
}

// ---- products -------------------------------------------------------------------
struct Frag8 { u32x4_t u[2]; };                               // a 16 x 128 operand
__device__ __forceinline__ Frag8 load_frag(const unsigned char *tile, int lane) {
  return Frag8{*(const u32x4_t *)(tile + lane * 16), *(const u32x4_t *)(tile + 1024 + lane * 16)};
}
__device__ __forceinline__ i32x8_t operand8(const Frag8 &f) {
  return i32x8_t{(int)f.u[0].x, (int)f.u[0].y, (int)f.u[0].z, (int)f.u[0].w, (int)f.u[1].x, (int)f.u[1].y, (int)f.u[1].z, (int)f.u[1].w};
}
// D[i][j] += sum over 128 k of a[i][k] b[j][k]; ea, eb: the lane's row's exponent + 127 in the lowest byte.  Lane (j = lane % 16) gets i = 4 (lane / 16) + 0 .. 3.
template <bool EXACT> __device__ __forceinline__ f32x4_t product(const Frag8 &a, uint32_t ea, const Frag8 &b, uint32_t eb, f32x4_t d) {
  if constexpr (!EXACT) return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(operand8(a), operand8(b), d, 0, 0, 0, (int)ea, 0, (int)eb);
  const float sa = __uint_as_float((ea & 0xFF) << 23), sb = __uint_as_float((eb & 0xFF) << 23);
#pragma unroll
  for (int u = 0; u < 2; u++)
#pragma unroll
    for (int h = 0; h < 2; h++) {
      const uint32_t a0 = a.u[u][2 * h], a1 = a.u[u][2 * h + 1], b0 = b.u[u][2 * h], b1 = b.u[u][2 * h + 1];
      const u32x4_t av{bf16_of_codes<false>(a0, sa), bf16_of_codes<true>(a0, sa), bf16_of_codes<false>(a1, sa), bf16_of_codes<true>(a1, sa)};
      const u32x4_t bv{bf16_of_codes<false>(b0, sb), bf16_of_codes<true>(b0, sb), bf16_of_codes<false>(b1, sb), bf16_of_codes<true>(b1, sb)};
      d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, av), __builtin_bit_cast(bf16x8_t, bv), d, 0, 0, 0);
    }
  return d;
}

// Four columns c0 .. c0 + 3 of a row of y; VEC: aligned to four elements
template <bool VEC> __device__ __forceinline__ void store4(float *y, int c0, int rows, f32x4_t v) {
  if (VEC && c0 + 4 <= rows) { *(f32x4_t *)(y + c0) = v; return; }
#pragma unroll
  for (int i = 0; i < 4; i++)
    if (c0 + i < rows) y[c0 + i] = v[i];
}
template <bool VEC> __device__ __forceinline__ void store4(bf16_t *y, int c0, int rows, f32x4_t v) {
  if (VEC && c0 + 4 <= rows) { *(u32x2_t *)(y + c0) = u32x2_t{pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w)}; return; }
#pragma unroll
  for (int i = 0; i < 4; i++)
    if (c0 + i < rows) y[c0 + i] = from_f32<bf16_t>(v[i]);
}

// ---- few tokens: weights streamed -----------------------------------------------
// A workgroup's eight wavefronts take an eighth of k each (contiguous bytes), the weights straight from memory into registers, and their sums are added up
// in the LDS in ascending order.
constexpr int kStreamWaves = 8;

__device__ __forceinline__ Frag8 stream_frag(const unsigned char *tile, int lane) {
  return Frag8{__builtin_nontemporal_load((const u32x4_t *)(tile + lane * 16)), __builtin_nontemporal_load((const u32x4_t *)(tile + 1024 + lane * 16))};
}
// A 16-row block of the weights, with its exponents
struct Weights8 {
  const unsigned char *tile;
  const uint32_t *exp;
  __device__ __forceinline__ Weights8(const Gemm8Args &a, const Packed8 &pw, int rb, int lane)
      : tile(a.w8 + (size_t)rb * pw.groups * kTile8), exp((const uint32_t *)(a.w8 + packed8_exps(pw)) + (size_t)rb * pw.quads * 16 + (lane & 15)) {}
};
// The wavefronts' sums of row block rb x T token tiles, in ascending order, into y
template <typename OUT, bool VEC, int T>
__device__ __forceinline__ void join_waves(const Gemm8Args &a, const f32x4_t (&acc)[T], f32x4_t (*part)[T][64], int rb) {
  static_assert(T <= kStreamWaves, "a wavefront each");
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int t = 0; t < T; t++) part[wave][t][lane] = acc[t];
  __syncthreads();
  if (wave >= T) return;
  f32x4_t s = part[0][wave][lane];
#pragma unroll
  for (int w = 1; w < kStreamWaves; w++) s += part[w][wave][lane];
  const int tok = wave * 16 + (lane & 15);
  if (tok < a.m) store4<VEC>((OUT *)a.y + (size_t)tok * a.ldy, rb * 16 + 4 * (lane >> 4), a.rows, s);
}

// Up to 16 tokens, one 16-row block a workgroup: four tiles on the way in each wavefront.  RAW: the workgroup puts its tokens into 8 bits itself, into the LDS, while its first
// weights are coming: [128 k][piece u][q][token] 16 bytes, then the exponents [128 k][token], MP (a power of two) tokens.  Else they are in a.x8.
constexpr int kFewRing = 4;
template <typename X, typename OUT, bool VEC, bool RAW>
__global__ __launch_bounds__(kStreamWaves * 64, 4) void gemm8_few_kernel(Gemm8Args a, int mp_log2) {
  constexpr bool kExact = sizeof(OUT) == 4;
  constexpr int R = kFewRing;
  __shared__ f32x4_t part[kStreamWaves][1][64];
  extern __shared__ __attribute__((aligned(16))) unsigned char tokens[];
  const Packed8 pw = packed8(a.rows, a.in);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r16 = lane & 15, q = lane >> 4;
  const Weights8 w(a, pw, blockIdx.x, lane);
  const int g0 = pw.groups * wave / kStreamWaves, n = pw.groups * (wave + 1) / kStreamWaves - g0;
  const unsigned char *exps = RAW ? tokens + ((size_t)pw.groups << (mp_log2 + 7)) : a.x8 + packed8_exps(packed8(a.m, a.in));
  const int tok = RAW ? r16 & ((1 << mp_log2) - 1) : r16;

  struct Slot { Frag8 w, x; uint32_t ew, ex; };
  auto load = [&](Slot &s, int i) __attribute__((always_inline)) {
    const int g = g0 + i;
    s.w = stream_frag(w.tile + (size_t)g * kTile8, lane);
    s.ew = w.exp[(g >> 2) * 16];
    if constexpr (!RAW) {
      s.x = load_frag(a.x8 + (size_t)g * kTile8, lane);
      s.ex = ((const uint32_t *)exps)[(g >> 2) * 16 + r16];
    }
  };
  f32x4_t acc[1] = {f32x4_t{0.f, 0.f, 0.f, 0.f}};
  auto compute = [&](Slot &s, int i) __attribute__((always_inline)) {
    const int g = g0 + i, sh = 8 * (g & 3);
    if constexpr (RAW) {
      const unsigned char *p = tokens + (((g * 8 + q) << mp_log2) + tok) * 16;
      s.x = Frag8{*(const u32x4_t *)p, *(const u32x4_t *)(p + (64 << mp_log2))};
      s.ex = exps[(g << mp_log2) + tok];
    } else s.ex >>= sh;
    acc[0] = product<kExact>(s.w, s.ew >> sh, s.x, s.ex, acc[0]);
  };
  Slot ring[R];
#pragma unroll
  for (int u = 0; u < R - 1; u++)
    if (u < n) load(ring[u], u);
  if constexpr (RAW) {
    const bool whole = ((uintptr_t)a.x & 15) == 0 && a.ldx % (16 / (int)sizeof(X)) == 0;
    const int units = a.m * pw.groups * 8;                    // of 16 k; eight lanes have a row's 128
    for (int i = threadIdx.x; i < (units + 63) / 64 * 64; i += kStreamWaves * 64) {   // (whole wavefronts)
      const int piece = i & 7, row = min(i >> 3, a.m * pw.groups - 1) / pw.groups, g = min(i >> 3, a.m * pw.groups - 1) - row * pw.groups, k0 = g * 128 + piece * 16;
      const X *p = (const X *)a.x + (int64_t)row * a.ldx + k0;
      float v[16];
      if (whole && k0 + 16 <= a.in) load16(p, v);
      else
#pragma unroll
        for (int j = 0; j < 16; j++) v[j] = k0 + j < a.in ? to_f32(p[j]) : 0.f;
      u32x4_t c;
      const int e = codes_of_eight_lanes(v, c);
      *(u32x4_t *)(tokens + (((g * 8 + piece) << mp_log2) + row) * 16) = c;
      if (piece == 0) ((unsigned char *)exps)[(g << mp_log2) + row] = (unsigned char)(e + 127);
    }
    __syncthreads();
  }
  int i = 0;
  for (; i + 2 * R - 1 <= n; i += R)                          // every load is in range: no branch, exact waits
#pragma unroll
    for (int u = 0; u < R; u++) {
      load(ring[(u + R - 1) % R], i + u + R - 1);
      __builtin_amdgcn_sched_barrier(0);
      compute(ring[u], i + u);
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
  for (int u = 0; u < 2 * R - 2; u++)
    if (i + u < n) {
      if (i + u + R - 1 < n) load(ring[(u + R - 1) % R], i + u + R - 1);
      __builtin_amdgcn_sched_barrier(0);
      compute(ring[u % R], i + u);
      __builtin_amdgcn_sched_barrier(0);
    }
  join_waves<OUT, VEC, 1>(a, acc, part, blockIdx.x);
}

// 17 to 64 tokens (16 T), one 16-row block a workgroup: a weight tile is read again, for the next 128 k, as soon as its products are under way, the
// tokens' (from L2) ahead of them.  (Two to eight row blocks a workgroup, for fewer reads of the tokens, took no less: 60 x 22016 x 4096 28 to 42 us.)
template <typename OUT, bool VEC, int T>
__global__ __launch_bounds__(kStreamWaves * 64, 2) void gemm8_stream_kernel(Gemm8Args a) {
  constexpr bool kExact = sizeof(OUT) == 4;
  __shared__ f32x4_t part[kStreamWaves][T][64];
  const Packed8 pw = packed8(a.rows, a.in), px = packed8(a.m, a.in);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r16 = lane & 15;
  const Weights8 w(a, pw, blockIdx.x, lane);
  const unsigned char *xt[T];
  const uint32_t *xe[T];
#pragma unroll
  for (int t = 0; t < T; t++) {
    const int tb = min(t, px.blocks - 1);
    xt[t] = a.x8 + (size_t)tb * px.groups * kTile8;
    xe[t] = (const uint32_t *)(a.x8 + packed8_exps(px)) + (size_t)tb * px.quads * 16 + r16;
  }
  const int g0 = pw.groups * wave / kStreamWaves, g1 = pw.groups * (wave + 1) / kStreamWaves;
  struct Tokens { Frag8 f[T]; uint32_t e[T]; };
  auto load_x = [&](Tokens &x, int g) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < T; t++) { x.f[t] = load_frag(xt[t] + (size_t)g * kTile8, lane); x.e[t] = xe[t][(g >> 2) * 16]; }
  };
  Frag8 wf;
  uint32_t we;
  auto load_w = [&](int g) __attribute__((always_inline)) { wf = stream_frag(w.tile + (size_t)g * kTile8, lane); we = w.exp[(g >> 2) * 16]; };
  f32x4_t acc[T];
#pragma unroll
  for (int t = 0; t < T; t++) acc[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  auto step = [&](Tokens &x, Tokens &next, int g) __attribute__((always_inline)) {
    const int ahead = min(g + 1, g1 - 1), sh = 8 * (g & 3);   // (the last one: once more, and not used)
    load_x(next, ahead);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int t = 0; t < T; t++) acc[t] = product<kExact>(wf, we >> sh, x.f[t], x.e[t] >> sh, acc[t]);
    __builtin_amdgcn_sched_barrier(0);
    load_w(ahead);
    __builtin_amdgcn_sched_barrier(0);
  };
  if (g0 < g1) {
    Tokens x[2];
    load_w(g0);
    load_x(x[0], g0);
    int g = g0;
    for (; g + 2 <= g1; g += 2) {
      step(x[0], x[1], g);
      step(x[1], x[0], g + 1);
    }
    if (g < g1) step(x[0], x[1], g);
  }
  join_waves<OUT, VEC, T>(a, acc, part, blockIdx.x);
}

template <typename OUT, bool VEC, int T>
hipError_t launch_stream(const Gemm8Args &a, hipStream_t st) {
  hipLaunchKernelGGL((gemm8_stream_kernel<OUT, VEC, T>), dim3((a.rows + 15) / 16), dim3(kStreamWaves * 64), 0, st, a);
  return hipGetLastError();
}

// ---- many tokens: tiles ------------------------------------------------------------
// A workgroup owns WM * TB * 32 tokens x WN * WB * 32 weight rows, a wavefront TB x WB blocks of 32 x 32 of them.  Both operands are copied straight into the LDS, 64 k
// (half a packed tile) at a time, STAGES (four or eight) deep, and read from there in the order of the operands of the 32 x 32 x 64 product (weights as A, so that a lane
// ends up with four consecutive columns of one token).  One barrier per stage: behind it the next stage is there for everybody and this stage's operands are in registers, so
// that its buffer takes the copies of STAGES stages on.
// Every stage buffer is an array of its own, which tells the compiler what a read depends on.  The barrier stands behind the products of a stage's first 32 tokens, which cover the
// wait for its last operands; operands of tokens are read again, for the next stage, as soon as their products are under way.  The next stage's weights and the copies are asked for
// behind later products, not at the barrier, where all wavefronts would ask and none multiply (us, 2048 x 24576 x 4096: 175 against 182; fp32 results 316 against 331).
template <int WM, int WN, int TB, int WB>
struct Tile8 {
  static constexpr int kWaves = WM * WN, kTok = WM * TB * 32, kRows = WN * WB * 32;
  static constexpr int kX = kTok * 64, kW = kRows * 64;       // bytes of a stage
  static constexpr int kXParts = kX / 1024, kWParts = kW / 1024;   // 1 KiB, 16 rows, each
  static constexpr int kXLoads = (kXParts + kWaves - 1) / kWaves, kWLoads = (kWParts + kWaves - 1) / kWaves;   // copies per wavefront and stage (some twice where they do not divide)
  // exponents: 64 bytes per 16-row block, tokens first; a wavefront copies those of four blocks (those past the end: the last again)
  static constexpr int kBlocks = (kTok + kRows) / 16, kE = kWaves * 256;
  static constexpr int kLoads = kXLoads + kWLoads + 1;
  static_assert(kBlocks <= 4 * kWaves, "exponents");
  static __device__ __forceinline__ int x_part(int wave, int i) { return kXParts % kWaves ? min(wave * kXLoads + i, kXParts - 1) : wave * kXLoads + i; }
  static __device__ __forceinline__ int w_part(int wave, int i) { return kWParts % kWaves ? min(wave * kWLoads + i, kWParts - 1) : wave * kWLoads + i; }
};

typedef __attribute__((ext_vector_type(16))) float f32x16_t;
typedef __attribute__((address_space(3))) void lds_void;
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_of(const void *base) {
  return __builtin_amdgcn_make_buffer_rsrc((void *)base, 0, 0x7FFFFFFF, 0x00027000);
}
// 16 bytes per lane from base + voff (lane) + soff (wave-uniform) straight into the LDS, to dst + 16 * lane; dst is wave-uniform
__device__ __forceinline__ void load_to_lds(__amdgpu_buffer_rsrc_t base, int voff, int soff, void *dst) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(base, (lds_void *)dst, 16, voff, soff, 0, 0);
}
// Workgroup barrier that waits for nothing else
__device__ __forceinline__ void wg_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

struct Half8 { u32x4_t u[2]; };                               // a 32 x 64 operand
__device__ __forceinline__ i32x8_t operand8(const Half8 &f) {
  return i32x8_t{(int)f.u[0].x, (int)f.u[0].y, (int)f.u[0].z, (int)f.u[0].w, (int)f.u[1].x, (int)f.u[1].y, (int)f.u[1].z, (int)f.u[1].w};
}
struct Wide8 { u32x4_t v[4]; };                               // the same as bf16 operands of 16 k
__device__ __forceinline__ Wide8 widen8(const Half8 &f, uint32_t e) {
  const float s = __uint_as_float(e << 23);
  Wide8 r;
#pragma unroll
  for (int i = 0; i < 4; i++) {
    const uint32_t a = f.u[i / 2][(i & 1) * 2], b = f.u[i / 2][(i & 1) * 2 + 1];
    r.v[i] = u32x4_t{bf16_of_codes<false>(a, s), bf16_of_codes<true>(a, s), bf16_of_codes<false>(b, s), bf16_of_codes<true>(b, s)};
  }
  return r;
}

template <typename OUT, bool VEC, int WM, int WN, int TB, int WB, int STAGES>
__global__ __launch_bounds__(WM * WN * 64, 2) void gemm8_tile_kernel(Gemm8Args a) {
  using L = Tile8<WM, WN, TB, WB>;
  constexpr bool kExact = sizeof(OUT) == 4;
  static_assert(STAGES == 4 || STAGES == 8, "written out below");
  constexpr int kMore = STAGES == 8;
  __shared__ __attribute__((aligned(1024))) unsigned char x0[L::kX], x1[L::kX], x2[L::kX], x3[L::kX], w0[L::kW], w1[L::kW], w2[L::kW], w3[L::kW];
  __shared__ __attribute__((aligned(1024))) unsigned char e0[L::kE], e1[L::kE], e2[L::kE], e3[L::kE];
  __shared__ __attribute__((aligned(1024))) unsigned char x4[kMore ? L::kX : 1], x5[kMore ? L::kX : 1], x6[kMore ? L::kX : 1], x7[kMore ? L::kX : 1];
  __shared__ __attribute__((aligned(1024))) unsigned char w4[kMore ? L::kW : 1], w5[kMore ? L::kW : 1], w6[kMore ? L::kW : 1], w7[kMore ? L::kW : 1];
  __shared__ __attribute__((aligned(1024))) unsigned char e4[kMore ? L::kE : 1], e5[kMore ? L::kE : 1], e6[kMore ? L::kE : 1], e7[kMore ? L::kE : 1];
  const Packed8 pw = packed8(a.rows, a.in), px = packed8(a.m, a.in);
  const int tok_tiles = (a.m + L::kTok - 1) / L::kTok, row_tiles = (a.row_end - a.row_begin + L::kRows - 1) / L::kRows;
  // ids 8 apart run on one XCD: the token tiles of a weight tile follow each other there
  const int row_tile = (int)blockIdx.x / 8 / tok_tiles * 8 + (int)blockIdx.x % 8, tok_tile = (int)blockIdx.x / 8 % tok_tiles;
  if (row_tile >= row_tiles) return;
  const int row0 = a.row_begin + row_tile * L::kRows;         // (a multiple of 16)
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 31, g = lane >> 5;
  const int wm = wave % WM, wn = wave / WM;
  const int n_stage = 2 * pw.groups;

  // what this wavefront copies: 16-row blocks of tokens and of weights (those past the end: the last one again), and a share of the exponents
  __amdgpu_buffer_rsrc_t xsrc[L::kXLoads], wsrc[L::kWLoads];
#pragma unroll
  for (int i = 0; i < L::kXLoads; i++)
    xsrc[i] = buffer_of(a.x8 + (size_t)min(tok_tile * (L::kTok / 16) + L::x_part(wave, i), px.blocks - 1) * px.groups * kTile8);
#pragma unroll
  for (int i = 0; i < L::kWLoads; i++)
    wsrc[i] = buffer_of(a.w8 + (size_t)min(row0 / 16 + L::w_part(wave, i), pw.blocks - 1) * pw.groups * kTile8);
  const int eb = min(wave * 4 + lane / 16, L::kBlocks - 1);
  const uint32_t *esrc = (const uint32_t *)(eb < L::kTok / 16 ? a.x8 + packed8_exps(px) + (size_t)min(tok_tile * (L::kTok / 16) + eb, px.blocks - 1) * px.quads * 64
                                                              : a.w8 + packed8_exps(pw) + (size_t)min(row0 / 16 + eb - L::kTok / 16, pw.blocks - 1) * pw.quads * 64) + lane % 16;
  auto copy = [&](unsigned char *x, unsigned char *w, unsigned char *e, int s) __attribute__((always_inline)) {
    s = min(s, n_stage - 1);                                  // past the end: the last stage again (never read)
#pragma unroll
    for (int i = 0; i < L::kWLoads; i++) load_to_lds(wsrc[i], lane * 16, s * 1024, w + L::w_part(wave, i) * 1024);
#pragma unroll
    for (int i = 0; i < L::kXLoads; i++) load_to_lds(xsrc[i], lane * 16, s * 1024, x + L::x_part(wave, i) * 1024);
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(esrc + (s >> 3) * 16), (lds_void *)(e + wave * 256), 4, 0, 0);
  };

  f32x16_t acc[WB][TB];
#pragma unroll
  for (int b = 0; b < WB; b++)
#pragma unroll
    for (int t = 0; t < TB; t++)
#pragma unroll
      for (int v = 0; v < 16; v++) acc[b][t][v] = 0.f;
  // lane (c, g) of a 32-row operand: row c % 16 of block c / 16, its pieces 2 g and 2 g + 1
  const int at = (c >> 4) * 1024 + (2 * g * 16 + (c & 15)) * 16, e_at = (c >> 4) * 64 + (c & 15) * 4;
  struct Operand { Half8 h; uint32_t e; };
  auto read_x = [&](Operand &o, const unsigned char *x, const unsigned char *e, int t, int s) __attribute__((always_inline)) {
    const unsigned char *p = x + (wm * TB + t) * 2048 + at;
    o = Operand{{*(const u32x4_t *)p, *(const u32x4_t *)(p + 256)}, e[(wm * TB + t) * 128 + e_at + ((s >> 1) & 3)]};
  };
  auto read_w = [&](Operand &o, const unsigned char *w, const unsigned char *e, int b, int s) __attribute__((always_inline)) {
    const unsigned char *p = w + (wn * WB + b) * 2048 + at;
    o = Operand{{*(const u32x4_t *)p, *(const u32x4_t *)(p + 256)}, e[(L::kTok / 32 + wn * WB + b) * 128 + e_at + ((s >> 1) & 3)]};
  };
  Operand xo[TB], wo[2][WB];
  // cw: weight operands of stage s (nw: the next one's); x, w, e: its buffers; xn, wn_, en: those of the next stage
  auto stage = [&](Operand (&cw)[WB], Operand (&nw)[WB], unsigned char *x, unsigned char *w, unsigned char *e, unsigned char *xn, unsigned char *wn_, unsigned char *en,
                   int s) __attribute__((always_inline)) {
    Wide8 ww[kExact ? WB : 1];
    if constexpr (kExact)
#pragma unroll
      for (int b = 0; b < WB; b++) ww[b] = widen8(cw[b].h, cw[b].e);
#pragma unroll
    for (int t = 0; t < TB; t++) {
      Wide8 xw;
      if constexpr (kExact) xw = widen8(xo[t].h, xo[t].e);
#pragma unroll
      for (int b = 0; b < WB; b++) {
        if constexpr (!kExact) acc[b][t] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand8(cw[b].h), operand8(xo[t].h), acc[b][t], 0, 0, 0, (int)cw[b].e, 0, (int)xo[t].e);
        else
#pragma unroll
          for (int i = 0; i < 4; i++)
            acc[b][t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, ww[b].v[i]), __builtin_bit_cast(bf16x8_t, xw.v[i]), acc[b][t], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
        if (t == 0 && b == WB - 1) {
          constexpr int kOpen = (STAGES - 2) * L::kLoads;     // copies that may still be under way
          __builtin_amdgcn_s_waitcnt(0x0070 | (kOpen & 15) | (kOpen >> 4 << 14));   // vmcnt(kOpen) lgkmcnt(0)
          wg_barrier();
        }
        if (TB == 1 ? b == WB - 1 : t == TB / 2 && b == 0) copy(x, w, e, s + STAGES);
        if (TB == 1 ? b == WB - 1 : t == 1 && b == 0)
#pragma unroll
          for (int n = 0; n < WB; n++) read_w(nw[n], wn_, en, n, s + 1);
        if (b == WB - 1) read_x(xo[t], xn, en, t, s + 1);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  };
  copy(x0, w0, e0, 0);
  copy(x1, w1, e1, 1);
  copy(x2, w2, e2, 2);
  copy(x3, w3, e3, 3);
  if constexpr (kMore) {
    copy(x4, w4, e4, 4);
    copy(x5, w5, e5, 5);
    copy(x6, w6, e6, 6);
    copy(x7, w7, e7, 7);
  }
  constexpr int kFirst = (STAGES - 1) * L::kLoads;
  static_assert(kFirst < 64, "what the wait can count");
  __builtin_amdgcn_s_waitcnt(0x0F70 | (kFirst & 15) | (kFirst >> 4 << 14));   // stage 0 here
  wg_barrier();
#pragma unroll
  for (int b = 0; b < WB; b++) read_w(wo[0][b], w0, e0, b, 0);
#pragma unroll
  for (int t = 0; t < TB; t++) read_x(xo[t], x0, e0, t, 0);
  int s = 0;
  for (; s + STAGES <= n_stage; s += STAGES) {
    stage(wo[0], wo[1], x0, w0, e0, x1, w1, e1, s);
    stage(wo[1], wo[0], x1, w1, e1, x2, w2, e2, s + 1);
    stage(wo[0], wo[1], x2, w2, e2, x3, w3, e3, s + 2);
    if constexpr (!kMore) stage(wo[1], wo[0], x3, w3, e3, x0, w0, e0, s + 3);
    else {
      stage(wo[1], wo[0], x3, w3, e3, x4, w4, e4, s + 3);
      stage(wo[0], wo[1], x4, w4, e4, x5, w5, e5, s + 4);
      stage(wo[1], wo[0], x5, w5, e5, x6, w6, e6, s + 5);
      stage(wo[0], wo[1], x6, w6, e6, x7, w7, e7, s + 6);
      stage(wo[1], wo[0], x7, w7, e7, x0, w0, e0, s + 7);
    }
  }
  if (s < n_stage) {                                          // stages come in pairs
    stage(wo[0], wo[1], x0, w0, e0, x1, w1, e1, s);
    stage(wo[1], wo[0], x1, w1, e1, x2, w2, e2, s + 1);
    if constexpr (kMore)
      if (s + 2 < n_stage) {
        stage(wo[0], wo[1], x2, w2, e2, x3, w3, e3, s + 2);
        stage(wo[1], wo[0], x3, w3, e3, x4, w4, e4, s + 3);
        if (s + 4 < n_stage) {
          stage(wo[0], wo[1], x4, w4, e4, x5, w5, e5, s + 4);
          stage(wo[1], wo[0], x5, w5, e5, x6, w6, e6, s + 5);
        }
      }
  }
  __builtin_amdgcn_s_waitcnt(0x0F70);                         // no copy into the LDS outlives the workgroup

  // Sums go through the LDS (the tokens' buffers, a share for each wavefront) into whole rows: a lane has four columns of one token, and stores of these touch 32 rows at a time.
  // Pieces of 16 bytes are permuted by the row, so that neither side meets in a bank.
  constexpr int kCols = WB * 32, kChunks = kCols / 4, kShare = 32 * kCols * 4, kPer = L::kX / kShare, kPerW = L::kW / kShare;
  static_assert(kPer >= 1 && (L::kWaves <= 4 * kPer || (kPerW >= 1 && L::kWaves - 4 * kPer <= 2 * kPerW)), "a share each");
  wg_barrier();                                               // everybody's operands are read
  unsigned char *mine = (wave / kPer == 0 ? x0 : wave / kPer == 1 ? x1 : wave / kPer == 2 ? x2 : x3) + wave % kPer * kShare;
  if constexpr (L::kWaves > 4 * kPer)                         // (the weights' buffers, too)
    if (const int more = wave - 4 * kPer; more >= 0) mine = (more / kPerW == 0 ? w0 : w1) + more % kPerW * kShare;
  const int col0 = row0 + wn * kCols;
#pragma unroll
  for (int t = 0; t < TB; t++) {
    const int tok0 = tok_tile * L::kTok + (wm * TB + t) * 32;
    wave_fence();                                             // (the 32 before have been read)
#pragma unroll
    for (int b = 0; b < WB; b++)
#pragma unroll
      for (int q = 0; q < 4; q++)
        *(f32x4_t *)(mine + c * kCols * 4 + ((b * 8 + 2 * q + g) ^ (c & (kChunks - 1))) * 16) = f32x4_t{acc[b][t][4 * q], acc[b][t][4 * q + 1], acc[b][t][4 * q + 2], acc[b][t][4 * q + 3]};
    wave_fence();
    if constexpr (VEC) {
      constexpr int kAtOnce = 64 / kChunks;
#pragma unroll
      for (int i = 0; i < 32; i += kAtOnce) {
        const int r = i + lane / kChunks, chunk = lane % kChunks;
        const f32x4_t v = *(const f32x4_t *)(mine + r * kCols * 4 + (chunk ^ (r & (kChunks - 1))) * 16);
        if (tok0 + r < a.m) store4<true>((OUT *)a.y + (size_t)(tok0 + r) * a.ldy, col0 + 4 * chunk, a.row_end, v);
      }
    } else {
      constexpr int kAtOnce = 64 / kCols;
#pragma unroll 8
      for (int i = 0; i < 32; i += kAtOnce) {
        const int r = i + lane / kCols, col = lane % kCols;
        const float v = *(const float *)(mine + r * kCols * 4 + ((col >> 2) ^ (r & (kChunks - 1))) * 16 + (col & 3) * 4);
        if (tok0 + r < a.m && col0 + col < a.row_end) ((OUT *)a.y)[(size_t)(tok0 + r) * a.ldy + col0 + col] = from_f32<OUT>(v);
      }
    }
  }
}

template <typename OUT, bool VEC, int WM, int WN, int TB, int WB, int STAGES>
hipError_t launch_tile(const Gemm8Args &a, hipStream_t st) {
  using L = Tile8<WM, WN, TB, WB>;
  const int64_t tok_tiles = (a.m + L::kTok - 1) / L::kTok, row_tiles = (a.row_end - a.row_begin + L::kRows - 1) / L::kRows;
  const int64_t grid = (row_tiles + 7) / 8 * 8 * tok_tiles;
  if (grid * L::kWaves * 64 >> 32) return hipErrorInvalidValue;   // (beyond any memory: the limit of a grid's threads)
  hipLaunchKernelGGL((gemm8_tile_kernel<OUT, VEC, WM, WN, TB, WB, STAGES>), dim3((unsigned)grid), dim3(L::kWaves * 64), 0, st, a);
  return hipGetLastError();
}

// The tile that a launch takes: the one whose workgroups, in rounds over the 256 compute units, are done first.  Measured (us for K = 4096, bf16 results; fp32 results take
// 1.4 to 1.9 times that for all of them): a round of one workgroup a unit, and a unit's time for each when there are more.  The table serves every K and both types: it compares shapes whose
// times grow alike with K; at other K it is not measured.
//   256 x 256: 56, one fits a unit (512 x 28672: 60 against 75 in 256 x 128)        256 x 128: 36, one (2048 x 4096: 36 against 50 in 256 x 256 and 42 in 128 x 128)
//   128 x 128: 24, or two in 41 (1024 x 4096: 24 against 33 in 256 x 128)           64 x 128: 16, or two in 30 (333 x 4096: 16 against 20 in 128 x 128)
//   64 x 64, eight stages deep: 11, or two in 17.5 (60 x 12288: 15 against 20 in 64 x 128)
//   64 x 96, eight stages deep: 14.3, one (60 x 22016, 230 tiles: 20.6 against 26 in 64 x 64, 64 x 128 and 128 x 128; 60 x 28672, 299 tiles: 33 against 28)
enum { kLargest = 0, kTiles8 = 6 };
struct TileCost { int tok, rows, fit; float one, fitting; };  // `fit` workgroups on a unit at once take `fitting`
constexpr TileCost kTileCosts[kTiles8] = {{256, 256, 1, 56.f, 56.f}, {256, 128, 1, 36.f, 36.f}, {128, 128, 2, 24.f, 41.f}, {64, 128, 2, 16.f, 30.f}, {64, 64, 2, 11.f, 17.5f}, {64, 96, 1, 14.3f, 14.3f}};
float tiles_cost(int shape, int m, int rows) {
  const TileCost &c = kTileCosts[shape];
  const int64_t tiles = (int64_t)((m + c.tok - 1) / c.tok) * ((rows + c.rows - 1) / c.rows), a_round = 256 * c.fit, left = tiles % a_round;
  return (float)(tiles / a_round) * c.fitting + (left == 0 ? 0.f : left <= 256 ? c.one : c.fitting);
}
struct Tiles8 { int shape; float cost; };
Tiles8 best_tiles(int m, int rows) {
  Tiles8 best{kLargest, tiles_cost(kLargest, m, rows)};
  for (int i = 1; i < kTiles8; i++)
    if (const float cost = tiles_cost(i, m, rows); cost < best.cost) best = Tiles8{i, cost};
  return best;
}
template <typename OUT, bool VEC> hipError_t launch_tiles(int shape, const Gemm8Args &a, hipStream_t st) {
  switch (shape) {
    case kLargest: return launch_tile<OUT, VEC, 2, 4, 4, 2, 4>(a, st);
    case 1: return launch_tile<OUT, VEC, 4, 2, 2, 2, 4>(a, st);
    case 2: return launch_tile<OUT, VEC, 2, 4, 2, 1, 4>(a, st);
    case 3: return launch_tile<OUT, VEC, 1, 4, 2, 1, 4>(a, st);
    case 4: return launch_tile<OUT, VEC, 2, 2, 1, 1, 8>(a, st);
    default: return launch_tile<OUT, VEC, 2, 3, 1, 1, 8>(a, st);
  }
}

// Up to 16 tokens: they are put into 8 bits by every workgroup for itself where that is little work each, or by a launch ahead (3.8 us), into scratch.  Measured (us, with the launch
// where there is one): 1 token, 22016 x 4096 19.3 against 23.1; 4 tokens, 4096 x 4096 7.3 against 9.8, but 28672 x 8192 47.9 against 46.6.
int few_tokens_log2(int m) {
  int mp = 0;
  while ((1 << mp) < m) mp++;
  return mp;
}
bool few_raw(int m, int in, int rows) {
  const Packed8 pw = packed8(rows, in);
  return m <= 16 && ((int64_t)pw.groups << (few_tokens_log2(m) + 7)) <= (pw.blocks <= 512 ? 1 << 15 : 1 << 13);
}
template <typename X, typename OUT, bool VEC>
hipError_t launch_few(Gemm8Args a, void *scratch, hipStream_t st) {
  const Packed8 pw = packed8(a.rows, a.in);
  if (few_raw(a.m, a.in, a.rows)) {
    const int mp = few_tokens_log2(a.m);
    hipLaunchKernelGGL((gemm8_few_kernel<X, OUT, VEC, true>), dim3(pw.blocks), dim3(kStreamWaves * 64), (unsigned)((pw.groups << (mp + 7)) + (pw.groups << mp)), st, a, mp);
    return hipGetLastError();
  }
  const hipError_t e = quant8((const X *)a.x, a.ldx, a.m, a.in, 0, scratch, st);
  if (e != hipSuccess) return e;
  a.x8 = (const unsigned char *)scratch;
  hipLaunchKernelGGL((gemm8_few_kernel<void, OUT, VEC, false>), dim3(pw.blocks), dim3(kStreamWaves * 64), 0, st, a, 0);
  return hipGetLastError();
}

template <typename X, typename OUT, bool VEC>
hipError_t launch_typed(Gemm8Args a, void *scratch, hipStream_t st) {
  if (a.m <= 16) return launch_few<X, OUT, VEC>(a, scratch, st);
  const hipError_t e = quant8((const X *)a.x, a.ldx, a.m, a.in, 0, scratch, st);
  if (e != hipSuccess) return e;
  a.x8 = (const unsigned char *)scratch;
  // 17 to 64 tokens through few rows: the weights straight into registers (us, 60 tokens: 4096 rows of 4096 9.1 against 11.1 in tiles of 64 x 64, of 11008 18.9 against 28.1;
  // 12288 rows of 4096 23.1 against 15.1)
  if (a.m <= 64 && a.rows <= 4096) return a.m <= 32 ? launch_stream<OUT, VEC, 2>(a, st) : launch_stream<OUT, VEC, 4>(a, st);
  a.row_begin = 0; a.row_end = a.rows;
  const Tiles8 all = best_tiles(a.m, a.rows);
  // whole rounds of the largest tile, and the rows that are left in what suits them: 2048 x 28672 x 4096 (3.5 rounds) 217 -> 205 us, 2048 x
  // 12288 x 4096 (1.5) 105 -> 94; 2048 x 22016 x 4096 (2.7) would take 177 instead of 164.  (The 3 us of another launch are against the costs of K = 4096.)
  const int64_t tok = (a.m + 255) / 256, in_rounds = tok * ((a.rows + 255) / 256) / 256 * 256 / tok * 256;
  if (in_rounds > 0 && in_rounds < a.rows) {
    const Tiles8 rest = best_tiles(a.m, a.rows - (int)in_rounds);
    if (tiles_cost(kLargest, a.m, (int)in_rounds) + rest.cost + 3.f < all.cost) {
      a.row_end = (int)in_rounds;
      const hipError_t first = launch_tiles<OUT, VEC>(kLargest, a, st);
      if (first != hipSuccess) return first;
      a.row_begin = a.row_end; a.row_end = a.rows;
      return launch_tiles<OUT, VEC>(rest.shape, a, st);
    }
  }
  return launch_tiles<OUT, VEC>(all.shape, a, st);
}

}  // namespace

hipError_t launch_pack_weight8(int dtype, const void *src, int rows, int in, void *dst, hipStream_t st) {
  return dtype == 1 ? quant8((const bf16_t *)src, in, rows, in, 1, dst, st) : quant8((const float *)src, in, rows, in, 1, dst, st);
}

uint64_t gemm8_scratch_bytes(int m, int in, int rows) { return few_raw(m, in, rows) ? 0 : packed8_bytes(packed8(m, in)); }

hipError_t launch_gemm8(int dtype, int out_dtype, const Gemm8Args &a, void *scratch, hipStream_t st) {
  const bool vec = ((uintptr_t)a.y & (out_dtype == 1 ? 7 : 15)) == 0 && a.ldy % 4 == 0;
#define SPEC_G8(X, OUT) (vec ? launch_typed<X, OUT, true>(a, scratch, st) : launch_typed<X, OUT, false>(a, scratch, st))
  if (dtype == 1) return out_dtype == 1 ? SPEC_G8(bf16_t, bf16_t) : SPEC_G8(bf16_t, float);
  return out_dtype == 1 ? SPEC_G8(float, bf16_t) : SPEC_G8(float, float);
#undef SPEC_G8
}

}  // namespace spec
