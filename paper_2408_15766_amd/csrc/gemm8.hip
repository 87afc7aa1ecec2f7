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
// A wavefront owns 8 rows x 128 k: lane = row * 8 + piece, 16 k each.  Rows beyond `rows` are written as zeros if `pad` (weights: the whole
// buffer is defined), else left out (their products are never stored).
template <typename T, bool VEC>
__global__ __launch_bounds__(256) void quant8_kernel(const T *x, int64_t ldx, int rows, int in, int pad, unsigned char *dst) {
  const Packed8 pk = packed8(rows, in);
  const int lane = threadIdx.x & 63, r8 = lane >> 3, piece = lane & 7;
  const int64_t wave = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
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
  float amax = 0.f;
#pragma unroll
  for (int i = 0; i < 16; i++) amax = fmaxf(amax, finite_abs(v[i]));
  amax = fmaxf(amax, dpp_f32<0xB1>(amax));                    // the row's eight lanes
  amax = fmaxf(amax, dpp_f32<0x4E>(amax));
  amax = fmaxf(amax, dpp_f32<0x141>(amax));
  const int e = exponent8(amax);
  const float down = pow2(-e);
  u32x4_t c;
#pragma unroll
  for (int i = 0; i < 4; i++) c[i] = codes4(v[4 * i] * down, v[4 * i + 1] * down, v[4 * i + 2] * down, v[4 * i + 3] * down);
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
  const int64_t grid = (waves + 3) / 4;
  if (grid > 0x7FFFFFFFll) return hipErrorInvalidValue;
  const bool vec = ((uintptr_t)x & 15) == 0 && ldx % (16 / (int)sizeof(T)) == 0;
  if (vec) hipLaunchKernelGGL((quant8_kernel<T, true>), dim3((unsigned)grid), dim3(256), 0, st, x, ldx, rows, in, pad, (unsigned char *)dst);
  else hipLaunchKernelGGL((quant8_kernel<T, false>), dim3((unsigned)grid), dim3(256), 0, st, x, ldx, rows, in, pad, (unsigned char *)dst);
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

// Weights streamed: a workgroup owns a 16-row block and up to 64 tokens, its eight wavefronts an eighth of k each, added up in the LDS in ascending order.
constexpr int kStreamWaves = 8, kStreamTiles = 4;
template <typename OUT, bool VEC>
__global__ __launch_bounds__(kStreamWaves * 64) void gemm8_stream_kernel(Gemm8Args a) {
  constexpr bool kExact = sizeof(OUT) == 4;
  __shared__ f32x4_t part[kStreamWaves][kStreamTiles][64];
  const Packed8 pw = packed8(a.rows, a.in), px = packed8(a.m, a.in);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int rb = blockIdx.x, t0 = blockIdx.y * kStreamTiles;
  const unsigned char *wt = a.w8 + (size_t)rb * pw.groups * kTile8;
  const uint32_t *we = (const uint32_t *)(a.w8 + packed8_exps(pw)) + (size_t)rb * pw.quads * 16 + (lane & 15);
  const int g0 = pw.groups * wave / kStreamWaves, g1 = pw.groups * (wave + 1) / kStreamWaves;
  f32x4_t acc[kStreamTiles];
#pragma unroll
  for (int t = 0; t < kStreamTiles; t++) acc[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  for (int g = g0; g < g1; g++) {
    const Frag8 w = load_frag(wt + (size_t)g * kTile8, lane);
    const uint32_t ew = we[(g >> 2) * 16] >> (8 * (g & 3));
#pragma unroll
    for (int t = 0; t < kStreamTiles; t++) {
      const int b = min(t0 + t, px.blocks - 1);
      const Frag8 x = load_frag(a.x8 + ((size_t)b * px.groups + g) * kTile8, lane);
      const uint32_t ex = ((const uint32_t *)(a.x8 + packed8_exps(px)))[((size_t)b * px.quads + (g >> 2)) * 16 + (lane & 15)] >> (8 * (g & 3));
      acc[t] = product<kExact>(w, ew, x, ex, acc[t]);
    }
  }
#pragma unroll
  for (int t = 0; t < kStreamTiles; t++) part[wave][t][lane] = acc[t];
  __syncthreads();
  if (threadIdx.x >= kStreamTiles * 64) return;
  f32x4_t s = part[0][wave][lane];
#pragma unroll
  for (int w = 1; w < kStreamWaves; w++) s += part[w][wave][lane];
  const int tok = (t0 + wave) * 16 + (lane & 15);
  if (tok < a.m) store4<VEC>((OUT *)a.y + (size_t)tok * a.ldy, rb * 16 + 4 * (lane >> 4), a.rows, s);
}

}  // namespace

hipError_t launch_pack_weight8(int dtype, const void *src, int rows, int in, void *dst, hipStream_t st) {
  return dtype == 1 ? quant8((const bf16_t *)src, in, rows, in, 1, dst, st) : quant8((const float *)src, in, rows, in, 1, dst, st);
}

hipError_t launch_gemm8(int dtype, const void *x, int64_t ldx, int out_dtype, Gemm8Args a, void *scratch, hipStream_t st) {
  a.x8 = (const unsigned char *)scratch;
  const hipError_t e = dtype == 1 ? quant8((const bf16_t *)x, ldx, a.m, a.in, 0, scratch, st) : quant8((const float *)x, ldx, a.m, a.in, 0, scratch, st);
  if (e != hipSuccess) return e;
  const bool vec = ((uintptr_t)a.y & (out_dtype == 1 ? 7 : 15)) == 0 && a.ldy % 4 == 0;
  const dim3 grid((a.rows + 15) / 16, (a.m + 16 * kStreamTiles - 1) / (16 * kStreamTiles));
  if (grid.y > 65535) return hipErrorInvalidValue;
#define SPEC_G8(OUT, VEC) hipLaunchKernelGGL((gemm8_stream_kernel<OUT, VEC>), grid, dim3(kStreamWaves * 64), 0, st, a)
  if (out_dtype == 1) { if (vec) SPEC_G8(bf16_t, true); else SPEC_G8(bf16_t, false); }
  else { if (vec) SPEC_G8(float, true); else SPEC_G8(float, false); }
#undef SPEC_G8
  return hipGetLastError();
}

}  // namespace spec
