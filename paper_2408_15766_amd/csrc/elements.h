// Elements of fp32 and bf16 tensors one or eight at a time, and angles: shared by the kernels that walk tensors of either type.
#pragma once
#include "common.h"

namespace spec {

// scale * (cos, sin) of x turns, by the series of sine and cosine to the 13th and 12th power (what is left out of them: under 4e-13 up to an eighth of a turn)
__device__ __forceinline__ float2 turn_of(double x, double scale) {
  const double q = rint(4.0 * x), t = fma(-0.25, q, x) * 6.283185307179586, u = t * t;   // a quarter turn's multiple, and at most an eighth beside it
  double s = fma(u, 1.0 / 6227020800.0, -1.0 / 39916800.0), c = fma(u, 1.0 / 479001600.0, -1.0 / 3628800.0);
  s = fma(u, s, 1.0 / 362880.0);
  c = fma(u, c, 1.0 / 40320.0);
  s = fma(u, s, -1.0 / 5040.0);
  c = fma(u, c, -1.0 / 720.0);
  s = fma(u, s, 1.0 / 120.0);
  c = fma(u, c, 1.0 / 24.0);
  s = fma(u, s, -1.0 / 6.0);
  c = fma(u, c, -0.5);
  s = fma(u * t, s, t) * scale;
  c = fma(u, c, 1.0) * scale;
  const int k = (int)(q - 4.0 * floor(0.25 * q));             // 0 .. 3
  const float cq = (float)((k & 1) ? s : c), sq = (float)((k & 1) ? c : s);
  return make_float2((k == 1 || k == 2) ? -cq : cq, (k >= 2) ? -sq : sq);
}

__device__ __forceinline__ float load1(const void *p, int64_t i, int bf16) { return bf16 ? to_f32(((const bf16_t *)p)[i]) : ((const float *)p)[i]; }
__device__ __forceinline__ void store1(void *p, int64_t i, int bf16, float v) {
  if (bf16) ((bf16_t *)p)[i] = from_f32<bf16_t>(v);
  else ((float *)p)[i] = v;
}
// Eight values as they are in memory (bf16: the first half only)
struct Eight { u32x4_t v[2]; };
__device__ __forceinline__ Eight load8(const void *p, int64_t i, int bf16) {
  Eight r;
  if (bf16) r.v[0] = *(const u32x4_t *)((const bf16_t *)p + i);
  else { r.v[0] = *(const u32x4_t *)((const float *)p + i); r.v[1] = *(const u32x4_t *)((const float *)p + i + 4); }
  return r;
}
__device__ __forceinline__ void widen8(const Eight &r, int bf16, float (&x)[8]) {
#pragma unroll
  for (int j = 0; j < 4; j++) {
    if (bf16) { x[2 * j] = __uint_as_float(r.v[0][j] << 16); x[2 * j + 1] = __uint_as_float(r.v[0][j] & 0xFFFF0000u); }
    else { x[j] = __uint_as_float(r.v[0][j]); x[4 + j] = __uint_as_float(r.v[1][j]); }
  }
}
__device__ __forceinline__ void store8(void *p, int64_t i, int bf16, const float (&x)[8]) {
  if (bf16) *(u32x4_t *)((bf16_t *)p + i) = u32x4_t{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7])};
  else {
    *(f32x4_t *)((float *)p + i) = f32x4_t{x[0], x[1], x[2], x[3]};
    *(f32x4_t *)((float *)p + i + 4) = f32x4_t{x[4], x[5], x[6], x[7]};
  }
}

// A field of the launch's arguments as a value of its own: a choice between two fields must not become a choice between their addresses (that
// would put the arguments into private memory).
template <typename V> __device__ __forceinline__ V pinned(V v) { asm("" : "+s"(v)); return v; }

}  // namespace spec
