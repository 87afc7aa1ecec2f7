// Rotary embedding of the heads of up to three tensors, forward and adjoint (include/spec_layer8.h).
//
// A workgroup owns one row: its threads first make the row's (cos, sin) table in the LDS, then walk the row's heads.  The angle in turns, pos * freq / 2 pi,
// is formed and brought to an eighth of a turn in 64 bits, sine and cosine of what is left in 32: their error does not grow with the position.
// Bound: memory (each element once in, once out).
#include "common.h"
#include "kernels.h"

namespace spec {

namespace {

constexpr int kRotaryThreads = 256;

// (cos, sin) of x turns
__device__ __forceinline__ float2 turn_of(double x) {
  const double q = rint(4.0 * x), r = fma(-0.25, q, x);       // a quarter turn's multiple, and at most an eighth beside it
  float s, c;
  sincosf((float)(r * 6.283185307179586), &s, &c);
  const int k = (int)(q - 4.0 * floor(0.25 * q));             // 0 .. 3
  const float cq = (k & 1) ? s : c, sq = (k & 1) ? c : s;
  return make_float2((k == 1 || k == 2) ? -cq : cq, (k >= 2) ? -sq : sq);
}

__device__ __forceinline__ float load1(const void *p, int64_t i, int dtype) { return dtype == 1 ? to_f32(((const bf16_t *)p)[i]) : ((const float *)p)[i]; }
__device__ __forceinline__ void store1(void *p, int64_t i, int dtype, float v) {
  if (dtype == 1) ((bf16_t *)p)[i] = from_f32<bf16_t>(v);
  else ((float *)p)[i] = v;
}

__global__ __launch_bounds__(kRotaryThreads) void rotary_kernel(RotaryArgs a) {
  __shared__ float2 table[kRotaryMaxPlanes];
  const int64_t row = blockIdx.x;
  const int half = a.rot / 2;
  const double pos = (double)(a.pos ? (int64_t)a.pos[row] : (int64_t)a.pos0 + row);
  for (int j = threadIdx.x; j < half; j += kRotaryThreads) {
    float2 cs = turn_of(pos * a.turns[j]);
    cs.x *= a.mscale; cs.y *= a.adjoint ? -a.mscale : a.mscale;
    table[j] = cs;
  }
  __syncthreads();
  for (int n = 0; n < a.n_parts; n++) {
    const RotaryPart &p = a.part[n];
    const int planes = p.turn ? half : 0, items = planes + a.hd - 2 * planes;
    for (int i = threadIdx.x; i < p.heads * items; i += kRotaryThreads) {
      const int h = i / items, it = i - h * items;
      const int64_t xi = row * p.ldx + h * p.hsx, oi = row * p.ldo + h * p.hso;
      if (it < planes) {
        const int da = a.interleaved ? 2 * it : it, db = a.interleaved ? da + 1 : it + half;
        const float u = load1(p.x, xi + da, p.dtype), v = load1(p.x, xi + db, p.dtype);
        store1(p.out, oi + da, p.out_dtype, rope_first(u, v, table[it]));
        store1(p.out, oi + db, p.out_dtype, rope_second(u, v, table[it]));
      } else {
        const int d = it + planes;
        store1(p.out, oi + d, p.out_dtype, load1(p.x, xi + d, p.dtype));
      }
    }
  }
}

}  // namespace

hipError_t launch_rotary(const RotaryArgs &a, hipStream_t st) {
  hipLaunchKernelGGL(rotary_kernel, dim3(a.rows), dim3(kRotaryThreads), 0, st, a);
  return hipGetLastError();
}

}  // namespace spec
