// Rotary embedding of the heads of up to three tensors, forward and adjoint (include/spec_layer8.h).
//
// A workgroup owns a few whole rows of one tensor.  Its threads ask for their first values, make the rows' (cos, sin) table in the LDS while these are coming, and
// turn.  The angle in turns, pos * freq / 2 pi, is formed and brought to an eighth of a turn in 64 bits, as are its sine and cosine and their product with mscale: the error does not grow
// with the position, and the table's entries are rounded once, to fp32.
// Bound: memory (each element once in, once out): 16-byte accesses, eight planes (or eight dims that pass) a step of a thread.
#include "common.h"
#include "elements.h"
#include "kernels.h"

namespace spec {

namespace {

constexpr int kRotaryThreads = 256, kRotaryTable = 1024;      // table entries of a workgroup

// n / d by the launch's d.x = ceil(2^32 / d): exact below 2^16 (d.y = d)
__device__ __forceinline__ uint32_t over(uint32_t n, uint2 d) { return d.y == 1 ? n : __umulhi(n, d.x); }

__device__ __forceinline__ RotaryPart pinned_part(const RotaryPart &p) {
  return RotaryPart{pinned(p.x), pinned(p.out), pinned(p.ldx), pinned(p.hsx), pinned(p.ldo), pinned(p.hso), pinned(p.heads), pinned(p.dtype), pinned(p.out_dtype), pinned(p.turn)};
}

// One tensor of some rows.  A thread's step: eight planes or eight dims that pass (VEC), else one; the items of a head are its planes' first, then the dims that pass.
template <bool VEC>
__global__ __launch_bounds__(kRotaryThreads) void rotary_kernel(RotaryArgs a) {
  __shared__ float2 table[kRotaryTable];
  constexpr int W = VEC ? 8 : 1;
  const RotaryPart p0 = pinned_part(a.part[0]), p1 = pinned_part(a.part[1]), p2 = pinned_part(a.part[2]);
  const uint2 h0 = make_uint2(pinned(a.head_items[0].x), pinned(a.head_items[0].y)), h1 = make_uint2(pinned(a.head_items[1].x), pinned(a.head_items[1].y)),
              h2 = make_uint2(pinned(a.head_items[2].x), pinned(a.head_items[2].y));
  const uint2 r0 = make_uint2(pinned(a.row_items[0].x), pinned(a.row_items[0].y)), r1 = make_uint2(pinned(a.row_items[1].x), pinned(a.row_items[1].y)),
              r2 = make_uint2(pinned(a.row_items[2].x), pinned(a.row_items[2].y));
  const int n = blockIdx.y;
  const RotaryPart p = n == 0 ? p0 : n == 1 ? p1 : p2;
  const uint2 head_items = n == 0 ? h0 : n == 1 ? h1 : h2, row_items = n == 0 ? r0 : n == 1 ? r1 : r2;
  const int64_t row0 = ((int64_t)blockIdx.z * gridDim.x + blockIdx.x) * a.rows_each;   // (from a.rows on: nothing to do)
  const int rows = (int)min((int64_t)a.rows_each, a.rows - row0), half = a.rot / 2, total = rows * (int)row_items.y;
  const bool pairs = !a.interleaved;                          // a turning step has its planes' partners half further on
  const int turning = !p.turn ? 0 : VEC && a.interleaved ? half / 4 : half / W;   // steps of a head that turn
  struct Step { int64_t x, o; int it, row; bool turn; };
  auto step_of = [&](int i) {
    Step s;
    s.row = (int)over(i, row_items);
    const int at = i - s.row * (int)row_items.y, h = (int)over(at, head_items);
    s.it = at - h * (int)head_items.y;
    s.turn = s.it < turning;
    const int d = s.turn ? (a.interleaved && !VEC ? 2 : W) * s.it : (p.turn ? a.rot : 0) + W * (s.it - turning);   // its first dim
    s.x = (row0 + s.row) * p.ldx + h * p.hsx + d;
    s.o = (row0 + s.row) * p.ldo + h * p.hso + d;
    return s;
  };
  struct Values { Eight u, v; };
  auto load = [&](const Step &s) {
    Values r;
    if constexpr (VEC) {
      r.u = load8(p.x, s.x, p.dtype);
      if (s.turn && pairs) r.v = load8(p.x, s.x + half, p.dtype);
    }
    return r;
  };
  const int first = threadIdx.x;
  Step s;
  Values val;
  if (first < total) { s = step_of(first); val = load(s); }
  if (p.turn)
    for (int j = threadIdx.x; j < rows * half; j += kRotaryThreads) {
      const int r = j / half, plane = j - r * half;
      const double pos = a.pos ? (double)a.pos[row0 + r] : (double)(a.pos0 + row0 + r);
      float2 cs = turn_of(pos * a.turns[plane], a.mscale);
      if (a.adjoint) cs.y = -cs.y;
      table[j] = cs;
    }
  __syncthreads();
  for (int i = first; i < total; i += kRotaryThreads) {
    const Step now = s;
    const Values cur = val;
    if (i + kRotaryThreads < total) { s = step_of(i + kRotaryThreads); val = load(s); }
    if constexpr (VEC) {
      float u[8];
      widen8(cur.u, p.dtype, u);
      if (now.turn && pairs) {
        const float2 *cs = table + now.row * half + 8 * now.it;
        float v[8], x[8], y[8];
        widen8(cur.v, p.dtype, v);
#pragma unroll
        for (int j = 0; j < 8; j++) { x[j] = rope_first(u[j], v[j], cs[j]); y[j] = rope_second(u[j], v[j], cs[j]); }
        store8(p.out, now.o, p.out_dtype, x);
        store8(p.out, now.o + half, p.out_dtype, y);
      } else if (now.turn) {
        const float2 *cs = table + now.row * half + 4 * now.it;
        float x[8];
#pragma unroll
        for (int j = 0; j < 4; j++) { x[2 * j] = rope_first(u[2 * j], u[2 * j + 1], cs[j]); x[2 * j + 1] = rope_second(u[2 * j], u[2 * j + 1], cs[j]); }
        store8(p.out, now.o, p.out_dtype, x);
      } else store8(p.out, now.o, p.out_dtype, u);
    } else {
      const float u = load1(p.x, now.x, p.dtype);
      if (now.turn) {
        const int64_t other = pairs ? half : 1;
        const float v = load1(p.x, now.x + other, p.dtype);
        const float2 cs = table[now.row * half + now.it];
        store1(p.out, now.o, p.out_dtype, rope_first(u, v, cs));
        store1(p.out, now.o + other, p.out_dtype, rope_second(u, v, cs));
      } else store1(p.out, now.o, p.out_dtype, u);
    }
  }
}

uint2 divisor(int d) { return make_uint2(d == 1 ? 0u : (uint32_t)(((1ull << 32) + d - 1) / d), (uint32_t)d); }

}  // namespace

hipError_t launch_rotary(RotaryArgs a, hipStream_t st) {
  // eight dims at a time where every access is a multiple of 16 bytes from a multiple of 16 bytes
  bool vec = a.hd % 8 == 0 && a.rot % (a.interleaved ? 8 : 16) == 0;
  for (int n = 0; n < a.n_parts; n++) {
    const RotaryPart &p = a.part[n];
    const int64_t ex = p.dtype ? 8 : 4, eo = p.out_dtype ? 8 : 4;
    vec = vec && ((uintptr_t)p.x & 15) == 0 && ((uintptr_t)p.out & 15) == 0 && p.ldx % ex == 0 && p.hsx % ex == 0 && p.ldo % eo == 0 && p.hso % eo == 0;
  }
  const int w = vec ? 8 : 1, half = a.rot / 2;
  int64_t most = 0;                                           // steps of a row of one tensor
  for (int n = 0; n < a.n_parts; n++) {
    const int of_head = a.part[n].turn ? (vec && a.interleaved ? half / 4 : half / w) + (a.hd - a.rot) / w : a.hd / w;
    const int64_t of_row = (int64_t)a.part[n].heads * of_head;
    if (of_row >= 1 << 16) {                                  // (the divisions: steps are numbered below 2^16; only more than 255 heads of 256 get here)
      RotaryArgs b = a;
      const int heads = a.part[n].heads / 2;
      b.part[n].heads = heads;
      const hipError_t e = launch_rotary(b, st);
      if (e != hipSuccess) return e;
      b.n_parts = 1;
      b.part[0] = a.part[n];
      b.part[0].heads -= heads;
      b.part[0].x = (const char *)a.part[n].x + heads * a.part[n].hsx * (a.part[n].dtype ? 2 : 4);
      b.part[0].out = (char *)a.part[n].out + heads * a.part[n].hso * (a.part[n].out_dtype ? 2 : 4);
      return launch_rotary(b, st);
    }
    a.head_items[n] = divisor(of_head);
    a.row_items[n] = divisor((int)of_row);
    most = of_row > most ? of_row : most;
  }
  // two steps a thread, if there are rows for it and the LDS holds their tables
  int each = (int)(2 * kRotaryThreads / most);
  each = each < 1 ? 1 : each > 32 ? 32 : each;
  if (half > 0 && each * half > kRotaryTable) each = kRotaryTable / half;
  while (each > 1 && a.rows / each < 256) each /= 2;          // (rather more workgroups than compute units)
  a.rows_each = each;
  const int64_t groups = ((int64_t)a.rows + each - 1) / each, deep = (groups + (1 << 23) - 1) >> 23;   // (a grid's dimension holds less than 2^32 threads)
  const dim3 grid((unsigned)((groups + deep - 1) / deep), a.n_parts, (unsigned)deep);
  if (vec) hipLaunchKernelGGL(rotary_kernel<true>, grid, dim3(kRotaryThreads), 0, st, a);
  else hipLaunchKernelGGL(rotary_kernel<false>, grid, dim3(kRotaryThreads), 0, st, a);
  return hipGetLastError();
}

}  // namespace spec
