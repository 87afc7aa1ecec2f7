// Norms of heads with the rotary embedding in the same pass, and their gradients (include/spec_step.h).
//
// A head is held by a group of 2^n lanes, each with the same dims of every head it meets: eight planes (16 dims) or eight dims that do
// not turn, four where eight do not fit the layout (a head of 72), else up to four single ones (then a wavefront holds the head, and
// takes five times as long).  So a weight is read once, the sums over a head are a few exchanges between neighbouring lanes, and a lane
// adds up its dims' share of the weights' gradient in registers over all its heads; the workgroup's shares meet in the LDS once, in a
// fixed order, the workgroups' in a second launch.  The rows' (cos, sin) table is made in the LDS as for the rotary embedding alone.
// All sums are fp32: the weights' gradient one head after the other in a lane, the head's mean times r^2 by four products.  In fp32 the
// results are 1.7e-7 of their norm off, those of the same formulas in torch's fp32 1.2e-7 (777 rows of 5 + 3 heads of 80).
// Bound: memory (forward: each element once in, once out; gradients: dy and x once in, dx once out).  Measured (4096 rows of 32 + 32
// heads of 128): forward in bf16 24.6 us (5.5 TB/s); gradients in bf16 38 us (5.2 TB/s) and 4 for the second launch (5 with eight
// threads to a dim), 52 with a fixed number of rows a workgroup, whose table was made again for each; in fp32 93 us (4.3 TB/s).  Rows of
// a tree (60, 32 + 8 + 8 heads) 5.5 us, a launch and two trips to memory.
#include "common.h"
#include "elements.h"
#include "kernels.h"

namespace spec {

namespace {

constexpr int kNormWg = 256, kNormTable = 1024;               // threads, and table entries of a workgroup
// Workgroups of a launch, shared out among the parts by their heads: as many as run at once, so that every one has about the same number
// of rows and their table is made once.  Forward calls have four to a compute unit.  Gradients have three in bf16 (161 and 163
// registers); of eight dims in fp32 (182, 189) or of mixed types (171) two run at once, so that 768 are a round and a half there.
constexpr int kGradGroups = 768, kForwardGroups = 1024;

// Sum over the aligned group of 2^n lanes that a lane is in; all 64 lanes take part
__device__ __forceinline__ float group_sum(float x, int group) {
  if (group >= 2) x += dpp_f32<0xB1>(x);                      // quad_perm [1,0,3,2]
  if (group >= 4) x += dpp_f32<0x4E>(x);                      // quad_perm [2,3,0,1]
  if (group >= 8) x += dpp_f32<0x141>(x);                     // the other quad of eight (mirrored: all lanes of a quad hold the same)
  if (group >= 16) x += dpp_f32<0x140>(x);                    // the other half of a row of sixteen
  if (group >= 32) x += __int_as_float(butterfly<16>(__float_as_int(x)));
  if (group >= 64) x += __int_as_float(butterfly<32>(__float_as_int(x)));
  return x;
}

// The dims of a lane.  W = 8 or 4: x[0 .. W - 1] are W consecutive dims, x[W ..] their planes' partners (half layout) or nothing.
// W = 1: up to four items a lane, item k: x[2 k] and, if it is a plane, x[2 k + 1].
enum { kIdle = 0, kPass = 1, kPairs = 2, kInterleaved = 3 };
template <int W> struct Dims { static constexpr int kItems = W > 1 ? 1 : 4, kElems = W > 1 ? 2 * W : 8; int kind[kItems], first[kItems], plane[kItems]; };
template <int W> __device__ __forceinline__ Dims<W> dims_of(int lane, int items, int group, int rot, bool interleaved) {
  Dims<W> r;
  const int half = rot / 2, planes = W > 1 && interleaved ? W / 2 : W, turning = half / planes;   // planes of a step, and steps that turn
#pragma unroll
  for (int k = 0; k < Dims<W>::kItems; k++) {
    const int it = lane + k * group;
    r.kind[k] = it >= items ? kIdle : it >= turning ? kPass : interleaved ? kInterleaved : kPairs;
    r.plane[k] = planes * it;
    r.first[k] = r.kind[k] == kPass ? rot + W * (it - turning) : interleaved ? 2 * r.plane[k] : r.plane[k];
  }
  return r;
}
// As they are in memory, then as numbers
struct Raw { u32x4_t a, b, c, d; };                           // W = 8: a and b (bf16: a), and the partners' c and d; W = 4: a, and c
template <int W> __device__ __forceinline__ Eight load_w(const void *p, int64_t i, int bf16) {
  if constexpr (W == 8) return load8(p, i, bf16);
  Eight r;
  if (bf16) { const u32x2_t v = *(const u32x2_t *)((const bf16_t *)p + i); r.v[0] = u32x4_t{v.x, v.y, 0u, 0u}; }
  else r.v[0] = *(const u32x4_t *)((const float *)p + i);
  return r;
}
template <int W> __device__ __forceinline__ Raw load_dims(const void *p, int64_t at, int bf16, const Dims<W> &m, int half) {
  const u32x4_t zero = {0u, 0u, 0u, 0u};
  Raw r{zero, zero, zero, zero};
  if constexpr (W > 1) {
    if (m.kind[0] != kIdle) { const Eight e = load_w<W>(p, at + m.first[0], bf16); r.a = e.v[0]; if (W == 8 && !bf16) r.b = e.v[1]; }
    if (m.kind[0] == kPairs) { const Eight e = load_w<W>(p, at + m.first[0] + half, bf16); r.c = e.v[0]; if (W == 8 && !bf16) r.d = e.v[1]; }
  } else {
    uint32_t x[8];
#pragma unroll
    for (int k = 0; k < 4; k++) {
      x[2 * k] = x[2 * k + 1] = 0u;
      if (m.kind[k] != kIdle) x[2 * k] = __float_as_uint(load1(p, at + m.first[k], bf16));
      if (m.kind[k] >= kPairs) x[2 * k + 1] = __float_as_uint(load1(p, at + m.first[k] + (m.kind[k] == kPairs ? half : 1), bf16));
    }
    r.a = u32x4_t{x[0], x[1], x[2], x[3]};
    r.b = u32x4_t{x[4], x[5], x[6], x[7]};
  }
  return r;
}
template <int W> __device__ __forceinline__ void widen_dims(const Raw &r, int bf16, float (&x)[Dims<W>::kElems]) {
  if constexpr (W > 1) {
    float a[8], b[8];
    widen8(Eight{{r.a, r.b}}, bf16, a);
    widen8(Eight{{r.c, r.d}}, bf16, b);
#pragma unroll
    for (int j = 0; j < W; j++) { x[j] = a[j]; x[W + j] = b[j]; }
  } else {
#pragma unroll
    for (int j = 0; j < 4; j++) { x[j] = __uint_as_float(r.a[j]); x[4 + j] = __uint_as_float(r.b[j]); }
  }
}
template <int W> __device__ __forceinline__ void store_w(void *p, int64_t i, int bf16, const float *x) {
  if constexpr (W == 8) {
    const float v[8] = {x[0], x[1], x[2], x[3], x[4], x[5], x[6], x[7]};
    store8(p, i, bf16, v);
  } else if (bf16) *(u32x2_t *)((bf16_t *)p + i) = u32x2_t{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3])};
  else *(f32x4_t *)((float *)p + i) = f32x4_t{x[0], x[1], x[2], x[3]};
}
template <int W> __device__ __forceinline__ void store_dims(void *p, int64_t at, int bf16, const Dims<W> &m, int half, const float (&x)[Dims<W>::kElems]) {
  if constexpr (W > 1) {
    if (m.kind[0] != kIdle) store_w<W>(p, at + m.first[0], bf16, x);
    if (m.kind[0] == kPairs) store_w<W>(p, at + m.first[0] + half, bf16, x + W);
  } else {
#pragma unroll
    for (int k = 0; k < 4; k++) {
      if (m.kind[k] != kIdle) store1(p, at + m.first[k], bf16, x[2 * k]);
      if (m.kind[k] >= kPairs) store1(p, at + m.first[k] + (m.kind[k] == kPairs ? half : 1), bf16, x[2 * k + 1]);
    }
  }
}
// Turned by the row's table (back: by the opposite angles).  INTER is for several dims at a time (two patterns behind one branch went to memory)
template <int W, bool INTER> __device__ __forceinline__ void turn_dims(float (&x)[Dims<W>::kElems], const Dims<W> &m, const float2 *cs, float back) {
  auto turn = [&](float &a, float &b, int plane) __attribute__((always_inline)) {
    const float2 c = make_float2(cs[plane].x, back * cs[plane].y);
    const float u = rope_first(a, b, c), v = rope_second(a, b, c);
    a = u; b = v;
  };
  if constexpr (W > 1 && !INTER) {
    if (m.kind[0] == kPairs) {
#pragma unroll
      for (int j = 0; j < W; j++) turn(x[j], x[W + j], m.plane[0] + j);
    }
  } else if constexpr (W > 1) {
    if (m.kind[0] == kInterleaved) {
#pragma unroll
      for (int j = 0; j < W / 2; j++) turn(x[2 * j], x[2 * j + 1], m.plane[0] + j);
    }
  } else {
#pragma unroll
    for (int k = 0; k < 4; k++)
      if (m.kind[k] >= kPairs) turn(x[2 * k], x[2 * k + 1], m.plane[k]);
  }
}

// Runs of rows_each rows of a part, every groups-th of them.  TYPE: of x (and dy) in all parts, or kAny: asked at each access (then one waits for the other).
enum { kFp32 = 0, kBf16 = 1, kAny = 2 };
template <int W, bool GRAD, bool INTER, int TYPE>
__global__ __launch_bounds__(kNormWg) void headnorm_kernel(HeadnormArgs a) {
  constexpr int E = Dims<W>::kElems;
  __shared__ float2 table[kNormTable];
  __shared__ float shares[GRAD ? kNormWg * E : 1];            // of dw: [element of a lane][thread]
  const int n = (int)blockIdx.x >= a.first[2] ? 2 : (int)blockIdx.x >= a.first[1] ? 1 : 0, wg = blockIdx.x - a.first[n];
  const HeadnormPart p = a.part[n];
  const int group = a.group, slots = kNormWg / group, lane = threadIdx.x & (group - 1), slot = threadIdx.x / group;
  const int half = a.rot / 2, heads = p.p.heads, hd = a.hd;
  const Dims<W> m = dims_of<W>(lane, a.items, group, a.rot, a.interleaved != 0);
  const bool normed = p.w != nullptr;
  const int y_type = TYPE == kAny ? p.p.dtype : TYPE, x_type = TYPE == kAny ? p.x_dtype : TYPE;
  float w[E], dw[E];                                          // 2 W of them, or four pairs
#pragma unroll
  for (int j = 0; j < E; j++) w[j] = dw[j] = 0.f;
  if (normed) {
    if (W > 1 && ((uintptr_t)p.w & 15) != 0) {                // (aligned to its type only)
#pragma unroll
      for (int j = 0; j < (W > 1 ? W : 0); j++) {
        if (m.kind[0] != kIdle) w[j] = load1(p.w, m.first[0] + j, p.w_dtype);
        if (m.kind[0] == kPairs) w[W + j] = load1(p.w, m.first[0] + half + j, p.w_dtype);
      }
    } else {
      widen_dims<W>(load_dims<W>(p.w, 0, p.w_dtype, m, half), W > 1 ? p.w_dtype : 0, w);
    }
#pragma unroll
    for (int j = 0; j < E; j++) w[j] += p.offset;             // (of absent dims: meets zeros)
  }
  const float each = 1.0f / (float)hd;
  const int rows_each = a.rows_each[n], groups = a.first[n + 1] - a.first[n];
  for (int64_t row0 = (int64_t)wg * rows_each; row0 < a.rows; row0 += (int64_t)groups * rows_each) {
    const int rows = (int)min((int64_t)rows_each, a.rows - row0), total = rows * heads;
    struct Place { int row; int64_t y, x, o; };
    auto place_of = [&](int i) {
      Place q;
      q.row = i / heads;
      const int h = i - q.row * heads;
      const int64_t r = row0 + q.row;
      q.y = r * p.p.ldx + h * p.p.hsx;
      q.o = r * p.p.ldo + h * p.p.hso;
      q.x = GRAD ? r * p.ld + h * p.hs : 0;
      return q;
    };
    Place next{0, 0, 0, 0};
    const u32x4_t zero = {0u, 0u, 0u, 0u};
    Raw ny{zero, zero, zero, zero}, nx{zero, zero, zero, zero};
    auto ask = [&](int i) {
      if (i >= total) return;                                 // (the last values again, never used)
      next = place_of(i);
      ny = load_dims<W>(p.p.x, next.y, y_type, m, half);
      if (GRAD && normed) nx = load_dims<W>(p.x, next.x, x_type, m, half);
    };
    ask(slot);
    __syncthreads();                                          // nobody reads the last rows' table any more
    if (p.p.turn)
      for (int j = threadIdx.x; j < rows * half; j += kNormWg) {
        const int r = j / half, plane = j - r * half;
        const double pos = a.pos ? (double)a.pos[row0 + r] : (double)(a.pos0 + row0 + r);
        table[j] = turn_of(pos * a.turns[plane], a.mscale);
      }
    __syncthreads();
    for (int i0 = 0; i0 < total; i0 += slots) {
      const int i = i0 + slot;
      const bool mine = i < total;
      const Place now = next;
      float y[E], x[E];
      widen_dims<W>(ny, y_type, y);
      if (GRAD && normed) widen_dims<W>(nx, x_type, x);
      ask(i + slots);
      const float2 *cs = table + (mine ? now.row : 0) * half;
      if constexpr (!GRAD) {
        if (normed) {
          float q = 0.f;
#pragma unroll
          for (int j = 0; j < E; j++) q = fmaf(y[j], y[j], q);
          const float r = 1.0f / sqrtf(fmaf(group_sum(q, group), each, a.eps));
#pragma unroll
          for (int j = 0; j < E; j++) y[j] = y[j] * r * w[j];
        }
        if (p.p.turn) turn_dims<W, INTER>(y, m, cs, 1.f);
      } else {
        if (p.p.turn) turn_dims<W, INTER>(y, m, cs, -1.f);
        if (normed) {
          float q = 0.f, s = 0.f;
#pragma unroll
          for (int j = 0; j < E; j++) { q = fmaf(x[j], x[j], q); s = fmaf(y[j] * w[j], x[j], s); }
          const float r = 1.0f / sqrtf(fmaf(group_sum(q, group), each, a.eps));
          const float along = group_sum(s, group) * each * r * r;
#pragma unroll
          for (int j = 0; j < E; j++) {
            if (mine) dw[j] = fmaf(y[j], x[j] * r, dw[j]);
            y[j] = r * fmaf(-x[j], along, y[j] * w[j]);
          }
        }
      }
      if (mine) store_dims<W>(p.p.out, now.o, p.p.out_dtype, m, half, y);
    }
  }
  if constexpr (GRAD) {
    if (p.dw == nullptr) return;
    // thread i adds up the slots' shares of element i % E of lane i / E, if that lane has it, and so on in steps of the threads
#pragma unroll
    for (int j = 0; j < E; j++) shares[j * kNormWg + threadIdx.x] = dw[j];
    __syncthreads();
    float *out = a.scratch + ((int64_t)n * kGradGroups + wg) * hd;
    for (int i = threadIdx.x; i < group * E; i += kNormWg) {
      const int l = i / E, j = i - l * E;
      const Dims<W> d = dims_of<W>(l, a.items, group, a.rot, a.interleaved != 0);
      int dim = -1;
      if constexpr (W > 1) {
        if (j < W ? d.kind[0] != kIdle : d.kind[0] == kPairs) dim = d.first[0] + (j < W ? j : half + j - W);
      } else {
#pragma unroll
        for (int k = 0; k < 4; k++)
          if (j >> 1 == k) {
            if (!(j & 1) && d.kind[k] != kIdle) dim = d.first[k];
            if ((j & 1) && d.kind[k] >= kPairs) dim = d.first[k] + (d.kind[k] == kPairs ? half : 1);
          }
      }
      if (dim < 0) continue;
      float sum = 0.f;
      for (int s = 0; s < slots; s++) sum += shares[j * kNormWg + s * group + l];
      out[dim] = sum;
    }
  }
}

// The workgroups' shares of dw: a thread adds up every kSlices-th in their order, then kSlices threads meet.
constexpr int kSlices = 32;
__global__ __launch_bounds__(32 * kSlices) void headnorm_dw_kernel(HeadnormArgs a) {
  __shared__ float sh[32 * kSlices];
  const HeadnormPart p = a.part[blockIdx.y];
  if (p.dw == nullptr) return;
  const int dim = blockIdx.x * 32 + (threadIdx.x & 31), slice = threadIdx.x >> 5;
  const float *share = a.scratch + (int64_t)blockIdx.y * kGradGroups * a.hd;
  const int groups = a.first[blockIdx.y + 1] - a.first[blockIdx.y];
  float s = 0.f;
  if (dim < a.hd) {
#pragma unroll 8
    for (int g = slice; g < groups; g += kSlices) s += share[(int64_t)g * a.hd + dim];
  }
  sh[threadIdx.x] = s;
  __syncthreads();
  if (slice != 0 || dim >= a.hd) return;
#pragma unroll
  for (int i = 1; i < kSlices; i++) s += sh[i * 32 + threadIdx.x];
  p.dw[dim] = s;
}

// Every access of `w` dims is a multiple of its size from one
bool whole(const void *p, int64_t ld, int64_t hs, int bf16, int w) {
  const int64_t bytes = bf16 ? 2 * w : 16, e = bytes / (bf16 ? 2 : 4);
  return ((uintptr_t)p & (bytes - 1)) == 0 && ld % e == 0 && hs % e == 0;
}
template <int W, bool GRAD, bool INTER> auto of_type(int type) {
  return type == kFp32 ? headnorm_kernel<W, GRAD, INTER, kFp32> : type == kBf16 ? headnorm_kernel<W, GRAD, INTER, kBf16> : headnorm_kernel<W, GRAD, INTER, kAny>;
}
template <int W> auto of_layout(bool grad, bool inter, int type) {
  return inter ? (grad ? of_type<W, true, true>(type) : of_type<W, false, true>(type)) : grad ? of_type<W, true, false>(type) : of_type<W, false, false>(type);
}

hipError_t launch(HeadnormArgs a, bool grad, hipStream_t st) {
  int w = 8, heads = 0;
  for (; w >= 4; w /= 2) {
    bool fits = a.hd % w == 0 && a.rot % (a.interleaved ? w : 2 * w) == 0;
    for (int n = 0; n < a.n_parts && fits; n++) {
      const HeadnormPart &p = a.part[n];
      fits = whole(p.p.x, p.p.ldx, p.p.hsx, p.p.dtype, w) && whole(p.p.out, p.p.ldo, p.p.hso, p.p.out_dtype, w) && (!grad || !p.w || whole(p.x, p.ld, p.hs, p.x_dtype, w));
    }
    if (fits) break;
  }
  if (w < 4) w = 1;
  for (int n = 0; n < a.n_parts; n++) heads += a.part[n].p.heads;
  const int half = a.rot / 2;
  a.items = a.interleaved && w > 1 ? a.hd / w : half / w + (a.hd - a.rot) / w;
  a.group = 1;
  while (a.group < (w > 1 ? a.items : 64)) a.group *= 2;
  const int slots = kNormWg / a.group, all = grad ? kGradGroups : kForwardGroups, most_rows = half > 0 ? kNormTable / half : 1024;
  a.first[0] = 0;
  for (int n = 0; n < 3; n++) {
    if (n >= a.n_parts) { a.first[n + 1] = 0x7FFFFFFF; a.rows_each[n] = 1; continue; }
    int64_t groups = (int64_t)all * a.part[n].p.heads / heads;
    groups = groups < 1 ? 1 : groups;
    int64_t each = (a.rows + groups - 1) / groups;
    const int64_t fill = slots / a.part[n].p.heads < a.rows / 512 ? slots / a.part[n].p.heads : a.rows / 512;   // (a lane group each, where there are rows for it)
    each = each < fill ? fill : each;
    each = each < 1 ? 1 : each > most_rows ? most_rows : each;
    const int64_t runs = (a.rows + each - 1) / each;
    a.rows_each[n] = (int)each;
    a.first[n + 1] = a.first[n] + (int)(runs < groups ? runs : groups);
  }
  const dim3 grid((unsigned)a.first[a.n_parts]);
  int type = a.part[0].p.dtype;
  for (int n = 0; n < a.n_parts; n++)
    if (a.part[n].p.dtype != type || (grad && a.part[n].w && a.part[n].x_dtype != type)) type = kAny;
  const auto kernel = w == 8 ? of_layout<8>(grad, a.interleaved, type) : w == 4 ? of_layout<4>(grad, a.interleaved, type)
                      : grad ? headnorm_kernel<1, true, false, kAny> : headnorm_kernel<1, false, false, kAny>;
  hipLaunchKernelGGL(kernel, grid, dim3(kNormWg), 0, st, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !grad) return e;
  bool any = false;
  for (int n = 0; n < a.n_parts; n++) any = any || a.part[n].dw != nullptr;
  if (!any) return hipSuccess;
  hipLaunchKernelGGL(headnorm_dw_kernel, dim3((a.hd + 31) / 32, a.n_parts), dim3(32 * kSlices), 0, st, a);
  return hipGetLastError();
}

}  // namespace

int headnorm_grad_groups() { return kGradGroups; }
hipError_t launch_headnorm(HeadnormArgs a, hipStream_t st) { return launch(a, false, st); }
hipError_t launch_headnorm_grad(HeadnormArgs a, hipStream_t st) { return launch(a, true, st); }

}  // namespace spec
