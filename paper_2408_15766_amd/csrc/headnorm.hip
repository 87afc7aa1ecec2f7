// Norms of heads with the rotary embedding in the same pass, and their gradients (include/spec_step.h).
//
// A head is held by a group of lanes (2^n, at most 32, or a wavefront where dims are taken one at a time), each with the same dims of every head it meets: eight planes (16 dims), or eight dims
// that do not turn.  So a weight is read once, the sums over a head are a few exchanges between neighbouring lanes, and a lane adds up its dims' share of the
// weights' gradient in registers over all its heads; the workgroup's shares meet in the LDS once, in a fixed order, the workgroups' in a second
// launch.  The rows' (cos, sin) table is made in the LDS as for the rotary embedding alone.
// Bound: memory (forward: each element once in, once out; gradients: dy and x once in, dx once out).
#include "common.h"
#include "elements.h"
#include "kernels.h"

namespace spec {

namespace {

constexpr int kNormWg = 256, kNormTable = 1024;               // threads, and table entries of a workgroup
// Workgroups of a launch, shared out among the parts by their heads: as many as run at once (gradients three to a compute unit, else four), so that every one has about the
// same number of rows and their table is made once.
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

// The dims of a lane.  VEC: x[0 .. 7] are eight consecutive dims, x[8 .. 15] their planes' partners (half layout) or nothing.  Else up to four items a lane, item k: x[2 k] and,
// if it is a plane, x[2 k + 1].
enum { kIdle = 0, kPass = 1, kPairs = 2, kInterleaved = 3 };
template <bool VEC> struct Dims { static constexpr int kItems = VEC ? 1 : 4, kElems = VEC ? 16 : 8; int kind[kItems], first[kItems], plane[kItems]; };
template <bool VEC> __device__ __forceinline__ Dims<VEC> dims_of(int lane, int items, int group, int rot, bool interleaved) {
  Dims<VEC> r;
  constexpr int W = VEC ? 8 : 1;
  const int half = rot / 2, turning = VEC && interleaved ? half / 4 : half / W;
#pragma unroll
  for (int k = 0; k < Dims<VEC>::kItems; k++) {
    const int it = lane + k * group;
    r.kind[k] = it >= items ? kIdle : it >= turning ? kPass : interleaved ? kInterleaved : kPairs;
    r.plane[k] = VEC && interleaved ? 4 * it : W * it;
    r.first[k] = r.kind[k] == kPass ? rot + W * (it - turning) : interleaved ? 2 * r.plane[k] : r.plane[k];
  }
  return r;
}
// As they are in memory, then as numbers
struct Raw { u32x4_t a, b, c, d; };                           // VEC: a and b (bf16: a), and the partners' c and d
template <bool VEC> __device__ __forceinline__ Raw load_dims(const void *p, int64_t at, int bf16, const Dims<VEC> &m, int half) {
  const u32x4_t zero = {0u, 0u, 0u, 0u};
  Raw r{zero, zero, zero, zero};
  if constexpr (VEC) {
    if (m.kind[0] != kIdle) { const Eight e = load8(p, at + m.first[0], bf16); r.a = e.v[0]; if (!bf16) r.b = e.v[1]; }
    if (m.kind[0] == kPairs) { const Eight e = load8(p, at + m.first[0] + half, bf16); r.c = e.v[0]; if (!bf16) r.d = e.v[1]; }
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
template <bool VEC> __device__ __forceinline__ void widen_dims(const Raw &r, int bf16, const Dims<VEC> &m, float (&x)[Dims<VEC>::kElems]) {
  if constexpr (VEC) {
    float a[8], b[8];
    widen8(Eight{{r.a, r.b}}, bf16, a);
    widen8(Eight{{r.c, r.d}}, bf16, b);
#pragma unroll
    for (int j = 0; j < 8; j++) { x[j] = a[j]; x[8 + j] = b[j]; }
  } else {
#pragma unroll
    for (int j = 0; j < 4; j++) { x[j] = __uint_as_float(r.a[j]); x[4 + j] = __uint_as_float(r.b[j]); }
  }
}
template <bool VEC> __device__ __forceinline__ void store_dims(void *p, int64_t at, int bf16, const Dims<VEC> &m, int half, const float (&x)[Dims<VEC>::kElems]) {
  if constexpr (VEC) {
    float a[8], b[8];
#pragma unroll
    for (int j = 0; j < 8; j++) { a[j] = x[j]; b[j] = x[8 + j]; }
    if (m.kind[0] != kIdle) store8(p, at + m.first[0], bf16, a);
    if (m.kind[0] == kPairs) store8(p, at + m.first[0] + half, bf16, b);
  } else {
#pragma unroll
    for (int k = 0; k < 4; k++) {
      if (m.kind[k] != kIdle) store1(p, at + m.first[k], bf16, x[2 * k]);
      if (m.kind[k] >= kPairs) store1(p, at + m.first[k] + (m.kind[k] == kPairs ? half : 1), bf16, x[2 * k + 1]);
    }
  }
}
// Turned by the row's table (back: by the opposite angles).  INTER is for eight dims at a time (two patterns behind one branch went to memory)
template <bool VEC, bool INTER> __device__ __forceinline__ void turn_dims(float (&x)[Dims<VEC>::kElems], const Dims<VEC> &m, const float2 *cs, float back) {
  if constexpr (VEC && !INTER) {
    if (m.kind[0] == kPairs) {
#pragma unroll
      for (int j = 0; j < 8; j++) {
        const float2 c = make_float2(cs[m.plane[0] + j].x, back * cs[m.plane[0] + j].y);
        const float u = rope_first(x[j], x[8 + j], c), v = rope_second(x[j], x[8 + j], c);
        x[j] = u; x[8 + j] = v;
      }
    }
  } else if constexpr (VEC) {
    if (m.kind[0] == kInterleaved) {
#pragma unroll
      for (int j = 0; j < 4; j++) {
        const float2 c = make_float2(cs[m.plane[0] + j].x, back * cs[m.plane[0] + j].y);
        const float u = rope_first(x[2 * j], x[2 * j + 1], c), v = rope_second(x[2 * j], x[2 * j + 1], c);
        x[2 * j] = u; x[2 * j + 1] = v;
      }
    }
  } else {
#pragma unroll
    for (int k = 0; k < 4; k++)
      if (m.kind[k] >= kPairs) {
        const float2 c = make_float2(cs[m.plane[k]].x, back * cs[m.plane[k]].y);
        const float u = rope_first(x[2 * k], x[2 * k + 1], c), v = rope_second(x[2 * k], x[2 * k + 1], c);
        x[2 * k] = u; x[2 * k + 1] = v;
      }
  }
}

// Runs of rows_each rows of a part, every groups-th of them.  TYPE: of x (and dy) in all parts, or kAny: asked at each access (then one waits for the other).
enum { kFp32 = 0, kBf16 = 1, kAny = 2 };
template <bool VEC, bool GRAD, bool INTER, int TYPE>
__global__ __launch_bounds__(kNormWg) void headnorm_kernel(HeadnormArgs a) {
  constexpr int E = Dims<VEC>::kElems;
  __shared__ float2 table[kNormTable];
  __shared__ float shares[GRAD ? kNormWg * E : 1];            // of dw: [element of a lane][thread]
  const int n = (int)blockIdx.x >= a.first[2] ? 2 : (int)blockIdx.x >= a.first[1] ? 1 : 0, wg = blockIdx.x - a.first[n];
  const HeadnormPart p = a.part[n];
  const int group = a.group, slots = kNormWg / group, lane = threadIdx.x & (group - 1), slot = threadIdx.x / group;
  const int half = a.rot / 2, heads = p.p.heads, hd = a.hd;
  const Dims<VEC> m = dims_of<VEC>(lane, a.items, group, a.rot, a.interleaved != 0);
  const bool normed = p.w != nullptr;
  const int y_type = TYPE == kAny ? p.p.dtype : TYPE, x_type = TYPE == kAny ? p.x_dtype : TYPE;
  float w[E], dw[E];
#pragma unroll
  for (int j = 0; j < E; j++) w[j] = dw[j] = 0.f;
  if (normed) {
    if (VEC && ((uintptr_t)p.w & 15) != 0) {                  // (aligned to its type only)
#pragma unroll
      for (int j = 0; j < 8; j++) {
        if (m.kind[0] != kIdle) w[j] = load1(p.w, m.first[0] + j, p.w_dtype);
        if (VEC && m.kind[0] == kPairs) w[E - 8 + j] = load1(p.w, m.first[0] + half + j, p.w_dtype);
      }
    } else {
      widen_dims<VEC>(load_dims<VEC>(p.w, 0, p.w_dtype, m, half), p.w_dtype, m, w);
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
      ny = load_dims<VEC>(p.p.x, next.y, y_type, m, half);
      if (GRAD && normed) nx = load_dims<VEC>(p.x, next.x, x_type, m, half);
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
      widen_dims<VEC>(ny, y_type, m, y);
      if (GRAD && normed) widen_dims<VEC>(nx, x_type, m, x);
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
        if (p.p.turn) turn_dims<VEC, INTER>(y, m, cs, 1.f);
      } else {
        if (p.p.turn) turn_dims<VEC, INTER>(y, m, cs, -1.f);
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
      if (mine) store_dims<VEC>(p.p.out, now.o, p.p.out_dtype, m, half, y);
    }
  }
  if constexpr (GRAD) {
    if (p.dw == nullptr) return;
    // thread t of the first `group` ones that has dims adds up the slots' shares of its elements
#pragma unroll
    for (int j = 0; j < E; j++) shares[j * kNormWg + threadIdx.x] = dw[j];
    __syncthreads();
    float *out = a.scratch + ((int64_t)n * kGradGroups + wg) * hd;
    for (int i = threadIdx.x; i < group * E; i += kNormWg) {
      const int l = i / E, j = i - l * E;
      const Dims<VEC> d = dims_of<VEC>(l, a.items, group, a.rot, a.interleaved != 0);
      int dim = -1;
      if constexpr (VEC) {
        if (j < 8 ? d.kind[0] != kIdle : d.kind[0] == kPairs) dim = d.first[0] + (j < 8 ? j : half + j - 8);
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

// The workgroups' shares of dw, in their order: a thread adds up every eighth, then eight threads meet.
__global__ __launch_bounds__(256) void headnorm_dw_kernel(HeadnormArgs a) {
  __shared__ float sh[256];
  const HeadnormPart p = a.part[blockIdx.y];
  if (p.dw == nullptr) return;
  const int dim = blockIdx.x * 32 + (threadIdx.x & 31), slice = threadIdx.x >> 5;
  const float *share = a.scratch + (int64_t)blockIdx.y * kGradGroups * a.hd;
  const int groups = a.first[blockIdx.y + 1] - a.first[blockIdx.y];
  float s = 0.f;
  if (dim < a.hd) {
#pragma unroll 8
    for (int g = slice; g < groups; g += 8) s += share[(int64_t)g * a.hd + dim];
  }
  sh[threadIdx.x] = s;
  __syncthreads();
  if (slice != 0 || dim >= a.hd) return;
#pragma unroll
  for (int i = 1; i < 8; i++) s += sh[i * 32 + threadIdx.x];
  p.dw[dim] = s;
}

bool eights(const void *p, int64_t ld, int64_t hs, int bf16) { const int64_t e = bf16 ? 8 : 4; return ((uintptr_t)p & 15) == 0 && ld % e == 0 && hs % e == 0; }

template <bool GRAD, bool INTER> auto of_type(int type) {
  return type == kFp32 ? headnorm_kernel<true, GRAD, INTER, kFp32> : type == kBf16 ? headnorm_kernel<true, GRAD, INTER, kBf16> : headnorm_kernel<true, GRAD, INTER, kAny>;
}

hipError_t launch(HeadnormArgs a, bool grad, hipStream_t st) {
  // eight dims at a time where every access is a multiple of 16 bytes from a multiple of 16 bytes
  bool vec = a.hd % 8 == 0 && a.rot % (a.interleaved ? 8 : 16) == 0;
  int heads = 0;
  for (int n = 0; n < a.n_parts; n++) {
    const HeadnormPart &p = a.part[n];
    vec = vec && eights(p.p.x, p.p.ldx, p.p.hsx, p.p.dtype) && eights(p.p.out, p.p.ldo, p.p.hso, p.p.out_dtype);
    if (grad && p.w) vec = vec && eights(p.x, p.ld, p.hs, p.x_dtype);
    heads += p.p.heads;
  }
  const int half = a.rot / 2;
  a.items = vec ? (a.interleaved ? a.hd / 8 : half / 8 + (a.hd - a.rot) / 8) : half + a.hd - a.rot;
  a.group = 1;
  while (a.group < (vec ? a.items : 64)) a.group *= 2;
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
  const auto kernel = !vec ? (grad ? headnorm_kernel<false, true, false, kAny> : headnorm_kernel<false, false, false, kAny>)
                      : a.interleaved ? (grad ? of_type<true, true>(type) : of_type<false, true>(type)) : (grad ? of_type<true, false>(type) : of_type<false, false>(type));
  hipLaunchKernelGGL(kernel, grid, dim3(kNormWg), 0, st, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !grad) return e;
  bool any = false;
  for (int n = 0; n < a.n_parts; n++) any = any || a.part[n].dw != nullptr;
  if (!any) return hipSuccess;
  hipLaunchKernelGGL(headnorm_dw_kernel, dim3((a.hd + 31) / 32, a.n_parts), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace

int headnorm_grad_groups() { return kGradGroups; }
hipError_t launch_headnorm(HeadnormArgs a, hipStream_t st) { return launch(a, false, st); }
hipError_t launch_headnorm_grad(HeadnormArgs a, hipStream_t st) { return launch(a, true, st); }

}  // namespace spec
