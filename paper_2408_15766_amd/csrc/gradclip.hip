// The norm of many gradients together, and the gradients brought down to a largest norm (include/spec_step.h).
//
// Two passes over the gradients with nothing between them: the first leaves kGradSums partial sums of squares, the second's workgroups each add these up (8 KB out of
// the L2) and scale.  A launch takes the addresses of up to kGradTensors tensors as arguments; they are cut into chunks of kGradChunk elements, counted from
// the 16-byte boundary at or before the tensor's first element, that the workgroups take in turn.  Squares are exact in 64 bits and added up there, so that
// the norm neither overflows nor depends on the number of elements.
// Bound: memory.  Measured: 236 M elements, sums 113 us in bf16 (4.2 TB/s, while the outputs of the pass before are still on their way
// out of the last-level cache; 73 where they are not), 172 in fp32 (5.5 TB/s); clipped from bf16 into fp32 273 us (5.2 TB/s), in bf16 155
// (6.1).  Half the loads in flight: sums 118, clipped 275.  Stores past the caches: clipped 328.
#include "common.h"
#include "elements.h"
#include "kernels.h"

namespace spec {

namespace {

constexpr int kGradThreads = 256, kGradUnroll = 8, kGradChunk = kGradThreads * kGradUnroll * 8;

struct Chunk { int tensor; int64_t first; };                  // first: the chunk's first element, from -7 on
__device__ __forceinline__ Chunk chunk_of(const GradArgs &a, int c) {
  int lo = 0, hi = a.n;                                       // the last tensor that begins at or before c
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (a.begin[mid] <= c) lo = mid; else hi = mid;
  }
  return Chunk{lo, (int64_t)(c - a.begin[lo]) * kGradChunk};
}

__device__ __forceinline__ double block_sum64(double x, double *sh) {   // four wavefronts; every thread gets the sum, in a fixed order
  for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = x;
  __syncthreads();
  return (sh[0] + sh[1]) + (sh[2] + sh[3]);
}

__global__ __launch_bounds__(kGradThreads) void grad_sums_kernel(GradArgs a) {
  __shared__ double sh[4];
  double sum[2] = {0.0, 0.0};
  for (int c = blockIdx.x; c < a.chunks; c += kGradSums) {
    const Chunk at = chunk_of(a, c);
    const GradTensor t = a.t[at.tensor];
    const int64_t n = t.count & kGradCount;
    const int bf16 = (t.count & kGradBf16) != 0;
    const int64_t first = at.first - (int64_t)(((uintptr_t)t.g & 15) >> (bf16 ? 1 : 2));
    Eight v[kGradUnroll];
    const bool whole = first >= 0 && first + kGradChunk <= n;
    if (whole) {
#pragma unroll
      for (int u = 0; u < kGradUnroll; u++) v[u] = load8(t.g, first + (int64_t)(u * kGradThreads + threadIdx.x) * 8, bf16);
#pragma unroll
      for (int u = 0; u < kGradUnroll; u++) {
        float x[8];
        widen8(v[u], bf16, x);
#pragma unroll
        for (int j = 0; j < 8; j++) sum[j & 1] = fma((double)x[j], (double)x[j], sum[j & 1]);
      }
    } else {
      for (int u = 0; u < kGradUnroll; u++) {
        const int64_t i = first + (int64_t)(u * kGradThreads + threadIdx.x) * 8;
        if (i >= n) break;
        float x[8];
        if (i >= 0 && i + 8 <= n) widen8(load8(t.g, i, bf16), bf16, x);
        else
          for (int j = 0; j < 8; j++) x[j] = i + j >= 0 && i + j < n ? load1(t.g, i + j, bf16) : 0.f;
#pragma unroll
        for (int j = 0; j < 8; j++) sum[j & 1] = fma((double)x[j], (double)x[j], sum[j & 1]);
      }
    }
  }
  const double all = block_sum64(sum[0] + sum[1], sh);
  if (threadIdx.x == 0) a.sums[blockIdx.x] = a.first ? all : a.sums[blockIdx.x] + all;
}

__global__ __launch_bounds__(kGradThreads) void grad_clip_kernel(GradArgs a) {
  __shared__ double sh[4];
  double part = 0.0;
#pragma unroll
  for (int i = 0; i < kGradSums / kGradThreads; i++) part += a.sums[i * kGradThreads + threadIdx.x];
  const double norm = sqrt(block_sum64(part, sh));
  if (a.norm != nullptr && blockIdx.x == 0 && threadIdx.x == 0) a.norm[0] = (float)norm;
  const double ratio = a.max_norm / (norm + 1e-6);
  // the factor as a number of [1/2, 1] times a power of two: below fp32's normal range it keeps its precision
  int down = 0;
  const float factor = ratio < 1.0 ? (float)frexp(ratio, &down) : ratio == ratio ? 1.f : (float)ratio;
  const bool none = factor == 1.f && down == 0;
  for (int b = blockIdx.x; b < a.chunks; b += gridDim.x) {
    const Chunk at = chunk_of(a, a.chunks - 1 - b);           // (last first: what the sums have read last is still in the last-level cache)
    const GradTensor t = a.t[at.tensor];
    if (t.out == t.g && none) continue;
    const int64_t n = t.count & kGradCount;
    const int bf16 = (t.count & kGradBf16) != 0, to_bf16 = (t.count & kGradToBf16) != 0;
    const int64_t first = at.first - (int64_t)(((uintptr_t)t.g & 15) >> (bf16 ? 1 : 2));
    const bool even = (((uintptr_t)t.out + (uintptr_t)first * (to_bf16 ? 2 : 4)) & 15) == 0;   // stores of 16 bytes are aligned
    if (even && first >= 0 && first + kGradChunk <= n) {
      Eight v[kGradUnroll];
#pragma unroll
      for (int u = 0; u < kGradUnroll; u++) v[u] = load8(t.g, first + (int64_t)(u * kGradThreads + threadIdx.x) * 8, bf16);
#pragma unroll
      for (int u = 0; u < kGradUnroll; u++) {
        float x[8];
        widen8(v[u], bf16, x);
#pragma unroll
        for (int j = 0; j < 8; j++) x[j] = ldexpf(x[j] * factor, down);
        store8(t.out, first + (int64_t)(u * kGradThreads + threadIdx.x) * 8, to_bf16, x);
      }
      continue;
    }
    for (int u = 0; u < kGradUnroll; u++) {
      const int64_t i = first + (int64_t)(u * kGradThreads + threadIdx.x) * 8;
      if (i >= n) break;
      float x[8];
      const bool eight = i >= 0 && i + 8 <= n;
      if (eight) widen8(load8(t.g, i, bf16), bf16, x);
      else
        for (int j = 0; j < 8; j++) x[j] = i + j >= 0 && i + j < n ? load1(t.g, i + j, bf16) : 0.f;
#pragma unroll
      for (int j = 0; j < 8; j++) x[j] = ldexpf(x[j] * factor, down);
      if (eight && even) store8(t.out, i, to_bf16, x);
      else
        for (int j = 0; j < 8; j++)
          if (i + j >= 0 && i + j < n) store1(t.out, i + j, to_bf16, x[j]);
    }
  }
}

}  // namespace

// Chunks of a tensor that starts at g, counted from the 16-byte boundary before it
int64_t grad_chunks(const void *g, int64_t n, int bf16) { return (n + (int64_t)(((uintptr_t)g & 15) >> (bf16 ? 1 : 2)) + kGradChunk - 1) / kGradChunk; }

hipError_t launch_grad_sums(const GradArgs &a, hipStream_t st) {
  hipLaunchKernelGGL(grad_sums_kernel, dim3(kGradSums), dim3(kGradThreads), 0, st, a);
  return hipGetLastError();
}
hipError_t launch_grad_clip(const GradArgs &a, hipStream_t st) {
  const int groups = a.chunks < 1 ? 1 : a.chunks < 2048 ? a.chunks : 2048;
  hipLaunchKernelGGL(grad_clip_kernel, dim3(groups), dim3(kGradThreads), 0, st, a);
  return hipGetLastError();
}

}  // namespace spec
