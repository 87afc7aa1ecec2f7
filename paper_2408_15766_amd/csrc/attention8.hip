// Attention over a cache of 64-token blocks in 8 bits with a bf16 window behind it, and the cache's store and load (include/spec_layer8.h).
#include "common.h"
#include "fp8.h"
#include "kernels.h"

namespace spec {

namespace {

// Where a block's codes lie.  Scores are taken as S^T = K Q^T and outputs as O^T = V^T P^T with 32 x 32 x 16 products; a wavefront reads 1 KiB at a time, lane
// (c = lane % 32, g = lane / 32) 16 bytes, which are its operands of two products:
//   keys  : piece (32 keys, 32 dims): key c, dims 16 g + 0 .. 15,
//   values: piece (32 keys, 32 dims): dim c, keys 4 g + {0..3, 8..11, 16..19, 24..27}: the keys whose weights the lane holds after the scores.
template <int HD> __device__ __forceinline__ int key_at(int t, int d) {   // token t, dim d
  return (t >> 5) * 32 * HD + (d >> 5) * 1024 + (((d >> 4) & 1) * 32 + (t & 31)) * 16 + (d & 15);
}
template <int HD> __device__ __forceinline__ int value_at(int t, int d) {
  return (t >> 5) * 32 * HD + (d >> 5) * 1024 + (((t >> 2) & 1) * 32 + (d & 31)) * 16 + ((t >> 3) & 3) * 4 + (t & 3);
}

__device__ __forceinline__ float code_to_f32(unsigned char c) { return __builtin_amdgcn_cvt_f32_fp8((int)c, 0); }

// A workgroup puts one head's keys or values of a block into 8 bits.
template <int HD>
__global__ __launch_bounds__(256) void kv8_store_kernel(const bf16_t *k, const bf16_t *v, int64_t ld, int hkv, unsigned char *cache8, int first_block) {
  __shared__ __attribute__((aligned(16))) unsigned char codes[kKv8Block * HD];
  __shared__ float sh[16];
  const int h = blockIdx.x >> 1, values = blockIdx.x & 1, blk = blockIdx.y;
  const bf16_t *src = (values ? v : k) + (int64_t)blk * kKv8Block * ld + (int64_t)h * HD;
  constexpr int kEach = kKv8Block * HD / 256;                 // consecutive values of a thread
  const int t = threadIdx.x * kEach / HD, d0 = threadIdx.x * kEach % HD;
  float x[kEach], amax = 0.f;
#pragma unroll
  for (int i = 0; i < kEach; i++) {
    x[i] = to_f32(src[t * ld + d0 + i]);
    amax = fmaxf(amax, finite_abs(x[i]));
  }
  const int e = exponent8(block_max(amax, sh));
  const float down = pow2(-e);
#pragma unroll
  for (int i = 0; i < kEach; i += 4) {
    const uint32_t c = codes4(x[i] * down, x[i + 1] * down, x[i + 2] * down, x[i + 3] * down);
#pragma unroll
    for (int j = 0; j < 4; j++) codes[values ? value_at<HD>(t, d0 + i + j) : key_at<HD>(t, d0 + i + j)] = (unsigned char)(c >> (8 * j));
  }
  __syncthreads();
  unsigned char *block = cache8 + (size_t)(first_block + blk) * kv8_block_bytes(hkv, HD);
  u32x4_t *dst = (u32x4_t *)(block + (size_t)(2 * h + values) * kKv8Block * HD);
  for (int i = threadIdx.x; i < kKv8Block * HD / 16; i += 256) dst[i] = ((const u32x4_t *)codes)[i];
  if (threadIdx.x == 0) block[(size_t)hkv * 2 * kKv8Block * HD + 2 * h + values] = (unsigned char)(e + 127);
}

template <int HD>
__global__ __launch_bounds__(256) void kv8_load_kernel(const unsigned char *cache8, int first_block, int hkv, bf16_t *k, bf16_t *v, int64_t ld) {
  const int h = blockIdx.x >> 1, values = blockIdx.x & 1, blk = blockIdx.y;
  const unsigned char *block = cache8 + (size_t)(first_block + blk) * kv8_block_bytes(hkv, HD);
  const unsigned char *src = block + (size_t)(2 * h + values) * kKv8Block * HD;
  const float up = pow2((int)block[(size_t)hkv * 2 * kKv8Block * HD + 2 * h + values] - 127);
  bf16_t *dst = (values ? v : k) + (int64_t)blk * kKv8Block * ld + (int64_t)h * HD;
  for (int i = threadIdx.x; i < kKv8Block * HD; i += 256) {
    const int t = i / HD, d = i % HD;
    dst[t * ld + d] = from_f32<bf16_t>(code_to_f32(src[values ? value_at<HD>(t, d) : key_at<HD>(t, d)]) * up);
  }
}

// A workgroup owns one query of one row: 256 keys at a time, a thread's key each, one running maximum and sum; then a thread's dim over these keys.
template <int HD>
__global__ __launch_bounds__(256) void attention8_kernel(Attn8Args a) {
  __shared__ float q[HD], w[256], sh[16], o_sh[256];
  __shared__ int row_of[256];                                 // window row of a key, -1: in the blocks, -2: not seen
  const int i = blockIdx.x, h = blockIdx.y, kvh = h / (a.hq / a.hkv), tid = threadIdx.x;
  const int deep = min(a.depth[i], a.max_depth);
  if (deep < 0) return;
  const int n8 = a.n_blocks * kKv8Block, keys = a.base + deep + 1;
  for (int d = tid; d < HD; d += 256) q[d] = a.q[(size_t)i * a.hq * HD + h * HD + d];
  const size_t block_bytes = kv8_block_bytes(a.hkv, HD);
  const unsigned char *exps = a.cache8 + (size_t)a.hkv * 2 * kKv8Block * HD + 2 * kvh;
  float m = -INFINITY, l = 0.f, o = 0.f;
  constexpr int kShares = 256 / HD;                           // threads that share a dim
  const int d = tid % HD, share = tid / HD;
  for (int p0 = 0; p0 < keys; p0 += 256) {
    __syncthreads();
    const int p = p0 + tid;
    int row = -2;
    float s = -INFINITY;
    if (p < keys) {
      if (p < n8) row = -1;
      else {
        row = (p < a.base || !a.anc) ? p - n8 : a.base - n8 + a.anc[(size_t)i * kAncStride + p - a.base];
        if (row < 0 || row >= a.win_rows) row = -2;
      }
      if (row != -2) {
        s = 0.f;
        if (row == -1) {
          const unsigned char *block = a.cache8 + (size_t)(p / kKv8Block) * block_bytes;
          const unsigned char *kc = block + (size_t)(2 * kvh) * kKv8Block * HD;
          for (int e = 0; e < HD; e++) s = fmaf(q[e], code_to_f32(kc[key_at<HD>(p % kKv8Block, e)]), s);
          s *= pow2((int)exps[(size_t)(p / kKv8Block) * block_bytes] - 127);
        } else {
          const bf16_t *kr = (const bf16_t *)a.kwin + (size_t)row * a.hkv * HD + kvh * HD;
          for (int e = 0; e < HD; e++) s = fmaf(q[e], to_f32(kr[e]), s);
        }
        s *= a.scale;
      }
    }
    row_of[tid] = row;
    const float m_new = fmaxf(m, block_max(s, sh));           // (a NaN score: its weight is NaN below)
    const float m_use = m_new == -INFINITY ? 0.f : m_new, turn = exp2_((m == -INFINITY ? m_use : m) - m_use);
    const float weight = row == -2 ? 0.f : exp2_(s - m_use);
    w[tid] = weight;
    l = l * turn + block_sum(weight, sh);
    m = m_new;
    o *= turn;
    __syncthreads();
    for (int t = share; t < 256 && p0 + t < keys; t += kShares) {
      const int r = row_of[t], p2 = p0 + t;
      if (r == -2) continue;
      float v;
      if (r == -1) {
        const unsigned char *block = a.cache8 + (size_t)(p2 / kKv8Block) * block_bytes;
        v = code_to_f32(block[(size_t)(2 * kvh + 1) * kKv8Block * HD + value_at<HD>(p2 % kKv8Block, d)]) *
            pow2((int)exps[(size_t)(p2 / kKv8Block) * block_bytes + 1] - 127);
      } else v = to_f32(((const bf16_t *)a.vwin)[(size_t)r * a.hkv * HD + kvh * HD + d]);
      o = fmaf(w[t], v, o);
    }
  }
  o_sh[tid] = o;
  __syncthreads();
  if (tid >= HD) return;
  for (int t = 1; t < kShares; t++) o += o_sh[t * HD + tid];
  ((bf16_t *)a.out)[(size_t)i * a.hq * HD + h * HD + tid] = from_f32<bf16_t>(l == 0.f ? 0.f : o / l);
}

}  // namespace

hipError_t launch_kv8_store(const void *k, const void *v, int64_t ld, int n_blocks, int hkv, int hd, void *cache8, int first_block, hipStream_t st) {
  for (int b = 0; b < n_blocks; b += 65535) {                 // (the grid's second dimension)
    const int n = n_blocks - b < 65535 ? n_blocks - b : 65535;
    const bf16_t *ks = (const bf16_t *)k + (int64_t)b * kKv8Block * ld, *vs = (const bf16_t *)v + (int64_t)b * kKv8Block * ld;
    if (hd == 128) hipLaunchKernelGGL(kv8_store_kernel<128>, dim3(2 * hkv, n), dim3(256), 0, st, ks, vs, ld, hkv, (unsigned char *)cache8, first_block + b);
    else hipLaunchKernelGGL(kv8_store_kernel<64>, dim3(2 * hkv, n), dim3(256), 0, st, ks, vs, ld, hkv, (unsigned char *)cache8, first_block + b);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_kv8_load(const void *cache8, int first_block, int n_blocks, int hkv, int hd, void *k, void *v, int64_t ld, hipStream_t st) {
  for (int b = 0; b < n_blocks; b += 65535) {
    const int n = n_blocks - b < 65535 ? n_blocks - b : 65535;
    bf16_t *ks = (bf16_t *)k + (int64_t)b * kKv8Block * ld, *vs = (bf16_t *)v + (int64_t)b * kKv8Block * ld;
    if (hd == 128) hipLaunchKernelGGL(kv8_load_kernel<128>, dim3(2 * hkv, n), dim3(256), 0, st, (const unsigned char *)cache8, first_block + b, hkv, ks, vs, ld);
    else hipLaunchKernelGGL(kv8_load_kernel<64>, dim3(2 * hkv, n), dim3(256), 0, st, (const unsigned char *)cache8, first_block + b, hkv, ks, vs, ld);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

size_t attention8_scratch_floats(int rows, int hq, int hkv, int hd, int n_blocks, int win_rows) {
  (void)rows; (void)hq; (void)hkv; (void)hd; (void)n_blocks; (void)win_rows;
  return 64;
}

hipError_t launch_attention8(const Attn8Args &a, hipStream_t st) {
  const dim3 grid(a.rows, a.hq);
  if (a.hd == 128) hipLaunchKernelGGL(attention8_kernel<128>, grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL(attention8_kernel<64>, grid, dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace spec
