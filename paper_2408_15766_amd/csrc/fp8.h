// 8-bit values: e4m3 codes and a power of two per block (include/spec_layer8.h states the format).
#pragma once
#include "common.h"

namespace spec {

constexpr int kExp8Least = -100;                              // (2^e and 2^-e stay normal numbers, and so does every value in bf16)

// Largest finite magnitude among the arguments' bits: not finite counts as nothing
__device__ __forceinline__ float finite_abs(float x) {
  const uint32_t b = __float_as_uint(x) & 0x7FFFFFFFu;
  return b < 0x7F800000u ? __uint_as_float(b) : 0.f;
}
// The block's exponent from its largest magnitude: the least e with amax <= 448 * 2^e = 1.75 * 2^(e + 8)
__device__ __forceinline__ int exponent8(float amax) {
  const uint32_t b = __float_as_uint(amax);
  const int e = (int)(b >> 23) - 127 - 8 + ((b & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return max(e, kExp8Least);
}
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }   // -126 <= e <= 127
// Four values, already divided by the block's 2^e, to codes, rounded to nearest even (v_cvt_pk_fp8_f32; infinities become NaN)
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d) {
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  r = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
  return (uint32_t)r;
}
// Two codes (the lower or upper half of w) times 2^e to bf16, exactly; s = 2^e
template <bool HI> __device__ __forceinline__ uint32_t bf16_of_codes(uint32_t w, float s) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, HI));
}
template <bool HI> __device__ __forceinline__ uint32_t f16_of_codes(uint32_t w, float s) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, s, HI));
}

// Orders this wavefront's LDS accesses for the compiler (the hardware keeps their order)
__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}
// Sixteen consecutive values to fp32; the pointer is aligned to 16 bytes
__device__ __forceinline__ void load16(const float *p, float (&x)[16]) {
#pragma unroll
  for (int i = 0; i < 4; i++) {
    const f32x4_t v = *(const f32x4_t *)(p + 4 * i);
    x[4 * i] = v.x; x[4 * i + 1] = v.y; x[4 * i + 2] = v.z; x[4 * i + 3] = v.w;
  }
}
__device__ __forceinline__ void load16(const bf16_t *p, float (&x)[16]) {
#pragma unroll
  for (int i = 0; i < 2; i++) {
    const u32x4_t v = *(const u32x4_t *)(p + 8 * i);
#pragma unroll
    for (int j = 0; j < 4; j++) {
      x[8 * i + 2 * j] = __uint_as_float(v[j] << 16);
      x[8 * i + 2 * j + 1] = __uint_as_float(v[j] & 0xFFFF0000u);
    }
  }
}

// ---- packed matrices -------------------------------------------------------------
// A [rows, in] matrix in 8 bits is cut into tiles of 16 rows x 128 k, 2 KiB each, those of a 16-row block one behind the other along k.  The 16 k
// from 64 u + 16 q on of row r are the 16 bytes at u * 1024 + (q * 16 + r) * 16: lane 16 q + r of a wavefront reads the pieces u = 0, 1 and holds the operand of a
// 16 x 16 x 128 product, and each half u is the operand of a 32 x 32 x 64 product over two such tiles (a sum does not depend on
// which k a lane holds, as long as both operands agree).  Rows and k are padded with zeros to whole tiles.  Behind the tiles: the exponents + 127, one byte
// per row and tile, [row block][ceil(tiles / 4)][16 rows][4 tiles]: a dword has a row's next four.
constexpr int kTile8 = 2048;
struct Packed8 { int blocks, groups, quads; };                // 16-row blocks, 128-k tiles of a row, and their dwords of exponents
__host__ __device__ inline Packed8 packed8(int rows, int in) { return Packed8{(rows + 15) / 16, (in + 127) / 128, (in + 511) / 512}; }
__host__ __device__ inline uint64_t packed8_exps(const Packed8 &p) { return (uint64_t)p.blocks * p.groups * kTile8; }   // where the exponents begin
__host__ __device__ inline uint64_t packed8_bytes(const Packed8 &p) { return packed8_exps(p) + (uint64_t)p.blocks * p.quads * 64; }

}  // namespace spec
