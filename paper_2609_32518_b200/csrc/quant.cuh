// 8-bit cache: e4m3 codes, a power of two (e8m0 byte) for every 32 neighbouring dims.  Device code shared by
// the append, the read and the attention.  A power of two, and not a float: codes times it are exact in bf16 (4 significant
// bits of 8), so that whoever decodes, into registers, a tile or memory, gets the same operand and rounds nothing.
#pragma once

#include <cuda_bf16.h>
#include <stdint.h>

#include "ptx.cuh"

namespace unstep {
namespace q8 {

constexpr int kBlock = 32;                       // dims that share a scale
constexpr uint32_t kNanByte = 255;
constexpr uint32_t kTooLarge = 0x7F780000u;      // 1.9375 * 2^127: from here on the code would read as 2^128
constexpr uint32_t kLeastByte = 3;               // 2^-124: its smallest code, 2^-9, is the smallest bf16

// Scale byte of a block by the bits of its largest magnitude: the least power of two with m <= 448 * 2^e, and 448 is 1.75 * 2^8, so
// that a mantissa above 0.75 (0x600000) needs one more than the exponent less 8.  The bits of a NaN and of an infinity
// are the largest of all.
__device__ __forceinline__ uint32_t scale_byte(uint32_t top_bits) {
  if (top_bits >= kTooLarge) return kNanByte;
  const int e = static_cast<int>((top_bits + 0x1FFFFFu) >> 23) - 8;
  return static_cast<uint32_t>(max(e, static_cast<int>(kLeastByte)));
}

__device__ __forceinline__ uint32_t cvt_e4m3x2(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}

// Larger of magnitudes, a NaN if one of them is: its bits are then above kTooLarge.
__device__ __forceinline__ float max_abs(float a, float b) {
  float d;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(fabsf(a)), "f"(fabsf(b)));
  return d;
}
__device__ __forceinline__ float max_abs(float a, float b, float c) {
  float d;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(fabsf(a)), "f"(fabsf(b)), "f"(fabsf(c)));
  return d;
}

// Quantises 8 values of a thread; the four threads of a block of 32 are neighbouring lanes that all come here.
__device__ __forceinline__ uint2 quantise8(const float* y, uint32_t* byte) {
  float top = max_abs(max_abs(max_abs(y[0], y[1], y[2]), y[3], y[4]), max_abs(y[5], y[6], y[7]));
  top = max_abs(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
  top = max_abs(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
  const uint32_t e = scale_byte(__float_as_uint(top));
  *byte = e;
  if (e == kNanByte) return make_uint2(0u, 0u);
  const float inverse = __uint_as_float((254u - e) << 23);   // 2^(127 - e), a product with it is exact
  const uint64_t inverse2 = ptx::pack_f32x2(inverse, inverse);
  uint32_t c[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float lo, hi;
    ptx::unpack_f32x2(ptx::mul_f32x2(ptx::pack_f32x2(y[2 * i], y[2 * i + 1]), inverse2), lo, hi);
    c[i] = cvt_e4m3x2(lo, hi);
  }
  return make_uint2(c[0] | c[1] << 16, c[2] | c[3] << 16);
}

// Four codes as two bf16 pairs of 2^-120 times their values: exponent and mantissa of e4m3, moved to the lowest exponent
// bits of bf16, subnormals included.  The upper bytes of the four bf16 (sign, three exponent bits) and the lower ones
// are made four at a time.
__device__ __forceinline__ uint2 spread4(uint32_t w) {
  const uint32_t upper = (w & 0x80808080u) | ((w >> 4) & 0x07070707u), lower = (w << 4) & 0xF0F0F0F0u;
  return make_uint2(__byte_perm(lower, upper, 0x5140), __byte_perm(lower, upper, 0x7362));
}
__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
  const __nv_bfloat162 r = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
  return *reinterpret_cast<const uint32_t*>(&r);
}

// What the spread codes of a block are multiplied by, 2^120 * 2^(E - 127): one bf16 factor up to E = 134, two beyond
// (a second one is 1 otherwise).  A block of E = 255 becomes NaN.
__device__ __forceinline__ bool one_factor(uint32_t byte) { return byte <= 134u; }
__device__ __forceinline__ uint32_t factor1(uint32_t byte) { return one_factor(byte) ? (byte + 120u) * 0x00800080u : 0x7B807B80u; }
__device__ __forceinline__ uint32_t factor2(uint32_t byte) {
  return one_factor(byte) ? 0x3F803F80u : (byte == kNanByte ? 0x7FC07FC0u : byte * 0x00800080u);
}

// 8 codes (two words) as 8 bf16.
__device__ __forceinline__ uint4 decode8(uint32_t w0, uint32_t w1, uint32_t f1) {
  const uint2 a = spread4(w0), b = spread4(w1);
  return make_uint4(mul_bf16x2(a.x, f1), mul_bf16x2(a.y, f1), mul_bf16x2(b.x, f1), mul_bf16x2(b.y, f1));
}
__device__ __forceinline__ uint4 mul8(uint4 x, uint32_t f) {
  return make_uint4(mul_bf16x2(x.x, f), mul_bf16x2(x.y, f), mul_bf16x2(x.z, f), mul_bf16x2(x.w, f));
}

}  // namespace q8
}  // namespace unstep
