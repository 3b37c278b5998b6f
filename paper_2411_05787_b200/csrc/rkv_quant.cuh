// The 8-bit cache format: e4m3 codes and one fp32 scale per block of 64 positions and KV head (K and V apart).
// value = code * scale.  The library writes scales that are powers of two, so that a product with a scale (or with a
// ratio of two) is exact in fp32 and a block can be encoded again under a larger scale without a second rounding of
// its normal codes; its readers take any finite scale.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "rkv_internal.h"

namespace rkv {

// Two codes -> two halves (exact: e4m3 has 3 mantissa bits and exponents -9 .. 8; NaN stays NaN).
__device__ __forceinline__ uint32_t e4m3x2_to_f16x2(uint16_t codes) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(codes));
  return h;
}
// Four codes -> two pairs of halves.
__device__ __forceinline__ void e4m3x4_to_f16x4(uint32_t codes, uint32_t& lo, uint32_t& hi) {
  asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\tcvt.rn.f16x2.e4m3x2 %1, h;\n\t}"
      : "=r"(lo), "=r"(hi)
      : "r"(codes));
}
__device__ __forceinline__ uint32_t codes_lo_f16x2(uint32_t w) { return e4m3x2_to_f16x2((uint16_t)(w & 0xffffu)); }
__device__ __forceinline__ uint32_t codes_hi_f16x2(uint32_t w) { return e4m3x2_to_f16x2((uint16_t)(w >> 16)); }
__device__ __forceinline__ float2 f16x2_to_float2(uint32_t h) { return __half22float2(*reinterpret_cast<__half2*>(&h)); }
// Two floats -> two codes, round to nearest even, magnitudes above 448 to 448, NaN to NaN.
__device__ __forceinline__ uint32_t encode2(float lo, float hi) {
  uint16_t c;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(c) : "f"(hi), "f"(lo));
  return c;
}

// Binary exponent of the smallest power of two s >= 2^-126 with magnitude <= 448 s, for a finite bf16 magnitude given
// by its bits (sign cleared): 448 = 1.75 * 2^8, so a = m 2^x needs 2^(x - 8) when m <= 1.75 and one more otherwise.
__device__ __forceinline__ int scale_exponent(uint32_t bits) {
  int e = (int)(bits >> 7) - 127 - 8 + ((bits & 0x7fu) > 0x60u ? 1 : 0);   // (a subnormal's x is too large here, but below the floor)
  return e < -126 ? -126 : e;
}
__device__ __forceinline__ float pow2f(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }   // -126 <= e <= 127

// Where a sequence's rows lie must suit the blocks: multiples of 64, inside the buffer.
__device__ __forceinline__ bool quant_layout_ok(int64_t roff, int cap, int n_kv_heads, int64_t n_rows) {
  return (((int)roff | cap) & (kQuantBlock - 1)) == 0 && roff >= 0 && cap >= 0 && roff + (int64_t)n_kv_heads * cap <= n_rows;
}

}  // namespace rkv
