// Sixteen consecutive values of a block to E4M3 codes with the block's power-of-two scale.
#pragma once

#include "common.cuh"

namespace bsr {

struct Codes16 { uint4 u; };

__device__ __forceinline__ void load_values16(const float* p, float* v) {
#pragma unroll
  for (int j = 0; j < 16; j += 4) load16(p + j, v + j);
}
__device__ __forceinline__ void load_values16(const bf16* p, float* v) {
  load16(p, v);
  load16(p + 8, v + 8);
}
// Bits of the largest magnitude among the finite values (magnitudes are ordered as their bits are).
__device__ __forceinline__ uint32_t finite_max16(const float* v) {
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < 16; ++j) {
    const uint32_t a = __float_as_uint(v[j]) & 0x7fffffffu;
    top = max(top, a < 0x7f800000u ? a : 0u);
  }
  return top;
}
// The scale's byte (exponent + 127): the least with max <= 448 * 2^e, 448 = 1.75 * 2^8; 127 for a block of zeros.
__device__ __forceinline__ uint32_t scale_byte(uint32_t top) {
  if (top == 0) return 127u;
  return (uint32_t)max(0, (int)(top >> 23) - 8 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0));
}
__device__ __forceinline__ Codes16 codes16(const float* v, uint32_t byte) {
  const float inv = __uint_as_float((254u - byte) << 23);      // 2^-e; byte <= 247
  Codes16 c;
  uint32_t* w = reinterpret_cast<uint32_t*>(&c.u);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    float t[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) t[i] = fmaf(v[4 * j + i], inv, v[4 * j + i] * 0.f);      // (infinities would saturate: NaN instead)
    uint16_t lo, hi;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(t[1]), "f"(t[0]));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(t[3]), "f"(t[2]));
    w[j] = (uint32_t)lo | (uint32_t)hi << 16;
  }
  return c;
}

}  // namespace bsr
