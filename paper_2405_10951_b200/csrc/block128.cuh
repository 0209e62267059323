// Sixteen consecutive values of a block, as they come from memory, to E4M3 codes with the block's power-of-two scale.
#pragma once

#include "common.cuh"

namespace bsr {

constexpr uint32_t F32_INF = 0x7f800000u;

template <typename T> struct Values16;
template <> struct Values16<float> {
  uint4 u[4];
  __device__ __forceinline__ void load(const float* p) {
#pragma unroll
    for (int j = 0; j < 4; ++j) u[j] = reinterpret_cast<const uint4*>(p)[j];
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int j = 0; j < 4; ++j) u[j] = make_uint4(0, 0, 0, 0);
  }
  __device__ __forceinline__ float get(int i) const {
    const uint4& q = u[i >> 2];
    return __uint_as_float((i & 3) == 0 ? q.x : (i & 3) == 1 ? q.y : (i & 3) == 2 ? q.z : q.w);
  }
  // Bits of the largest magnitude as a float (magnitudes are ordered as their bits are, infinities and NaN above all numbers).
  __device__ __forceinline__ uint32_t top() const {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) m = max(m, __float_as_uint(get(i)) & 0x7fffffffu);
    return m;
  }
};
template <> struct Values16<bf16> {
  uint4 u[2];
  __device__ __forceinline__ void load(const bf16* p) {
    u[0] = reinterpret_cast<const uint4*>(p)[0];
    u[1] = reinterpret_cast<const uint4*>(p)[1];
  }
  __device__ __forceinline__ void zero() { u[0] = u[1] = make_uint4(0, 0, 0, 0); }
  __device__ __forceinline__ uint32_t word(int j) const {
    const uint4& q = u[j >> 2];
    return (j & 3) == 0 ? q.x : (j & 3) == 1 ? q.y : (j & 3) == 2 ? q.z : q.w;
  }
  __device__ __forceinline__ float get(int i) const { return __uint_as_float(i & 1 ? word(i >> 1) & 0xffff0000u : word(i >> 1) << 16); }
  __device__ __forceinline__ uint32_t top() const {
    uint32_t m = 0;                              // two magnitudes a word
#pragma unroll
    for (int j = 0; j < 8; ++j) m = __vmaxu2(m, word(j) & 0x7fff7fffu);
    return max(m << 16, m & 0xffff0000u);
  }
};
// The same over the finite values alone.
template <typename T> __device__ __forceinline__ uint32_t finite_top(const Values16<T>& v) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const uint32_t a = __float_as_uint(v.get(i)) & 0x7fffffffu;
    m = max(m, a < F32_INF ? a : 0u);
  }
  return m;
}
// The scale's byte (exponent + 127): the least with max <= 448 * 2^e, 448 = 1.75 * 2^8; 127 for a block of zeros.
__device__ __forceinline__ uint32_t scale_byte(uint32_t top) {
  if (top == 0) return 127u;
  return (uint32_t)max(0, (int)(top >> 23) - 8 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0));
}
// finite: whether the block's values all are (an infinity would saturate: it becomes NaN like the others).
template <typename T> __device__ __forceinline__ uint4 codes16(const Values16<T>& v, uint32_t byte, bool finite) {
  const float inv = __uint_as_float((254u - byte) << 23);      // 2^-e; byte <= 247
  uint32_t w[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    float t[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      t[i] = v.get(4 * j + i) * inv;
      if (!finite && (__float_as_uint(v.get(4 * j + i)) & 0x7fffffffu) >= F32_INF) t[i] = __uint_as_float(0x7fffffffu);
    }
    uint16_t lo, hi;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(t[1]), "f"(t[0]));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(t[3]), "f"(t[2]));
    w[j] = (uint32_t)lo | (uint32_t)hi << 16;
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

}  // namespace bsr
