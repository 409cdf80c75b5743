// kv8.cuh -- caches held in 8 bits: e4m3 codes, and for each block of `block` consecutive rows of a page and head
// a scale 2^e in e8m0 (the byte e + 127). An element is code * 2^e.
//
// e is the smallest in [-32, 32] with top <= 448 * 2^e, top the block's largest magnitude, so no code saturates
// below 448 * 2^32 and the rounding to a code is off by at most 2^-4 of an element (2^-10 * 2^e below 2^-6 * 2^e).
// Powers of two make every rescaling but that rounding exact: a score takes the key block's scale as a factor, and
// a numerator the value block's as an addend of its exponent. The bound on e keeps the products of such factors
// inside fp32. A byte outside it counts as the nearer end.
#pragma once
#include <cuda_fp8.h>

#include "device_common.cuh"

namespace trident {

constexpr int kScaleLo = -32, kScaleHi = 32;

__device__ __forceinline__ int scale_exp(uint32_t byte) { return min(max((int)byte - 127, kScaleLo), kScaleHi); }
__device__ __forceinline__ float exp2_int(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }  // -126 .. 127

// The exponent for a largest magnitude (not NaN; infinite: 32). 448 = 1.75 * 2^8: a mantissa above 0.75 carries.
__device__ __forceinline__ int scale_for(float top) {
  const int e = (int)((__float_as_uint(top) + 0x1fffffu) >> 23) - 127 - 8;
  return min(max(e, kScaleLo), kScaleHi);
}

// Two values to codes (x in the low byte), rounded to nearest; +-448 beyond the range, NaN stays NaN.
__device__ __forceinline__ uint32_t codes2(float x, float y) {
  uint16_t w;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(w) : "f"(y), "f"(x));
  return w;
}
__device__ __forceinline__ uint32_t codes4(const float* v) { return codes2(v[0], v[1]) | codes2(v[2], v[3]) << 16; }

// Two codes as halves, exactly.
__device__ __forceinline__ uint32_t halves2(uint32_t codes) {
  uint32_t h;
  asm("{ .reg .b16 lo, hi; mov.b32 {lo, hi}, %1; cvt.rn.f16x2.e4m3x2 %0, lo; }" : "=r"(h) : "r"(codes));
  return h;
}
__device__ __forceinline__ uint32_t halves2_hi(uint32_t codes) {  // of the upper 16 bits
  uint32_t h;
  asm("{ .reg .b16 lo, hi; mov.b32 {lo, hi}, %1; cvt.rn.f16x2.e4m3x2 %0, hi; }" : "=r"(h) : "r"(codes));
  return h;
}
__device__ __forceinline__ float2 values2(uint32_t halves) {
  __half2 h;
  memcpy(&h, &halves, 4);
  return __half22float2(h);
}
__device__ __forceinline__ float code_value(const void* cache, int64_t at) {
  return values2(halves2(reinterpret_cast<const uint8_t*>(cache)[at])).x;
}

__device__ __forceinline__ uint8_t* scale_at(const PagedScale& s, int64_t page, int h, int block) {
  return s.base + page * s.page + (int64_t)h * s.head + (int64_t)block * s.block;
}

}  // namespace trident
