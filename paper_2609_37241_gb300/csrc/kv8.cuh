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

// Two values to e5m2, x in the low byte, and back.
__device__ __forceinline__ uint32_t e5m2x2(float x, float y) {
  uint16_t w;
  asm("cvt.rn.satfinite.e5m2x2.f32 %0, %1, %2;" : "=h"(w) : "f"(y), "f"(x));
  return w;
}
__device__ __forceinline__ float2 e5m2_values(uint32_t two) {
  uint32_t h;
  asm("cvt.rn.f16x2.e5m2x2 %0, %1;" : "=r"(h) : "h"((uint16_t)two));
  return values2(h);
}

// A row of q beside codes, in 8-bit products: the row times a power of two that takes its largest element to [2^7, 2^8),
// as a sum of 8-bit pieces, each the rounding of what the ones before leave: e4m3 first, then e5m2, whose range goes on
// below (a rounding to 4 bits leaves at most 8 units of a bf16's last place, which 3 bits hold). Two pieces hold a bf16
// element exactly where it is at least 2^-13 of the row's largest, three an fp16 element; a smaller one is off by 2^-21
// of the largest at most.
template <int DT> __host__ __device__ constexpr int q_pieces() { return DT == DT_BF16 ? 2 : 3; }
// bits: of the largest magnitude as fp32 (a NaN counts as the largest). A row that is not finite becomes all NaN.
__device__ __forceinline__ int q_shift(uint32_t bits) { return 134 - (int)min(max(bits >> 23, 14u), 254u); }
__device__ __forceinline__ float q_up(uint32_t bits) {
  return bits >= 0x7f800000u ? __uint_as_float(0x7fffffffu) : exp2_int(q_shift(bits));
}
__device__ __forceinline__ float q_down(uint32_t bits) { return exp2_int(-q_shift(bits)); }
// The next piece of four elements, which become what it leaves of them.
__device__ __forceinline__ uint32_t q_piece(float* y, int piece) {
  uint32_t u[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    u[k] = piece == 0 ? codes2(y[2 * k], y[2 * k + 1]) : e5m2x2(y[2 * k], y[2 * k + 1]);
    const float2 held = piece == 0 ? values2(halves2(u[k])) : e5m2_values(u[k]);
    y[2 * k] -= held.x;
    y[2 * k + 1] -= held.y;
  }
  return u[0] | u[1] << 16;
}

__device__ __forceinline__ uint8_t* scale_at(const PagedScale& s, int64_t page, int h, int block) {
  return s.base + page * s.page + (int64_t)h * s.head + (int64_t)block * s.block;
}

}  // namespace trident
