// rope_paged.cuh -- what the RoPE kernels that append to paged caches share: which elements a lane holds, the
// pairs that they make, where a head-row comes from.
#pragma once
#include "device_common.cuh"

namespace trident {

constexpr uint32_t kErrSlot = 0x4u;  // TRIDENT_DEVERR_SLOT

// Element offsets of lane l's two vectors in a head-row.
template <bool INTER>
__device__ __forceinline__ void lane_vectors(const RopePagedParams& p, int l, int* a, int* b) {
  const int pairs = p.R / 16;  // lanes that rotate
  if (l >= pairs || INTER) {
    *a = 16 * l;
    *b = 16 * l + 8;
  } else {
    *a = 8 * l;
    *b = p.R / 2 + 8 * l;
  }
}

__device__ __forceinline__ const char* paged_src(const RopePagedParams& p, int64_t t, int hh) {
  const int64_t rb = (int64_t)p.D * 2;
  return hh < p.Hq ? row_ptr(p.q, t, p.q_rs, 2) + hh * rb
       : hh < p.Hq + p.Hkv ? row_ptr(p.k, t, p.k_rs, 2) + (hh - p.Hq) * rb
                           : row_ptr(p.v, t, p.v_rs, 2) + (hh - p.Hq - p.Hkv) * rb;
}

// Eight values of vectors x and y as the first and second members of the lane's pairs, and back.
template <bool INTER>
__device__ __forceinline__ void pairs_of(const float* x, const float* y, bool rot, F2* A, F2* B) {
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    if (INTER && rot) {
      const float* s = q < 2 ? x + 4 * q : y + 4 * (q - 2);
      A[q] = f2_pack(s[0], s[2]);
      B[q] = f2_pack(s[1], s[3]);
    } else {
      A[q] = f2_pack(x[2 * q], x[2 * q + 1]);
      B[q] = f2_pack(y[2 * q], y[2 * q + 1]);
    }
  }
}
template <bool INTER>
__device__ __forceinline__ void pairs_back(const F2* A, const F2* B, bool rot, float* x, float* y) {
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    float a0, a1, b0, b1;
    f2_unpack(A[q], &a0, &a1);
    f2_unpack(B[q], &b0, &b1);
    if (INTER && rot) {
      float* s = q < 2 ? x + 4 * q : y + 4 * (q - 2);
      s[0] = a0; s[1] = b0; s[2] = a1; s[3] = b1;
    } else {
      x[2 * q] = a0; x[2 * q + 1] = a1;
      y[2 * q] = b0; y[2 * q + 1] = b1;
    }
  }
}

// A lane's sines and cosines for position pos, times the call's magnitude; fq: its frequencies.
__device__ __forceinline__ void paged_freqs(const RopePagedParams& p, int lane, bool rot, float4* fq) {
#pragma unroll
  for (int q = 0; q < 4; ++q)
    fq[q] = rot ? *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(p.freqs) + 16 * lane + 4 * q)
                : make_float4(0.f, 0.f, 0.f, 0.f);
}
__device__ __forceinline__ void paged_angles(const RopePagedParams& p, int32_t pos, const float4* fq, RopeAngles* an) {
  rope_angles(pos, fq, an);
  const F2 m = f2_pack(p.mag, p.mag);
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    an->sn[q] = f2_mul(an->sn[q], m);
    an->ns[q] = f2_mul(an->ns[q], m);
    an->cs[q] = f2_mul(an->cs[q], m);
  }
}

// A lane's 16 elements of a q or k row, normalised (QKNORM, gam the row's weights) and rotated. Every lane of the
// row's LPG calls it; `on`: the lane holds elements.
template <int DT, int LPG, bool QKNORM, bool INTER>
__device__ __forceinline__ void paged_row_math(const RopePagedParams& p, const uint4& lo, const uint4& hi, const float* gam,
                                               const RopeAngles& an, bool on, bool rot, int va, int vb, float* x, float* y) {
  F2 A[4], B[4];
  unpack<DT>(lo, x);
  unpack<DT>(hi, y);
  if (QKNORM) {
    float ss = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) ss = fmaf(x[e], x[e], fmaf(y[e], y[e], ss));
    if (!on) ss = 0.f;
    const unsigned mask = LPG == 32 ? 0xffffffffu : (((1u << LPG) - 1u) << ((threadIdx.x & 31) & ~(LPG - 1)));
#pragma unroll
    for (int o = LPG / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(mask, ss, o, LPG);
    const float inv = rsqrtf(ss * p.inv_D + p.eps);
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const float4 ga = *reinterpret_cast<const float4*>(gam + va + 4 * q);
      const float4 gb = *reinterpret_cast<const float4*>(gam + vb + 4 * q);
      x[4 * q] *= inv * ga.x; x[4 * q + 1] *= inv * ga.y; x[4 * q + 2] *= inv * ga.z; x[4 * q + 3] *= inv * ga.w;
      y[4 * q] *= inv * gb.x; y[4 * q + 1] *= inv * gb.y; y[4 * q + 2] *= inv * gb.z; y[4 * q + 3] *= inv * gb.w;
    }
  }
  pairs_of<INTER>(x, y, rot, A, B);
  if (rot) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const F2 a = A[q], b = B[q];
      A[q] = f2_fma(a, an.cs[q], f2_mul(b, an.ns[q]));
      B[q] = f2_fma(b, an.cs[q], f2_mul(a, an.sn[q]));
    }
  }
  pairs_back<INTER>(A, B, rot, x, y);
}

}  // namespace trident
