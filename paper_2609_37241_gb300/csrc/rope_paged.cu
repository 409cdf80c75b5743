// rope_paged.cu -- RoPE over part of each head, in either pairing, with the append to a paged cache,
// optionally after per-head q/k RMSNorm.
//
// As rope.cu: a token has NH = Hq + 2 Hkv head-rows, a warp takes an item of consecutive head-rows of
// one token, D / 16 lanes per head-row. A lane holds two 16-byte vectors with both members of its eight
// pairs -- (i, i + R/2): the vectors at 8l and R/2 + 8l; (2i, 2i+1): those at 16l and 16l + 8 -- so a
// rotation needs no other lane, and its sines and cosines serve all rows of the item. The lanes past
// R / 16 hold what passes through. The frequency table and the slots are the caller's tensors, which
// the launch before may have written: they are read after the launch wait, by plain loads.
//
// Angles: pos < 2^24 is exact in fp32 and rope_sincos' first reduction step, fma(-k, A, pos * f), is
// exact for every such angle with f <= 1 (k A and pos * f are multiples of 2^-9 where they pass 2^15, and their
// difference is small), so what remains is the error of the hardware sine, about 1e-6. Frequencies above 1
// take it further: the reduced angle is within 1e-6 up to angles of 2^26, 1.3e-5 at 2^30 (checked on the CPU).
#include "device_common.cuh"

namespace trident {
namespace {

constexpr uint32_t kErrSlot = 0x4u;  // TRIDENT_DEVERR_SLOT
constexpr int kRopePagedThreads = 64;

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

// The row of a token in a paged cache (slot valid).
__device__ __forceinline__ char* paged_row(const PagedCache& c, const FastDiv& page, int32_t slot, int h) {
  const uint32_t pg = fast_div((uint32_t)slot, page.magic, page.shift);
  const uint32_t at = (uint32_t)slot - pg * (uint32_t)page.d;
  return reinterpret_cast<char*>(c.base) + ((int64_t)pg * c.page + (int64_t)h * c.head + (int64_t)at * c.row) * 2;
}

// Where head-row hh of token t goes; NULL: nowhere (a padding token's k or v).
__device__ __forceinline__ char* paged_dst(const RopePagedParams& p, int64_t t, int hh, int32_t slot) {
  if (hh < p.Hq) return row_ptr(p.q_out, t, p.o_rs, 2) + (int64_t)hh * p.D * 2;
  if (slot < 0) return nullptr;
  const bool is_v = hh >= p.Hq + p.Hkv;
  return paged_row(is_v ? p.vc : p.kc, p.page, slot, hh - p.Hq - (is_v ? p.Hkv : 0));
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

// R rows per lane group; every load they need is issued first.
template <int DT, int LPG, bool QKNORM, bool INTER, int R>
__global__ void __launch_bounds__(kRopePagedThreads) rope_paged_kernel(const RopePagedParams p) {
  pdl_prologue();
  constexpr int GW = 32 / LPG;
  const int l = (threadIdx.x & 31) % LPG, lane = min(l, p.D / 16 - 1);
  const bool on = l == lane;
  const int64_t item = (int64_t)blockIdx.x * (kRopePagedThreads / 32) + threadIdx.x / 32;
  if (item >= p.T * p.ipt) return;
  const uint32_t tok = fast_div((uint32_t)item, p.ipt_magic, p.ipt_shift);
  const int64_t t = tok;
  const int first = (int)((uint32_t)item - tok * (uint32_t)p.ipt) * p.rpi, end = min(p.NH, first + p.rpi);
  const int hh0 = first + (threadIdx.x & 31) / LPG;
  int va, vb;
  lane_vectors<INTER>(p, lane, &va, &vb);
  uint4 lo[R], hi[R];
#pragma unroll
  for (int j = 0; j < R; ++j) {  // groups past the item's end load its last row and drop it
    const char* src = paged_src(p, t, min(hh0 + j * GW, end - 1));
    lo[j] = ld16(src + va * 2);
    hi[j] = ld16(src + vb * 2);
  }
  const int32_t pos = p.pos[t];
  int32_t slot = p.slot[t];
  const bool rot = lane < p.R / 16;
  float4 fq[4];
#pragma unroll
  for (int q = 0; q < 4; ++q)
    fq[q] = rot ? *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(p.freqs) + 16 * lane + 4 * q)
                : make_float4(0.f, 0.f, 0.f, 0.f);
  if (pos < 0 || pos >= kPosLimit) {
    if ((threadIdx.x & 31) == 0) atomicOr(p.err, kErrPos);
    return;
  }
  if (slot >= p.slots) {
    if ((threadIdx.x & 31) == 0) atomicOr(p.err, kErrSlot);
    slot = -1;
  }
  RopeAngles an;
  rope_angles(pos, fq, &an);
  {
    const F2 m = f2_pack(p.mag, p.mag);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      an.sn[q] = f2_mul(an.sn[q], m);
      an.ns[q] = f2_mul(an.ns[q], m);
      an.cs[q] = f2_mul(an.cs[q], m);
    }
  }
#pragma unroll
  for (int j = 0; j < R; ++j) {
    const int hh = hh0 + j * GW;
    const bool live = on && hh < end;
    char* dst = hh < end ? paged_dst(p, t, hh, slot) : nullptr;
    if (hh >= p.Hq + p.Hkv) {  // bit copy into the cache
      if (live && dst) {
        st16(dst + va * 2, lo[j]);
        st16(dst + vb * 2, hi[j]);
      }
      continue;
    }
    float x[8], y[8];
    F2 A[4], B[4];
    unpack<DT>(lo[j], x);
    unpack<DT>(hi[j], y);
    if (QKNORM) {
      float ss = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) ss = fmaf(x[e], x[e], fmaf(y[e], y[e], ss));
      if (!on) ss = 0.f;
      const unsigned mask =
          LPG == 32 ? 0xffffffffu : (((1u << LPG) - 1u) << ((threadIdx.x & 31) & ~(LPG - 1)));
#pragma unroll
      for (int o = LPG / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(mask, ss, o, LPG);
      const float inv = rsqrtf(ss * p.inv_D + p.eps);
      const float* gam = hh < p.Hq ? p.gamma_q : p.gamma_k;
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
    if (live && dst) {
      st16(dst + va * 2, pack<DT>(x));
      st16(dst + vb * 2, pack<DT>(y));
    }
  }
}

// Any alignment, any even R: one warp per head-row, scalar accesses.
template <int DT, bool QKNORM, bool INTER>
__global__ void __launch_bounds__(kThreads) rope_paged_generic_kernel(const RopePagedParams p) {
  pdl_prologue();
  const int lane = threadIdx.x & 31;
  const int64_t total = p.T * p.NH, nwarps = (int64_t)gridDim.x * (kThreads / 32);
  for (int64_t unit = ((int64_t)blockIdx.x * kThreads + threadIdx.x) / 32; unit < total; unit += nwarps) {
    const int64_t t = unit / p.NH;
    const int hh = (int)(unit - t * p.NH);
    const int32_t pos = p.pos[t];
    int32_t slot = p.slot[t];
    if (pos < 0 || pos >= kPosLimit) {
      if (lane == 0) atomicOr(p.err, kErrPos);
      continue;
    }
    if (slot >= p.slots) {
      if (lane == 0) atomicOr(p.err, kErrSlot);
      slot = -1;
    }
    const void* src = paged_src(p, t, hh);
    void* dst = paged_dst(p, t, hh, slot);
    if (!dst) continue;
    if (hh >= p.Hq + p.Hkv) {  // bit copy into the cache
      for (int j = lane; j < p.D; j += 32)
        reinterpret_cast<uint16_t*>(dst)[j] = reinterpret_cast<const uint16_t*>(src)[j];
      continue;
    }
    const float* gam = hh < p.Hq ? p.gamma_q : p.gamma_k;
    float inv = 1.f;
    if (QKNORM) {
      float ss = 0.f;
      for (int j = lane; j < p.D; j += 32) {
        const float v = load_elem<DT>(src, j);
        ss = fmaf(v, v, ss);
      }
      inv = rsqrtf(warp_sum(ss) * p.inv_D + p.eps);
    }
    for (int i = lane; i < p.R / 2; i += 32) {
      const int a = INTER ? 2 * i : i, b = INTER ? 2 * i + 1 : i + p.R / 2;
      float x = load_elem<DT>(src, a), y = load_elem<DT>(src, b);
      if (QKNORM) {
        x *= inv * gam[a];
        y *= inv * gam[b];
      }
      float sn, cs;
      rope_sincos((float)pos, p.freqs[i].x, p.freqs[i].y, &sn, &cs);
      sn *= p.mag;
      cs *= p.mag;
      store_elem<DT>(dst, a, fmaf(x, cs, -y * sn));
      store_elem<DT>(dst, b, fmaf(y, cs, x * sn));
    }
    for (int j = p.R + lane; j < p.D; j += 32) {
      const float v = load_elem<DT>(src, j);
      store_elem<DT>(dst, j, QKNORM ? v * (inv * gam[j]) : v);
    }
  }
}

template <int DT, int LPG, bool QK, bool INTER>
void pick_rows(KernelEntry* out) {
  out->any_fn[0] = (const void*)rope_paged_kernel<DT, LPG, QK, INTER, 1>;
  out->any_fn[1] = (const void*)rope_paged_kernel<DT, LPG, QK, INTER, 2>;
  out->any_fn[2] = (const void*)rope_paged_kernel<DT, LPG, QK, INTER, 3>;
  out->any_fn[3] = (const void*)rope_paged_kernel<DT, LPG, QK, INTER, 4>;
}

template <int DT, bool QK, bool INTER>
void pick(int32_t variant, int32_t D, KernelEntry* out) {
  if (variant == 1) out->fn = (const void*)rope_paged_generic_kernel<DT, QK, INTER>;
  else if (D <= 64) pick_rows<DT, 4, QK, INTER>(out);
  else if (D <= 128) pick_rows<DT, 8, QK, INTER>(out);
  else pick_rows<DT, 16, QK, INTER>(out);
}

}  // namespace

// Rows per lane group at most: one up to three items (of one row each) per SM, three beyond, four from
// kRopePagedMany such items of three per SM on; the kernel is that of the rows that the item split leaves to
// a group. Measured, one / two / three / four rows at most: 200 tokens of 32 + 8 + 8 heads of 128 with q/k
// norm 3.56 / 3.49 / 3.82 / 3.93 us, 1000 tokens 8.20 / 6.40 / 6.33 / 7.26, 3333 (half of the head) 22.1 / 17.8
// / 16.4 / 16.3, 8192 without the norm 50.2 / 32.7 / 32.9 / 31.3 (0.95 of the 6.79 TB/s copy rate).
constexpr int64_t kRopePagedMany = 120;
int rope_paged_plan(RopePagedParams* p, int32_t* threads, int64_t* blocks, int32_t sms) {
  const int lanes = p->D <= 64 ? 4 : p->D <= 128 ? 8 : 16, groups = 32 / lanes;
  RopeSplit r = rope_split(p->NH, groups, 1);
  if (p->T * r.ipt > 3 * (int64_t)sms) r = rope_split(p->NH, groups, 3);
  if (r.rpi > groups && p->T * r.ipt > kRopePagedMany * sms) r = rope_split(p->NH, groups, 4);
  const int e = r.rpi / groups - 1;
  p->ipt = r.ipt;
  p->rpi = r.rpi;
  p->ipt_magic = r.magic;
  p->ipt_shift = r.shift;
  *threads = kRopePagedThreads;
  *blocks = (p->T * r.ipt + kRopePagedThreads / 32 - 1) / (kRopePagedThreads / 32);
  return e;
}

bool rope_paged_kernel(int32_t dtype, int32_t variant, int32_t D, int32_t R, bool qknorm, bool inter,
                       KernelEntry* out, const char** why) {
  if (dtype != DT_BF16 && dtype != DT_FP16) { *why = "RoPE supports bf16 and fp16"; return false; }
  if (variant != 1 && (D % 16 != 0 || R % 16 != 0 || D < 32 || D > 256)) {
    *why = "vector paged RoPE supports D in 32 .. 256 and R that are multiples of 16";
    return false;
  }
  out->kind = KK_ROPE_PAGED;
  out->vec = variant == 1 ? 1 : 8;
  if (dtype == DT_BF16) {
    if (qknorm) inter ? pick<DT_BF16, true, true>(variant, D, out) : pick<DT_BF16, true, false>(variant, D, out);
    else inter ? pick<DT_BF16, false, true>(variant, D, out) : pick<DT_BF16, false, false>(variant, D, out);
  } else {
    if (qknorm) inter ? pick<DT_FP16, true, true>(variant, D, out) : pick<DT_FP16, true, false>(variant, D, out);
    else inter ? pick<DT_FP16, false, true>(variant, D, out) : pick<DT_FP16, false, false>(variant, D, out);
  }
  if (!out->fn) out->fn = out->any_fn[0];
  return true;
}

}  // namespace trident
