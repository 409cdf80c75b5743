// rope_paged8.cu -- RoPE over part of each head with the append to a paged cache held in 8 bits (kv8.cuh).
//
// A block's scale needs the largest magnitude of all of its rows before the first code can be written. Rows of one
// block come from consecutive tokens with consecutive slots (a run), so a run is one team's: it takes its rows,
// rotates them in fp32, agrees on the largest magnitude and writes the codes, reading k and v once. A run that
// begins with its block's first row begins the block anew; another goes on with it, and where its own rows need a
// larger scale, the block's other rows are rounded to that one (read and written again: the smaller the block and
// the longer it lives, the rarer).
//
// q has no such ties: other blocks of the grid rotate it a few rows at a time, as rope_paged.cu does.
#include <type_traits>

#include "kv8.cuh"
#include "rope_paged.cuh"

namespace trident {
namespace {

// Is token t the first of a run; the run that it begins has run_length tokens.
__device__ __forceinline__ bool slot_valid(const RopePagedParams& p, int32_t slot) { return slot >= 0 && slot < p.slots; }
__device__ __forceinline__ int32_t in_block(const RopePaged8Params& p, int32_t slot) {
  return slot - (int32_t)fast_div((uint32_t)slot, p.block.magic, p.block.shift) * p.block.d;
}
__device__ __forceinline__ bool run_starts(const RopePaged8Params& p, int64_t t, int32_t slot) {
  if (!slot_valid(p.r, slot)) return false;
  return t == 0 || p.r.slot[t - 1] != slot - 1 || in_block(p, slot) == 0;
}
__device__ __forceinline__ bool pos_valid(int32_t pos) { return pos >= 0 && pos < kPosLimit; }

// A slot's block: its scale and its first row (kv head h).
struct Block8 {
  uint8_t* scale;
  uint8_t* row0;
  int64_t row;  // bytes from row to row
};
__device__ __forceinline__ Block8 block_of(const RopePaged8Params& p, bool is_v, int32_t slot, int h) {
  const PagedCache& c = is_v ? p.r.vc : p.r.kc;
  const uint32_t pg = fast_div((uint32_t)slot, p.r.page.magic, p.r.page.shift);
  const uint32_t at = (uint32_t)slot - pg * (uint32_t)p.r.page.d;
  const uint32_t blk = fast_div(at, p.block.magic, p.block.shift);
  Block8 b;
  b.scale = scale_at(is_v ? p.vs : p.ks, pg, h, (int)blk);
  b.row0 = reinterpret_cast<uint8_t*>(c.base) + (int64_t)pg * c.page + (int64_t)h * c.head + (int64_t)blk * p.block.d * c.row;
  b.row = c.row;
  return b;
}

// ---------------------------------------------------------------- any alignment, any even R
// Element j of a q or k row, normalised by inv * gam[j] and rotated.
template <int DT, bool QKNORM, bool INTER>
__device__ __forceinline__ float row_elem(const RopePagedParams& p, const void* src, int j, int32_t pos, float inv,
                                          const float* gam) {
  auto at = [&](int i) {
    const float v = load_elem<DT>(src, i);
    return QKNORM ? v * (inv * gam[i]) : v;
  };
  if (j >= p.R) return at(j);
  const int i = INTER ? j / 2 : (j < p.R / 2 ? j : j - p.R / 2);
  const int a = INTER ? 2 * i : i, b = INTER ? 2 * i + 1 : i + p.R / 2;
  float sn, cs;
  rope_sincos((float)pos, p.freqs[i].x, p.freqs[i].y, &sn, &cs);
  sn *= p.mag;
  cs *= p.mag;
  const float x = at(a), y = at(b);
  return j == a ? fmaf(x, cs, -y * sn) : fmaf(y, cs, x * sn);
}

// One warp per (token, head-row); a kv head-row has work where its token begins a run, and then takes all of it.
template <int DT, bool QKNORM, bool INTER>
__global__ void __launch_bounds__(kThreads) rope_paged8_generic_kernel(const RopePaged8Params p8) {
  pdl_prologue();
  const RopePagedParams& p = p8.r;
  const int lane = threadIdx.x & 31;
  const int64_t total = p.T * p.NH, nwarps = (int64_t)gridDim.x * (kThreads / 32);
  for (int64_t unit = ((int64_t)blockIdx.x * kThreads + threadIdx.x) / 32; unit < total; unit += nwarps) {
    const int64_t t = unit / p.NH;
    const int hh = (int)(unit - t * p.NH);
    const bool is_q = hh < p.Hq, is_v = hh >= p.Hq + p.Hkv;
    const float* gam = is_q ? p.gamma_q : p.gamma_k;
    auto inverse = [&](const void* src) {
      if (!QKNORM || is_v) return 1.f;
      float ss = 0.f;
      for (int j = lane; j < p.D; j += 32) {
        const float v = load_elem<DT>(src, j);
        ss = fmaf(v, v, ss);
      }
      return rsqrtf(warp_sum(ss) * p.inv_D + p.eps);
    };
    const int32_t pos = p.pos[t], slot = p.slot[t];
    if (!pos_valid(pos) && lane == 0) atomicOr(p.err, kErrPos);
    if (is_q) {
      if (!pos_valid(pos)) continue;
      const void* src = paged_src(p, t, hh);
      char* dst = row_ptr(p.q_out, t, p.o_rs, 2) + (int64_t)hh * p.D * 2;
      const float inv = inverse(src);
      // in place: a pair's elements are read and written by one lane
      for (int i = lane; i < p.R / 2; i += 32) {
        const int a = INTER ? 2 * i : i, b = INTER ? 2 * i + 1 : i + p.R / 2;
        const float x = row_elem<DT, QKNORM, INTER>(p, src, a, pos, inv, gam);
        const float y = row_elem<DT, QKNORM, INTER>(p, src, b, pos, inv, gam);
        store_elem<DT>(dst, a, x);
        store_elem<DT>(dst, b, y);
      }
      for (int j = p.R + lane; j < p.D; j += 32) store_elem<DT>(dst, j, row_elem<DT, QKNORM, INTER>(p, src, j, pos, inv, gam));
      continue;
    }
    if (slot >= p.slots && lane == 0) atomicOr(p.err, kErrSlot);
    if (!run_starts(p8, t, slot)) continue;
    const int first = in_block(p8, slot);
    int n = 1;
    while (t + n < p.T && first + n < p8.block.d && p.slot[t + n] == slot + n) ++n;
    const Block8 blk = block_of(p8, is_v, slot, hh - p.Hq - (is_v ? p.Hkv : 0));
    auto elem = [&](const void* src, int j, int32_t at, float inv) {
      return is_v ? load_elem<DT>(src, j) : row_elem<DT, QKNORM, INTER>(p, src, j, at, inv, gam);
    };
    float top = 0.f;
    for (int i = 0; i < n; ++i) {
      const int32_t at = p.pos[t + i];
      if (!pos_valid(at)) continue;
      const void* src = paged_src(p, t + i, hh);
      const float inv = inverse(src);
      for (int j = lane; j < p.D; j += 32) top = fmaxf(top, fabsf(elem(src, j, at, inv)));
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    int e = scale_for(top);
    if (first > 0) {
      const int old = scale_exp(*blk.scale);
      e = max(e, old);
      if (e > old)
        for (int r = 0; r < p8.block.d; ++r) {
          if (r >= first && r < first + n) continue;
          uint8_t* row = blk.row0 + r * blk.row;
          for (int j = lane; j < p.D; j += 32) row[j] = (uint8_t)codes2(code_value(row, j) * exp2_int(old - e), 0.f);
        }
    }
    __syncwarp();  // the old scale has been read by every lane
    if (lane == 0) *blk.scale = (uint8_t)(e + 127);
    for (int i = 0; i < n; ++i) {
      const int32_t at = p.pos[t + i];
      if (!pos_valid(at)) continue;
      const void* src = paged_src(p, t + i, hh);
      const float inv = inverse(src);
      uint8_t* row = blk.row0 + (first + i) * blk.row;
      for (int j = lane; j < p.D; j += 32) row[j] = (uint8_t)codes2(elem(src, j, at, inv) * exp2_int(-e), 0.f);
    }
  }
}

}  // namespace

bool rope_paged8_kernel(int32_t dtype, int32_t variant, int32_t D, int32_t R, bool qknorm, bool inter,
                        KernelEntry* out, const char** why) {
  if (dtype != DT_BF16 && dtype != DT_FP16) { *why = "RoPE supports bf16 and fp16"; return false; }
  out->kind = KK_ROPE_PAGED8;
  if (variant != 1) {
    *why = "no vector kernel yet";
    return false;
  }
  out->vec = 1;
  auto pick = [&](auto dt) {
    constexpr int DT = decltype(dt)::value;
    return qknorm ? (inter ? (const void*)rope_paged8_generic_kernel<DT, true, true> : (const void*)rope_paged8_generic_kernel<DT, true, false>)
                  : (inter ? (const void*)rope_paged8_generic_kernel<DT, false, true> : (const void*)rope_paged8_generic_kernel<DT, false, false>);
  };
  out->fn = dtype == DT_BF16 ? pick(std::integral_constant<int, DT_BF16>()) : pick(std::integral_constant<int, DT_FP16>());
  return true;
}

}  // namespace trident
