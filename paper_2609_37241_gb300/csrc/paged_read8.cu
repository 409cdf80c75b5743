// paged_read8.cu -- rows of a paged cache held in 8 bits (kv8.cuh), read back in the activation type.
#include "kv8.cuh"

namespace trident {
namespace {

constexpr uint32_t kErrTable = 0x10u;  // TRIDENT_DEVERR_TABLE

// Where token t of the call lies: its page and row there. false: past the last request, or *bad (no such place).
struct Place { int64_t page; int32_t row; };
__device__ __forceinline__ bool place_of(const PagedRead8Params& p, int64_t t, Place* at, bool* bad) {
  *bad = false;
  if (p.B == 0 || t >= p.cu[p.B]) return false;
  int64_t b = 0, n = p.B;  // the last request that starts at or before t, by 32 lanes
  while (n > 1) {
    const int64_t step = (n + 31) / 32, mine = (int64_t)(threadIdx.x & 31) * step;
    const unsigned le = __ballot_sync(0xffffffffu, mine < n && p.cu[b + mine] <= t);
    const int last = le ? 31 - __clz(le) : 0;
    b += last * step;
    n = min(step, n - last * step);
  }
  const int64_t pos = (int64_t)p.first[b] + (t - p.cu[b]);
  if (t < p.cu[b] || pos < 0 || pos >= p.M * (int64_t)p.page.d) {
    *bad = true;
    return false;
  }
  const uint32_t pg = fast_div((uint32_t)pos, p.page.magic, p.page.shift);
  at->page = p.table[b * p.table_rs + pg];
  at->row = (int32_t)((uint32_t)pos - pg * (uint32_t)p.page.d);
  *bad = at->page < 0 || at->page >= p.P;
  return !*bad;
}

// Any alignment: one warp per token, an element per lane at a time.
template <int DT>
__global__ void __launch_bounds__(kThreads) paged_read8_generic_kernel(const PagedRead8Params p) {
  pdl_prologue();
  const int lane = threadIdx.x & 31;
  const int64_t nwarps = (int64_t)gridDim.x * (kThreads / 32);
  for (int64_t t = ((int64_t)blockIdx.x * kThreads + threadIdx.x) / 32; t < p.T; t += nwarps) {
    Place at{0, 0};
    bool bad = false;
    const bool live = place_of(p, t, &at, &bad);
    if (!live && !bad) continue;
    if (bad && lane == 0) atomicOr(p.err, kErrTable);
    const int block = (int)fast_div((uint32_t)at.row, p.block.magic, p.block.shift);
    for (int x = 0; x < 2; ++x) {
      const PagedCache& c = x ? p.vc : p.kc;
      char* out = row_ptr(x ? p.v_out : p.k_out, t, x ? p.v_rs : p.k_rs, 2);
      for (int h = 0; h < p.Hkv; ++h) {
        const float f = live ? exp2_int(scale_exp(*scale_at(x ? p.vs : p.ks, at.page, h, block))) : 0.f;
        const int64_t src = at.page * c.page + h * c.head + at.row * c.row;
        for (int j = lane; j < p.D; j += 32) store_elem<DT>(out, (int64_t)h * p.D + j, live ? code_value(c.base, src + j) * f : 0.f);
      }
    }
  }
}

// 16-byte aligned rows, D a multiple of 16: one warp per token, 16 codes per lane at a time, four of them in flight.
// Bound: HBM (a byte read for two written); the search, the page and the scales are short chains of loads that other
// warps of the SM cover. Measured on a GB300: 24 requests of 1024 to 8192 tokens, 8 heads of 128, fp16 123 us (5.9 TB/s,
// 0.87 of the copy rate), 500 tokens 3.4 us.
template <int DT>
__global__ void __launch_bounds__(kThreads) paged_read8_vec_kernel(const PagedRead8Params p, const FastDiv vecs) {
  pdl_prologue();
  const int lane = threadIdx.x & 31;
  const int64_t t = ((int64_t)blockIdx.x * kThreads + threadIdx.x) / 32;
  if (t >= p.T) return;
  Place at{0, 0};
  bool bad = false;
  const bool live = place_of(p, t, &at, &bad);
  if (!live && !bad) return;
  if (bad && lane == 0) atomicOr(p.err, kErrTable);
  const int block = (int)fast_div((uint32_t)at.row, p.block.magic, p.block.shift);
  const uint8_t* src[2] = {reinterpret_cast<const uint8_t*>(p.kc.base) + at.page * p.kc.page + at.row * p.kc.row,
                           reinterpret_cast<const uint8_t*>(p.vc.base) + at.page * p.vc.page + at.row * p.vc.row};
  char* dst[2] = {row_ptr(p.k_out, t, p.k_rs, 2), row_ptr(p.v_out, t, p.v_rs, 2)};
  const int n = p.Hkv * vecs.d;  // vectors of a token's k
  for (int i0 = lane; i0 < n; i0 += 64) {
    uint4 c[4];
    uint32_t sc[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int i = i0 + (e >> 1) * 32;
      c[e] = make_uint4(0, 0, 0, 0);
      sc[e] = 127;
      if (i < n && live) {
        const int h = (int)fast_div((uint32_t)i, vecs.magic, vecs.shift);
        c[e] = ld16(src[e & 1] + (int64_t)h * (e & 1 ? p.vc.head : p.kc.head) + (i - h * vecs.d) * 16);
        sc[e] = *scale_at(e & 1 ? p.vs : p.ks, at.page, h, block);
      }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int i = i0 + (e >> 1) * 32;
      if (i >= n) continue;
      const float f = exp2_int(scale_exp(sc[e]));
      const uint32_t w[4] = {c[e].x, c[e].y, c[e].z, c[e].w};
      float v[16];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float2 a = values2(halves2(w[k])), b = values2(halves2_hi(w[k]));
        v[4 * k] = a.x * f; v[4 * k + 1] = a.y * f; v[4 * k + 2] = b.x * f; v[4 * k + 3] = b.y * f;
      }
      st16(dst[e & 1] + i * 32, pack<DT>(v));
      st16(dst[e & 1] + i * 32 + 16, pack<DT>(v + 8));
    }
  }
}

}  // namespace

bool paged_read8_kernel(int32_t dtype, int32_t variant, int32_t D, KernelEntry* out, const char** why) {
  if (dtype != DT_BF16 && dtype != DT_FP16) { *why = "reading a cache back supports bf16 and fp16"; return false; }
  out->kind = KK_PAGED_READ8;
  if (variant != 1) {
    if (D % 16 != 0) { *why = "the vector kernel supports D that are multiples of 16"; return false; }
    out->vec = 16;
    out->fn = dtype == DT_BF16 ? (const void*)paged_read8_vec_kernel<DT_BF16> : (const void*)paged_read8_vec_kernel<DT_FP16>;
    return true;
  }
  out->vec = 1;
  out->fn = dtype == DT_BF16 ? (const void*)paged_read8_generic_kernel<DT_BF16> : (const void*)paged_read8_generic_kernel<DT_FP16>;
  return true;
}

}  // namespace trident
