// attn.cu -- attention of each request's last rows over its cache pages, any alignment (the formulas
// are in attn_common.cuh), and the choice of the kernels.
#include "attn_common.cuh"

namespace trident {
namespace {

// Any alignment and head size up to 512: one warp per (row, head), a key per lane for the scores, then
// the lanes split D for the product with v.
template <int DT>
__global__ void __launch_bounds__(kThreads) attn_generic_kernel(const PagedAttnParams p) {
  pdl_prologue();
  const int lane = threadIdx.x & 31;
  const int64_t unit = ((int64_t)blockIdx.x * kThreads + threadIdx.x) / 32;
  if (unit >= p.T * p.Hq) return;
  const int64_t t = unit / p.Hq;
  const int h = (int)(unit - t * p.Hq), hk = (int)fast_div((uint32_t)h, p.group.magic, p.group.shift);
  // the request of row t: the last one that starts at or before it
  int64_t lo = 0, hi = p.B;
  while (hi - lo > 1) {
    const int64_t mid = (lo + hi) / 2;
    if (p.cu[mid] <= t) lo = mid;
    else hi = mid;
  }
  bool ok = p.B > 0;
  Request r{0, 0, 0};
  if (ok) r = attn_request(p, lo, &ok);
  if (unit == 0)  // one warp looks every request's numbers over
    for (int64_t b = lane; b < p.B; b += 32) attn_request(p, b, &ok);
  const bool mine = t >= r.q0 && t < r.q0 + r.n;
  const int64_t seen = mine ? max((int64_t)0, min((int64_t)r.kv, r.kv - r.n + (t - r.q0) + 1)) : 0;
  const char* q = row_ptr(p.q, t, p.q_rs, 2) + (int64_t)h * p.D * 2;
  float m = -INFINITY, l = 0.f, acc[16];
#pragma unroll
  for (int e = 0; e < 16; ++e) acc[e] = 0.f;
  for (int64_t j0 = 0; j0 < seen; j0 += 32) {
    const int64_t j = j0 + lane;
    float s = -INFINITY;
    int64_t vat = 0;
    if (j < seen) {
      const uint32_t pg = fast_div((uint32_t)j, p.page.magic, p.page.shift);
      const int64_t at = (uint32_t)j - pg * (uint32_t)p.page.d;
      int64_t page = p.table[lo * p.table_rs + pg];
      if (page < 0 || page >= p.P) {
        ok = false;
        page = 0;
      }
      const int64_t kat = page * p.kc.page + hk * p.kc.head + at * p.kc.row;
      vat = page * p.vc.page + hk * p.vc.head + at * p.vc.row;
      float d = 0.f;
      for (int e = 0; e < p.D; ++e) d = fmaf(load_elem<DT>(q, e), load_elem<DT>(p.kc.base, kat + e), d);
      s = d * (p.scale * kLog2e);
    }
    float top = s;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    const float m2 = fmaxf(m, top), old = exp2f(m - m2);  // the first key of a chunk is always seen
    const float e = exp2f(s - m2);
    l = l * old + warp_sum(e);
    m = m2;
#pragma unroll
    for (int x = 0; x < 16; ++x) acc[x] *= old;
    const int n = (int)min((int64_t)32, seen - j0);
    for (int k = 0; k < n; ++k) {
      const float pk = __shfl_sync(0xffffffffu, e, k);
      const int64_t at = __shfl_sync(0xffffffffu, vat, k);
#pragma unroll
      for (int x = 0; x < 16; ++x)
        if (lane + 32 * x < p.D) acc[x] = fmaf(pk, load_elem<DT>(p.vc.base, at + lane + 32 * x), acc[x]);
    }
  }
  const float inv = attn_inverse(l);
  char* out = row_ptr(p.out, t, p.o_rs, 2) + (int64_t)h * p.D * 2;
#pragma unroll
  for (int x = 0; x < 16; ++x)
    if (lane + 32 * x < p.D) store_elem<DT>(out, lane + 32 * x, acc[x] * inv);
  if (lane == 0) p.lse[t * p.Hq + h] = attn_lse(m, l);
  if (!ok) atomicOr(p.err, kErrTable);
}

}  // namespace

// The kernel of few rows takes 16 of them (tokens x heads of a group) to a unit and reads the keys again for
// every further 16; the tile kernel reads them once, but its units cost more to begin and to end. Measured,
// few rows / tile kernel (us, D 128, 4 heads to a group, where nothing else is said): 32 requests of 32 rows
// over 8000 keys 311 / 184, of 20 rows over 1000 47 / 50; 16 of 128 over 2000 126 / 43, of 32 over 4000
// 73 / 61; 8 of 64 over 1500 34 / 29, of 32 over 3000 35 / 42; 4 of 24 over 500 14 / 17; D 64, 48 of 7 to 35
// rows over 400 to 3000 28 / 44, 16 of 64 over 3000 53 / 40; D 256, 8 of 32 over 4000 57 / 56. So the bound is
// by a request's elements read again: kReread. A single request does not fill the memory's rate with them:
// 96 rows over 1000 keys 14.6 / 18.5, over 2000 17.8 / 19.8, 256 over 1000 20.7 / 22.8, 400 over 1000
// 24.7 / 22.9; D 64, 210 over 2000 12.5 / 17.7; so there it is kRereadOne.
constexpr int64_t kReread = 4000 * 128, kRereadOne = 20000 * 128;

// The lengths are on the device, so the choice goes by what T, B and the table's width (keys) leave
// possible where every request has a row: both kernels, unless no request can then pass the bound, or there is
// one request only. So a call of no more rows than requests is taken for a decode step, for which a second launch
// that finds nothing would cost 4 us. A request of many rows beside empty ones (idle slots) is right there, but
// slow: 400 rows over 8000 keys among 512 requests 276 us, with 200 rows of padding 60, in a call of two 56.
// Pages that do not divide a tile's keys (or are no multiple of them), or hold fewer than the eight rows of a
// swizzle atom, and groups of more than 128 heads stay with the kernel of few rows.
AttnPlan attn_plan(const AttnEntry& tile, int64_t T, int64_t B, int64_t G, int64_t D, int64_t ps, int64_t keys) {
  const bool fits = tile.fn && G <= 128 && ps % 8 == 0 && (tile.keys % ps == 0 || ps % tile.keys == 0);
  const int64_t most = T > B ? T - B + 1 : 1;  // rows of a request, if every one has some
  AttnPlan pl;
  pl.reread = ((B == 1 ? kRereadOne : kReread) + D - 1) / D;
  pl.tile = fits && ((most * G + 15) / 16 - 1) * keys >= pl.reread;
  pl.rows = !pl.tile || B > 1;
  return pl;
}

// per_sm blocks on every SM; at most kMaxAttnBlocks, whose parts two rounds of kFanIn join.
int32_t attn_blocks(const AttnEntry& e, int32_t sms) {
  return sms * e.per_sm < kMaxAttnBlocks ? sms * e.per_sm : kMaxAttnBlocks;
}

int64_t attn_slots_floats(const AttnEntry& e, int32_t sms) {
  return e.fn ? 2 * (int64_t)attn_blocks(e, sms) * e.slot_floats : 0;
}

bool paged_attn_kernel(int32_t dtype, int32_t variant, int32_t D, KernelEntry* out, const char** why) {
  if (dtype != DT_BF16 && dtype != DT_FP16) { *why = "paged attention supports bf16 and fp16"; return false; }
  out->kind = KK_PAGED_ATTN;
  if (variant != 1) {
    if (!attn_rows_entry(dtype, D, &out->attn_rows)) {
      *why = "vector paged attention supports D in {64, 128, 256}";
      return false;
    }
    attn_tile_entry(dtype, D, &out->attn_tile);
    out->vec = 8;
    out->fn = out->attn_rows.fn;
    return true;
  }
  out->vec = 1;
  out->fn = dtype == DT_BF16 ? (const void*)attn_generic_kernel<DT_BF16> : (const void*)attn_generic_kernel<DT_FP16>;
  return true;
}

}  // namespace trident
