// page_map.cu -- cache pages, positions and slots of a batch's new tokens, from its lengths.
//
// With c_b cached and n_b new tokens of request b and pages of ps tokens: have = ceil(c / ps),
// need = ceil((c + n) / ps); the pages have .. need-1 are the next entries of the free list, in
// request order, so page j of request b is free[head + off_b + j - have], off_b the exclusive sum of
// need - have. New token i of b stands at position c + i, on page (c + i) / ps of its table.
//
// Bound: latency (a decode step of 64 requests moves 2 KB). One launch, no exchange between blocks:
// every block reads all lengths (they sit in L2 after the first), a run of consecutive requests per thread,
// and scans the runs' sums -- the call hands out all or nothing, so it has to know the totals before its
// first write -- then each thread writes one token: it finds the token's run by binary search in the sums in
// shared memory and walks the run's requests (two for 512 requests). The table entry of a new page is
// written by the thread of the page's first token, which always is new. On a GB300, back to back: 64
// requests 2.4 us, 512 requests with 20000 new tokens 3.2 us.
#include "device_common.cuh"

namespace trident {
namespace {

constexpr uint32_t kErrPages = 0x8u;   // TRIDENT_DEVERR_PAGES
constexpr uint32_t kErrTable = 0x10u;  // TRIDENT_DEVERR_TABLE
constexpr int kMapWarps = kMapThreads / 32;

// Pages that hold n tokens (n >= 0; n + ps - 1 may pass 2^31, not 2^32).
__device__ __forceinline__ uint32_t pages_of(int32_t n, const FastDiv& page) {
  return fast_div((uint32_t)n + (uint32_t)(page.d - 1), page.magic, page.shift);
}

__device__ __forceinline__ unsigned long long warp_scan(unsigned long long v) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned long long u = __shfl_up_sync(0xffffffffu, v, o);
    if ((threadIdx.x & 31) >= o) v += u;
  }
  return v;
}

// Lengths in shared memory up to this many requests; beyond, a run's are read again.
constexpr int kMapStaged = 4096;

__global__ void __launch_bounds__(kMapThreads) page_map_kernel(const PageMapParams p) {
  __shared__ unsigned long long s_warp[2][kMapWarps];
  __shared__ int s_bad[kMapWarps];
  __shared__ int32_t s_tok[kMapThreads + 1], s_page[kMapThreads];  // tokens and pages before a run
  __shared__ int2 s_req[kMapStaged];                               // (cached, new) of a request
  pdl_prologue();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int64_t run = (p.B + kMapThreads - 1) / kMapThreads, b0 = tid * run, b1 = min(b0 + run, p.B);
  const bool staged = p.B <= kMapStaged;

  unsigned long long tokens = 0, pages = 0;
  bool bad = false;
  for (int64_t b = b0; b < b1; ++b) {
    const int32_t c = p.ctx[b], n = p.fresh[b];
    if (staged) s_req[b] = make_int2(c, n);
    if (c < 0 || n < 0 || n > INT32_MAX - c) {
      bad = true;
      continue;
    }
    const uint32_t need = pages_of(c + n, p.page);
    bad |= (int64_t)need > p.M;
    tokens += (uint32_t)n;
    pages += need - pages_of(c, p.page);
  }
  const unsigned long long own_tokens = tokens, own_pages = pages;
  tokens = warp_scan(tokens);
  pages = warp_scan(pages);
  bad = __any_sync(0xffffffffu, bad);
  if (lane == 31) {
    s_warp[0][warp] = tokens;
    s_warp[1][warp] = pages;
    s_bad[warp] = bad;
  }
  const int32_t head = *p.free_head;
  __syncthreads();
  unsigned long long all_tokens = 0, all_pages = 0;
#pragma unroll
  for (int w = 0; w < kMapWarps; ++w) {
    if (w < warp) {
      tokens += s_warp[0][w];
      pages += s_warp[1][w];
    }
    all_tokens += s_warp[0][w];
    all_pages += s_warp[1][w];
    bad |= s_bad[w] != 0;
  }
  bad |= head < 0 || head > p.F || all_tokens > (unsigned long long)p.N ||
         all_pages > (unsigned long long)(p.F - head);
  const int32_t total = bad ? 0 : (int32_t)all_tokens;
  s_tok[tid + 1] = bad ? 0 : (int32_t)tokens;
  s_page[tid] = bad ? 0 : (int32_t)(pages - own_pages);
  if (tid == 0) s_tok[0] = 0;
  if (blockIdx.x == 0 && tid == 0) {
    if (bad) atomicOr(p.err, kErrPages);
    *p.head_out = bad ? head : head + (int32_t)all_pages;
    p.cu[0] = 0;
  }
  if (tid % gridDim.x == blockIdx.x) {  // the blocks share the requests' outputs
    int32_t at = bad ? 0 : (int32_t)(tokens - own_tokens);
    for (int64_t b = b0; b < b1; ++b) {
      const int32_t c = p.ctx[b], n = bad ? 0 : p.fresh[b];
      at += n;
      p.cu[b + 1] = at;
      p.kv[b] = c + n;
    }
  }
  __syncthreads();

  const int64_t t1 = min((int64_t)(blockIdx.x + 1) * kMapTokens, p.N);
  for (int64_t t = (int64_t)blockIdx.x * kMapTokens + tid; t < t1; t += kMapThreads) {
    if (t >= total) {  // padding
      p.pos[t] = 0;
      p.slot[t] = -1;
      continue;
    }
    int r = 0;  // the last run that starts at or before t: it is not empty
#pragma unroll
    for (int step = kMapThreads / 2; step > 0; step >>= 1)
      if (s_tok[r + step] <= t) r += step;
    int32_t at = s_tok[r], page_at = head + s_page[r];  // its request's first token, and first new page's entry
    int64_t b = r * run;
    int2 req;
    uint32_t have;
    while (true) {  // ends inside the run, which holds t
      req = staged ? s_req[b] : make_int2(p.ctx[b], p.fresh[b]);
      have = pages_of(req.x, p.page);
      if (t < (int64_t)at + req.y) break;
      at += req.y;
      page_at += (int32_t)(pages_of(req.x + req.y, p.page) - have);
      ++b;
    }
    const int32_t pos = req.x + (int32_t)(t - at);
    const uint32_t j = fast_div((uint32_t)pos, p.page.magic, p.page.shift);
    const uint32_t in_page = (uint32_t)pos - j * (uint32_t)p.page.d;
    int32_t* entry = p.table + b * p.table_rs + j;
    int32_t page;
    if (j < have) {
      page = *entry;
    } else {
      page = p.free_pages[(int64_t)page_at + (j - have)];
      if (in_page == 0) *entry = page;
    }
    int64_t slot = (int64_t)page * p.page.d + in_page;
    if (slot < 0 || slot > INT32_MAX) {
      atomicOr(p.err, kErrTable);
      slot = -1;
    }
    p.pos[t] = pos;
    p.slot[t] = (int32_t)slot;
  }
}

}  // namespace

const void* page_map_entry() { return (const void*)page_map_kernel; }

}  // namespace trident
