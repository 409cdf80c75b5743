// page_map.cu -- cache pages, positions and slots of a batch's new tokens, from its lengths.
//
// With c_b cached and n_b new tokens of request b and pages of ps tokens: have = ceil(c / ps),
// need = ceil((c + n) / ps); the pages have .. need-1 are the next entries of the free list, in
// request order, so page j of request b is free[head + off_b + j - have], off_b the exclusive sum of
// need - have. New token i of b stands at position c + i, on page (c + i) / ps of its table.
//
// Bound: latency (a decode step of 64 requests moves 2 KB). One launch, no exchange between blocks:
// every block reads all lengths (they sit in L2 after the first), sums them -- the call hands out all
// or nothing, so it has to know the totals before its first write -- and then walks the requests in
// chunks of one per thread with a block scan, writing the tokens of its own 1024 that fall into the
// chunk. A token finds its request by binary search in the chunk's sums in shared memory. The table
// entry of a new page is written by the thread of the page's first token, which always is new.
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

__global__ void __launch_bounds__(kMapThreads) page_map_kernel(const PageMapParams p) {
  __shared__ unsigned long long s_warp[2][kMapWarps];
  __shared__ int s_bad[kMapWarps];
  __shared__ int32_t s_cu[kMapThreads + 1], s_off[kMapThreads], s_ctx[kMapThreads];
  pdl_prologue();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;

  // totals of the whole batch
  unsigned long long tokens = 0, pages = 0;
  bool bad = false;
  for (int64_t b = tid; b < p.B; b += kMapThreads) {
    const int32_t c = p.ctx[b], n = p.fresh[b];
    if (c < 0 || n < 0 || n > INT32_MAX - c) {
      bad = true;
      continue;
    }
    const uint32_t need = pages_of(c + n, p.page);
    bad |= (int64_t)need > p.M;
    tokens += (uint32_t)n;
    pages += need - pages_of(c, p.page);
  }
  tokens = __shfl_sync(0xffffffffu, warp_scan(tokens), 31);
  pages = __shfl_sync(0xffffffffu, warp_scan(pages), 31);
  bad = __any_sync(0xffffffffu, bad);
  if (lane == 0) {
    s_warp[0][warp] = tokens;
    s_warp[1][warp] = pages;
    s_bad[warp] = bad;
  }
  __syncthreads();
  tokens = pages = 0;
#pragma unroll
  for (int w = 0; w < kMapWarps; ++w) {
    tokens += s_warp[0][w];
    pages += s_warp[1][w];
    bad |= s_bad[w] != 0;
  }
  const int32_t head = *p.free_head;
  bad |= head < 0 || head > p.F || tokens > (unsigned long long)p.N || pages > (unsigned long long)(p.F - head);
  if (blockIdx.x == 0 && tid == 0) {
    if (bad) atomicOr(p.err, kErrPages);
    *p.head_out = bad ? head : head + (int32_t)pages;
    p.cu[0] = 0;
  }

  const int64_t t0 = (int64_t)blockIdx.x * kMapTokens, t1 = min(t0 + kMapTokens, p.N);
  const int64_t total = bad ? 0 : (int64_t)tokens;
  for (int64_t t = max(t0, total) + tid; t < t1; t += kMapThreads) {  // padding
    p.pos[t] = 0;
    p.slot[t] = -1;
  }
  // chunks of one request per thread; `run`: (tokens, pages) of the chunks before, in 32 bits each
  unsigned long long run = 0;
  for (int64_t b0 = 0; b0 < p.B; b0 += kMapThreads) {
    const int64_t b = b0 + tid;
    int32_t c = 0, n = 0;
    uint32_t have = 0, fresh = 0;
    if (b < p.B) {
      c = p.ctx[b];
      n = bad ? 0 : p.fresh[b];
      if (!bad) {
        have = pages_of(c, p.page);
        fresh = pages_of(c + n, p.page) - have;
      }
    }
    const unsigned long long own = ((unsigned long long)(uint32_t)n << 32) | fresh;
    unsigned long long sum = warp_scan(own);
    __syncthreads();  // the totals, or the chunk before, have been read
    if (lane == 31) s_warp[0][warp] = sum;
    __syncthreads();
    unsigned long long before = run, chunk = 0;
#pragma unroll
    for (int w = 0; w < kMapWarps; ++w) {
      if (w < warp) before += s_warp[0][w];
      chunk += s_warp[0][w];
    }
    sum += before;
    s_cu[tid + 1] = (int32_t)(sum >> 32);
    // page j of the request is entry s_off + j of the free list
    s_off[tid] = (int32_t)(head + (int32_t)((sum - own) & 0xffffffffu) - (int32_t)have);
    s_ctx[tid] = c;
    if (tid == 0) s_cu[0] = (int32_t)(run >> 32);
    if (b < p.B && b0 / kMapThreads % gridDim.x == blockIdx.x) {  // a block per chunk writes its requests
      p.cu[b + 1] = (int32_t)(sum >> 32);
      p.kv[b] = c + n;
    }
    __syncthreads();
    const int64_t lo = max(t0, (int64_t)(run >> 32));
    run += chunk;
    const int64_t hi = min(min(t1, total), (int64_t)(run >> 32));
    for (int64_t t = lo + tid; t < hi; t += kMapThreads) {
      int r = 0;  // the last request of the chunk that starts at or before t and is not empty
#pragma unroll
      for (int step = kMapThreads / 2; step > 0; step >>= 1)
        if (s_cu[r + step] <= t) r += step;
      const int32_t pos = s_ctx[r] + (int32_t)(t - s_cu[r]);
      const uint32_t j = fast_div((uint32_t)pos, p.page.magic, p.page.shift);
      const uint32_t at = (uint32_t)pos - j * (uint32_t)p.page.d;
      int32_t* entry = p.table + (b0 + r) * p.table_rs + j;
      int32_t page;
      if (j < pages_of(s_ctx[r], p.page)) {
        page = *entry;
      } else {
        page = p.free_pages[(int64_t)s_off[r] + j];
        if (at == 0) *entry = page;
      }
      int64_t slot = (int64_t)page * p.page.d + at;
      if (slot < 0 || slot > INT32_MAX) {
        atomicOr(p.err, kErrTable);
        slot = -1;
      }
      p.pos[t] = pos;
      p.slot[t] = (int32_t)slot;
    }
  }
}

}  // namespace

const void* page_map_entry() { return (const void*)page_map_kernel; }

}  // namespace trident
