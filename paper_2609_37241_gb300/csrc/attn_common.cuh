// attn_common.cuh -- what the paged attention kernels share: a request's rows and keys, the split of a
// call's work over the blocks, and the joining of partial results.
//
// Row i of request b's n rows stands at position kv - n + i and sees the keys up to there:
//   s_j = scale * q . k_j,  m = max s_j,  l = sum exp(s_j - m),  out = sum exp(s_j - m) v_j / l,
//   lse = m + log l.
// Scores are kept in units of log 2 (scale * log2(e) folded in), so that each exponential is one exp2.
//
// Split. A unit is one tile of a (request, kv head)'s rows (row r: token r / G, head r mod G of the
// group); its keys come in tiles. The units' key tiles, one after the other over the whole call, are cut
// into equal runs, one per block: a ragged batch, one long request and a long prompt then all load the
// blocks evenly, from lengths that only the device knows. A unit that a cut goes through is joined from
// its fragments' (m, l, unnormalised out) in the workspace by the block that finishes last -- in
// fragment order, so that the result does not depend on which one that is; above kFanIn fragments in two
// levels, since one block reading hundreds would take longer than the attention itself.
#pragma once
#include "attn_count.h"
#include "device_common.cuh"

namespace trident {

constexpr uint32_t kErrTable = 0x10u;  // TRIDENT_DEVERR_TABLE
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// Request b's rows [q0, q0 + n) and keys; lengths out of range give none and set *ok = false.
struct Request { int32_t q0, n, kv; };
__device__ __forceinline__ Request attn_request(const PagedAttnParams& p, int64_t b, bool* ok) {
  const int32_t c0 = p.cu[b], c1 = p.cu[b + 1], kv = p.kv[b];
  const int64_t most = p.M * p.page.d;
  Request r{c0, c1 - c0, kv};
  if (c0 < 0 || c1 < c0 || c1 > p.T || (b == 0 && c0 != 0)) {
    *ok = false;
    r.q0 = r.n = 0;
  }
  if (kv < 0 || kv > most) {
    *ok = false;
    r.kv = kv < 0 ? 0 : (int32_t)most;
  }
  return r;
}


// Workspace: the words that are zero between calls first, as many for every version (kAttnWords), so that any of
// them can use a workspace after another: the counters of both kernels and the start word. Then, for each
// kernel, two slots of rows * (D + 2) floats per block: slot 2c for the unit that a block's run starts within,
// 2c + 1 for the one that it ends within.
__host__ __device__ constexpr int64_t attn_slot_floats(int rows, int D) { return (int64_t)rows * (D + 2); }

// kUp: the numerators are taken against the running maximum less kUp, so that they reach 2^kUp, and with a maximum
// that is 2^8 behind 2^(kUp + 8). fp16 holds nothing below 2^-25: with 7 a key counts in the product with v down to
// 2^-32 of the largest, not 2^-25, while the sum counts every one; 2^15 is within its range. In bf16 it would
// change nothing. m in what follows is that level, and lse = m + log2 l whatever it is.
template <int DT> struct ActType;
template <> struct ActType<DT_BF16> {
  static constexpr float kUp = 0.f;
  static __device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    __nv_bfloat162 b = __floats2bfloat162_rn(lo, hi);
    uint32_t w;
    memcpy(&w, &b, 4);
    return w;
  }
};
template <> struct ActType<DT_FP16> {
  static constexpr float kUp = 7.f;
  static __device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    __half2 b = __floats2half2_rn(lo, hi);
    uint32_t w;
    memcpy(&w, &b, 4);
    return w;
  }
};

// The level of a largest score, c * score in units of log 2.
template <int DT>
__device__ __forceinline__ float attn_level(float c, float score) {
  if constexpr (ActType<DT>::kUp == 0.f) return c * score;
  else return fmaf(c, score, -ActType<DT>::kUp);
}

__device__ __forceinline__ float fast_exp2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// What a row's sum l of numerators and its maximum make of it; l is 0 where the row sees no key, and NaN where a
// score was NaN or +inf: then so are out and lse.
__device__ __forceinline__ float attn_inverse(float l) { return l == 0.f ? 0.f : 1.f / l; }
__device__ __forceinline__ float attn_lse(float m, float l) { return l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2; }

// Rows past the last request: out 0, lse -inf.
template <int NT>
__device__ __forceinline__ void attn_fill_tail(const PagedAttnParams& p) {
  const int32_t last = p.B > 0 ? p.cu[p.B] : 0;
  const int64_t t0 = last < 0 ? 0 : last;
  for (int64_t t = t0 + blockIdx.x; t < p.T; t += gridDim.x) {
    char* out = row_ptr(p.out, t, p.o_rs, 2);
    for (int64_t e = threadIdx.x; e < (int64_t)p.Hq * p.D / 8; e += NT) st16(out + e * 16, make_uint4(0, 0, 0, 0));
    for (int h = threadIdx.x; h < p.Hq; h += NT) p.lse[t * p.Hq + h] = -INFINITY;
  }
}

// Does this launch take the request? Where both kernels run, by the keys that the kernel of few rows would
// read again for row tiles after the first: the tile kernel's from p.reread of them on.
__device__ __forceinline__ bool attn_takes(const PagedAttnParams& p, const Request& r) {
  if (p.part == ATTN_ALL) return r.n > 0;
  const int64_t again = (((int64_t)r.n * p.G + 15) / 16 - 1) * r.kv;
  return r.n > 0 && (again >= p.reread) == (p.part == ATTN_MANY);
}

// One block's share of the call: tiles per block and this block's run [lo, hi). whole: a unit per block
// instead, all of it, where there are at most as many units as blocks and none is longer than an even run
// and what a cut costs (a partial written, counted and joined: about kTileJoin tiles' time); per, lo and
// hi then count units.
struct AttnShare {
  int64_t per, lo, hi, total;
  bool whole;
  bool others;  // ATTN_FEW: some requests are the other kernel's
};

// Cost::of(p, r): the key tiles of all of request r's units, at least one per unit so that a unit
// without keys is written too. WHOLE: whole units are a choice, with Cost::units and Cost::longest, the
// request's units and the tiles of the longest. NT: threads of the block.
template <int NT, class Cost, bool WHOLE>
struct AttnSplit {
  struct Smem {
    long long warp[NT / 32], units[NT / 32];
    int32_t longest[NT / 32];
    int hit;                // the request that holds the run's first tile (at most NT requests)
    long long pre[NT + 1];  // tiles (units) before each request of the current chunk, from the call's start
    int32_t q0[NT], n[NT], kv[NT];
  };

  // Inclusive sum over the block's threads and the block's total; a barrier before the words are used again.
  // others: is set where any thread's is (one barrier for both).
  static __device__ __forceinline__ long long block_scan(Smem& s, long long v, long long* all, bool* others) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long u = __shfl_up_sync(0xffffffffu, v, o);
      if ((int)(threadIdx.x & 31) >= o) v += u;
    }
    if ((threadIdx.x & 31) == 31) s.warp[threadIdx.x >> 5] = v;
    *others = __syncthreads_or(*others) != 0;
    long long total = 0;
#pragma unroll
    for (int w = 0; w < NT / 32; ++w) {
      if (w < (int)(threadIdx.x >> 5)) v += s.warp[w];
      total += s.warp[w];
    }
    *all = total;
    return v;
  }

  // The block's share; with at most NT requests their chunk is filled as well.
  static __device__ __forceinline__ AttnShare share(const PagedAttnParams& p, Smem& s) {
    bool ok = true, others = false;
    long long own = 0, own_units = 0;
    int32_t longest = 0;
    Request r{0, 0, 0};
    for (int64_t b = threadIdx.x; b < p.B; b += NT) {
      r = attn_request(p, b, &ok);
      if (!attn_takes(p, r)) {
        others |= r.n > 0;
        continue;
      }
      own += Cost::of(p, r);
      if constexpr (WHOLE) {
        own_units += Cost::units(p, r);
        longest = max(longest, Cost::longest(p, r));
      }
    }
    if (!ok && blockIdx.x == 0) atomicOr(p.err, kErrTable);
    if (threadIdx.x == 0) s.hit = 0;
    long long units = own_units;
    if constexpr (WHOLE) {
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) {
        units += __shfl_xor_sync(0xffffffffu, units, o);
        longest = max(longest, __shfl_xor_sync(0xffffffffu, longest, o));
      }
      if ((threadIdx.x & 31) == 0) {
        s.units[threadIdx.x >> 5] = units;
        s.longest[threadIdx.x >> 5] = longest;
      }
    }
    long long sum;
    long long upto = block_scan(s, own, &sum, &others);
    const int64_t even = (uint64_t)sum >> 31 ? (sum + gridDim.x - 1) / gridDim.x
                                             : (int64_t)(((uint32_t)sum + gridDim.x - 1) / gridDim.x);
    AttnShare a;
    a.others = others;
    a.whole = false;
    a.total = sum;
    a.per = even > p.min_tiles ? even : p.min_tiles;
    if constexpr (WHOLE) {
      units = 0;
#pragma unroll
      for (int w = 0; w < NT / 32; ++w) {
        units += s.units[w];
        longest = max(longest, s.longest[w]);
      }
      if (units <= gridDim.x && longest <= even + kTileJoin) {  // the same in every thread
        a.whole = true;
        a.total = units;
        a.per = 1;
        own = own_units;
        __syncthreads();
        upto = block_scan(s, own, &sum, &others);
      }
    }
    a.lo = min(a.total, (int64_t)blockIdx.x * a.per);
    a.hi = min(a.total, a.lo + a.per);
    if (p.B <= NT) fill(s, r, own, upto, a.lo);
    return a;
  }

  // Fills the chunk of NT requests from b0 on (share has filled the only one of at most NT requests); run:
  // the tiles before it. Returns those after it.
  static __device__ __forceinline__ int64_t chunk(const PagedAttnParams& p, Smem& s, int64_t b0, int64_t run, const AttnShare& a) {
    if (p.B <= NT) return a.total;
    const int64_t b = b0 + threadIdx.x;
    bool ok = true, others = false;
    Request r{0, 0, 0};
    if (b < p.B) r = attn_request(p, b, &ok);
    long long own = 0;
    if (attn_takes(p, r)) {
      own = Cost::of(p, r);
      if constexpr (WHOLE)
        if (a.whole) own = Cost::units(p, r);
    }
    long long all;
    __syncthreads();  // the chunk before has been read
    const long long upto = block_scan(s, own, &all, &others);
    fill(s, r, own, run + upto, -1);
    return run + all;
  }
  static __device__ __forceinline__ void fill(Smem& s, const Request& r, long long own, long long upto, int64_t lo) {
    s.q0[threadIdx.x] = r.q0;
    s.n[threadIdx.x] = r.n;
    s.kv[threadIdx.x] = r.kv;
    s.pre[threadIdx.x + 1] = upto;
    if (threadIdx.x == 0) s.pre[0] = upto - own;
    if (upto - own <= lo && lo < upto) s.hit = threadIdx.x;
    __syncthreads();
  }

  // The last request of the chunk with pre[r] <= x (pre[0] <= x < the chunk's end): it holds tile x.
  static __device__ __forceinline__ int find(const PagedAttnParams& p, const Smem& s, const AttnShare& a, int64_t x) {
    if (p.B <= NT && x == a.lo) return s.hit;
    int r = 0, end = NT;
    while (end - r > 1) {
      const int mid = (r + end) / 2;
      if (s.pre[mid] <= x) r = mid;
      else end = mid;
    }
    return r;
  }
};

__device__ __forceinline__ int64_t attn_div(int64_t a, int64_t b) {  // a, b >= 0
  return ((uint64_t)a | (uint64_t)b) >> 32 ? a / b : (int64_t)((uint32_t)a / (uint32_t)b);
}

// A fragment's place: unit tiles [u0, u1) of the call, cut into runs of `per` tiles.
struct AttnCuts {
  int64_t first, last;  // blocks that hold a part of the unit
  __device__ __forceinline__ bool whole() const { return first == last; }
  __device__ __forceinline__ int64_t slot(int64_t block) const { return block == first ? 2 * block + 1 : 2 * block; }
};

// A block of either kernel as attn_count.h's start word sees it.
struct AttnStartBlock {
  uint32_t* word;
  __device__ __forceinline__ void sync() const { __syncthreads(); }
  __device__ __forceinline__ bool any(bool x) const { return __syncthreads_or(x) != 0; }
  __device__ __forceinline__ bool leader() const { return threadIdx.x == 0; }
  __device__ __forceinline__ bool first() const { return blockIdx.x == 0; }
  __device__ __forceinline__ void wait_before() const { pdl_wait(); }
  __device__ __forceinline__ uint32_t start_word() const {
    uint32_t x;
    asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(x) : "l"(word) : "memory");
    return x;
  }
  __device__ __forceinline__ void set_start_word(uint32_t x) const {
    asm volatile("st.release.gpu.global.u32 [%0], %1;" :: "l"(word), "r"(x) : "memory");
  }
};

// The block as attn_count.h sees it: NT threads at named barrier BAR, their words in shared memory.
template <int BAR, int NT>
__device__ __forceinline__ void attn_sync() {
  asm volatile("bar.sync %0, %1;" :: "n"(BAR), "n"(NT) : "memory");
}
template <int BAR, int NT>
struct AttnBlock {
  volatile int* words;          // kAttnAnswers of them
  const volatile int* abort;    // set where a wait ran out; NULL: a kernel that waits for nothing
  __device__ __forceinline__ void sync() const { attn_sync<BAR, NT>(); }
  __device__ __forceinline__ bool leader() const { return threadIdx.x == 0; }
  __device__ __forceinline__ void fence() const { __threadfence(); }
  __device__ __forceinline__ uint32_t look(uint32_t* c) const { return *reinterpret_cast<volatile uint32_t*>(c); }
  __device__ __forceinline__ uint32_t add(uint32_t* c) const { return atomicAdd(c, 1u); }
  __device__ __forceinline__ void zero(uint32_t* c) const { *c = 0u; }
  __device__ __forceinline__ bool failed() const { return abort && *abort != 0; }
  __device__ __forceinline__ void tell(AttnWord w, bool x) const { words[w] = x; }
  __device__ __forceinline__ bool told(AttnWord w) const { return words[w] != 0; }
};

}  // namespace trident
