// attn_tile.cuh -- paged attention for requests of many rows: what does not depend on how the cache holds its elements.
// A Core (attn_tile.cu: 16 bits, attn_tile8.cu: 8) loads q and the tiles of keys, issues the products and has a
// softmax; here are barriers and tensor instructions, the units and their split over the blocks, and the ends of
// fragments.
//
// A unit is NT tiles of 128 rows (tokens x the G heads of a group, so that all of them share the keys' loads) against
// tiles of KEYS keys; per block NT softmax warpgroups, NT warps that issue tcgen05.mma (a Core's work()), and the Core's
// other warps. TMEM columns: NT x KEYS of scores S (the numerators P in their first half) and NT x D of O.
//
// Every wait is bounded (params.polls polls, kBulkWaitPolls by default): a wait that runs out sets
// TRIDENT_DEVERR_TIMEOUT and a flag that ends the block's other waits; the warps then let their copies
// and products in flight finish (bounded again), free the TMEM and return without further writes.
#pragma once
#include <cuda.h>

#include "attn_common.cuh"

namespace trident {

constexpr float kTileLazy = 8.f;
constexpr int kFrags = 32;  // fragments listed at a time

// ---------------------------------------------------------------- barriers, TMA, tcgen05
__device__ __forceinline__ uint32_t smem_at(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void mb_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" :: "r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mb_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" :: "r"(bar) : "memory");
}
__device__ __forceinline__ void mb_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" :: "r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool mb_try(uint32_t bar, uint32_t parity) {
  uint32_t done;
  asm volatile("{ .reg .pred q; mbarrier.try_wait.parity.shared::cta.b64 q, [%1], %2; selp.u32 %0, 1, 0, q; }"
               : "=r"(done) : "r"(bar), "r"(parity) : "memory");
  return done != 0;
}
// Bounded wait; false when it ran out or another wait of the block did.
__device__ __forceinline__ bool mb_wait(uint32_t bar, uint32_t parity, uint32_t polls, volatile int* abort) {
  for (uint32_t i = 0; i < polls; ++i) {
    if (mb_try(bar, parity)) return true;
    if ((i & 15) == 15 && *abort) return false;
  }
  *abort = 1;
  return false;
}
// Bounded wait on the way out, whatever the flag says.
__device__ __forceinline__ void mb_drain(uint32_t bar, uint32_t parity) {
  for (uint32_t i = 0; i < kBulkWaitPolls; ++i)
    if (mb_try(bar, parity)) return;
}
__device__ __forceinline__ void tma_4d(uint32_t dst, const CUtensorMap* map, int c0, int c1, int c2, int c3, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
               " [%0], [%1, {%2, %3, %4, %5}], [%6];"
               :: "r"(dst), "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(bar) : "memory");
}
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void tc_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" :: "r"(bar) : "memory");
}
// One lane of the warp, the same one each time.
__device__ __forceinline__ bool elect_one() {
  uint32_t is;
  asm volatile("{ .reg .pred q; elect.sync _|q, 0xffffffff; selp.u32 %0, 1, 0, q; }" : "=r"(is));
  return is != 0;
}
// D = A B (+ D where add): A and B by descriptor, or A in TMEM.
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t add) {
  asm volatile("{ .reg .pred p; setp.ne.u32 p, %4, 0; tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p; }"
               :: "r"(d), "l"(a), "l"(b), "r"(idesc), "r"(add) : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t add) {
  asm volatile("{ .reg .pred p; setp.ne.u32 p, %4, 0; tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p; }"
               :: "r"(d), "r"(a), "l"(b), "r"(idesc), "r"(add) : "memory");
}
// Shared-memory operand descriptor, 128-byte swizzle (layout code 2, bits 61-63; version 1, bits 46-48):
// start, leading and stride byte offsets in units of 16. The start is in the low word's first 14 bits, so
// a step inside a tile is an addition there.
__device__ __forceinline__ uint32_t desc_lo(uint32_t at, uint32_t leading) { return (at >> 4) | ((leading >> 4) << 16); }
__device__ __forceinline__ uint64_t desc128(uint32_t lo) {  // stride: 1024, eight rows of 128 bytes
  constexpr uint32_t hi = (1024u >> 4) | (1u << 14) | (2u << 29);
  return ((uint64_t)hi << 32) | lo;
}
// Instruction descriptor of kind::f16: fp32 accumulators, A and B of the activation type, both K-major
// unless b_mn, M x N.
template <int DT>
__host__ __device__ constexpr uint32_t idesc_of(int M, int N, bool b_mn) {
  return (1u << 4) | ((DT == DT_BF16 ? 1u : 0u) << 7) | ((DT == DT_BF16 ? 1u : 0u) << 10) | ((b_mn ? 1u : 0u) << 16) |
         ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}

#define TC_R8(r, k) "=r"(r[k]), "=r"(r[k + 1]), "=r"(r[k + 2]), "=r"(r[k + 3]), "=r"(r[k + 4]), "=r"(r[k + 5]), "=r"(r[k + 6]), "=r"(r[k + 7])
#define TC_W8(r, k) "+r"(r[k]), "+r"(r[k + 1]), "+r"(r[k + 2]), "+r"(r[k + 3]), "+r"(r[k + 4]), "+r"(r[k + 5]), "+r"(r[k + 6]), "+r"(r[k + 7])
#define TC_I8(r, k) "r"(r[k]), "r"(r[k + 1]), "r"(r[k + 2]), "r"(r[k + 3]), "r"(r[k + 4]), "r"(r[k + 5]), "r"(r[k + 6]), "r"(r[k + 7])
// 32 columns of the warp's 32 lanes: lane i, register k = column k.
__device__ __forceinline__ void tc_ld32(uint32_t at, uint32_t* r) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
               "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
               : TC_R8(r, 0), TC_R8(r, 8), TC_R8(r, 16), TC_R8(r, 24) : "r"(at) : "memory");
}
__device__ __forceinline__ void tc_st32(uint32_t at, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
               "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};"
               :: TC_I8(r, 0), TC_I8(r, 8), TC_I8(r, 16), TC_I8(r, 24), "r"(at) : "memory");
}

// Waits for the loads before it, as what brings the values of these N registers: a use of them depends on the wait, so
// that no compiler may move it between a load and the wait.
template <int N>
__device__ __forceinline__ void tc_wait_ld(uint32_t* r) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int i = 0; i < N; i += 8) asm volatile("" : TC_W8(r, i));
}
__device__ __forceinline__ void tc_st16(uint32_t at, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};"
               :: TC_I8(r, 0), TC_I8(r, 8), "r"(at) : "memory");
}
__device__ __forceinline__ F2 f2_add(F2 a, F2 b) {
  F2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}

// ---------------------------------------------------------------- units
// sum of floor((a i + b) / m) for i < n (the Euclid-like reduction of lattice-point counts), for
// a n + b + m < 2^32.
__device__ __forceinline__ int64_t floor_sum(uint32_t n, uint32_t m, uint32_t a, uint32_t b) {
  int64_t total = 0;
  while (n > 0) {
    if (a >= m) {
      total += (int64_t)n * (n - 1) / 2 * (a / m);
      a %= m;
    }
    if (b >= m) {
      total += (int64_t)n * (b / m);
      b %= m;
    }
    const uint32_t y = a * n + b;  // the last term's numerator is y - a
    if (y < m) break;
    n = y / m;
    b = y % m;
    const uint32_t t = m;
    m = a;
    a = t;
  }
  return total;
}

// Row tile k of a request: tokens [k R, (k + 1) R) of its n, R = ROWS / G whole tokens. It sees
// kv - n + min(n, (k + 1) R) keys (its last token's).
template <int ROWS, int KEYS>
struct TileCost {
  static __device__ __forceinline__ int32_t sees(const PagedAttnParams& p, const Request& r, int32_t k) {
    const int64_t i = min((int64_t)r.n, (int64_t)(k + 1) * p.tokens);
    return (int32_t)max((int64_t)0, min((int64_t)r.kv, (int64_t)r.kv - r.n + i));
  }
  static __device__ __forceinline__ int32_t key_tiles(int32_t keys) {
    return keys > KEYS ? (int32_t)(((uint32_t)keys + KEYS - 1) / KEYS) : 1;
  }
  static __device__ __forceinline__ int32_t row_tiles(const PagedAttnParams& p, const Request& r) {
    return (int32_t)(((uint32_t)r.n + (uint32_t)(p.tokens - 1)) / (uint32_t)p.tokens);
  }
  // Key tiles of the first k row tiles of one kv head; all of them end at a whole R (last: but the k-th).
  static __device__ __forceinline__ int64_t before(const PagedAttnParams& p, const Request& r, int32_t k, bool last) {
    const int32_t c = r.kv - r.n;
    int64_t total = 0;
    if (last) total = key_tiles(sees(p, r, --k));
    if (c < 0) {
      for (int32_t i = 0; i < k; ++i) total += key_tiles(sees(p, r, i));
      return total;
    }
    // sum of ceil((c + (i + 1) R) / KEYS); whole multiples of KEYS taken out with constant divisors
    const uint32_t R = (uint32_t)p.tokens, b = (uint32_t)c + R + KEYS - 1;
    return total + (int64_t)k * (b / KEYS) + (int64_t)k * (k - 1) / 2 * (R / KEYS) + floor_sum(k, KEYS, R % KEYS, b % KEYS);
  }
  static __device__ __forceinline__ int64_t units(const PagedAttnParams& p, const Request& r) {
    return (int64_t)p.Hkv * row_tiles(p, r);
  }
  static __device__ __forceinline__ int32_t longest(const PagedAttnParams&, const Request& r) { return key_tiles(r.kv); }
  static __device__ __forceinline__ int64_t of(const PagedAttnParams& p, const Request& r) {
    return (int64_t)p.Hkv * before(p, r, row_tiles(p, r), true);
  }
};

struct Frag {
  int64_t b, first, last;  // request; blocks that share the unit
  int32_t q0, n, kv, h, tok0, rows, limit;
  int32_t t0, t1;          // key tiles
};

// C: a Core's constants -- DT, D, NT, KEYS, the threads besides the softmax's (OTHERS, whole warpgroups) and the registers
// of both. The launch gives every thread LAUNCH_REGS; SOFT * SOFT_REGS + OTHERS * OTHER_REGS is below that in total.
template <class C>
struct TileShape {
  static constexpr int DT = C::DT, D = C::D, NT = C::NT, KEYS = C::KEYS;
  static constexpr int ROWS = 128 * NT;
  static constexpr int SOFT = 128 * NT;        // softmax threads
  static constexpr int THREADS = SOFT + C::OTHERS;
  static constexpr int LAUNCH_REGS = 65536 / THREADS / 8 * 8;
  static_assert(SOFT * C::SOFT_REGS + C::OTHERS * C::OTHER_REGS <= THREADS * (LAUNCH_REGS < 255 ? LAUNCH_REGS : 248), "register split");
  static constexpr int S_COL = 0, O_COL = NT * KEYS;
  static_assert(NT * (KEYS + D) <= 512, "TMEM columns");
  static constexpr int MMA_WARP = SOFT / 32;
  using Cost = TileCost<ROWS, KEYS>;
  using Split = AttnSplit<THREADS, Cost, true>;
  // Shared memory of every Core.
  struct Common {
    alignas(8) uint64_t q_full[NT], s_full[NT], p_half[NT], p_full[NT], o_full[NT], drain;
    uint32_t tmem;
    volatile int abort, words[kAttnAnswers];
    int count;
    long long x;
    Frag frag[kFrags];
    typename Split::Smem split;
  };
};

// K: the Core. K::Smem derives from Common; K::init sets its own barriers; load_q and softmax are a softmax warpgroup's;
// K::work is a fragment's part of any other warp, with K::Other as its state, and K::leave its way out.
template <class K, class C>
struct TileFrame : TileShape<C> {
  using T = TileShape<C>;
  using T::DT; using T::D; using T::NT; using T::KEYS; using T::ROWS; using T::SOFT; using T::THREADS;
  using T::S_COL; using T::O_COL; using T::MMA_WARP;
  using typename T::Cost; using typename T::Split;
  using Smem = typename C::Smem;

  struct Soft {
    uint32_t s = 0, o = 0;  // tiles and fragments waited for
    uint32_t tiles = 0;     // key tiles up to the end of the fragment under way, those of units without this warpgroup's rows too
    bool q_ready = false;   // the next fragment's q has been loaded
  };
  // The two warpgroups take turns (named barriers 2 and 3; every thread passes them as often, whatever
  // failed): one makes the numerators of its tile while the other's products run. Without turns they fall
  // into step, both in their softmax and then both waiting for the tensor cores.
  static __device__ __forceinline__ void turn_wait(int x) { asm volatile("bar.sync %0, 256;" :: "r"(2 + x) : "memory"); }
  static __device__ __forceinline__ void turn_pass(int x) { asm volatile("bar.arrive %0, 256;" :: "r"(3 - x) : "memory"); }

  // Row r's place in out, and in lse (*at).
  static __device__ __forceinline__ char* out_row(const PagedAttnParams& p, const Frag& f, int r, int64_t* at) {
    const int32_t k = (int32_t)fast_div((uint32_t)r, p.group.magic, p.group.shift);
    const int64_t t = f.q0 + f.tok0 + k;
    const int h = f.h * p.G + r - k * p.G;
    *at = t * p.Hq + h;
    return row_ptr(p.out, t, p.o_rs, 2) + (int64_t)h * D * 2;
  }
  static __device__ __forceinline__ void put_lse(const PagedAttnParams& p, int64_t at, float m, float l) {
    p.lse[at] = attn_lse(m, l);
  }

  // The finished accumulator to out, or unnormalised to a workspace slot: m[ROWS], l[ROWS], then for every
  // four columns the rows' float4 side by side, so that a warp writes 512 bytes at a time.
  static __device__ __forceinline__ void finish(const PagedAttnParams& p, uint32_t tmem, const Frag& f, int x, float m,
                                                float l, float* slot) {
    const uint32_t oc = tmem + (((threadIdx.x >> 5) & 3) << 21) + O_COL + x * D;
    const int r = x * 128 + (threadIdx.x & 127);
    const bool live = r < f.rows;
    const float inv = attn_inverse(l);
    int64_t at = 0;
    char* out = live ? out_row(p, f, r, &at) : nullptr;
#pragma unroll 1
    for (int i = 0; i < D / 32; ++i) {
      uint32_t o[32];
      tc_ld32(oc + i * 32, o);
      tc_wait_ld<32>(o);
      if (live && slot) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          *reinterpret_cast<uint4*>(slot + 2 * ROWS + ((i * 8 + e) * ROWS + r) * 4) =
              make_uint4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
      } else if (live) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float v[8];
#pragma unroll
          for (int q = 0; q < 8; ++q) v[q] = __uint_as_float(o[8 * e + q]) * inv;
          st16(out + (i * 32 + e * 8) * 2, pack<DT>(v));
        }
      }
      __syncwarp();
    }
    tc_before();
    if (!live) return;
    if (slot) {
      slot[r] = m;
      slot[ROWS + r] = l;
    } else {
      put_lse(p, at, m, l);
    }
  }

  // Joins n slots, a thread per row, to out or (unnormalised) to dst, the first of them. own >= 0: slot
  // `own` is this block's accumulator in TMEM with its m and l.
  template <bool OWN, class At>
  static __device__ __forceinline__ void join(const PagedAttnParams& p, uint32_t tmem, const Frag& f, int x, int n, At at,
                                              float* dst, int own, float m_own, float l_own) {
    const int row = x * 128 + (threadIdx.x & 127), r = min(row, f.rows - 1);  // rows past the unit do the last's again
    const bool live = row < f.rows;
    const uint32_t oc = tmem + (((threadIdx.x >> 5) & 3) << 21) + O_COL + x * D;
    float m = OWN ? m_own : -INFINITY;
#pragma unroll 1
    for (int i = 0; i < n; i += 4) {  // four slots' maxima at a time (the last one's again past it)
      float z[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) z[e] = __ldcg(at(min(i + e, n - 1)) + r);
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (!OWN || min(i + e, n - 1) != own) m = fmaxf(m, z[e]);
    }
    const float base = m == -INFINITY ? 0.f : m;
    int64_t at_row = 0;
    char* out = out_row(p, f, r, &at_row);
    float l = 0.f;
    // 64 columns at a time, a slot at a time with all of its loads in flight: little code, which a block that
    // seldom comes here first has to fetch.
#pragma unroll 1
    for (int c = 0; c < D; c += 64) {
      float v[64];
#pragma unroll
      for (int e = 0; e < 64; ++e) v[e] = 0.f;
      l = 0.f;
#pragma unroll 1
      for (int i = 0; i < n; ++i) {
        if (OWN && i == own) {
          const float w = fast_exp2(m_own - base);
          l = fmaf(w, l_own, l);
#pragma unroll
          for (int d = 0; d < 64; d += 32) {
            uint32_t o[32];
            __syncwarp();
            tc_ld32(oc + c + d, o);
            tc_wait_ld<32>(o);
#pragma unroll
            for (int e = 0; e < 32; ++e) v[d + e] = fmaf(w, __uint_as_float(o[e]), v[d + e]);
          }
          continue;
        }
        const float* z = at(i);
        const float w = fast_exp2(__ldcg(z + r) - base);
        l = fmaf(w, __ldcg(z + ROWS + r), l);
        const float4* q = reinterpret_cast<const float4*>(z + 2 * ROWS) + c / 4 * ROWS + r;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const float4 a = __ldcg(q + e * ROWS);
          v[4 * e] = fmaf(w, a.x, v[4 * e]);
          v[4 * e + 1] = fmaf(w, a.y, v[4 * e + 1]);
          v[4 * e + 2] = fmaf(w, a.z, v[4 * e + 2]);
          v[4 * e + 3] = fmaf(w, a.w, v[4 * e + 3]);
        }
      }
      if (!live) continue;
      if (dst) {
#pragma unroll
        for (int e = 0; e < 16; ++e)
          *reinterpret_cast<float4*>(dst + 2 * ROWS + ((c / 4 + e) * ROWS + r) * 4) =
              make_float4(v[4 * e], v[4 * e + 1], v[4 * e + 2], v[4 * e + 3]);
      } else {
        const float inv = attn_inverse(l);
#pragma unroll
        for (int e = 0; e < 64; ++e) v[e] *= inv;
#pragma unroll
        for (int e = 0; e < 8; ++e) st16(out + (c + e * 8) * 2, pack<DT>(v + 8 * e));
      }
    }
    if (OWN) tc_before();
    if (!live) return;
    if (dst) {  // the group's first slot, whose m and l this thread has read
      dst[r] = m;
      dst[ROWS + r] = l;
    } else {
      put_lse(p, at_row, m, l);
    }
  }

  // One fragment of a softmax warpgroup. Both warpgroups pass the same named barriers, whatever failed.
  static __device__ __forceinline__ bool soft_fragment(const PagedAttnParams& p, Smem& s, uint32_t tmem, const Frag& f,
                                                       const Frag* next, int x, Soft& st, bool ok, float* slots,
                                                       uint32_t* counters) {
    constexpr int64_t SLOT = attn_slot_floats(ROWS, D);
    const int r = x * 128 + (threadIdx.x & 127);
    if (f.limit == 0) {  // no keys: never split
      if (ok && r < f.rows) {
        int64_t at;
        char* out = out_row(p, f, r, &at);
        for (int d = 0; d < D / 8; ++d) st16(out + d * 16, make_uint4(0, 0, 0, 0));
        put_lse(p, at, 0.f, 0.f);
      }
      return ok;
    }
    const AttnCuts cut{f.first, f.last};
    float* mine = cut.whole() ? nullptr : slots + cut.slot(blockIdx.x) * SLOT;
    const int n = (int)(cut.last - cut.first + 1), i0 = (int)(blockIdx.x - cut.first);
    const int groups = (n + kFanIn - 1) / kFanIn, gr = i0 / kFanIn, size = min(kFanIn, n - gr * kFanIn);
    const int64_t g0 = cut.first + (int64_t)gr * kFanIn;
    auto slot = [&](int64_t block) { return slots + cut.slot(block) * SLOT; };
    auto in_group = [&](int i) { return slot(g0 + i); };
    uint32_t* counter = counters + cut.slot(g0);
    const bool used = x == 0 || f.rows > 128;
    float m = -INFINITY, l = 0.f;
    st.tiles += (uint32_t)(f.t1 - f.t0);
    if (used) {
      if (ok && !st.q_ready) K::load_q(p, s, f, x);
      ok = K::softmax(p, s, tmem, f, x, st, ok, &m, &l);
      // the next unit's q before this one's end: its first scores are made meanwhile
      st.q_ready = ok && next && next->limit > 0 && (x == 0 || next->rows > 128);
      if (st.q_ready) K::load_q(p, s, *next, x);
    }
    // A unit that goes on past this block's run: the blocks after this one began with it, so they mostly are
    // done. Then this one's part is the last and is joined from TMEM without a turn through the workspace.
    const AttnBlock<1, SOFT> block{s.words, &s.abort};
    if (f.last > blockIdx.x && groups == 1 && attn_is_last(block, counter, (uint32_t)size)) {
      if (used && ok) join<true>(p, tmem, f, x, size, in_group, nullptr, i0, m, l);
      if (block.leader()) block.zero(counter);
      return ok;
    }
    if (used && ok) finish(p, tmem, f, x, m, l, mine);
    if (cut.whole()) return ok;
    if (attn_completes(block, counter, (uint32_t)size)) {
      if (used) join<false>(p, tmem, f, x, size, in_group, groups > 1 ? slot(g0) : nullptr, -1, 0.f, 0.f);
      if (groups > 1 && attn_completes(block, counters + 2 * gridDim.x + cut.slot(cut.first), (uint32_t)groups) && used)
        join<false>(p, tmem, f, x, groups, [&](int i) { return slot(cut.first + (int64_t)i * kFanIn); }, nullptr, -1, 0.f, 0.f);
    }
    return ok;
  }

  // ------------------------------------------------------------ the block
  // The place of tile x is looked for once, by a warp: its lanes try 32 row tiles at a time. The units after
  // it follow one another.
  static __device__ __forceinline__ void list(const PagedAttnParams& p, Smem& s, int64_t b0, int64_t x, int64_t run,
                                              const AttnShare& a) {
    int count = 0;
    const int64_t end = min(a.hi, run);
    const int32_t R = p.tokens;
    int rq = Split::find(p, s.split, a, x);
    Request r{s.split.q0[rq], s.split.n[rq], s.split.kv[rq]};
    int32_t nm = Cost::row_tiles(p, r), h, k = 0;
    int64_t start = s.split.pre[rq];  // the unit's first tile
    {
      const int64_t head = attn_div(s.split.pre[rq + 1] - start, p.Hkv);
      h = (int32_t)attn_div(x - start, head);
      start += h * head;
      int64_t at = 0;
      int32_t step = 1;
      while (step < nm) step *= 32;
      if (a.whole) {
        k = (int32_t)(x - start);
        at = k;
        step = 0;
      }
      for (step /= 32; step > 0; step /= 32) {  // before(k) <= x - start < before(k + 32 step)
        const int32_t mine = k + (int32_t)(threadIdx.x & 31) * step;
        const int64_t y = mine < nm ? Cost::before(p, r, mine, false) : INT64_MAX;
        const int last = 31 - __clz(__ballot_sync(0xffffffffu, y <= x - start));
        k += last * step;
        at = __shfl_sync(0xffffffffu, y, last);
      }
      start += at;
    }
    while (true) {
      Frag& f = s.frag[count++];
      f.b = b0 + rq;
      f.q0 = r.q0;
      f.n = r.n;
      f.kv = r.kv;
      f.h = h;
      f.tok0 = k * R;
      f.rows = min(R, r.n - k * R) * p.G;
      f.limit = Cost::sees(p, r, k);
      const int32_t nt = Cost::key_tiles(f.limit);
      f.t0 = a.whole ? 0 : (int32_t)(x - start);
      f.t1 = a.whole ? nt : (int32_t)min((int64_t)nt, f.t0 + (a.hi - x));
      f.first = start >= a.lo ? (int64_t)blockIdx.x : attn_div(start, a.per);
      f.last = a.whole || start + nt <= a.hi ? (int64_t)blockIdx.x : attn_div(start + nt - 1, a.per);
      x += a.whole ? 1 : f.t1 - f.t0;
      if (x >= end || count == kFrags) break;
      start = x;  // the unit ended inside the run: the next one
      if (++k == nm) {
        k = 0;
        if (++h == p.Hkv) {
          h = 0;
          do ++rq;
          while (s.split.pre[rq + 1] <= x);
          r = Request{s.split.q0[rq], s.split.n[rq], s.split.kv[rq]};
          nm = Cost::row_tiles(p, r);
        }
      }
    }
    s.count = count;
    s.x = x;
  }

  // Lists the fragments of the block's run, kFrags at a time, and has every warp go through them. All warps
  // pass the same block barriers, each role from its own copy of this loop.
  template <bool LISTS, class Body>
  static __device__ __forceinline__ void fragments(const PagedAttnParams& p, Smem& s, const AttnShare& a, Body body) {
    int64_t run = 0, x = a.lo;
    for (int64_t b0 = 0; b0 < p.B && x < a.hi; b0 += THREADS) {
      run = Split::chunk(p, s.split, b0, run, a);
      while (x < a.hi && x < run) {
        if (LISTS && threadIdx.x < 32) list(p, s, b0, x, run, a);
        __syncthreads();
        const int count = s.count;
        x = s.x;
        for (int i = 0; i < count; ++i) body(s.frag[i], i + 1 < count ? &s.frag[i + 1] : nullptr);
        __syncwarp();
        __syncthreads();
      }
    }
  }

  static __device__ __forceinline__ void run(const PagedAttnParams& p, const CUtensorMap* mk, const CUtensorMap* mv, Smem& s) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (warp == MMA_WARP) {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" :: "r"(smem_at(&s.tmem)) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
      if (lane == 0) {
        K::init(s);
        mb_init(smem_at(&s.drain), NT);
        for (int x = 0; x < NT; ++x) {
          mb_init(smem_at(&s.q_full[x]), 128);
          mb_init(smem_at(&s.s_full[x]), 1);
          mb_init(smem_at(&s.p_half[x]), 128);
          mb_init(smem_at(&s.p_full[x]), 128);
          mb_init(smem_at(&s.o_full[x]), 1);
        }
        s.abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
      }
      __syncwarp();
      tc_before();
    }
    pdl_trigger();
    bool work = true;
    const AttnStartBlock start{p.start};
    if (p.part == ATTN_ALL) {
      pdl_wait();
    } else {
      work = attn_starts(start);
      asm volatile("fence.proxy.async.global;" ::: "memory");  // the TMA loads, behind what the word or the wait brought
    }
    __syncthreads();
    tc_after();
    const uint32_t tmem = s.tmem;
    AttnShare a{};
    if (work) a = Split::share(p, s.split);
    uint32_t* counters = p.counters;
    float* slots = p.slots;
    typename K::Other other;
    bool ok = true;
    if (warp < MMA_WARP) {
      if constexpr (C::SOFT_REGS > T::LAUNCH_REGS) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" :: "n"(C::SOFT_REGS));
      Soft so;
      fragments<true>(p, s, a, [&](const Frag& f, const Frag* next) {
        ok = soft_fragment(p, s, tmem, f, next, warp / 4, so, ok, slots, counters);
      });
    } else {
      if constexpr (C::SOFT_REGS > T::LAUNCH_REGS) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" :: "n"(C::OTHER_REGS));
      const bool one = elect_one();
      fragments<false>(p, s, a, [&](const Frag& f, const Frag*) {
        if (f.limit > 0 && ok) ok = K::work(p, mk, mv, s, tmem, f, warp, other, one);
      });
    }
    if (p.part == ATTN_ALL) attn_fill_tail<THREADS>(p);
    else attn_ends(start);
    // the way out: every copy and product of the block has to be done before its memory is given back
    K::leave(p, s, warp, other, ok);
    if (warp >= MMA_WARP && warp < MMA_WARP + NT) {
      if (elect_one()) tc_commit(smem_at(&s.drain));  // warps without products of their own commit nothing, at once
      mb_drain(smem_at(&s.drain), 0);
    }
    __syncwarp();
    tc_before();
    __syncthreads();
    tc_after();
    if (threadIdx.x == 0 && s.abort) atomicOr(p.err, kErrTimeout);
    if (warp == MMA_WARP)
      asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" :: "r"(tmem) : "memory");
  }
};

template <class K>
__global__ void __launch_bounds__(K::THREADS, 1)
attn_tile_kernel(const __grid_constant__ PagedAttnParams p, const __grid_constant__ CUtensorMap mk,
                 const __grid_constant__ CUtensorMap mv) {
  extern __shared__ __align__(128) char smem[];
  char* at = smem + (1024 - (smem_at(smem) & 1023)) % 1024;  // swizzle atoms start at multiples of 1024
  K::run(p, &mk, &mv, *reinterpret_cast<typename K::Smem*>(at));
}

template <class K>
void attn_tile_pick(AttnEntry* e) {
  e->fn = (const void*)attn_tile_kernel<K>;
  e->threads = K::THREADS;
  e->smem = sizeof(typename K::Smem) + 1024;
  e->per_sm = 1;
  e->slot_floats = attn_slot_floats(K::ROWS, K::D);
  e->keys = K::KEYS;
  e->rows = K::ROWS;
  static_assert(sizeof(typename K::Smem) + 1024 <= 232448, "shared memory of a block");
}

}  // namespace trident
