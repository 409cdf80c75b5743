// attn_rows.cuh -- paged attention for requests of few rows: what does not depend on how the cache holds its
// elements. A Core (attn_rows.cu: 16 bits, attn_rows8.cu: 8) has a warp go through its share of a fragment's keys;
// here are a call's units, the split over the blocks, and the joining of warps and blocks.
//
// A unit's 16 rows (of mma.m16n8k16) read every key once. Every warp is a stream of its own: it takes a fourth of each
// tile's keys, keeps a ring of stages of them filled by cp.async and never waits for another warp until the
// fragment's end, where the four warps' (m, l, out) are joined in shared memory.
#pragma once
#include "attn_common.cuh"

namespace trident {

constexpr int kRowsThreads = 128;
constexpr int kRowsTile = 16;   // rows of a unit
// The running maximum moves only when a score passes it by 2^kRowsLazy, so that the accumulators are seldom rescaled.
constexpr float kRowsLazy = 8.f;

template <int DT>
__device__ __forceinline__ void mma16816(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
  if constexpr (DT == DT_BF16)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void ldsm4(uint32_t* r, uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t* r, uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void cp16(uint32_t dst, const void* src, bool live) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" :: "r"(dst), "l"(src), "r"(live ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" :: "r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" :: "n"(N) : "memory"); }

// A fragment of a unit: 16 rows from r0 of request (q0, n, kv), kv head h, key tiles [t0, t1).
struct Unit {
  int64_t b, first, last;                 // request; blocks that share the unit
  int32_t q0, n, kv, h, r0, rows, limit;  // rows: of the 16 that exist; limit: keys that the last one sees
  int32_t t0, t1;
};

// Every row tile counted with all of the request's keys: exact for decode steps, a little unequal where a
// long chunk comes this way; and with kUnitTiles for its beginning and end, which take a block as long as
// that many tiles do (a block of many short units would otherwise be the last: 48 requests of about 3 rows of
// D 64, the slowest block 38.9 us, the median one 28.7; with tiles of 128 keys 3 is still the best of 1 to 3).
// A cut in these tiles moves to the unit's beginning.
constexpr int kUnitTiles = 3;
template <int KEYS>
struct RowsCost {
  static __device__ __forceinline__ int64_t row_tiles(const PagedAttnParams& p, int32_t n) {
    return ((int64_t)n * p.G + kRowsTile - 1) / kRowsTile;
  }
  static __device__ __forceinline__ int64_t key_tiles(int32_t kv) {
    return kv > KEYS ? ((int64_t)kv + KEYS - 1) / KEYS : 1;
  }
  static __device__ __forceinline__ int64_t of(const PagedAttnParams& p, const Request& r) {
    return p.Hkv * row_tiles(p, r.n) * (key_tiles(r.kv) + kUnitTiles);
  }
};

// Core: DT, D; G with KEYS (of a tile), RING (bytes), PASS (rows that the warps join at a time: a float4 per thread) and
// LDO (a row's floats there); Extra, its own shared memory; State, what a warp holds between a fragment's first loads
// and its last product; start() those loads, body() the rest, spill() a row's elements of the accumulators.
template <class Core>
struct RowsKernel {
  static constexpr int DT = Core::DT, D = Core::D;
  using G = typename Core::G;
  using Cost = RowsCost<G::KEYS>;
  using Split = AttnSplit<kRowsThreads, Cost, false>;
  struct Smem {
    alignas(128) char ring[G::RING];
    typename Core::Extra extra;
    alignas(16) float part[4][G::PASS][G::LDO];
    typename Split::Smem split;
    float m[4][16], l[4][16];
    volatile int words[kAttnAnswers];
  };

  // Four elements of a row over slots at(i), i < n, in their order, eight at a time whose m, l and elements
  // come in one round of loads; slot `own` is the part (a0, l0, m0) itself, as if it had gone through it.
  template <class At>
  static __device__ __forceinline__ void add_slots(float4& a, float& l, float& m, int row, int d, int n, At at, int own,
                                                   const float4& a0, float l0, float m0) {
    a = make_float4(0.f, 0.f, 0.f, 0.f);
    l = 0.f;
    m = -INFINITY;
    for (int i0 = 0; i0 < n; i0 += 8) {
      float4 v[8];
      float ms[8], ls[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int i = min(i0 + e, n - 1);
        const float* z = at(i);
        v[e] = a0;
        ms[e] = m0;
        ls[e] = l0;
        if (i != own) {
          ms[e] = __ldcg(z + row);
          ls[e] = __ldcg(z + kRowsTile + row);
          v[e] = __ldcg(reinterpret_cast<const float4*>(z + 2 * kRowsTile + row * D + d));
        }
      }
      float m2 = m;
#pragma unroll
      for (int e = 0; e < 8; ++e) m2 = fmaxf(m2, ms[e]);
      const float base = m2 == -INFINITY ? 0.f : m2, old = fast_exp2(m - base);
      m = m2;
      l *= old;
      a.x *= old; a.y *= old; a.z *= old; a.w *= old;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (i0 + e >= n) continue;
        const float f = fast_exp2(ms[e] - base);
        l = fmaf(f, ls[e], l);
        a.x = fmaf(f, v[e].x, a.x); a.y = fmaf(f, v[e].y, a.y); a.z = fmaf(f, v[e].z, a.z); a.w = fmaf(f, v[e].w, a.w);
      }
    }
  }

  // Joins the four warps of a fragment, PASS rows at a time: into out and lse; unnormalised into a workspace
  // slot; or, where it is the unit's last part, with the n - 1 other slots `at(i)`, i != own, into out and lse.
  template <class At>
  static __device__ __forceinline__ void join_warps(const PagedAttnParams& p, Smem& s, const Unit& u, const float* m,
                                                    const float* l, const float (*o)[4], float* slot, int n, int own, At at) {
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
#pragma unroll
    for (int k = 0; k < 2; ++k)
      if (t == 0) {
        s.m[w][g + 8 * k] = m[k];
        s.l[w][g + 8 * k] = l[k];
      }
    for (int p0 = 0; p0 < u.rows; p0 += G::PASS) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int row = g + 8 * k;
        if (row >= p0 && row < p0 + G::PASS) {
          Core::spill(s.part[w][row - p0], o, k, t);
        }
      }
      __syncthreads();
      const int at_row = threadIdx.x / (D / 4), row = p0 + at_row, d = threadIdx.x % (D / 4) * 4;
      if (row < u.rows) {
        float mm = -INFINITY, ll = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) mm = fmaxf(mm, s.m[i][row]);
        const float base = mm == -INFINITY ? 0.f : mm;
        float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float f = fast_exp2(s.m[i][row] - base);
          const float4 v = *reinterpret_cast<const float4*>(&s.part[i][at_row][d]);
          ll = fmaf(f, s.l[i][row], ll);
          a.x = fmaf(f, v.x, a.x); a.y = fmaf(f, v.y, a.y); a.z = fmaf(f, v.z, a.z); a.w = fmaf(f, v.w, a.w);
        }
        if (n > 0) {
          const float4 a0 = a;
          const float l0 = ll, m0 = mm;
          add_slots(a, ll, mm, row, d, n, at, own, a0, l0, m0);
        }
        if (slot) {
          *reinterpret_cast<float4*>(slot + 2 * kRowsTile + row * D + d) = a;
          if (d == 0) {
            slot[row] = mm;
            slot[kRowsTile + row] = ll;
          }
        } else {
          put(p, u, row, d, a, mm, ll);
        }
      }
      __syncthreads();
    }
  }

  // Four elements of a finished row.
  static __device__ __forceinline__ void put(const PagedAttnParams& p, const Unit& u, int row, int d, const float4& a,
                                             float m, float l) {
    const int32_t r = u.r0 + row, i = (int32_t)fast_div((uint32_t)r, p.group.magic, p.group.shift);
    const int64_t t = u.q0 + i;
    const int h = u.h * p.G + (r - i * p.G);
    const float inv = attn_inverse(l);
    uint2 v;
    v.x = ActType<DT>::pack2(a.x * inv, a.y * inv);
    v.y = ActType<DT>::pack2(a.z * inv, a.w * inv);
    *reinterpret_cast<uint2*>(row_ptr(p.out, t, p.o_rs, 2) + ((int64_t)h * D + d) * 2) = v;
    if (d == 0) p.lse[t * p.Hq + h] = attn_lse(m, l);
  }

  // Joins n workspace slots, `at(i)` the i-th, into out and lse or into dst, the first of them.
  template <class At>
  static __device__ __forceinline__ void join_slots(const PagedAttnParams& p, Smem& s, const Unit& u, int n, At at,
                                                    float* dst) {
    for (int e0 = 0; e0 < u.rows * (D / 4); e0 += kRowsThreads) {  // whole rounds: see the barrier below
      const int e = e0 + threadIdx.x, row = min(e / (D / 4), u.rows - 1), d = e % (D / 4) * 4;
      const bool live = e < u.rows * (D / 4);
      float m, l;
      float4 a;
      add_slots(a, l, m, row, d, n, at, -1, make_float4(0.f, 0.f, 0.f, 0.f), 0.f, 0.f);
      if (dst) __syncthreads();  // dst is one of the slots: its m and l are read by all threads of the row first
      if (!live) continue;
      if (dst) {
        *reinterpret_cast<float4*>(dst + 2 * kRowsTile + row * D + d) = a;
        if (d == 0) {
          dst[row] = m;
          dst[kRowsTile + row] = l;
        }
      } else {
        put(p, u, row, d, a, m, l);
      }
    }
  }

  // The end of a fragment whose keys are done.
  static __device__ __forceinline__ void finish(const PagedAttnParams& p, Smem& s, const Unit& u, const float* m,
                                                const float* l, const float (*o)[4]) {
    uint32_t* counters = p.counters;
    float* slots = p.slots;
    constexpr int64_t SLOT = attn_slot_floats(kRowsTile, D);
    const AttnCuts cut{u.first, u.last};
    const int n = (int)(cut.last - cut.first + 1), f = (int)(blockIdx.x - cut.first);
    const int groups = (n + kFanIn - 1) / kFanIn, gr = f / kFanIn;
    const int64_t g0 = cut.first + (int64_t)gr * kFanIn;
    const int size = min(kFanIn, n - gr * kFanIn);
    uint32_t* counter = counters + cut.slot(g0);
    auto slot = [&](int64_t block) { return slots + cut.slot(block) * SLOT; };
    auto in_group = [&](int i) { return slot(g0 + i); };
    // A unit that goes on past this block's run: the blocks after this one began with it, so they mostly are
    // done, and this part is joined with theirs without a turn through the workspace.
    const AttnBlock<0, kRowsThreads> block{s.words, nullptr};
    const bool last = u.last > blockIdx.x && groups == 1 && attn_is_last(block, counter, (uint32_t)size);
    const bool done = cut.whole() || last;
    join_warps(p, s, u, m, l, o, done ? nullptr : slot(blockIdx.x), last ? size : 0, f, in_group);
    if (last && block.leader()) block.zero(counter);
    if (done) return;
    if (attn_completes(block, counter, (uint32_t)size)) {
      join_slots(p, s, u, size, in_group, groups > 1 ? slot(g0) : nullptr);
      if (groups > 1 && attn_completes(block, counters + 2 * gridDim.x + cut.slot(cut.first), (uint32_t)groups))
        join_slots(p, s, u, groups, [&](int i) { return slot(cut.first + (int64_t)i * kFanIn); }, nullptr);
    }
  }

  static __device__ __forceinline__ void run(const PagedAttnParams& p, Smem& s) {
    const AttnShare a = Split::share(p, s.split);
    if (p.part == ATTN_FEW) {
      const AttnStartBlock block{p.start};
      attn_sets_start(block, a.others);
      pdl_trigger();
    }
    bool bad = false;
    int64_t run = 0, x = a.lo;
    for (int64_t b0 = 0; b0 < p.B && x < a.hi; b0 += kRowsThreads) {
      run = Split::chunk(p, s.split, b0, run, a);
      const int64_t end = min(a.hi, run);
      if (x >= end) continue;
      // the unit that holds x; those after it follow one another
      int rq = Split::find(p, s.split, a, x);
      Unit u;
      int64_t start_of;  // its first tile, of kUnitTiles + nt
      int32_t nt, nm, mt;
      auto request_of = [&]() {
        u.b = b0 + rq;
        u.q0 = s.split.q0[rq];
        u.n = s.split.n[rq];
        u.kv = s.split.kv[rq];
        nt = (int32_t)Cost::key_tiles(u.kv);
        nm = (int32_t)Cost::row_tiles(p, u.n);
      };
      request_of();
      {
        const int64_t unit = attn_div(x - s.split.pre[rq], nt + kUnitTiles);
        start_of = s.split.pre[rq] + unit * (nt + kUnitTiles);
        u.h = (int32_t)attn_div(unit, nm);
        mt = (int32_t)(unit - (int64_t)u.h * nm);
      }
      // This block's part of the unit at x; false where its run ends before the unit's keys.
      auto part = [&]() {
        const int64_t keys = start_of + kUnitTiles;
        u.t0 = (int32_t)max((int64_t)0, x - keys);
        u.t1 = (int32_t)min((int64_t)nt, a.hi - keys);
        u.first = keys >= a.lo ? (int64_t)blockIdx.x : attn_div(keys, a.per);
        u.last = keys + nt <= a.hi ? (int64_t)blockIdx.x : attn_div(keys + nt - 1, a.per);
        u.r0 = mt * kRowsTile;
        u.rows = (int32_t)min((int64_t)kRowsTile, (int64_t)u.n * p.G - u.r0);
        const int32_t ilast = (int32_t)fast_div((uint32_t)(u.r0 + u.rows - 1), p.group.magic, p.group.shift);
        u.limit = max(0, min(u.kv, u.kv - u.n + ilast + 1));
        x = keys + nt;
        return u.t1 > u.t0;
      };
      typename Core::State st;
      st.buf = 0;
      bool more = part();
      if (more) Core::start(p, s.ring, s.extra, u, st, &bad);
      if (G::QS) __syncthreads();  // q in shared memory
      while (more) {
        float m[2], l[2], o[D / 8][4];
        Core::body(p, s.ring, s.extra, u, st, m, l, o, &bad);
        const Unit done = u;
        more = x < end;
        if (more) {
          start_of = x;
          if (++mt == nm) {
            mt = 0;
            if (++u.h == p.Hkv) {
              u.h = 0;
              do ++rq;
              while (s.split.pre[rq + 1] <= x);
              request_of();
            }
          }
          more = part();
          if (more) Core::start(p, s.ring, s.extra, u, st, &bad);
        }
        finish(p, s, done, m, l, o);
      }
      x = max(x, end);  // a last unit of which only the beginning's tiles were this block's
    }
    attn_fill_tail<kRowsThreads>(p);
    if (bad) atomicOr(p.err, kErrTable);
  }
};

}  // namespace trident
