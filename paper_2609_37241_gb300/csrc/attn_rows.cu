// attn_rows.cu -- paged attention for requests of few rows: decode steps, drafted tokens.
//
// Bound: HBM. A unit's 16 rows (of mma.m16n8k16; a decode step of G = 4 fills four) read every key once,
// 4 flops per byte and used row, so the legacy tensor instructions suffice and their padding rows cost
// nothing that the memory does not wait for. What matters is bytes in flight, so every warp is a stream
// of its own: it takes 16 keys of each 64-key tile, keeps a ring of NS stages (16 rows of k and of v)
// filled by cp.async and never waits for another warp until the fragment's end, where the four warps'
// (m, l, out) are joined in shared memory. Any page size and any strides: cp.async copies 16 bytes to
// where the swizzle puts them (chunk ^ row mod 8: ldmatrix reads eight rows from eight bank groups).
// Rows past the unit's last visible key are filled with zeros, not read.
//
// The running maximum moves only when a score passes it by 2^kLazy, so that the accumulators are seldom
// rescaled; the numerators stay below 2^kLazy, which fp16 and the fp32 sums hold easily. The numerators
// are rounded to the activation type for the product with v, the sum is taken before that.
#include "attn_common.cuh"

namespace trident {
namespace {

constexpr int kRowsThreads = 128;
constexpr int kRowsTile = 16;   // rows of a unit
constexpr int kRowsKeys = 64;   // keys of a tile, 16 per warp
constexpr float kLazy = 8.f;

template <int D>
struct RowsGeom {
  static constexpr int CH = D / 8;              // 16-byte chunks per row
  static constexpr int HALF = 16 * D * 2;       // bytes of a stage's k (and of its v)
  static constexpr int STAGE = 2 * HALF;
  static constexpr int NS = D == 64 ? 6 : 3;    // stages per warp: 24 KB in flight, D 256 48 KB
  static constexpr int RING = 4 * NS * STAGE;
  static constexpr int PER_SM = D == 256 ? 1 : 2;
  // after the ring's use, in its place: out of four warps, 16 rows each; then the joins' weights
  static constexpr int LDO = D + 4;
};

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
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" :: "n"(N) : "memory"); }

// A unit: 16 rows from r0 of request (q0, n, kv), kv head h.
struct Unit {
  int64_t b;
  int32_t q0, n, kv, h, r0, rows, limit;  // rows: of the 16 that exist; limit: keys that the last one sees
};

// Every row tile counted with all of the request's keys: exact for decode steps, a little unequal where a
// long chunk comes this way.
struct RowsCost {
  static __device__ __forceinline__ int64_t row_tiles(const PagedAttnParams& p, int32_t n) {
    return ((int64_t)n * p.G + kRowsTile - 1) / kRowsTile;
  }
  static __device__ __forceinline__ int64_t key_tiles(int32_t kv) {
    return kv > kRowsKeys ? ((int64_t)kv + kRowsKeys - 1) / kRowsKeys : 1;
  }
  static __device__ __forceinline__ int64_t units(const PagedAttnParams& p, const Request& r) {
    return (int64_t)p.Hkv * row_tiles(p, r.n);
  }
  static __device__ __forceinline__ int32_t longest(const PagedAttnParams&, const Request& r) { return (int32_t)key_tiles(r.kv); }
  static __device__ __forceinline__ int64_t of(const PagedAttnParams& p, const Request& r) {
    return units(p, r) * key_tiles(r.kv);
  }
};

template <int DT, int D>
struct RowsKernel {
  using G = RowsGeom<D>;
  using Split = AttnSplit<kRowsThreads, RowsCost>;
  struct Smem {
    alignas(128) char ring[G::RING];
    typename Split::Smem split;
    float m[4][16], l[4][16];
    int last;
  };

  // Issues the copies of 16 keys from j0 on into a stage.
  static __device__ __forceinline__ void load(const PagedAttnParams& p, const Unit& u, const char* kb, const char* vb,
                                              int32_t j0, uint32_t stage, bool* bad) {
    const int lane = threadIdx.x & 31;
    constexpr int RPI = 32 / G::CH > 0 ? 32 / G::CH : 1;  // rows per instruction (D 256: one)
    constexpr int ITER = 16 / RPI;
    const int c = lane % G::CH, rr = lane / G::CH;
    const int32_t* table = p.table + u.b * p.table_rs;
    if (p.page.d % 16 == 0) {  // one page for all 16 rows
      const uint32_t pg = fast_div((uint32_t)j0, p.page.magic, p.page.shift);
      const uint32_t at = (uint32_t)j0 - pg * (uint32_t)p.page.d;
      int64_t page = table[pg];
      if (page < 0 || page >= p.P) {
        *bad = true;
        page = 0;
      }
      const char* ks = kb + (page * p.kc.page + (int64_t)(at + rr) * p.kc.row + c * 8) * 2;
      const char* vs = vb + (page * p.vc.page + (int64_t)(at + rr) * p.vc.row + c * 8) * 2;
      const int64_t kstep = RPI * p.kc.row * 2, vstep = RPI * p.vc.row * 2;
#pragma unroll
      for (int i = 0; i < ITER; ++i) {
        const int r = rr + i * RPI;
        const bool live = j0 + r < u.limit;
        const uint32_t dst = stage + r * (D * 2) + ((c ^ (r & 7)) << 4);
        cp16(dst, live ? ks + i * kstep : kb, live);
        cp16(dst + G::HALF, live ? vs + i * vstep : vb, live);
      }
    } else {
#pragma unroll 2
      for (int i = 0; i < ITER; ++i) {
        const int r = rr + i * RPI;
        const bool live = j0 + r < u.limit;
        int64_t ko = 0, vo = 0;
        if (live) {
          const uint32_t j = (uint32_t)(j0 + r), pg = fast_div(j, p.page.magic, p.page.shift);
          const int64_t at = j - pg * (uint32_t)p.page.d;
          int64_t page = table[pg];
          if (page < 0 || page >= p.P) {
            *bad = true;
            page = 0;
          }
          ko = (page * p.kc.page + at * p.kc.row + c * 8) * 2;
          vo = (page * p.vc.page + at * p.vc.row + c * 8) * 2;
        }
        const uint32_t dst = stage + r * (D * 2) + ((c ^ (r & 7)) << 4);
        cp16(dst, kb + ko, live);
        cp16(dst + G::HALF, vb + vo, live);
      }
    }
  }

  // Key tiles [t0, t1) of a unit; leaves every warp's m, l and unnormalised out in shared memory.
  static __device__ __forceinline__ void fragment(const PagedAttnParams& p, Smem& s, const Unit& u, int64_t t0,
                                                  int64_t t1, bool* bad) {
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const char* kb = reinterpret_cast<const char*>(p.kc.base) + (int64_t)u.h * p.kc.head * 2;
    const char* vb = reinterpret_cast<const char*>(p.vc.base) + (int64_t)u.h * p.vc.head * 2;
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(s.ring) + w * (G::NS * G::STAGE);
    // this warp's 16-key groups: keys 16 (4 x + w), x in [t0, t1), up to the limit
    const int32_t first = (int32_t)t0 * kRowsKeys + 16 * w;
    const int32_t upto = (int32_t)min((int64_t)u.limit, t1 * kRowsKeys);
    const int groups = first < upto ? (upto - first + kRowsKeys - 1) / kRowsKeys : 0;
#pragma unroll
    for (int i = 0; i < G::NS - 1; ++i) {
      if (i < groups) load(p, u, kb, vb, first + i * kRowsKeys, ring + i * G::STAGE, bad);
      cp_commit();
    }
    // rows g and g + 8 of the unit: q and how far they see
    uint32_t qf[D / 16][4];
    int32_t see[2];
    {
      const char* src[2];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int32_t r = u.r0 + min(g + 8 * k, u.rows - 1);
        const int32_t i = (int32_t)fast_div((uint32_t)r, p.group.magic, p.group.shift);
        see[k] = u.kv - u.n + i + 1;
        src[k] = row_ptr(p.q, u.q0 + i, p.q_rs, 2) + ((int64_t)u.h * p.G + (r - i * p.G)) * D * 2;
      }
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          qf[kk][e] = *reinterpret_cast<const uint32_t*>(src[e & 1] + (kk * 16 + (e >> 1) * 8 + 2 * t) * 2);
    }
    const float c = p.scale * kLog2e;
    float o[D / 8][4];
#pragma unroll
    for (int i = 0; i < D / 8; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[i][e] = 0.f;
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
    const int mi = lane >> 3, mr = lane & 7;
    for (int x = 0; x < groups; ++x) {
      cp_wait<G::NS - 2>();
      __syncwarp();  // all lanes' copies have landed, and the stage refilled below has been read
      {
        const int y = x + G::NS - 1;
        if (y < groups) load(p, u, kb, vb, first + y * kRowsKeys, ring + (y % G::NS) * G::STAGE, bad);
        cp_commit();
      }
      const uint32_t st = ring + (x % G::NS) * G::STAGE;
      float sc[2][4] = {};
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk) {
        uint32_t kf[4];
        const int key = (mi >> 1) * 8 + mr, ch = kk * 2 + (mi & 1);
        ldsm4(kf, st + key * (D * 2) + ((ch ^ (key & 7)) << 4));
        mma16816<DT>(sc[0], qf[kk], kf[0], kf[1]);
        mma16816<DT>(sc[1], qf[kk], kf[2], kf[3]);
      }
      const int32_t j0 = first + x * kRowsKeys;
      if (j0 + 16 > min(see[0], see[1]))  // some key is hidden from a row
#pragma unroll
        for (int nt = 0; nt < 2; ++nt)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (j0 + nt * 8 + 2 * t + (e & 1) >= see[e >> 1]) sc[nt][e] = -INFINITY;
      float top[2];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        top[k] = fmaxf(fmaxf(sc[0][2 * k], sc[0][2 * k + 1]), fmaxf(sc[1][2 * k], sc[1][2 * k + 1]));
        top[k] = fmaxf(top[k], __shfl_xor_sync(0xffffffffu, top[k], 1));
        top[k] = c * fmaxf(top[k], __shfl_xor_sync(0xffffffffu, top[k], 2));
      }
      if (__any_sync(0xffffffffu, top[0] > m[0] + kLazy || top[1] > m[1] + kLazy)) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const float m2 = fmaxf(m[k], top[k]);
          const float f = m2 == -INFINITY ? 1.f : fast_exp2(m[k] - m2);
          m[k] = m2;
          l[k] *= f;
#pragma unroll
          for (int i = 0; i < D / 8; ++i) {
            o[i][2 * k] *= f;
            o[i][2 * k + 1] *= f;
          }
        }
      }
      uint32_t pf[4];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const float base = m[k] == -INFINITY ? 0.f : m[k];
#pragma unroll
        for (int nt = 0; nt < 2; ++nt) {
          const float e0 = fast_exp2(fmaf(sc[nt][2 * k], c, -base)), e1 = fast_exp2(fmaf(sc[nt][2 * k + 1], c, -base));
          l[k] += e0 + e1;
          pf[2 * nt + k] = ActType<DT>::pack2(e0, e1);
        }
      }
#pragma unroll
      for (int dd = 0; dd < D / 16; ++dd) {
        uint32_t vf[4];
        const int key = (mi & 1) * 8 + mr, ch = dd * 2 + (mi >> 1);
        ldsm4t(vf, st + G::HALF + key * (D * 2) + ((ch ^ (key & 7)) << 4));
        mma16816<DT>(o[2 * dd], pf, vf[0], vf[1]);
        mma16816<DT>(o[2 * dd + 1], pf, vf[2], vf[3]);
      }
    }
    cp_wait<0>();
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      l[k] += __shfl_xor_sync(0xffffffffu, l[k], 1);
      l[k] += __shfl_xor_sync(0xffffffffu, l[k], 2);
    }
    __syncthreads();  // every warp is done with its ring: the partial outs take its place
    float* so = reinterpret_cast<float*>(s.ring);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int row = g + 8 * k;
      if (row < u.rows) {
        if (t == 0) {
          s.m[w][row] = m[k];
          s.l[w][row] = l[k];
        }
#pragma unroll
        for (int i = 0; i < D / 8; ++i)
          *reinterpret_cast<float2*>(so + (w * 16 + row) * G::LDO + i * 8 + 2 * t) = make_float2(o[i][2 * k], o[i][2 * k + 1]);
      }
    }
    __syncthreads();
  }

  // Joins the four warps of a fragment: into out and lse, or unnormalised into a workspace slot.
  static __device__ __forceinline__ void join_warps(const PagedAttnParams& p, Smem& s, const Unit& u, float* slot) {
    const float* so = reinterpret_cast<const float*>(s.ring);
    for (int e = threadIdx.x; e < u.rows * (D / 4); e += kRowsThreads) {
      const int row = e / (D / 4), d = e % (D / 4) * 4;
      float m = -INFINITY;
#pragma unroll
      for (int w = 0; w < 4; ++w) m = fmaxf(m, s.m[w][row]);
      const float base = m == -INFINITY ? 0.f : m;
      float l = 0.f;
      float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const float f = fast_exp2(s.m[w][row] - base);
        const float4 v = *reinterpret_cast<const float4*>(so + (w * 16 + row) * G::LDO + d);
        l = fmaf(f, s.l[w][row], l);
        a.x = fmaf(f, v.x, a.x); a.y = fmaf(f, v.y, a.y); a.z = fmaf(f, v.z, a.z); a.w = fmaf(f, v.w, a.w);
      }
      if (slot) {
        *reinterpret_cast<float4*>(slot + 2 * kRowsTile + row * D + d) = a;
        if (d == 0) {
          slot[row] = m;
          slot[kRowsTile + row] = l;
        }
      } else {
        put(p, u, row, d, a, m, l);
      }
    }
  }

  // Four elements of a finished row.
  static __device__ __forceinline__ void put(const PagedAttnParams& p, const Unit& u, int row, int d, const float4& a,
                                             float m, float l) {
    const int32_t r = u.r0 + row, i = (int32_t)fast_div((uint32_t)r, p.group.magic, p.group.shift);
    const int64_t t = u.q0 + i;
    const int h = u.h * p.G + (r - i * p.G);
    const float inv = l > 0.f ? 1.f / l : 0.f;
    uint2 v;
    v.x = ActType<DT>::pack2(a.x * inv, a.y * inv);
    v.y = ActType<DT>::pack2(a.z * inv, a.w * inv);
    *reinterpret_cast<uint2*>(row_ptr(p.out, t, p.o_rs, 2) + ((int64_t)h * D + d) * 2) = v;
    if (d == 0) p.lse[t * p.Hq + h] = l > 0.f ? (m + log2f(l)) * kLn2 : -INFINITY;
  }

  // Joins n workspace slots, `at(i)` the i-th; as join_warps otherwise (dst may be the first of them).
  template <class At>
  static __device__ __forceinline__ void join_slots(const PagedAttnParams& p, Smem& s, const Unit& u, int n, At at,
                                                    float* dst) {
    for (int e = threadIdx.x; e < u.rows * (D / 4); e += kRowsThreads) {
      const int row = e / (D / 4), d = e % (D / 4) * 4;
      float m = -INFINITY;
#pragma unroll 4
      for (int i = 0; i < n; ++i) m = fmaxf(m, __ldcg(at(i) + row));
      const float base = m == -INFINITY ? 0.f : m;
      float l = 0.f;
      float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
      for (int i = 0; i < n; ++i) {
        const float* z = at(i);
        const float f = fast_exp2(__ldcg(z + row) - base);
        const float4 v = __ldcg(reinterpret_cast<const float4*>(z + 2 * kRowsTile + row * D + d));
        l = fmaf(f, __ldcg(z + kRowsTile + row), l);
        a.x = fmaf(f, v.x, a.x); a.y = fmaf(f, v.y, a.y); a.z = fmaf(f, v.z, a.z); a.w = fmaf(f, v.w, a.w);
      }
      if (dst) {
        *reinterpret_cast<float4*>(dst + 2 * kRowsTile + row * D + d) = a;
        if (d == 0) {
          s.m[0][row] = m;
          s.l[0][row] = l;
        }
      } else {
        put(p, u, row, d, a, m, l);
      }
    }
    if (dst) {  // m and l last (dst is a slot, whose m and l every thread of the row reads)
      __syncthreads();
      if (threadIdx.x < u.rows) {
        dst[threadIdx.x] = s.m[0][threadIdx.x];
        dst[kRowsTile + threadIdx.x] = s.l[0][threadIdx.x];
      }
    }
  }

  static __device__ __forceinline__ void run(const PagedAttnParams& p, Smem& s) {
    const AttnShare a = Split::share(p, s.split);
    attn_fill_tail<kRowsThreads>(p);
    uint32_t* counters = reinterpret_cast<uint32_t*>(p.work);
    float* slots = p.work + attn_counters(gridDim.x);
    constexpr int64_t SLOT = attn_slot_floats(kRowsTile, D);
    bool bad = false;
    int64_t run = 0, x = a.lo;
    for (int64_t b0 = 0; b0 < p.B && x < a.hi; b0 += kRowsThreads) {
      run = Split::chunk(p, s.split, b0, run, a);
      while (x < a.hi && x < run) {
        const int rq = Split::find(s.split, x);
        Unit u;
        u.b = b0 + rq;
        u.q0 = s.split.q0[rq];
        u.n = s.split.n[rq];
        u.kv = s.split.kv[rq];
        const int64_t nt = RowsCost::key_tiles(u.kv), nm = RowsCost::row_tiles(p, u.n);
        const int64_t rel = x - s.split.pre[rq], unit = rel / nt, t0 = rel - unit * nt;
        const int64_t t1 = min(nt, t0 + a.hi - x);
        u.h = (int32_t)(unit / nm);
        u.r0 = (int32_t)(unit - u.h * nm) * kRowsTile;
        u.rows = (int32_t)min((int64_t)kRowsTile, (int64_t)u.n * p.G - u.r0);
        const int32_t ilast = (int32_t)fast_div((uint32_t)(u.r0 + u.rows - 1), p.group.magic, p.group.shift);
        u.limit = max(0, min(u.kv, u.kv - u.n + ilast + 1));
        fragment(p, s, u, t0, t1, &bad);
        const int64_t start = x - t0;  // the unit's first tile
        AttnCuts cut{start / a.per, (start + nt - 1) / a.per};
        if (cut.whole()) {
          join_warps(p, s, u, nullptr);
        } else {
          float* mine = slots + cut.slot(blockIdx.x) * SLOT;
          join_warps(p, s, u, mine);
          const int n = (int)(cut.last - cut.first + 1), f = (int)(blockIdx.x - cut.first);
          const int groups = (n + kFanIn - 1) / kFanIn, gr = f / kFanIn;
          const int64_t g0 = cut.first + (int64_t)gr * kFanIn;
          const int size = min(kFanIn, n - gr * kFanIn);
          auto slot = [&](int64_t block) { return slots + cut.slot(block) * SLOT; };
          if (attn_completes<0, kRowsThreads>(&s.last, threadIdx.x == 0, counters + cut.slot(g0), size)) {
            join_slots(p, s, u, size, [&](int i) { return slot(g0 + i); }, groups > 1 ? slot(g0) : nullptr);
            if (groups > 1 && attn_completes<0, kRowsThreads>(&s.last, threadIdx.x == 0,
                                                            counters + 2 * gridDim.x + cut.slot(cut.first), groups))
              join_slots(p, s, u, groups, [&](int i) { return slot(cut.first + (int64_t)i * kFanIn); }, nullptr);
          }
        }
        __syncthreads();  // the shared partial outs have been read
        x += t1 - t0;
      }
    }
    if (bad) atomicOr(p.err, kErrTable);
  }
};

template <int DT, int D>
__global__ void __launch_bounds__(kRowsThreads, RowsGeom<D>::PER_SM) attn_rows_kernel(const PagedAttnParams p) {
  extern __shared__ __align__(128) char smem[];
  // After the tile kernel of the same call, which waits for everything before it and only then lets this
  // launch start, nothing has to be waited for: the two write different rows. This grid then must not be
  // over before that one, so the wait comes last.
  pdl_trigger();
  if (!p.beside) pdl_wait();
  using K = RowsKernel<DT, D>;
  K::run(p, *reinterpret_cast<typename K::Smem*>(smem));
  if (p.beside) pdl_wait();
}

template <int DT, int D>
void pick(AttnEntry* e) {
  e->fn = (const void*)attn_rows_kernel<DT, D>;
  e->threads = kRowsThreads;
  e->smem = sizeof(typename RowsKernel<DT, D>::Smem);
  e->per_sm = RowsGeom<D>::PER_SM;
  e->slot_floats = attn_slot_floats(kRowsTile, D);
}

}  // namespace

bool attn_rows_entry(int32_t dtype, int32_t D, AttnEntry* e) {
  *e = AttnEntry{};
  if (D == 64) dtype == DT_BF16 ? pick<DT_BF16, 64>(e) : pick<DT_FP16, 64>(e);
  else if (D == 128) dtype == DT_BF16 ? pick<DT_BF16, 128>(e) : pick<DT_FP16, 128>(e);
  else if (D == 256) dtype == DT_BF16 ? pick<DT_BF16, 256>(e) : pick<DT_FP16, 256>(e);
  return e->fn != nullptr;
}

}  // namespace trident
