// attn_rows.cu -- paged attention for requests of few rows: decode steps, drafted tokens.
//
// Bound: HBM. A unit's 16 rows (of mma.m16n8k16; a decode step of G = 4 fills four) read every key once,
// 4 flops per byte and used row, so the legacy tensor instructions suffice and their padding rows cost
// nothing that the memory does not wait for. What matters is bytes in flight, so every warp is a stream
// of its own: it takes a fourth of each tile's keys (16 of 64; heads of 64: 32 of 128), keeps a ring of NS
// stages of them filled by cp.async and never waits for another warp until the fragment's end, where the four
// warps' (m, l, out) are joined in shared memory. Any page size and any strides: cp.async copies 16 bytes to
// where the swizzle puts them (chunk ^ row mod 8: ldmatrix reads eight rows from eight bank groups).
// Rows past the unit's last visible key are filled with zeros, not read.
//
// The running maximum moves only when a score passes it by 2^kLazy, so that the accumulators are seldom
// rescaled; the numerators stay below 2^kLazy (fp16: 2^15, ActType::kUp), which the type and the fp32 sums hold.
// They are rounded to the activation type for the product with v, the sum is taken before that.
//
// Measured on a GB300 (32 q heads on 8 kv heads of 128 where nothing else is said; of the 6.79 TB/s copy
// rate): 64 requests of 1000 to 8000 keys 178 us (0.99), 3 of 131071 keys 242 us (0.98), 64 of 4000 keys with
// 4 kv heads of 256 161 us (0.96); one request of 1000 keys 8.5 us, four dependent rounds of loads and the
// join of its parts.
#include "attn_common.cuh"

namespace trident {
namespace {

constexpr int kRowsThreads = 128;
constexpr int kRowsTile = 16;   // rows of a unit
constexpr float kLazy = 8.f;

template <int D>
struct RowsGeom {
  static constexpr int CH = D / 8;              // 16-byte chunks per row
  // 16-key groups that a warp takes at a time. Heads of 64: two, since the fixed part of a step (waits, the
  // maximum's exchange, page numbers) and its chain of dependent instructions bound it before the memory does:
  // 48 requests of about 3 rows 37.5 -> 30.8 us, 200 decode steps of 1700 keys 125 -> 113 us.
  static constexpr int KG = D == 64 ? 2 : 1;
  static constexpr int KEYS = 64 * KG;          // keys of a tile, a fourth of them per warp
  static constexpr int HALF = 16 * KG * D * 2;  // bytes of a stage's k (and of its v)
  static constexpr int STAGE = 2 * HALF;
  static constexpr int NS = 3;                  // stages per warp: 24 KB, D 256 48 KB
  static constexpr int RING = 4 * NS * STAGE;
  static constexpr int PER_SM = D == 256 ? 1 : 2;
  static constexpr int PASS = 512 / D;          // rows that the warps join at a time: a float4 per thread
  static constexpr int LDO = D + 4;
  // q in registers; for D 256, whose accumulators fill them, in shared memory, a buffer for the fragment under
  // way and one for the next
  static constexpr bool QS = D > 128;
  static constexpr int QREG = QS ? 1 : D / 16, QBUF = QS ? 16 * D * 2 : 16;
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

template <int DT, int D>
struct RowsKernel {
  using G = RowsGeom<D>;
  static constexpr int KG = G::KG, KEYS = G::KEYS, WARP = 16 * KG;  // WARP: keys of a tile that are one warp's
  using Cost = RowsCost<KEYS>;
  using Split = AttnSplit<kRowsThreads, Cost, false>;
  struct Smem {
    alignas(128) char ring[G::RING];
    alignas(128) char q[2][G::QBUF];
    alignas(16) float part[4][G::PASS][G::LDO];
    typename Split::Smem split;
    float m[4][16], l[4][16];
    volatile int words[kAttnAnswers];
  };

  // The table's entry for the lane's row (lane mod WARP) of the keys from j0 on. It is asked for a stage
  // before its copies are issued, so that they do not wait for it.
  static __device__ __forceinline__ int32_t entry(const PagedAttnParams& p, const Unit& u, int32_t j0) {
    const uint32_t j = (uint32_t)min(j0 + (int32_t)(threadIdx.x & (WARP - 1)), u.limit - 1);
    return p.table[u.b * p.table_rs + fast_div(j, p.page.magic, p.page.shift)];
  }

  // Issues the copies of WARP keys from j0 on into a stage; page: what entry() gave for them.
  static __device__ __forceinline__ void load(const PagedAttnParams& p, const Unit& u, const char* kb, const char* vb,
                                              int32_t j0, int32_t page, uint32_t stage, bool* bad) {
    const int lane = threadIdx.x & 31;
    constexpr int RPI = 32 / G::CH > 0 ? 32 / G::CH : 1;  // rows per instruction (D 256: one)
    constexpr int ITER = 16 / RPI;  // for 16 rows
    const int c = lane % G::CH, rr = lane / G::CH;
    if (page < 0 || page >= p.P) {
      *bad = true;
      page = 0;
    }
    const uint32_t j = (uint32_t)min(j0 + (lane & (WARP - 1)), u.limit - 1);
    const int32_t at = (int32_t)(j - fast_div(j, p.page.magic, p.page.shift) * (uint32_t)p.page.d);
    if (p.page.d % 16 == 0) {  // one page for 16 rows
      const int64_t kstep = RPI * p.kc.row * 2, vstep = RPI * p.vc.row * 2;
#pragma unroll
      for (int h = 0; h < KG; ++h) {
        const int32_t at0 = __shfl_sync(0xffffffffu, at, 16 * h);
        const int32_t pg = KG == 1 ? page : __shfl_sync(0xffffffffu, page, 16 * h);
        const char* ks = kb + ((int64_t)pg * p.kc.page + (int64_t)(at0 + rr) * p.kc.row + c * 8) * 2;
        const char* vs = vb + ((int64_t)pg * p.vc.page + (int64_t)(at0 + rr) * p.vc.row + c * 8) * 2;
#pragma unroll
        for (int i = 0; i < ITER; ++i) {
          const int r = 16 * h + rr + i * RPI;
          const bool live = j0 + r < u.limit;
          const uint32_t dst = stage + r * (D * 2) + ((c ^ (r & 7)) << 4);
          cp16(dst, live ? ks + i * kstep : kb, live);
          cp16(dst + G::HALF, live ? vs + i * vstep : vb, live);
        }
      }
    } else {  // each row's place from the lane that looked it up
      const int64_t ko = ((int64_t)page * p.kc.page + (int64_t)at * p.kc.row) * 2;
      const int64_t vo = ((int64_t)page * p.vc.page + (int64_t)at * p.vc.row) * 2;
#pragma unroll
      for (int i = 0; i < KG * ITER; ++i) {
        const int r = rr + i * RPI;
        const bool live = j0 + r < u.limit;
        const int64_t kr = __shfl_sync(0xffffffffu, ko, r), vr = __shfl_sync(0xffffffffu, vo, r);
        const uint32_t dst = stage + r * (D * 2) + ((c ^ (r & 7)) << 4);
        cp16(dst, live ? kb + kr + c * 16 : kb, live);
        cp16(dst + G::HALF, live ? vb + vr + c * 16 : vb, live);
      }
    }
  }

  // What a warp holds of a fragment between its first loads and its last product.
  struct State {
    const char *kb, *vb;
    int32_t first, groups;  // its groups of WARP keys: from first + KEYS x on, x < groups
    int32_t page;           // entry() of the next group to copy
    int32_t see[2];         // keys that rows g and g + 8 see
    uint32_t q[G::QREG][4];
    int32_t buf;            // QS: which buffer q is in
  };

  // Starts a fragment: q, and the copies of the first NS - 1 stages. The ring is the warp's own, so this comes
  // before the fragment before has been joined.
  static __device__ __forceinline__ void start(const PagedAttnParams& p, Smem& s, const Unit& u, State& st, bool* bad) {
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    auto q_row = [&](int row, int32_t* i) {
      const int32_t r = u.r0 + min(row, u.rows - 1);
      *i = (int32_t)fast_div((uint32_t)r, p.group.magic, p.group.shift);
      return row_ptr(p.q, u.q0 + *i, p.q_rs, 2) + ((int64_t)u.h * p.G + (r - *i * p.G)) * D * 2;
    };
    const char* src[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      int32_t i;
      src[k] = q_row(g + 8 * k, &i);
      st.see[k] = u.kv - u.n + i + 1;
    }
    if constexpr (G::QS) {  // read after the next block barrier
      st.buf ^= 1;
#pragma unroll
      for (int e = 0; e < 16 * G::CH / kRowsThreads; ++e) {
        const int at = threadIdx.x + e * kRowsThreads, row = at / G::CH, ch = at % G::CH;
        int32_t i;
        st16(s.q[st.buf] + row * (D * 2) + ((ch ^ (row & 7)) << 4), ld16(q_row(row, &i) + ch * 16));
      }
    } else {
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          st.q[kk][e] = *reinterpret_cast<const uint32_t*>(src[e & 1] + (kk * 16 + (e >> 1) * 8 + 2 * t) * 2);
    }
    st.kb = reinterpret_cast<const char*>(p.kc.base) + (int64_t)u.h * p.kc.head * 2;
    st.vb = reinterpret_cast<const char*>(p.vc.base) + (int64_t)u.h * p.vc.head * 2;
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(s.ring) + w * (G::NS * G::STAGE);
    st.first = u.t0 * KEYS + WARP * w;
    const int32_t upto = (int32_t)min((int64_t)u.limit, (int64_t)u.t1 * KEYS);
    st.groups = st.first < upto ? (upto - st.first + KEYS - 1) / KEYS : 0;
    int32_t page[G::NS];
#pragma unroll
    for (int i = 0; i < G::NS; ++i) page[i] = i < st.groups ? entry(p, u, st.first + i * KEYS) : 0;
#pragma unroll
    for (int i = 0; i < G::NS - 1; ++i) {
      if (i < st.groups) load(p, u, st.kb, st.vb, st.first + i * KEYS, page[i], ring + i * G::STAGE, bad);
      cp_commit();
    }
    st.page = page[G::NS - 1];
  }

  // The warp's keys of a fragment: m, l (of rows g and g + 8) and the unnormalised out.
  static __device__ __forceinline__ void body(const PagedAttnParams& p, Smem& s, const Unit& u, State& st, float* m,
                                              float* l, float (*o)[4], bool* bad) {
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, t = lane & 3;
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(s.ring) + w * (G::NS * G::STAGE);
    const float c = p.scale * kLog2e;
#pragma unroll
    for (int i = 0; i < D / 8; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[i][e] = 0.f;
    m[0] = m[1] = -INFINITY;
    l[0] = l[1] = 0.f;
    const int mi = lane >> 3, mr = lane & 7;
    const uint32_t q_at = (uint32_t)__cvta_generic_to_shared(s.q[st.buf & 1]);
    for (int x = 0; x < st.groups; ++x) {
      cp_wait<G::NS - 2>();
      __syncwarp();  // all lanes' copies have landed, and the stage refilled below has been read
      {
        const int y = x + G::NS - 1;
        if (y < st.groups) {
          const int32_t page = st.page;
          if (y + 1 < st.groups) st.page = entry(p, u, st.first + (y + 1) * KEYS);
          load(p, u, st.kb, st.vb, st.first + y * KEYS, page, ring + (y % G::NS) * G::STAGE, bad);
        }
        cp_commit();
      }
      const uint32_t at = ring + (x % G::NS) * G::STAGE;
      float sc[2 * KG][4] = {}, odd[2 * KG][4] = {};  // two chains of products, half as long
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk) {
        uint32_t qf[4];
        if constexpr (G::QS) {
          const int row = (mi & 1) * 8 + mr, qch = kk * 2 + (mi >> 1);
          ldsm4(qf, q_at + row * (D * 2) + ((qch ^ (row & 7)) << 4));
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) qf[e] = st.q[kk][e];
        }
#pragma unroll
        for (int h = 0; h < KG; ++h) {
          uint32_t kf[4];
          const int key = 16 * h + (mi >> 1) * 8 + mr, ch = kk * 2 + (mi & 1);
          ldsm4(kf, at + key * (D * 2) + ((ch ^ (key & 7)) << 4));
          mma16816<DT>(kk & 1 ? odd[2 * h] : sc[2 * h], qf, kf[0], kf[1]);
          mma16816<DT>(kk & 1 ? odd[2 * h + 1] : sc[2 * h + 1], qf, kf[2], kf[3]);
        }
      }
#pragma unroll
      for (int nt = 0; nt < 2 * KG; ++nt)
#pragma unroll
        for (int e = 0; e < 4; ++e) sc[nt][e] += odd[nt][e];
      const int32_t j0 = st.first + x * KEYS;
      if (j0 + WARP > min(st.see[0], st.see[1]))  // some key is hidden from a row
#pragma unroll
        for (int nt = 0; nt < 2 * KG; ++nt)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (j0 + nt * 8 + 2 * t + (e & 1) >= st.see[e >> 1]) sc[nt][e] = -INFINITY;
      float top[2];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        top[k] = fmaxf(sc[0][2 * k], sc[0][2 * k + 1]);
#pragma unroll
        for (int nt = 1; nt < 2 * KG; ++nt) top[k] = fmaxf(top[k], fmaxf(sc[nt][2 * k], sc[nt][2 * k + 1]));
        top[k] = fmaxf(top[k], __shfl_xor_sync(0xffffffffu, top[k], 1));
        top[k] = attn_level<DT>(c, fmaxf(top[k], __shfl_xor_sync(0xffffffffu, top[k], 2)));
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
      uint32_t pf[KG][4];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const float base = m[k] == -INFINITY ? 0.f : m[k];
#pragma unroll
        for (int nt = 0; nt < 2 * KG; ++nt) {
          const float e0 = fast_exp2(fmaf(sc[nt][2 * k], c, -base)), e1 = fast_exp2(fmaf(sc[nt][2 * k + 1], c, -base));
          l[k] += e0 + e1;
          pf[nt / 2][2 * (nt & 1) + k] = ActType<DT>::pack2(e0, e1);
        }
      }
#pragma unroll
      for (int h = 0; h < KG; ++h)
#pragma unroll
        for (int dd = 0; dd < D / 16; ++dd) {
          uint32_t vf[4];
          const int key = 16 * h + (mi & 1) * 8 + mr, ch = dd * 2 + (mi >> 1);
          ldsm4t(vf, at + G::HALF + key * (D * 2) + ((ch ^ (key & 7)) << 4));
          mma16816<DT>(o[2 * dd], pf[h], vf[0], vf[1]);
          mma16816<DT>(o[2 * dd + 1], pf[h], vf[2], vf[3]);
        }
    }
    cp_wait<0>();
    __syncwarp();  // the ring has been read by all lanes
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      l[k] += __shfl_xor_sync(0xffffffffu, l[k], 1);
      l[k] += __shfl_xor_sync(0xffffffffu, l[k], 2);
    }
  }

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
#pragma unroll
          for (int i = 0; i < D / 8; ++i)
            *reinterpret_cast<float2*>(&s.part[w][row - p0][i * 8 + 2 * t]) = make_float2(o[i][2 * k], o[i][2 * k + 1]);
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
      State st;
      st.buf = 0;
      bool more = part();
      if (more) start(p, s, u, st, &bad);
      if (G::QS) __syncthreads();
      while (more) {
        float m[2], l[2], o[D / 8][4];
        body(p, s, u, st, m, l, o, &bad);
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
          if (more) start(p, s, u, st, &bad);
        }
        finish(p, s, done, m, l, o);
      }
      x = max(x, end);  // a last unit of which only the beginning's tiles were this block's
    }
    attn_fill_tail<kRowsThreads>(p);
    if (bad) atomicOr(p.err, kErrTable);
  }
};

template <int DT, int D>
__global__ void __launch_bounds__(kRowsThreads, RowsGeom<D>::PER_SM) attn_rows_kernel(const PagedAttnParams p) {
  extern __shared__ __align__(128) char smem[];
  if (p.part == ATTN_ALL) pdl_trigger();
  pdl_wait();
  using K = RowsKernel<DT, D>;
  K::run(p, *reinterpret_cast<typename K::Smem*>(smem));
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
