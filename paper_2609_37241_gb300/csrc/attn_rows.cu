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
#include "attn_rows.cuh"

namespace trident {
namespace {

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

template <int DT_, int D_>
struct Rows16 {
  static constexpr int DT = DT_, D = D_;
  using G = RowsGeom<D>;
  static constexpr int KG = G::KG, KEYS = G::KEYS, WARP = 16 * KG;  // WARP: keys of a tile that are one warp's
  struct Extra {
    alignas(128) char q[2][G::QBUF];
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
  static __device__ __forceinline__ void start(const PagedAttnParams& p, char* ring_, Extra& s, const Unit& u, State& st,
                                               bool* bad) {
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
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(ring_) + w * (G::NS * G::STAGE);
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
  static __device__ __forceinline__ void body(const PagedAttnParams& p, char* ring_, Extra& s, const Unit& u, State& st, float* m,
                                              float* l, float (*o)[4], bool* bad) {
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, t = lane & 3;
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(ring_) + w * (G::NS * G::STAGE);
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
      if (__any_sync(0xffffffffu, top[0] > m[0] + kRowsLazy || top[1] > m[1] + kRowsLazy)) {
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

  // Row k of the lane's two, its elements of the accumulators, to a row of floats.
  static __device__ __forceinline__ void spill(float* row, const float (*o)[4], int k, int t) {
#pragma unroll
    for (int i = 0; i < D / 8; ++i) *reinterpret_cast<float2*>(row + i * 8 + 2 * t) = make_float2(o[i][2 * k], o[i][2 * k + 1]);
  }
};

template <int DT, int D>
__global__ void __launch_bounds__(kRowsThreads, RowsGeom<D>::PER_SM) attn_rows_kernel(const PagedAttnParams p) {
  extern __shared__ __align__(128) char smem[];
  if (p.part == ATTN_ALL) pdl_trigger();
  pdl_wait();
  using K = RowsKernel<Rows16<DT, D>>;
  K::run(p, *reinterpret_cast<typename K::Smem*>(smem));
}

template <int DT, int D>
void pick(AttnEntry* e) {
  e->fn = (const void*)attn_rows_kernel<DT, D>;
  e->threads = kRowsThreads;
  e->smem = sizeof(typename RowsKernel<Rows16<DT, D>>::Smem);
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
