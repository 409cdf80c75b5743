// attn_rows8.cu -- paged attention over caches held in 8 bits (kv8.cuh) for requests of few rows: decode steps,
// drafted tokens.
//
// Bound: HBM, a byte per element of k and v. As in the kernel of 16 bits (attn_rows.cu) every warp streams its keys
// through a ring of its own, 32 at a time (heads of 256: 16), and the products are m16n8k16 of halves: a code is a half
// exactly, so k and v become operands by one conversion per two codes, in registers, and no scale touches them:
//   k   ldmatrix gives a lane four consecutive codes of a key, two halves2 for one product whose 16 elements are taken
//       in the order (4t, 4t + 1 | 4t + 2, 4t + 3); q is held in that order
//   v   ldmatrix.trans moves pairs of codes: a lane gets the codes (2g, 2g + 1) of two keys, and a byte permutation
//       makes of them those keys' code 2g and code 2g + 1, operands of two products
//   q   bf16 rows are scaled by a power of two to a largest element in [2^13, 2^14), so that halves hold them exactly
//       down to 2^-27 of it
// (m16n8k32 of 8 bits takes k's codes as they are, with q in two 8-bit pieces, but was slower: 64 decode steps 127 us for
// 103.)
// The scales 2^ek of k and 2^ev of v enter with the scores: with s the score in units of log 2, t = 2^ek s' + ev, the
// running maximum m is of t, numerators 2^(t - m) hold v's scale already, and l takes them times 2^-ev. The numerators
// are halves: the largest is 2^7 at least (with a maximum that is 2^8 behind 2^15), so each is off by 2^-11 of itself down to
// 2^-21 of the largest and by 2^-32 of the largest below. In bf16 calls too: rounded to bf16, as over a 16-bit cache, every
// numerator would lose three bits more. What that costs is a floor. A column gets a key's numerator times a code, at most
// 448, so what it can lose is n keys * 448 * 2^-32 of the largest numerator: of one key 2^-13 of half the smallest step of a
// code in that numerator's block, which is what the cache itself is off by there. It shows in columns where that block's
// codes are 0 or cancel: they get what blocks with numerators of 2^-28 of the largest add, and not what those of 2^-40 do.
//
// Measured on a GB300 (32 q heads on 8 kv heads of 128 where nothing else is said; of the 6.77 TB/s copy rate): 64
// requests of 1000 to 8000 keys 101 us (0.88; the copies alone, with no products, 97), 3 of 131071 keys with a scale for
// each token 139 us (0.86), one request of 1000 keys 8.9 us. The 64 requests with heads of 256 199 us (0.89; these spill 24 to
// 32 bytes of registers), of 64 73 us (0.60). 48 requests of about 3 rows, 28 heads on 4 of 64, over 400 to
// 3000 keys 30 us: a warp's steps of 32 keys are too short for the memory and bound by their dependent instructions;
// units of 32 rows, which read the keys once, not twice, are longer and fewer, and took 36.
#include "attn_rows.cuh"
#include "kv8.cuh"

namespace trident {
namespace {

template <int D>
struct Rows8Geom {
  static constexpr int CH = D / 16;               // 16-byte chunks per row
  static constexpr int KG = D == 256 ? 1 : 2;     // 16-key groups that a warp takes at a time
  static constexpr int KEYS = 64 * KG;            // keys of a tile, a fourth of them per warp
  static constexpr int HALF = 16 * KG * D;        // bytes of a stage's k (and of its v)
  static constexpr int STAGE = 2 * HALF;
  static constexpr int NS = D == 256 ? 2 : 3;  // stages per warp: 12 KB, D 128 24, D 256 16
  static constexpr int RING = 4 * NS * STAGE;
  static constexpr int PER_SM = 2;
  static constexpr int PASS = 512 / D;
  static constexpr int LDO = D + 4;
  static constexpr bool QS = D > 128;             // q in shared memory (attn_rows.cu)
  static constexpr int QREG = QS ? 1 : D / 16, QBUF = QS ? 16 * D * 2 : 16;
  // Where chunk c of row r is: eight rows of a chunk in eight bank groups.
  static __device__ __forceinline__ uint32_t at(int r, int c) {
    return r * D + ((D == 64 ? c ^ ((r >> 1) & 3) : c ^ (r & 7)) << 4);
  }
};

// Two elements of q as halves: fp16 as they are, bf16 times f.
template <int DT>
__device__ __forceinline__ uint32_t q_halves(uint32_t w, float f) {
  if constexpr (DT == DT_FP16) return w;
  return ActType<DT_FP16>::pack2(__uint_as_float(w << 16) * f, __uint_as_float(w & 0xffff0000u) * f);
}
// The larger of top and the magnitudes of two elements, as bf16 bits.
__device__ __forceinline__ uint32_t top_bits(uint32_t top, uint32_t w) {
  return max(top, max(w & 0x7fffu, (w >> 16) & 0x7fffu));
}
// The exponent x for which a row with largest magnitude `bits` is held as q * 2^x.
__device__ __forceinline__ int half_shift(uint32_t bits) { return 140 - (int)min(max(bits >> 7, 14u), 254u); }

template <int DT_, int D_>
struct Rows8 {
  static constexpr int DT = DT_, D = D_;
  using G = Rows8Geom<D>;
  static constexpr int KG = G::KG, KEYS = G::KEYS, WARP = 16 * KG;  // WARP: keys of a tile that are one warp's
  struct Extra {
    alignas(128) char q[2][G::QBUF];
    float q_factor[2][16];               // QS: the rows' 2^-x
    alignas(16) float2 scale[4][G::NS][WARP];  // of a warp's keys: 2^ek, ev
  };

  // The table's entry for the lane's row (lane mod WARP) of the keys from j0 on. It is asked for a stage
  // before its copies are issued, so that they do not wait for it.
  static __device__ __forceinline__ int32_t entry(const PagedAttnParams& p, const Unit& u, int32_t j0) {
    const uint32_t j = (uint32_t)min(j0 + (int32_t)(threadIdx.x & (WARP - 1)), u.limit - 1);
    return p.table[u.b * p.table_rs + fast_div(j, p.page.magic, p.page.shift)];
  }

  struct Scales { uint32_t k, v; };

  // Issues the copies of WARP keys from j0 on into a stage; page: what entry() gave for them.
  static __device__ __forceinline__ void load(const PagedAttnParams& p, const Unit& u, const char* kb, const char* vb,
                                                  int32_t j0, int32_t page, uint32_t stage, bool* bad) {
    const int lane = threadIdx.x & 31;
    constexpr int RPI = 32 / G::CH;     // rows per instruction
    constexpr int ITER = 16 / RPI;      // for 16 rows
    const int c = lane % G::CH, rr = lane / G::CH;
    if (page < 0 || page >= p.P) {
      *bad = true;
      page = 0;
    }
    const uint32_t j = (uint32_t)min(j0 + (lane & (WARP - 1)), u.limit - 1);
    const int32_t at = (int32_t)(j - fast_div(j, p.page.magic, p.page.shift) * (uint32_t)p.page.d);
    if (p.page.d % 16 == 0) {  // one page for 16 rows
      const int64_t kstep = RPI * p.kc.row, vstep = RPI * p.vc.row;
#pragma unroll
      for (int h = 0; h < KG; ++h) {
        const int32_t at0 = __shfl_sync(0xffffffffu, at, 16 * h);
        const int32_t pg = KG == 1 ? page : __shfl_sync(0xffffffffu, page, 16 * h);
        const char* ks = kb + (int64_t)pg * p.kc.page + (int64_t)(at0 + rr) * p.kc.row + c * 16;
        const char* vs = vb + (int64_t)pg * p.vc.page + (int64_t)(at0 + rr) * p.vc.row + c * 16;
        if (j0 + WARP <= u.limit) {
#pragma unroll
          for (int i = 0; i < ITER; ++i) {
            const uint32_t dst = stage + G::at(16 * h + rr + i * RPI, c);
            cp16(dst, ks);
            cp16(dst + G::HALF, vs);
            ks += kstep;
            vs += vstep;
          }
          continue;
        }
#pragma unroll
        for (int i = 0; i < ITER; ++i) {
          const int r = 16 * h + rr + i * RPI;
          const bool live = j0 + r < u.limit;
          const uint32_t dst = stage + G::at(r, c);
          cp16(dst, live ? ks + i * kstep : kb, live);
          cp16(dst + G::HALF, live ? vs + i * vstep : vb, live);
        }
      }
    } else {  // each row's place from the lane that looked it up
      const int64_t ko = (int64_t)page * p.kc.page + (int64_t)at * p.kc.row;
      const int64_t vo = (int64_t)page * p.vc.page + (int64_t)at * p.vc.row;
#pragma unroll
      for (int i = 0; i < KG * ITER; ++i) {
        const int r = rr + i * RPI;
        const bool live = j0 + r < u.limit;
        const int64_t kr = __shfl_sync(0xffffffffu, ko, r), vr = __shfl_sync(0xffffffffu, vo, r);
        const uint32_t dst = stage + G::at(r, c);
        cp16(dst, live ? kb + kr + c * 16 : kb, live);
        cp16(dst + G::HALF, live ? vb + vr + c * 16 : vb, live);
      }
    }
  }

  // Asks for the scales of the lane's key (past the last key that key's). They come back behind the copies that were
  // issued before them, so they are asked for before a stage's copies and used behind the wait for the stage before.
  static __device__ __forceinline__ Scales scales(const PagedAttnParams& p, const Unit& u, int32_t j0, int32_t page) {
    if (page < 0 || page >= p.P) page = 0;  // load() says so
    const uint32_t j = (uint32_t)min(j0 + (int32_t)(threadIdx.x & (WARP - 1)), u.limit - 1);
    const int32_t at = (int32_t)(j - fast_div(j, p.page.magic, p.page.shift) * (uint32_t)p.page.d);
    const int block = (int)fast_div((uint32_t)at, p.block.magic, p.block.shift);
    return {*scale_at(p.ks, page, u.h, block), *scale_at(p.vs, page, u.h, block)};
  }
  static __device__ __forceinline__ void put_scales(float2* to, const Scales& sc) {
    const int lane = threadIdx.x & 31, ek = scale_exp(sc.k), ev = scale_exp(sc.v);
    if (WARP == 32 || lane < WARP) to[lane & (WARP - 1)] = make_float2(exp2_int(ek), (float)ev);
  }

  // What a warp holds of a fragment between its first loads and its last product.
  struct State {
    const char *kb, *vb;
    int32_t first, groups;  // its groups of WARP keys: from first + KEYS x on, x < groups
    int32_t page;           // entry() of the next group to copy
    int32_t see[2];         // keys that rows g and g + 8 see
    uint32_t q[G::QREG][4];
    float factor[2];        // rows g and g + 8: score of the held q times this, in units of log 2
    Scales scale[G::NS - 1];  // of the first groups
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
    const float c = p.scale * kLog2e;
    if constexpr (G::QS) {  // read after the next block barrier; a warp holds whole rows
      static_assert(!G::QS || D == 256, "a row's eighths of a warp");
      st.buf ^= 1;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int row = w + e * 4;
        int32_t i;
        const uint4 v = ld16(q_row(row, &i) + lane * 16);
        float f = 1.f;
        if constexpr (DT == DT_BF16) {
          uint32_t top = top_bits(top_bits(top_bits(top_bits(0, v.x), v.y), v.z), v.w);
          top = __reduce_max_sync(0xffffffffu, top);
          f = exp2_int(half_shift(top));
          if (lane == 0) s.q_factor[st.buf][row] = c * exp2_int(-half_shift(top));
        }
        // elements 8 lane ..: of a product's 16, each four give their first two to the first eight, the others to the last
        char* at = s.q[st.buf] + row * (D * 2);
        const int ch = lane & ~1, half = lane & 1;
        *reinterpret_cast<uint2*>(at + ((ch ^ (row & 7)) << 4) + half * 8) = make_uint2(q_halves<DT>(v.x, f), q_halves<DT>(v.z, f));
        *reinterpret_cast<uint2*>(at + (((ch + 1) ^ (row & 7)) << 4) + half * 8) = make_uint2(q_halves<DT>(v.y, f), q_halves<DT>(v.w, f));
      }
      st.factor[0] = st.factor[1] = c;
    } else {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        uint32_t top = 0;
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) {
          const uint2 v = *reinterpret_cast<const uint2*>(src[k] + (kk * 16 + 4 * t) * 2);
          st.q[kk][k] = v.x;
          st.q[kk][k + 2] = v.y;
          if (DT == DT_BF16) top = top_bits(top_bits(top, v.x), v.y);
        }
        st.factor[k] = c;
        if constexpr (DT == DT_BF16) {
          top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
          top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
          const float f = exp2_int(half_shift(top));
          st.factor[k] = c * exp2_int(-half_shift(top));
#pragma unroll
          for (int kk = 0; kk < D / 16; ++kk) {
            st.q[kk][k] = q_halves<DT>(st.q[kk][k], f);
            st.q[kk][k + 2] = q_halves<DT>(st.q[kk][k + 2], f);
          }
        }
      }
    }
    st.kb = reinterpret_cast<const char*>(p.kc.base) + (int64_t)u.h * p.kc.head;
    st.vb = reinterpret_cast<const char*>(p.vc.base) + (int64_t)u.h * p.vc.head;
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(ring_) + w * (G::NS * G::STAGE);
    st.first = u.t0 * KEYS + WARP * w;
    const int32_t upto = (int32_t)min((int64_t)u.limit, (int64_t)u.t1 * KEYS);
    st.groups = st.first < upto ? (upto - st.first + KEYS - 1) / KEYS : 0;
    int32_t page[G::NS];
#pragma unroll
    for (int i = 0; i < G::NS; ++i) page[i] = i < st.groups ? entry(p, u, st.first + i * KEYS) : 0;
#pragma unroll
    for (int i = 0; i < G::NS - 1; ++i) {
      st.scale[i] = {127, 127};
      if (i < st.groups) st.scale[i] = scales(p, u, st.first + i * KEYS, page[i]);
    }
#pragma unroll
    for (int i = 0; i < G::NS - 1; ++i) {
      if (i < st.groups) load(p, u, st.kb, st.vb, st.first + i * KEYS, page[i], ring + i * G::STAGE, bad);
      cp_commit();
    }
    st.page = page[G::NS - 1];
  }

  // The warp's keys of a fragment: m, l (of rows g and g + 8) and the unnormalised out. o[2 c], o[2 c + 1]: of columns
  // 16 c + 4t, 16 c + 4t + 2 and of those after them.
  static __device__ __forceinline__ void body(const PagedAttnParams& p, char* ring_, Extra& s, const Unit& u, State& st, float* m,
                                              float* l, float (*o)[4], bool* bad) {
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, t = lane & 3, g = lane >> 2;
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(ring_) + w * (G::NS * G::STAGE);
#pragma unroll
    for (int i = 0; i < D / 8; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[i][e] = 0.f;
    m[0] = m[1] = -INFINITY;
    l[0] = l[1] = 0.f;
    const int mi = lane >> 3, mr = lane & 7;
    const uint32_t q_at = (uint32_t)__cvta_generic_to_shared(s.q[st.buf & 1]);
    float factor[2] = {st.factor[0], st.factor[1]};
    if (G::QS && DT == DT_BF16) {
      factor[0] = s.q_factor[st.buf & 1][g];
      factor[1] = s.q_factor[st.buf & 1][g + 8];
    }
#pragma unroll
    for (int i = 0; i < G::NS - 1; ++i) put_scales(s.scale[w][i], st.scale[i]);
    Scales next{127, 127};  // of group x + NS - 2
    for (int x = 0; x < st.groups; ++x) {
      cp_wait<G::NS - 2>();
      __syncwarp();  // all lanes' copies and words have landed, and the stage and the words written below have been read
      {
        if (x > 0) put_scales(s.scale[w][(x + G::NS - 2) % G::NS], next);
        if (G::NS == 2) __syncwarp();
        const int y = x + G::NS - 1;
        if (y < st.groups) {
          const int32_t page = st.page;
          next = scales(p, u, st.first + y * KEYS, page);
          if (y + 1 < st.groups) st.page = entry(p, u, st.first + (y + 1) * KEYS);
          load(p, u, st.kb, st.vb, st.first + y * KEYS, page, ring + (y % G::NS) * G::STAGE, bad);
        }
        cp_commit();
      }
      const uint32_t at = ring + (x % G::NS) * G::STAGE;
      float sc[2 * KG][4] = {};
#pragma unroll
      for (int kk = 0; kk < D / 16; kk += 2) {
        uint32_t qf[2][4];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          if constexpr (G::QS) {
            const int row = (mi & 1) * 8 + mr, qch = (kk + i) * 2 + (mi >> 1);
            ldsm4(qf[i], q_at + row * (D * 2) + ((qch ^ (row & 7)) << 4));
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) qf[i][e] = st.q[kk + i][e];
          }
        }
#pragma unroll
        for (int h = 0; h < KG; ++h) {
          uint32_t kf[4];  // keys 0-7, 8-15 of chunk kk, the same of chunk kk + 1
          const int key = 16 * h + (mi & 1) * 8 + mr, ch = kk + (mi >> 1);
          ldsm4(kf, at + G::at(key, ch));
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int n = 0; n < 2; ++n)
              mma16816<DT_FP16>(sc[2 * h + n], qf[i], halves2(kf[2 * i + n]), halves2_hi(kf[2 * i + n]));
        }
      }
      // scores with the blocks' scales: t, in sc; f: 2^-ev
      float f[2 * KG][2];
#pragma unroll
      for (int nt = 0; nt < 2 * KG; ++nt) {
        const float4 k = *reinterpret_cast<const float4*>(&s.scale[w][x % G::NS][nt * 8 + 2 * t]);
        f[nt][0] = fast_exp2(-k.y);
        f[nt][1] = fast_exp2(-k.w);
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          sc[nt][2 * r] = fmaf(sc[nt][2 * r], factor[r] * k.x, k.y);
          sc[nt][2 * r + 1] = fmaf(sc[nt][2 * r + 1], factor[r] * k.z, k.w);
        }
      }
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
        top[k] = fmaxf(top[k], __shfl_xor_sync(0xffffffffu, top[k], 2)) - ActType<DT_FP16>::kUp;
      }
      if (__any_sync(0xffffffffu, top[0] > m[0] + kRowsLazy || top[1] > m[1] + kRowsLazy)) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const float m2 = fmaxf(m[k], top[k]);
          const float f2 = m2 == -INFINITY ? 1.f : fast_exp2(m[k] - m2);
          m[k] = m2;
          l[k] *= f2;
#pragma unroll
          for (int i = 0; i < D / 8; ++i) {
            o[i][2 * k] *= f2;
            o[i][2 * k + 1] *= f2;
          }
        }
      }
      uint32_t pf[KG][4];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const float base = m[k] == -INFINITY ? 0.f : m[k];
#pragma unroll
        for (int nt = 0; nt < 2 * KG; ++nt) {
          const float e0 = fast_exp2(sc[nt][2 * k] - base), e1 = fast_exp2(sc[nt][2 * k + 1] - base);
          l[k] = fmaf(e0, f[nt][0], fmaf(e1, f[nt][1], l[k]));
          pf[nt / 2][2 * (nt & 1) + k] = ActType<DT_FP16>::pack2(e0, e1);
        }
      }
#pragma unroll
      for (int h = 0; h < KG; ++h)
#pragma unroll
        for (int c = 0; c < D / 16; c += 2) {
          uint32_t vf[4];  // keys 0-7, 8-15 of chunk c, the same of chunk c + 1
          const int key = 16 * h + (mi & 1) * 8 + mr, ch = c + (mi >> 1);
          ldsm4t(vf, at + G::HALF + G::at(key, ch));
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const uint32_t a = __byte_perm(vf[2 * i], 0, 0x3120), b = __byte_perm(vf[2 * i + 1], 0, 0x3120);
            mma16816<DT_FP16>(o[2 * (c + i)], pf[h], halves2(a), halves2(b));
            mma16816<DT_FP16>(o[2 * (c + i) + 1], pf[h], halves2_hi(a), halves2_hi(b));
          }
        }
    }
    cp_wait<0>();
    __syncwarp();  // the ring and the words have been read by all lanes
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      l[k] += __shfl_xor_sync(0xffffffffu, l[k], 1);
      l[k] += __shfl_xor_sync(0xffffffffu, l[k], 2);
    }
  }

  // Row k of the lane's two, its elements of the accumulators, to a row of floats.
  static __device__ __forceinline__ void spill(float* row, const float (*o)[4], int k, int t) {
#pragma unroll
    for (int c = 0; c < D / 16; ++c)
      *reinterpret_cast<float4*>(row + 16 * c + 4 * t) =
          make_float4(o[2 * c][2 * k], o[2 * c + 1][2 * k], o[2 * c][2 * k + 1], o[2 * c + 1][2 * k + 1]);
  }
};

template <int DT, int D>
__global__ void __launch_bounds__(kRowsThreads, Rows8Geom<D>::PER_SM) attn_rows8_kernel(const PagedAttnParams p) {
  extern __shared__ __align__(128) char smem[];
  if (p.part == ATTN_ALL) pdl_trigger();
  pdl_wait();
  using K = RowsKernel<Rows8<DT, D>>;
  K::run(p, *reinterpret_cast<typename K::Smem*>(smem));
}

template <int DT, int D>
void pick(AttnEntry* e) {
  e->fn = (const void*)attn_rows8_kernel<DT, D>;
  e->threads = kRowsThreads;
  e->smem = sizeof(typename RowsKernel<Rows8<DT, D>>::Smem);
  e->per_sm = Rows8Geom<D>::PER_SM;
  e->slot_floats = attn_slot_floats(kRowsTile, D);
  static_assert(Rows8Geom<D>::PER_SM * (sizeof(typename RowsKernel<Rows8<DT, D>>::Smem) + 1024) <= 233472, "shared memory of an SM");
}

}  // namespace

bool attn_rows8_entry(int32_t dtype, int32_t D, AttnEntry* e) {
  *e = AttnEntry{};
  if (D == 64) dtype == DT_BF16 ? pick<DT_BF16, 64>(e) : pick<DT_FP16, 64>(e);
  else if (D == 128) dtype == DT_BF16 ? pick<DT_BF16, 128>(e) : pick<DT_FP16, 128>(e);
  else if (D == 256) dtype == DT_BF16 ? pick<DT_BF16, 256>(e) : pick<DT_FP16, 256>(e);
  return e->fn != nullptr;
}

}  // namespace trident
