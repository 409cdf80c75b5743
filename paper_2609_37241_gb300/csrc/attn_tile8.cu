// attn_tile8.cu -- paged attention over caches held in 8 bits (kv8.cuh) for requests of many rows: chunks of a prompt.
//
// Bound: the tensor cores, as in the kernel of 16 bits (attn_tile.cu), whose frame this is. What the codes change:
//   scores   k's tiles are operands as they are: 8-bit products (kind::f8f6f4) run at twice the 16-bit rate, and q is a
//            sum of 8-bit pieces (kv8.cuh). Two passes over k's codes cost what one 16-bit product does; k is never
//            converted.
//   out      v's tiles become halves: a warpgroup reads a tile's codes, copied into the upper half of its ring slot, and
//            writes the halves over the whole slot, in the swizzle that the products read. 16 + 16 + 32 KB of shared
//            memory traffic per 128 keys of 128 elements (copy in, read, write) beside the products' own 192.
//   softmax  the scales 2^ek, 2^ev of k and v enter with the scores: t = 2^ek s' + ev in units of log 2, the running
//            maximum is of t, numerators 2^(t - m) are halves and hold v's scale, the sum takes them times 2^-ev
//            (attn_rows8.cu has the reasons and what a column can lose by it). Where a scale's block is 16 keys or more,
//            the 16 scores of a group share the factors: the group's maximum is taken before they are applied. Else each
//            key has its own.
// Warps: NT softmax warpgroups, NT warps that issue products, two that load (k, v), four that convert v and look up the
// scales.
//
// Measured on a GB300 (32 q heads on 8 kv heads of 128, graphs of 30 calls, over a 16-bit cache beside it in parentheses):
// 8192 rows after 8192 keys 1165 us (950) or 1415 TFLOP/s, 0.82 of cuBLAS' sustained rate (back to back for longer, at the
// power limit, 1196 (1051)), 2048 rows after 6144 keys 203 us (156), with heads of 64 155 (126), of 256 556 (460). Registers
// (-Xptxas -v): 248 to 330 bytes of spill stores and 368 to 468 of loads for heads of 64 and 128, 196 and 316 for heads of 256
// (the 16-bit kernel: 140 to 148 and 248 to 280; none); what they cost has not been taken apart. Without the
// conversions it is 6% shorter, without half of the scores' products 5%: what bounds it is the chain of a tile's scores,
// softmax and products, in which every access to shared memory waits beside the products' (a wait that has nothing to
// wait for takes 200 cycles). Built and measured against this one, 8192 rows after 8192 keys: the conversions by two warps
// of a block of 384 threads 1600 to 1740 us, by the softmax warpgroups between their tiles 1450, one warp issuing all
// products 1600, scores read from TMEM twice so that a row needs fewer registers 2390.
#include "attn_tile.cuh"
#include "kv8.cuh"

namespace trident {
namespace {

__device__ __forceinline__ void mma_ss8(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t add) {
  asm volatile("{ .reg .pred p; setp.ne.u32 p, %4, 0; tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p; }"
               :: "r"(d), "l"(a), "l"(b), "r"(idesc), "r"(add) : "memory");
}
// Instruction descriptor of kind::f8f6f4: A e4m3 or e5m2, B e4m3, both K-major, fp32 accumulators.
__host__ __device__ constexpr uint32_t idesc8_of(int M, int N, bool e5m2) {
  return (1u << 4) | ((e5m2 ? 1u : 0u) << 7) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}
template <int DT_, int D_, int NT_, int KEYS_, int KS_, int VS_>
struct Tile8Shape {
  static constexpr int DT = DT_, D = D_, NT = NT_, KEYS = KEYS_;
  static constexpr int KS = KS_, VS = VS_;     // ring slots of k and of v
  static constexpr int OTHERS = 256;           // mma, load and idle warps; the converting warpgroup
  static constexpr int OTHER_REGS = NT == 2 ? 56 : 88, SOFT_REGS = NT == 2 ? 200 : 232;
  static constexpr int PIECES = q_pieces<DT>();
  static constexpr int QP = 128 * D;           // bytes of a piece of a q tile
  static constexpr int KB = KEYS * D;          // ... of a k tile
  static constexpr int VB = KEYS * D * 2;      // ... of a v tile as halves; its codes come to the upper half
  struct Smem : TileShape<Tile8Shape>::Common {
    alignas(1024) char q[NT * PIECES * QP];
    alignas(1024) char k[KS * KB];
    alignas(1024) char v[VS * VB];
    alignas(16) float4 scale[VS + 1][KEYS];    // of a tile's keys: 2^ek, ev, 2^-ev
    float q_factor[NT * 128];                  // 2^-x of the rows
    alignas(8) uint64_t k_full[KS], k_empty[KS], v_raw[VS], v_full[VS], v_empty[VS], scale_full[VS + 1], raw_read;
  };
};

template <class C>
struct Tile8 : TileFrame<Tile8<C>, C> {
  using F = TileFrame<Tile8<C>, C>;
  using F::DT; using F::D; using F::NT; using F::KEYS; using F::S_COL; using F::O_COL; using F::MMA_WARP;
  using typename F::Smem; using typename F::Soft;
  using F::turn_wait; using F::turn_pass;
  static constexpr int KS = C::KS, VS = C::VS, PIECES = C::PIECES, QP = C::QP, KB = C::KB, VB = C::VB;
  static constexpr int CW = D < 128 ? D : 128;       // bytes of a row in one swizzled part: 64 or 128
  static constexpr int QPART = 128 * CW, KPART = KEYS * CW;
  static constexpr int VHALF = KEYS * 128;           // bytes of 64 columns of halves
  static constexpr int LOAD_WARP = MMA_WARP + NT, CONVERT_WARP = MMA_WARP + 4;
  static constexpr float kLeast = 0x1p-94f;          // a row's factor at least: masked scores are infinite, and one that 2^-32 takes to 0 would make them NaN

  static __device__ __forceinline__ void init(Smem& s) {
    for (int i = 0; i < KS; ++i) {
      mb_init(smem_at(&s.k_full[i]), 1);
      mb_init(smem_at(&s.k_empty[i]), NT);
    }
    for (int i = 0; i < VS; ++i) {
      mb_init(smem_at(&s.v_raw[i]), 1);
      mb_init(smem_at(&s.v_full[i]), 128);
      mb_init(smem_at(&s.v_empty[i]), NT);
    }
    for (int i = 0; i <= VS; ++i) mb_init(smem_at(&s.scale_full[i]), 128);
    mb_init(smem_at(&s.raw_read), 128);
  }

  // Shared-memory operand descriptor of a K-major tile of codes: rows of CW bytes in the swizzle of that width (layout
  // code 2: 128 bytes, 4: 64), groups of eight rows CW * 8 bytes apart.
  static __device__ __forceinline__ uint64_t desc8(uint32_t lo) {
    constexpr uint32_t hi = ((uint32_t)(CW * 8) >> 4) | (1u << 14) | ((CW == 128 ? 2u : 4u) << 29);
    return ((uint64_t)hi << 32) | lo;
  }

  // ------------------------------------------------------------ load warps, one for k and one for v
  struct Load {
    uint32_t tiles = 0;      // tiles loaded so far
    bool bad = false;
  };
  static __device__ __forceinline__ bool load(const PagedAttnParams& p, const CUtensorMap* map, Smem& s, const Frag& f,
                                              bool is_v, Load& st) {
    const int lane = threadIdx.x & 31;
    const int32_t* table = p.table + f.b * p.table_rs;
    const int ps = p.page.d, box = min(ps, KEYS);       // rows of a box
    const int32_t limit = f.limit, t1 = f.t1, h = f.h;
    // the page of the lane's box in tile t, and its row there; read a tile ahead
    auto locate = [&](int32_t t, int32_t* at) {
      const int32_t j = t * KEYS + lane * box;
      int32_t page = 0;
      *at = 0;
      if (lane * box < KEYS && j < limit) {
        const uint32_t pg = fast_div((uint32_t)j, p.page.magic, p.page.shift);
        *at = (int32_t)((uint32_t)j - pg * (uint32_t)ps);
        page = table[pg];
        if (page < 0 || page >= p.P) {
          st.bad = true;
          page = 0;
        }
      }
      return page;
    };
    int32_t at, at_next, page = locate(f.t0, &at), page_next = 0;
    for (int32_t t = f.t0; t < t1; ++t, page = page_next, at = at_next) {
      page_next = at_next = 0;
      if (t + 1 < t1) page_next = locate(t + 1, &at_next);
      const int boxes = (min(KEYS, limit - t * KEYS) + box - 1) / box;
      const uint32_t n = is_v ? VS : KS, slot = st.tiles % n, use = st.tiles / n;
      const uint32_t empty = smem_at(is_v ? &s.v_empty[slot] : &s.k_empty[slot]);
      const uint32_t bar = smem_at(is_v ? &s.v_raw[slot] : &s.k_full[slot]);
      if (!__all_sync(0xffffffffu, mb_wait(empty, (use & 1) ^ 1, p.polls, &s.abort))) return false;
      if (lane == 0) mb_expect(bar, (uint32_t)(boxes * box * D));
      __syncwarp();
      if (lane < boxes) {
        if (is_v) {
          tma_4d(smem_at(s.v + slot * VB + VB / 2) + lane * box * D, map, 0, at, h, page, bar);
        } else {
#pragma unroll
          for (int c = 0; c < D / CW; ++c) tma_4d(smem_at(s.k + slot * KB) + c * KPART + lane * box * CW, map, c * CW, at, h, page, bar);
        }
      }
      __syncwarp();
      ++st.tiles;
    }
    return true;
  }

  // ------------------------------------------------------------ the converting warpgroup
  struct Convert {
    uint32_t tiles = 0;
    bool bad = false;
  };
  static __device__ __forceinline__ bool convert(const PagedAttnParams& p, Smem& s, const Frag& f, Convert& st) {
    const int i = threadIdx.x & 127;
    const int32_t limit = f.limit, t1 = f.t1;
    // the scales' bytes of key i of tile t; read two tiles ahead. Past the limit: 1.
    auto bytes = [&](int32_t t) {
      const int32_t j = t * KEYS + i;
      if (i >= KEYS || j >= limit) return 127u | 127u << 8;
      const uint32_t pg = fast_div((uint32_t)j, p.page.magic, p.page.shift);
      int64_t page = p.table[f.b * p.table_rs + pg];
      if (page < 0 || page >= p.P) {
        st.bad = true;
        page = 0;
      }
      const int block = (int)fast_div((uint32_t)j - pg * (uint32_t)p.page.d, p.block.magic, p.block.shift);
      return (uint32_t)*scale_at(p.ks, page, f.h, block) | (uint32_t)*scale_at(p.vs, page, f.h, block) << 8;
    };
    // Factors of the n-th tile. Their slots are one more than v's: that of tile n + 1 is free when tile n's v slot is.
    auto factors = [&](uint32_t n, uint32_t b) {
      if (i < KEYS) {
        const int ek = scale_exp(b & 255u), ev = scale_exp(b >> 8);
        s.scale[n % (VS + 1)][i] = make_float4(exp2_int(ek), (float)ev, exp2_int(-ev), 0.f);
      }
      mb_arrive(smem_at(&s.scale_full[n % (VS + 1)]));
    };
    factors(st.tiles, bytes(f.t0));
    uint32_t b = f.t0 + 1 < t1 ? bytes(f.t0 + 1) : 0;
    for (int32_t t = f.t0; t < t1; ++t) {
      const int32_t valid = min(KEYS, limit - t * KEYS), upto = (valid + 15) & ~15;
      const uint32_t slot = st.tiles % VS, use = st.tiles / VS, turn = st.tiles;
      ++st.tiles;
      if (!__all_sync(0xffffffffu, mb_wait(smem_at(&s.v_empty[slot]), (use & 1) ^ 1, p.polls, &s.abort))) return false;
      if (t + 1 < t1) factors(turn + 1, b);
      if (t + 2 < t1) b = bytes(t + 2);
      if (!__all_sync(0xffffffffu, mb_wait(smem_at(&s.v_raw[slot]), use & 1, p.polls, &s.abort))) return false;
      // 16 codes at a time: vectors i, i + 128, ... of the tile, D / 16 to a row. The slot is written when all are read.
      constexpr int VECS = KEYS * D / 16 / 128, CH = D / 16;
      const char* raw = s.v + slot * VB + VB / 2;
      uint4 c[VECS];
#pragma unroll
      for (int e = 0; e < VECS; ++e) {
        const int at = i + e * 128;
        c[e] = at / CH < valid ? *reinterpret_cast<const uint4*>(raw + at * 16) : make_uint4(0, 0, 0, 0);
      }
      mb_arrive(smem_at(&s.raw_read));
      if (!__all_sync(0xffffffffu, mb_wait(smem_at(&s.raw_read), turn & 1, p.polls, &s.abort))) return false;
      char* out = s.v + slot * VB;
#pragma unroll
      for (int e = 0; e < VECS; ++e) {
        const int at = i + e * 128, row = at / CH, ch = at % CH;
        if (row >= upto) continue;
        const uint4 lo = make_uint4(halves2(c[e].x), halves2_hi(c[e].x), halves2(c[e].y), halves2_hi(c[e].y));
        const uint4 hi = make_uint4(halves2(c[e].z), halves2_hi(c[e].z), halves2(c[e].w), halves2_hi(c[e].w));
        // columns 16 ch .. of a row: chunks 2 (ch mod 4) and the next of half ch / 4. The halves are banks apart by nothing,
        // so lanes of an odd half write their chunks in the other order.
        char* dst = out + (ch / 4) * VHALF + row * 128;
        const int k0 = 2 * (ch % 4), odd = D > 64 ? (ch / 4) & 1 : 0;
        *reinterpret_cast<uint4*>(dst + (((k0 + odd) ^ (row & 7)) << 4)) = odd ? hi : lo;
        *reinterpret_cast<uint4*>(dst + (((k0 + 1 - odd) ^ (row & 7)) << 4)) = odd ? lo : hi;
      }
      fence_async();
      mb_arrive(smem_at(&s.v_full[slot]));
    }
    return true;
  }

  // ------------------------------------------------------------ mma warps, one per q tile
  struct Mma {
    uint32_t tiles = 0;       // key tiles consumed so far
    uint32_t px = 0, qx = 0;  // p and q tiles waited for
  };
  static __device__ __forceinline__ void qk(uint32_t q_lo, uint32_t k_lo, uint32_t d) {
    constexpr int STEPS = CW / 32;
#pragma unroll
    for (int piece = 0; piece < PIECES; ++piece)
#pragma unroll
      for (int k = 0; k < D / 32; ++k)
        mma_ss8(d, desc8(q_lo + ((piece * QP + k / STEPS * QPART + k % STEPS * 32) >> 4)),
                desc8(k_lo + ((k / STEPS * KPART + k % STEPS * 32) >> 4)), piece == 0 ? idesc8_of(128, KEYS, false) : idesc8_of(128, KEYS, true),
                piece + k > 0);
  }
  // Half of P V: 16-key steps [HALF * KEYS / 32, ...), at most `steps` of the tile's.
  template <int HALF>
  static __device__ __forceinline__ void pv(uint32_t p_col, uint32_t v_lo, uint32_t d, int steps, bool add) {
    constexpr uint32_t id = idesc_of<DT_FP16>(128, D, true);
    constexpr int N = KEYS / 32, K0 = HALF * N;
    if (steps >= K0 + N) {
#pragma unroll
      for (int k = K0; k < K0 + N; ++k) mma_ts(d, p_col + k * 8, desc128(v_lo + k * (2048 >> 4)), id, k > 0 || add);
    } else {
      for (int k = K0; k < steps; ++k) mma_ts(d, p_col + k * 8, desc128(v_lo + k * (2048 >> 4)), id, k > 0 || add);
    }
  }
  static __device__ __forceinline__ bool mma(const PagedAttnParams& p, Smem& s, uint32_t tmem, const Frag& f, int x, Mma& st,
                                             bool one) {
    const int32_t t0 = f.t0, t1 = f.t1, limit = f.limit;
    const uint32_t q_lo = desc_lo(smem_at(s.q + x * PIECES * QP), 16), k_lo = desc_lo(smem_at(s.k), 16),
                   v_lo = desc_lo(smem_at(s.v), VHALF);
    const uint32_t sc = tmem + S_COL + x * KEYS, oc = tmem + O_COL + x * D;
    auto wait = [&](uint64_t* bar, uint32_t parity) {
      return __all_sync(0xffffffffu, mb_wait(smem_at(bar), parity, p.polls, &s.abort));
    };
    auto k_ready = [&](uint32_t i) { return wait(&s.k_full[i % KS], (i / KS) & 1) && wait(&s.scale_full[i % (VS + 1)], (i / (VS + 1)) & 1); };
    auto v_ready = [&](uint32_t i) { return wait(&s.v_full[i % VS], (i / VS) & 1); };
    uint32_t i = st.tiles;
    st.tiles += (uint32_t)(t1 - t0);
    if (x > 0 && f.rows <= 128 * x) {  // nothing to do but to give the slots back
      for (; i < st.tiles; ++i) {
        if (!k_ready(i) || !v_ready(i)) return false;
        if (one) {
          mb_arrive(smem_at(&s.k_empty[i % KS]));
          mb_arrive(smem_at(&s.v_empty[i % VS]));
        }
      }
      return true;
    }
    if (!wait(&s.q_full[x], st.qx++ & 1) || !k_ready(i)) return false;
    tc_after();
    if (one) {
      qk(q_lo, k_lo + i % KS * (KB >> 4), sc);
      tc_commit(smem_at(&s.s_full[x]));
      tc_commit(smem_at(&s.k_empty[i % KS]));
    }
    for (int32_t t = t0; t < t1; ++t, ++i) {
      const uint32_t parity = st.px++ & 1;
      const bool more = t + 1 < t1, add = t > t0;
      const int steps = (min(KEYS, limit - t * KEYS) + 15) / 16;
      const uint32_t v_at = v_lo + i % VS * (VB >> 4), k_at = k_lo + (i + 1) % KS * (KB >> 4);
      if (!v_ready(i) || (more && !k_ready(i + 1))) return false;
      if (!wait(&s.p_half[x], parity)) return false;
      tc_after();
      if (one) pv<0>(sc, v_at, oc, steps, add);
      if (!wait(&s.p_full[x], parity)) return false;
      tc_after();
      if (one) {
        pv<1>(sc, v_at, oc, steps, add);
        if (more) {
          qk(q_lo, k_at, sc);
          tc_commit(smem_at(&s.s_full[x]));
          tc_commit(smem_at(&s.k_empty[(i + 1) % KS]));
        } else {
          tc_commit(smem_at(&s.o_full[x]));
        }
        tc_commit(smem_at(&s.v_empty[i % VS]));
      }
    }
    return true;
  }

  // ------------------------------------------------------------ softmax warpgroup
  // Loads this warpgroup's q rows, 16 bytes per lane and D / 8 lanes per row, and writes their pieces into the swizzled
  // tiles and their factors.
  static __device__ __forceinline__ void load_q(const PagedAttnParams& p, Smem& s, const Frag& f, int x) {
    constexpr int CH = D / 8, RPI = 32 / CH, ITER = 32 / RPI;
    const int w = (threadIdx.x >> 5) & 3, lane = threadIdx.x & 31, c = lane % CH, rr = lane / CH;
    constexpr int BATCH = 8;  // loads in flight, none behind a branch: rows past the unit load its last and drop it
#pragma unroll 1
    for (int i = 0; i < ITER; i += BATCH) {
      uint4 v[BATCH];
#pragma unroll
      for (int e = 0; e < BATCH; ++e) {
        const int r = min(x * 128 + w * 32 + (i + e) * RPI + rr, f.rows - 1);
        const int32_t k = (int32_t)fast_div((uint32_t)r, p.group.magic, p.group.shift);
        v[e] = ld16(row_ptr(p.q, f.q0 + f.tok0 + k, p.q_rs, 2) + ((int64_t)(f.h * p.G + r - k * p.G) * D + c * 8) * 2);
      }
#pragma unroll
      for (int e = 0; e < BATCH; ++e) {
        const int row = w * 32 + (i + e) * RPI + rr;
        float y[8];
        if (x * 128 + row >= f.rows) v[e] = make_uint4(0, 0, 0, 0);
        unpack<DT>(v[e], y);
        uint32_t bits = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) bits = max(bits, __float_as_uint(y[k]) & 0x7fffffffu);
#pragma unroll
        for (int o = CH / 2; o > 0; o >>= 1) bits = max(bits, __shfl_xor_sync(0xffffffffu, bits, o));
        const float up = q_up(bits);
#pragma unroll
        for (int k = 0; k < 8; ++k) y[k] *= up;
        const int ch = c >> 1;
        char* dst = s.q + x * PIECES * QP + (ch / (CW / 16)) * QPART + row * CW +
                    ((ch % (CW / 16) ^ (CW == 128 ? row & 7 : (row >> 1) & 3)) << 4) + (c & 1) * 8;
#pragma unroll
        for (int piece = 0; piece < PIECES; ++piece)
          *reinterpret_cast<uint2*>(dst + piece * QP) = make_uint2(q_piece(y, piece), q_piece(y + 4, piece));
        if (c == 0) s.q_factor[x * 128 + row] = q_down(bits);
      }
    }
    fence_async();
    mb_arrive(smem_at(&s.q_full[x]));
  }

  template <bool GROUPS>
  static __device__ __forceinline__ bool softmax_of(const PagedAttnParams& p, Smem& s, uint32_t tmem, const Frag& f, int x,
                                                    Soft& st, bool ok, float* m_out, float* l_out) {
    const uint32_t lanes = tmem + (((threadIdx.x >> 5) & 3) << 21);  // TMEM lane 32 * (warp mod 4)
    const uint32_t sc = lanes + S_COL + x * KEYS, oc = lanes + O_COL + x * D;
    // Rows past the unit's (their q is zeros, their results go nowhere) see what its last one does, as in attn_tile.cu.
    const int r = min(x * 128 + (int)(threadIdx.x & 127), f.rows - 1);
    const int32_t see = f.kv - f.n + f.tok0 + (int32_t)fast_div((uint32_t)r, p.group.magic, p.group.shift) + 1;
    const bool turns = NT == 2 && f.rows > 128;
    const int32_t t0 = f.t0, t1 = f.t1;
    float m = -INFINITY, l = 0.f, c = 0.f;
    if (turns && x == 1) turn_pass(1);
    for (int32_t t = t0; t < t1; ++t) {
      ok = ok && __all_sync(0xffffffffu, mb_wait(smem_at(&s.s_full[x]), st.s & 1, st.s == 0 ? p.first_polls : p.polls, &s.abort));
      const float4* scale = s.scale[(st.tiles - (uint32_t)(t1 - t)) % (VS + 1)];
      ++st.s;
      uint32_t a[KEYS];
      if (turns) turn_wait(x);
      auto pass = [&]() {
        if (turns && (x == 0 || t + 1 < t1)) turn_pass(x);
      };
      float base = 0.f;
      F2 sum = f2_pack(0.f, 0.f);
      // numerators of half the tile's keys, to the columns of its scores; the turn ends inside the second half
      auto half = [&](int h) {
        uint32_t w[KEYS / 4];
#pragma unroll
        for (int g = 0; g < KEYS / 32; ++g) {
          const int e0 = h * (KEYS / 2) + 16 * g;
          F2 part = f2_pack(0.f, 0.f);
          F2 mul, add;
          float out = 1.f;
          if (GROUPS) {
            const float4 k = scale[e0];
            mul = f2_pack(c * k.x, c * k.x);
            add = f2_pack(k.y - base, k.y - base);
            out = k.z;
          } else {
            mul = f2_pack(1.f, 1.f);
            add = f2_pack(-base, -base);
          }
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int e = e0 + 2 * i;
            float u, v;
            const F2 z = f2_pack(__uint_as_float(a[e]), __uint_as_float(a[e + 1]));
            f2_unpack(GROUPS ? f2_fma(z, mul, add) : f2_add(z, add), &u, &v);
            u = fast_exp2(u);
            v = fast_exp2(v);
            if (GROUPS) part = f2_add(part, f2_pack(u, v));
            else part = f2_fma(f2_pack(u, v), f2_pack(scale[e].z, scale[e + 1].z), part);
            w[8 * g + i] = ActType<DT_FP16>::pack2(u, v);
          }
          sum = f2_fma(part, f2_pack(out, out), sum);
          if (h == 1 && g == 0) pass();
        }
#pragma unroll
        for (int k = 0; k < KEYS / 64; ++k) tc_st16(sc + h * (KEYS / 4) + k * 16, w + k * 16);
        tc_wait_st();
        tc_before();
        mb_arrive(smem_at(h == 0 ? &s.p_half[x] : &s.p_full[x]));
      };
      if (ok) {
        if (t == t0) c = fmaxf(p.scale * kLog2e * s.q_factor[x * 128 + (threadIdx.x & 127)], kLeast);  // what load_q wrote, behind s_full
        tc_after();
#pragma unroll
        for (int i = 0; i < KEYS / 32; ++i) tc_ld32(sc + i * 32, a + i * 32);
        tc_wait_ld<KEYS>(a);
        const int32_t left = see - t * KEYS;  // keys of the tile that the row sees
        if (!GROUPS) {
#pragma unroll
          for (int i = 0; i < KEYS; ++i) {
            const float4 k = scale[i];
            a[i] = __float_as_uint(fmaf(__uint_as_float(a[i]), c * k.x, k.y));
          }
        }
        if (left < KEYS) {
#pragma unroll
          for (int i = 0; i < KEYS; ++i)
            if (i >= left) a[i] = 0xff800000u;  // -inf
        }
        float hi = -INFINITY;
#pragma unroll
        for (int g = 0; g < KEYS / 16; ++g) {  // three-operand maxima
          float top[2] = {fmaxf(__uint_as_float(a[16 * g]), __uint_as_float(a[16 * g + 1])),
                          fmaxf(__uint_as_float(a[16 * g + 2]), __uint_as_float(a[16 * g + 3]))};
#pragma unroll
          for (int i = 4; i < 16; i += 2)
            top[i / 2 & 1] = fmaxf(fmaxf(top[i / 2 & 1], __uint_as_float(a[16 * g + i])), __uint_as_float(a[16 * g + i + 1]));
          const float z = fmaxf(top[0], top[1]);
          if (GROUPS) {
            const float4 k = scale[16 * g];
            hi = fmaxf(hi, fmaf(z, c * k.x, k.y));
          } else {
            hi = fmaxf(hi, z);
          }
        }
        hi -= ActType<DT_FP16>::kUp;
        if (__any_sync(0xffffffffu, hi > m + kTileLazy)) {
          const float m2 = fmaxf(m, hi);
          const float g = m2 == -INFINITY ? 1.f : fast_exp2(m - m2);
          m = m2;
          l *= g;
          if (t > t0) {
#pragma unroll 1
            for (int i = 0; i < D / 32; ++i) {
              uint32_t o[32];
              tc_ld32(oc + i * 32, o);
              tc_wait_ld<32>(o);
#pragma unroll
              for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * g);
              tc_st32(oc + i * 32, o);
            }
          }
        }
        base = m == -INFINITY ? 0.f : m;
        half(0);  // its products start while the second half's numerators are made
        half(1);
        float s0, s1;
        f2_unpack(sum, &s0, &s1);
        l += s0 + s1;
      } else {
        pass();
      }
    }
    *m_out = m;
    *l_out = l;
    ok = ok && __all_sync(0xffffffffu, mb_wait(smem_at(&s.o_full[x]), st.o & 1, p.polls, &s.abort));
    ++st.o;
    tc_after();
    return ok;
  }
  static __device__ __forceinline__ bool softmax(const PagedAttnParams& p, Smem& s, uint32_t tmem, const Frag& f, int x,
                                                 Soft& st, bool ok, float* m_out, float* l_out) {
    return p.block.d % 16 == 0 ? softmax_of<true>(p, s, tmem, f, x, st, ok, m_out, l_out)
                               : softmax_of<false>(p, s, tmem, f, x, st, ok, m_out, l_out);
  }

  // ------------------------------------------------------------ the other warps
  struct Other {
    Load load;
    Mma mma;
    Convert convert;
  };
  static __device__ __forceinline__ bool work(const PagedAttnParams& p, const CUtensorMap* mk, const CUtensorMap* mv, Smem& s,
                                              uint32_t tmem, const Frag& f, int warp, Other& st, bool one) {
    if (warp >= CONVERT_WARP) return convert(p, s, f, st.convert);
    if (warp >= LOAD_WARP && warp < LOAD_WARP + 2) return load(p, warp == LOAD_WARP ? mk : mv, s, f, warp > LOAD_WARP, st.load);
    return warp >= LOAD_WARP || mma(p, s, tmem, f, warp - MMA_WARP, st.mma, one);
  }
  static __device__ __forceinline__ void leave(const PagedAttnParams& p, Smem& s, int warp, const Other& st, bool ok) {
    if (st.load.bad || st.convert.bad) atomicOr(p.err, kErrTable);
    if (warp < LOAD_WARP || warp >= LOAD_WARP + 2) return;
    const uint32_t tiles = st.load.tiles, n = warp > LOAD_WARP ? VS : KS;
    for (uint32_t i = tiles > n ? tiles - n : 0; i < tiles; ++i) {
      const uint32_t slot = i % n;
      mb_drain(smem_at(warp > LOAD_WARP ? &s.v_raw[slot] : &s.k_full[slot]), (i / n) & 1);
      if (ok) mb_drain(smem_at(warp > LOAD_WARP ? &s.v_empty[slot] : &s.k_empty[slot]), (i / n) & 1);
    }
  }
};

template <int DT, int D, int NT, int KEYS, int KS, int VS>
void pick(AttnEntry* e) {
  attn_tile_pick<Tile8<Tile8Shape<DT, D, NT, KEYS, KS, VS>>>(e);
  e->kv8 = true;
}

}  // namespace

bool attn_tile8_entry(int32_t dtype, int32_t D, AttnEntry* e) {
  *e = AttnEntry{};
  if (D == 64) dtype == DT_BF16 ? pick<DT_BF16, 64, 2, 128, 4, 4>(e) : pick<DT_FP16, 64, 2, 128, 4, 4>(e);
  else if (D == 128) dtype == DT_BF16 ? pick<DT_BF16, 128, 2, 128, 2, 3>(e) : pick<DT_FP16, 128, 2, 128, 2, 2>(e);
  else if (D == 256) dtype == DT_BF16 ? pick<DT_BF16, 256, 1, 64, 3, 3>(e) : pick<DT_FP16, 256, 1, 64, 2, 2>(e);
  return e->fn != nullptr;
}

}  // namespace trident
