// attn_tile.cu -- paged attention for requests of many rows: chunks of a prompt.
//
// Bound: the tensor cores. A unit is NT tiles of 128 rows (tokens x the G heads of a group, so that all of
// them share the keys' loads) against tiles of KEYS keys; per block NT softmax warpgroups, NT warps that
// issue tcgen05.mma and two that load:
//   load     two warps, k and v tiles by TMA, a box per page, into rings of KEYS x D slots in the 128-byte
//            swizzle; a unit's last v tile gets zeros in the rows past the last key up to the next 16 (a pool's
//            unused rows may hold NaN, and 0 * NaN would reach the sums)
//   mma      S_x = Q_x K^T into TMEM, then for each tile O_x += P_x V with P_x from TMEM; the tiles take
//            turns, so that one tile's products run while the other tile's softmax does
//   softmax  a thread per row, so no exchange between lanes: 128 scores from TMEM, running maximum and
//            sum, numerators rounded to the activation type back into the columns of S_x
// The running maximum moves only when a score passes it by 2^kLazy; then the row's accumulator in TMEM is
// rescaled by its own thread, which may touch it because S_x of the next tile is issued after P_x V.
// TMEM columns: NT x KEYS of S (P in their first half) and NT x D of O.
//
// Every wait is bounded (params.polls polls, kBulkWaitPolls by default): a wait that runs out sets
// TRIDENT_DEVERR_TIMEOUT and a flag that ends the block's other waits; the warps then let their copies
// and products in flight finish (bounded again), free the TMEM and return without further writes.
//
// Measured on a GB300 (32 q heads on 8 kv heads of 128): 8192 rows after 8192 keys 1035 to 1066 us back to back
// (1593 to 1547 TFLOP/s, 0.94 to 0.92 of cuBLAS' sustained rate, at the power limit); 2048 rows after 6144 keys
// 155 us in a graph of 30 calls, 166 longer, 1000 after 3096 55 us; 2048 after 6144 with heads of 64 126 us, of 256
// 456 us. 128 keys
// of a unit take 1.26 us, about 2500 cycles, 2048 of them the products at the full rate; what is more is the
// chain of a tile's scores, softmax and products. Before its first tile a block takes 6 us (lengths, its share,
// q), a cut part 4 us to write and 2.5 us to count, the last one 8 us to join.
#include "attn_tile.cuh"

namespace trident {
namespace {

template <int DT_, int D_, int NT_, int KEYS_, int SLOTS_>
struct Tile16Shape {
  static constexpr int DT = DT_, D = D_, NT = NT_, KEYS = KEYS_, SLOTS = SLOTS_;
  static constexpr int OTHERS = 128;           // mma, load and idle warps: a warpgroup, for setmaxnreg
  // Registers: a softmax row takes its 128 scores and their numerators' words, the other warps few.
  static constexpr int OTHER_REGS = 88, SOFT_REGS = NT == 2 ? 208 : 232;
  static constexpr int QB = 128 * D * 2;       // bytes of a q tile
  static constexpr int KB = KEYS * D * 2;      // ... of a k or v tile
  struct Smem : TileShape<Tile16Shape>::Common {
    alignas(1024) char q[NT * QB];
    alignas(1024) char ring[SLOTS * KB];
    alignas(8) uint64_t full[SLOTS], empty[SLOTS], raw;
  };
};

template <class C>
struct Tile16 : TileFrame<Tile16<C>, C> {
  using F = TileFrame<Tile16<C>, C>;
  using F::DT; using F::D; using F::NT; using F::KEYS; using F::S_COL; using F::O_COL; using F::MMA_WARP;
  using typename F::Smem; using typename F::Soft;
  using F::turn_wait; using F::turn_pass;
  static constexpr int SLOTS = C::SLOTS, QB = C::QB, KB = C::KB;
  static constexpr int KS = SLOTS / 2;         // ring slots of k, and as many of v after them
  static constexpr int QHALF = 128 * 128, KHALF = KEYS * 128;  // bytes of 64 columns
  static constexpr int LOAD_WARP = MMA_WARP + NT;

  static __device__ __forceinline__ void init(Smem& s) {
    for (int i = 0; i < SLOTS; ++i) {
      mb_init(smem_at(&s.full[i]), 1);
      mb_init(smem_at(&s.empty[i]), NT);
    }
    mb_init(smem_at(&s.raw), 1);
  }

  // ------------------------------------------------------------ load warps, one for k and one for v
  struct Load {
    uint32_t tiles = 0;      // tiles loaded so far
    uint32_t raws = 0;       // v tiles with a wait of their own
    bool bad = false;
  };
  static __device__ __forceinline__ void arrive_lane0(uint32_t bar) {
    if ((threadIdx.x & 31) == 0) mb_arrive(bar);
    __syncwarp();
  }
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
      const int32_t valid = min(KEYS, limit - t * KEYS);
      const int boxes = (valid + box - 1) / box;
      const uint32_t slot = st.tiles % KS + (is_v ? KS : 0), use = st.tiles / KS;
      if (!__all_sync(0xffffffffu, mb_wait(smem_at(&s.empty[slot]), (use & 1) ^ 1, p.polls, &s.abort))) return false;
      const bool tail = is_v && valid % 16 != 0;
      const uint32_t bar = smem_at(tail ? &s.raw : &s.full[slot]), dst = smem_at(s.ring + slot * KB);
      if (lane == 0) mb_expect(bar, (uint32_t)(boxes * box * D * 2));
      __syncwarp();
      if (lane < boxes) {
#pragma unroll
        for (int c = 0; c < D / 64; ++c) tma_4d(dst + c * KHALF + lane * box * 128, map, c * 64, at, h, page, bar);
      }
      __syncwarp();
      ++st.tiles;
      if (tail) {  // zeros from the last key to the next 16
        const uint32_t parity = st.raws++ & 1;
        if (!__all_sync(0xffffffffu, mb_wait(bar, parity, p.polls, &s.abort))) {
          mb_drain(bar, parity);
          arrive_lane0(smem_at(&s.full[slot]));
          return false;
        }
        const int rows = 16 - valid % 16;
        for (int e = lane; e < rows * (D / 8); e += 32) {
          const int r = valid + e / (D / 8), c = e % (D / 8);
          *reinterpret_cast<uint4*>(s.ring + slot * KB + (c / 8) * KHALF + r * 128 + (c % 8) * 16) = make_uint4(0, 0, 0, 0);
        }
        fence_async();
        __syncwarp();
        arrive_lane0(smem_at(&s.full[slot]));
      }
    }
    return true;
  }

  // ------------------------------------------------------------ mma warps, one per q tile
  struct Mma {
    uint32_t tiles = 0;       // key tiles consumed so far
    uint32_t px = 0, qx = 0;  // p and q tiles waited for
  };
  static __device__ __forceinline__ void qk(uint32_t q_lo, uint32_t k_lo, uint32_t d) {
    constexpr uint32_t id = idesc_of<DT>(128, KEYS, false);
#pragma unroll
    for (int k = 0; k < D / 16; ++k)
      mma_ss(d, desc128(q_lo + ((k / 4 * QHALF + k % 4 * 32) >> 4)), desc128(k_lo + ((k / 4 * KHALF + k % 4 * 32) >> 4)), id,
             k > 0);
  }
  // Half of P V: 16-key steps [HALF * KEYS / 32, ...), at most `steps` of the tile's.
  template <int HALF>
  static __device__ __forceinline__ void pv(uint32_t p_col, uint32_t v_lo, uint32_t d, int steps, bool add) {
    constexpr uint32_t id = idesc_of<DT>(128, D, true);
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
    const uint32_t q_lo = desc_lo(smem_at(s.q + x * QB), 16), k_lo = desc_lo(smem_at(s.ring), 16),
                   v_lo = desc_lo(smem_at(s.ring), KHALF);
    const uint32_t sc = tmem + S_COL + x * KEYS, oc = tmem + O_COL + x * D;
    auto wait = [&](uint64_t* bar, uint32_t parity) {
      return __all_sync(0xffffffffu, mb_wait(smem_at(bar), parity, p.polls, &s.abort));
    };
    uint32_t i = st.tiles;
    auto k_slot = [](uint32_t i) { return i % KS; };
    auto v_slot = [](uint32_t i) { return KS + i % KS; };
    auto ready = [&](uint32_t slot, uint32_t i) { return wait(&s.full[slot], (i / KS) & 1); };
    st.tiles += (uint32_t)(t1 - t0);
    if (x > 0 && f.rows <= 128 * x) {  // nothing to do but to give the slots back
      for (; i < st.tiles; ++i) {
        if (!ready(k_slot(i), i) || !ready(v_slot(i), i)) return false;
        if (one) {
          mb_arrive(smem_at(&s.empty[k_slot(i)]));
          mb_arrive(smem_at(&s.empty[v_slot(i)]));
        }
      }
      return true;
    }
    if (!wait(&s.q_full[x], st.qx++ & 1) || !ready(k_slot(i), i)) return false;
    tc_after();
    if (one) {
      qk(q_lo, k_lo + k_slot(i) * (KB >> 4), sc);
      tc_commit(smem_at(&s.s_full[x]));
      tc_commit(smem_at(&s.empty[k_slot(i)]));
    }
    for (int32_t t = t0; t < t1; ++t, ++i) {
      const uint32_t parity = st.px++ & 1;
      const bool more = t + 1 < t1, add = t > t0;
      const int steps = (min(KEYS, limit - t * KEYS) + 15) / 16;
      const uint32_t v_at = v_lo + v_slot(i) * (KB >> 4), k_at = k_lo + k_slot(i + 1) * (KB >> 4);
      if (!ready(v_slot(i), i) || (more && !ready(k_slot(i + 1), i + 1))) return false;
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
          tc_commit(smem_at(&s.empty[k_slot(i + 1)]));
        } else {
          tc_commit(smem_at(&s.o_full[x]));
        }
        tc_commit(smem_at(&s.empty[v_slot(i)]));
      }
    }
    return true;
  }

  // ------------------------------------------------------------ softmax warpgroup
  // Loads this warpgroup's q rows into the swizzled tile: 16 bytes per lane, D / 8 lanes per row.
  static __device__ __forceinline__ void load_q(const PagedAttnParams& p, Smem& s, const Frag& f, int x) {
    constexpr int CH = D / 8, RPI = 32 / CH > 0 ? 32 / CH : 1, ITER = 32 / RPI;
    const int w = (threadIdx.x >> 5) & 3, lane = threadIdx.x & 31, c = lane % CH, rr = lane / CH;
    constexpr int BATCH = ITER < 16 ? ITER : 16;  // loads in flight, none behind a branch: rows past the unit load its last and drop it
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
        if (x * 128 + row >= f.rows) v[e] = make_uint4(0, 0, 0, 0);
        *reinterpret_cast<uint4*>(s.q + x * QB + (c / 8) * QHALF + row * 128 + (((c % 8) ^ (row & 7)) << 4)) = v[e];
      }
    }
    fence_async();
    mb_arrive(smem_at(&s.q_full[x]));
  }

  static __device__ __forceinline__ bool softmax(const PagedAttnParams& p, Smem& s, uint32_t tmem, const Frag& f, int x,
                                                 Soft& st, bool ok, float* m_out, float* l_out) {
    const uint32_t lanes = tmem + (((threadIdx.x >> 5) & 3) << 21);  // TMEM lane 32 * (warp mod 4)
    const uint32_t sc = lanes + S_COL + x * KEYS, oc = lanes + O_COL + x * D;
    // Rows past the unit's (their q is zeros, their results go nowhere) see what its last one does: a row that
    // sees less has every tile's scores masked, and the turn waits for that (1.75 us per tile instead of 1.25).
    const int r = min(x * 128 + (int)(threadIdx.x & 127), f.rows - 1);
    const int32_t see = f.kv - f.n + f.tok0 + (int32_t)fast_div((uint32_t)r, p.group.magic, p.group.shift) + 1;
    const float c = p.scale * kLog2e;
    const bool turns = NT == 2 && f.rows > 128;
    const int32_t t0 = f.t0, t1 = f.t1;
    float m = -INFINITY, l = 0.f;
    if (turns && x == 1) turn_pass(1);
    for (int32_t t = t0; t < t1; ++t) {
      ok = ok && __all_sync(0xffffffffu, mb_wait(smem_at(&s.s_full[x]), st.s & 1, st.s == 0 ? p.first_polls : p.polls, &s.abort));
      ++st.s;
      uint32_t a[KEYS];
      if (turns) turn_wait(x);
      F2 sum[2] = {f2_pack(0.f, 0.f), f2_pack(0.f, 0.f)};
      F2 cc = f2_pack(c, c), mm = cc;
      auto pass = [&]() {
        if (turns && (x == 0 || t + 1 < t1)) turn_pass(x);
      };
      // numerators of half the tile's keys, to the columns of its scores; the turn ends inside the second half
      auto half = [&](int h) {
        uint32_t w[KEYS / 4];
#pragma unroll
        for (int i = 0; i < KEYS / 4; ++i) {
          const int e = h * (KEYS / 2) + 2 * i;
          float u, v;
          f2_unpack(f2_fma(f2_pack(__uint_as_float(a[e]), __uint_as_float(a[e + 1])), cc, mm), &u, &v);
          u = fast_exp2(u);
          v = fast_exp2(v);
          sum[i & 1] = f2_add(sum[i & 1], f2_pack(u, v));
          w[i] = ActType<DT>::pack2(u, v);
          if (h == 1 && i == KEYS / 16 - 1) pass();
        }
#pragma unroll
        for (int k = 0; k < KEYS / 64; ++k) tc_st16(sc + h * (KEYS / 4) + k * 16, w + k * 16);
        tc_wait_st();
        tc_before();
        mb_arrive(smem_at(h == 0 ? &s.p_half[x] : &s.p_full[x]));
      };
      if (ok) {
        tc_after();
#pragma unroll
        for (int i = 0; i < KEYS / 32; ++i) tc_ld32(sc + i * 32, a + i * 32);
        tc_wait_ld<KEYS>(a);
        const int32_t left = see - t * KEYS;  // keys of the tile that the row sees
        if (left < KEYS) {
#pragma unroll
          for (int i = 0; i < KEYS; ++i)
            if (i >= left) a[i] = 0xff800000u;  // -inf
        }
        float top[4];  // three-operand maxima
#pragma unroll
        for (int i = 0; i < 4; ++i) top[i] = fmaxf(__uint_as_float(a[2 * i]), __uint_as_float(a[2 * i + 1]));
#pragma unroll
        for (int i = 8; i < KEYS; i += 2)
          top[i / 2 & 3] = fmaxf(fmaxf(top[i / 2 & 3], __uint_as_float(a[i])), __uint_as_float(a[i + 1]));
        const float hi = attn_level<DT>(c, fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])));
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
        const float base = m == -INFINITY ? 0.f : m;
        mm = f2_pack(-base, -base);
        half(0);  // its products start while the second half's numerators are made
        half(1);
        float s0, s1;
        f2_unpack(f2_add(sum[0], sum[1]), &s0, &s1);
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

  // ------------------------------------------------------------ the other warps
  struct Other {
    Load load;
    Mma mma;
  };
  static __device__ __forceinline__ bool work(const PagedAttnParams& p, const CUtensorMap* mk, const CUtensorMap* mv, Smem& s,
                                              uint32_t tmem, const Frag& f, int warp, Other& st, bool one) {
    if (warp >= LOAD_WARP && warp < LOAD_WARP + 2) return load(p, warp == LOAD_WARP ? mk : mv, s, f, warp > LOAD_WARP, st.load);
    return warp >= LOAD_WARP || mma(p, s, tmem, f, warp - MMA_WARP, st.mma, one);
  }
  static __device__ __forceinline__ void leave(const PagedAttnParams& p, Smem& s, int warp, const Other& st, bool ok) {
    if (warp < LOAD_WARP || warp >= LOAD_WARP + 2) return;
    const Load& ld = st.load;
    for (uint32_t i = ld.tiles > KS ? ld.tiles - KS : 0; i < ld.tiles; ++i) {
      const uint32_t slot = i % KS + (warp > LOAD_WARP ? KS : 0);
      mb_drain(smem_at(&s.full[slot]), (i / KS) & 1);
      if (ok) mb_drain(smem_at(&s.empty[slot]), (i / KS) & 1);
    }
    if (ld.bad) atomicOr(p.err, kErrTable);
  }
};

template <int DT, int D, int NT, int KEYS, int SLOTS>
void pick(AttnEntry* e) {
  attn_tile_pick<Tile16<Tile16Shape<DT, D, NT, KEYS, SLOTS>>>(e);
}

}  // namespace

bool attn_tile_entry(int32_t dtype, int32_t D, AttnEntry* e) {
  *e = AttnEntry{};
  if (D == 64) dtype == DT_BF16 ? pick<DT_BF16, 64, 2, 128, 8>(e) : pick<DT_FP16, 64, 2, 128, 8>(e);
  else if (D == 128) dtype == DT_BF16 ? pick<DT_BF16, 128, 2, 128, 4>(e) : pick<DT_FP16, 128, 2, 128, 4>(e);
  else if (D == 256) dtype == DT_BF16 ? pick<DT_BF16, 256, 1, 64, 4>(e) : pick<DT_FP16, 256, 1, 64, 4>(e);
  return e->fn != nullptr;
}

}  // namespace trident
