// rope_paged8.cu -- RoPE over part of each head with the append to a paged cache held in 8 bits (kv8.cuh).
//
// A block's scale needs the largest magnitude of all of its rows before the first code can be written. Rows of one
// block come from consecutive tokens with consecutive slots (a run), so a run is one team's: it takes its rows,
// rotates them in fp32, agrees on the largest magnitude and writes the codes, reading k and v once (runs of more than 64
// rows, 32 of heads above 128: twice). A run that
// begins with its block's first row begins the block anew; another goes on with it, and where its own rows need a
// larger scale, the block's other rows are rounded to that one (read and written again: the smaller the block and
// the longer it lives, the rarer).
//
// q has no such ties: other blocks of the grid rotate it a few rows at a time, as rope_paged.cu does.
#include <type_traits>

#include "kv8.cuh"
#include "rope_paged.cuh"

namespace trident {
namespace {

// Is token t the first of a run; the run that it begins has run_length tokens.
__device__ __forceinline__ bool slot_valid(const RopePagedParams& p, int32_t slot) { return slot >= 0 && slot < p.slots; }
__device__ __forceinline__ int32_t in_block(const RopePaged8Params& p, int32_t slot) {
  return slot - (int32_t)fast_div((uint32_t)slot, p.block.magic, p.block.shift) * p.block.d;
}
__device__ __forceinline__ bool run_starts(const RopePaged8Params& p, int64_t t, int32_t slot) {
  if (!slot_valid(p.r, slot)) return false;
  return t == 0 || p.r.slot[t - 1] != slot - 1 || in_block(p, slot) == 0;
}
__device__ __forceinline__ bool pos_valid(int32_t pos) { return pos >= 0 && pos < kPosLimit; }

// A slot's block: its scale and its first row (kv head h).
struct Block8 {
  uint8_t* scale;
  uint8_t* row0;
  int64_t row;  // bytes from row to row
};
__device__ __forceinline__ Block8 block_of(const RopePaged8Params& p, bool is_v, int32_t slot, int h) {
  const PagedCache& c = is_v ? p.r.vc : p.r.kc;
  const uint32_t pg = fast_div((uint32_t)slot, p.r.page.magic, p.r.page.shift);
  const uint32_t at = (uint32_t)slot - pg * (uint32_t)p.r.page.d;
  const uint32_t blk = fast_div(at, p.block.magic, p.block.shift);
  Block8 b;
  b.scale = scale_at(is_v ? p.vs : p.ks, pg, h, (int)blk);
  b.row0 = reinterpret_cast<uint8_t*>(c.base) + (int64_t)pg * c.page + (int64_t)h * c.head + (int64_t)blk * p.block.d * c.row;
  b.row = c.row;
  return b;
}

// ---------------------------------------------------------------- any alignment, any even R
// Element j of a q or k row, normalised by inv * gam[j] and rotated.
template <int DT, bool QKNORM, bool INTER>
__device__ __forceinline__ float row_elem(const RopePagedParams& p, const void* src, int j, int32_t pos, float inv,
                                          const float* gam) {
  auto at = [&](int i) {
    const float v = load_elem<DT>(src, i);
    return QKNORM ? v * (inv * gam[i]) : v;
  };
  if (j >= p.R) return at(j);
  const int i = INTER ? j / 2 : (j < p.R / 2 ? j : j - p.R / 2);
  const int a = INTER ? 2 * i : i, b = INTER ? 2 * i + 1 : i + p.R / 2;
  float sn, cs;
  rope_sincos((float)pos, p.freqs[i].x, p.freqs[i].y, &sn, &cs);
  sn *= p.mag;
  cs *= p.mag;
  const float x = at(a), y = at(b);
  return j == a ? fmaf(x, cs, -y * sn) : fmaf(y, cs, x * sn);
}

// One warp per (token, head-row); a kv head-row has work where its token begins a run, and then takes all of it.
template <int DT, bool QKNORM, bool INTER>
__global__ void __launch_bounds__(kThreads) rope_paged8_generic_kernel(const RopePaged8Params p8) {
  pdl_prologue();
  const RopePagedParams& p = p8.r;
  const int lane = threadIdx.x & 31;
  const int64_t total = p.T * p.NH, nwarps = (int64_t)gridDim.x * (kThreads / 32);
  for (int64_t unit = ((int64_t)blockIdx.x * kThreads + threadIdx.x) / 32; unit < total; unit += nwarps) {
    const int64_t t = unit / p.NH;
    const int hh = (int)(unit - t * p.NH);
    const bool is_q = hh < p.Hq, is_v = hh >= p.Hq + p.Hkv;
    const float* gam = is_q ? p.gamma_q : p.gamma_k;
    auto inverse = [&](const void* src) {
      if (!QKNORM || is_v) return 1.f;
      float ss = 0.f;
      for (int j = lane; j < p.D; j += 32) {
        const float v = load_elem<DT>(src, j);
        ss = fmaf(v, v, ss);
      }
      return rsqrtf(warp_sum(ss) * p.inv_D + p.eps);
    };
    const int32_t pos = p.pos[t], slot = p.slot[t];
    if (!pos_valid(pos) && lane == 0) atomicOr(p.err, kErrPos);
    if (is_q) {
      if (!pos_valid(pos)) continue;
      const void* src = paged_src(p, t, hh);
      char* dst = row_ptr(p.q_out, t, p.o_rs, 2) + (int64_t)hh * p.D * 2;
      const float inv = inverse(src);
      // in place: a pair's elements are read and written by one lane
      for (int i = lane; i < p.R / 2; i += 32) {
        const int a = INTER ? 2 * i : i, b = INTER ? 2 * i + 1 : i + p.R / 2;
        const float x = row_elem<DT, QKNORM, INTER>(p, src, a, pos, inv, gam);
        const float y = row_elem<DT, QKNORM, INTER>(p, src, b, pos, inv, gam);
        store_elem<DT>(dst, a, x);
        store_elem<DT>(dst, b, y);
      }
      for (int j = p.R + lane; j < p.D; j += 32) store_elem<DT>(dst, j, row_elem<DT, QKNORM, INTER>(p, src, j, pos, inv, gam));
      continue;
    }
    if (slot >= p.slots && lane == 0) atomicOr(p.err, kErrSlot);
    if (!run_starts(p8, t, slot)) continue;
    const int first = in_block(p8, slot);
    int n = 1;
    while (t + n < p.T && first + n < p8.block.d && p.slot[t + n] == slot + n) ++n;
    const Block8 blk = block_of(p8, is_v, slot, hh - p.Hq - (is_v ? p.Hkv : 0));
    auto elem = [&](const void* src, int j, int32_t at, float inv) {
      return is_v ? load_elem<DT>(src, j) : row_elem<DT, QKNORM, INTER>(p, src, j, at, inv, gam);
    };
    float top = 0.f;
    for (int i = 0; i < n; ++i) {
      const int32_t at = p.pos[t + i];
      if (!pos_valid(at)) continue;
      const void* src = paged_src(p, t + i, hh);
      const float inv = inverse(src);
      for (int j = lane; j < p.D; j += 32) top = fmaxf(top, fabsf(elem(src, j, at, inv)));
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    int e = scale_for(top);
    if (first > 0) {
      const int old = scale_exp(*blk.scale);
      e = max(e, old);
      if (e > old)
        for (int r = 0; r < p8.block.d; ++r) {
          if (r >= first && r < first + n) continue;
          uint8_t* row = blk.row0 + r * blk.row;
          for (int j = lane; j < p.D; j += 32) row[j] = (uint8_t)codes2(code_value(row, j) * exp2_int(old - e), 0.f);
        }
    }
    __syncwarp();  // the old scale has been read by every lane
    if (lane == 0) *blk.scale = (uint8_t)(e + 127);
    for (int i = 0; i < n; ++i) {
      const int32_t at = p.pos[t + i];
      if (!pos_valid(at)) continue;
      const void* src = paged_src(p, t + i, hh);
      const float inv = inverse(src);
      uint8_t* row = blk.row0 + (first + i) * blk.row;
      for (int j = lane; j < p.D; j += 32) row[j] = (uint8_t)codes2(elem(src, j, at, inv) * exp2_int(-e), 0.f);
    }
  }
}

// ---------------------------------------------------------------- 16-byte aligned rows
// A head-row by LPG lanes with two vectors of eight elements each (rope_paged.cuh), GW head-rows per warp at a time,
// PASS times: ROWS rows of one head whose loads are issued together and whose values stay in shared memory between the
// largest magnitude and the codes (in registers they left an SM twelve warps). Teams:
//   TEAM 1  blocks of at most ROWS rows. A warp looks a window of tokens over and takes whole runs, as many as its
//           rows hold: 16 decode steps or a block of a prompt cost the same round of loads.
//   TEAM 4  larger blocks. The thread block's warps share a run, TEAM * ROWS rows at a time; a longer one is read and
//           rotated twice. Runs come one after the other, so decode steps, whose runs are of one row, leave three of four
//           warps without work: measured below.
// Thread blocks past kv_blocks rotate q, items of R heads per lane group as rope_paged.cu. They come in as the append's
// blocks end: that waits for its chains, q for the memory.
//
// Measured on a GB300 (32 + 8 + 8 heads of 128, bf16, blocks of 16): 64 decode steps with q/k norm 4.5 us (windows of 16
// tokens, four rows after one another per warp: 7.7), one prompt of 8192 tokens 44 us (0.62 of the copy rate; q in a launch
// of its own 49, append blocks spread among q's 45), of which q's 134 MB would take 21 alone; the append is bound by its
// chain of loads, rotation (a token's sines and cosines once per kv head), maximum and codes. 3333 tokens, half of the
// head, blocks of 32: 25 us (one head of q per lane group 32, three 26).
// Decode steps by teams, 64 / 512 steps of these heads with q/k norm: blocks of 1 or 16 rows (a warp's) 4.2 to 4.5 / 8.4 to
// 9.5 us, of 32 or 64 (a thread block's) 9.5 / 35; heads of 256, blocks of 8 5.8 / 16, of 16 and more 9.6 / 36. The team goes
// by the block's size though a run may be shorter.
constexpr int kRope8Threads = 128;

template <int DT, int LPG, bool INTER, int TEAM>
struct Append8 {
  static constexpr int GW = 32 / LPG, PASS = LPG == 4 ? 2 : 4, ROWS = GW * PASS, CAP = TEAM * ROWS;
  static_assert(TEAM > 1 || CAP <= 16, "a warp's look at its tokens reaches past its rows");
  struct Smem {
    float4 x[4][PASS * 4][32];  // the lanes' values between the largest magnitude and the codes, 16 per row
    float top[4][16];
    int32_t grown[4][16];
  };
  // What a lane holds of a head-row.
  struct Lane {
    int l, va, vb;
    bool on, rot;
    float4 fq[4];
  };

  static __device__ __forceinline__ float group_max(float v) {
#pragma unroll
    for (int o = LPG / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
  }

  // Rows r(j) < n of the run tokens a + r: their values, to the lane's words of s.x, and each row's largest magnitude to
  // m(j, .) (0: no such row, or skipped for its position). Returns the rows that count, a bit each. All loads are
  // issued first and wait in the same words; then a row at a time, so that few registers leave the SM many warps.
  template <class Row, class Most>
  static __device__ __forceinline__ unsigned values(const RopePaged8Params& p8, Smem& s, const Lane& ln, int64_t a, int n, int hh,
                                                    Row row, Most most) {
    const RopePagedParams& p = p8.r;
    const bool is_v = hh >= p.Hq + p.Hkv;
    uint4* mine = reinterpret_cast<uint4*>(&s.x[threadIdx.x >> 5][0][threadIdx.x & 31]);  // word i: mine[32 i]
    const int g = (threadIdx.x & 31) / LPG;
    int32_t pos[PASS];
    {
      uint4 lo[PASS], hi[PASS];
#pragma unroll
      for (int j = 0; j < PASS; ++j) {
        const int64_t t = a + min(row(j), n - 1);
        const char* src = paged_src(p, t, hh);
        lo[j] = ld16(src + ln.va * 2);
        hi[j] = ld16(src + ln.vb * 2);
        pos[j] = p.pos[t];
      }
#pragma unroll
      for (int j = 0; j < PASS; ++j) {
        mine[128 * j] = lo[j];
        mine[128 * j + 32] = hi[j];
      }
    }
    unsigned live = 0;
#pragma unroll
    for (int j = 0; j < PASS; ++j) {
      if (row(j) >= n) continue;
      if (pos_valid(pos[j])) live |= 1u << j;
      else if (ln.l == 0) atomicOr(p.err, kErrPos);
    }
#pragma unroll 1
    for (int j = 0; j < PASS && row(j) - g < n; ++j) {
      const uint4 lo = mine[128 * j], hi = mine[128 * j + 32];
      float x[16];
      if (is_v) {
        unpack<DT>(lo, x);
        unpack<DT>(hi, x + 8);
      } else {
        int32_t at = pos[0];
#pragma unroll
        for (int k = 1; k < PASS; ++k)
          if (j == k) at = pos[k];
        RopeAngles an;
        paged_angles(p, live >> j & 1u ? at : 0, ln.fq, &an);
        if (p.gamma_k) paged_row_math<DT, LPG, true, INTER>(p, lo, hi, p.gamma_k, an, ln.on, ln.rot, ln.va, ln.vb, x, x + 8);
        else paged_row_math<DT, LPG, false, INTER>(p, lo, hi, nullptr, an, ln.on, ln.rot, ln.va, ln.vb, x, x + 8);
      }
      float top = 0.f;
#pragma unroll
      for (int e = 0; e < 16; ++e) top = fmaxf(top, fabsf(x[e]));
#pragma unroll
      for (int e = 0; e < 4; ++e)
        *reinterpret_cast<float4*>(&mine[128 * j + 32 * e]) = make_float4(x[4 * e], x[4 * e + 1], x[4 * e + 2], x[4 * e + 3]);
      most(j, group_max(ln.on && (live >> j & 1u) ? top : 0.f));
    }
    return live;
  }

  static __device__ __forceinline__ void put(const Smem& s, const Lane& ln, uint8_t* row, int j, int e) {
    const float f = exp2_int(-e);
    float y[16];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float4 v = s.x[threadIdx.x >> 5][4 * j + i][threadIdx.x & 31];
      y[4 * i] = v.x * f; y[4 * i + 1] = v.y * f; y[4 * i + 2] = v.z * f; y[4 * i + 3] = v.w * f;
    }
    const uint2 a = make_uint2(codes4(y), codes4(y + 4)), b = make_uint2(codes4(y + 8), codes4(y + 12));
    if (ln.vb == ln.va + 8) {
      st16(row + ln.va, make_uint4(a.x, a.y, b.x, b.y));
    } else {
      *reinterpret_cast<uint2*>(row + ln.va) = a;
      *reinterpret_cast<uint2*>(row + ln.vb) = b;
    }
  }

  // The block's rows outside [first, first + n) to a scale 2^by larger; `who` of `of` threads.
  static __device__ __forceinline__ void rescale(const RopePaged8Params& p, const Block8& b, int first, int n, int by, int who, int of) {
    const int vecs = p.r.D / 16;
    const float f = exp2_int(-by);
    for (int i = who; i < (p.block.d - n) * vecs; i += of) {
      int r = i / vecs;
      uint8_t* at = b.row0 + (int64_t)(r < first ? r : r + n) * b.row + (i - r * vecs) * 16;
      const uint4 v = ld16(at);
      const uint32_t w[4] = {v.x, v.y, v.z, v.w};
      uint32_t u[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float2 c = values2(halves2(w[k])), d = values2(halves2_hi(w[k]));
        u[k] = codes2(c.x * f, c.y * f) | codes2(d.x * f, d.y * f) << 16;
      }
      st16(at, make_uint4(u[0], u[1], u[2], u[3]));
    }
  }

  // A warp's window [t0, end) of tokens, head-row hh.
  static __device__ __forceinline__ void window(const RopePaged8Params& p8, Smem& s, const Lane& ln, int64_t t0, int64_t end, int hh) {
    const RopePagedParams& p = p8.r;
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, g = lane / LPG;
    const bool is_v = hh >= p.Hq + p.Hkv;
    const int h = hh - p.Hq - (is_v ? p.Hkv : 0);
    int64_t a = t0;
    while (a < end) {
      // 32 tokens from a on: which begin a run, which go on with one
      const bool in = a + lane < p.T;
      const int32_t slot = in ? p.slot[a + lane] : -1;
      int32_t before = __shfl_up_sync(0xffffffffu, slot, 1);
      if (lane == 0) before = a > 0 ? p.slot[a - 1] : -2;
      const bool valid = slot_valid(p, slot);
      if (slot >= p.slots && a + lane < end) atomicOr(p.err, kErrSlot);
      const bool begins = valid && (before != slot - 1 || in_block(p8, slot) == 0 || (a == 0 && lane == 0));
      const unsigned starts = __ballot_sync(0xffffffffu, begins), on = __ballot_sync(0xffffffffu, valid && !begins);
      const unsigned mine = end - a < 32 ? starts & ((1u << (end - a)) - 1u) : starts;
      if (mine == 0) {
        a += 32;
        continue;
      }
      if (!(mine & 1u)) {
        a += __ffs(mine) - 1;
        continue;
      }
      // whole runs from a on that fit the rows; none that begins past the window
      // the last of rows 1 .. CAP that does not go on with a run: no run is longer than a block, which CAP rows hold
      int n = max(1, 31 - __clz(~on & ((2u << CAP) - 1u)));
      n = (int)min((int64_t)n, p.T - a);
      const unsigned past = starts & ~mine;
      if (past) n = min(n, __ffs(past) - 1);
      auto row = [&](int j) { return j * GW + g; };
      // each row's run: its first row and the one past its last; its block, and that block's scale
      int first[PASS], stop[PASS], old[PASS];
      int32_t at[PASS];
      bool has[PASS];
#pragma unroll
      for (int j = 0; j < PASS; ++j) {
        const int r = min(row(j), n - 1);
        at[j] = __shfl_sync(0xffffffffu, slot, r);
        has[j] = row(j) < n && ((starts | on) >> r & 1u);
        const unsigned upto = starts & ((2u << r) - 1u);
        first[j] = upto ? 31 - __clz(upto) : 0;
        stop[j] = r + 1 + (__ffs(~(on >> (r + 1))) - 1);
        old[j] = kScaleLo;
        if (has[j] && in_block(p8, at[j]) > row(j) - first[j])  // the block was begun by an earlier call
          old[j] = scale_exp(*block_of(p8, is_v, at[j], h).scale);
      }
      const unsigned live = values(p8, s, ln, a, n, hh, row, [&](int j, float top) {
        if (ln.l == 0) s.top[w][row(j)] = row(j) < n ? top : 0.f;
      });
      __syncwarp();
#pragma unroll
      for (int j = 0; j < PASS; ++j) {
        float top = 0.f;
        for (int i = first[j] + ln.l; i < stop[j] && i < CAP; i += LPG) top = fmaxf(top, s.top[w][i]);
        const int e = max(old[j], scale_for(group_max(top)));
        const bool lead = has[j] && row(j) == first[j];
        const int by = lead && in_block(p8, at[j]) > 0 ? e - old[j] : 0;
        if (ln.l == 0) s.grown[w][row(j)] = by;
        if (!has[j]) continue;
        const Block8 blk = block_of(p8, is_v, at[j], h);
        if (lead && ln.l == 0) *blk.scale = (uint8_t)(e + 127);
        if ((live >> j & 1u) && ln.on) put(s, ln, blk.row0 + in_block(p8, at[j]) * blk.row, j, e);
      }
      __syncwarp();
      unsigned grown = __ballot_sync(0xffffffffu, lane < n && s.grown[w][min(lane, CAP - 1)] > 0);
      for (; grown; grown &= grown - 1) {
        const int r = __ffs(grown) - 1;
        const int32_t sl = __shfl_sync(0xffffffffu, slot, r);
        const int len = __ffs(~(on >> (r + 1)));
        rescale(p8, block_of(p8, is_v, sl, h), in_block(p8, sl), len, s.grown[w][r], lane, 32);
      }
      __syncwarp();
      a += n;
    }
  }

  // The same by the whole thread block, a run at a time.
  static __device__ __forceinline__ void windows_of_team(const RopePaged8Params& p8, Smem& s, const Lane& ln, int64_t t0, int64_t end,
                                                         int hh) {
    const RopePagedParams& p = p8.r;
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, g = lane / LPG;
    const bool is_v = hh >= p.Hq + p.Hkv;
    const int h = hh - p.Hq - (is_v ? p.Hkv : 0);
    for (int64_t base = t0; base < end; base += 32) {
      // the runs that begin among 32 tokens (every warp looks for itself)
      const int64_t t = base + lane;
      const int32_t slot = t < end ? p.slot[t] : -1;
      if (slot >= p.slots && w == 0) atomicOr(p.err, kErrSlot);
      unsigned starts = __ballot_sync(0xffffffffu, t < end && run_starts(p8, t, slot));
      for (; starts; starts &= starts - 1) {
        const int64_t a = base + __ffs(starts) - 1;
        const int32_t s0 = __shfl_sync(0xffffffffu, slot, __ffs(starts) - 1);
        const int at = in_block(p8, s0), most = (int)min((int64_t)(p8.block.d - at), p.T - a);
        int n = 1;  // the run's tokens
        while (n < most) {
          const bool goes = n + lane < most && p.slot[a + n + lane] == s0 + n + lane;
          const unsigned stop = __ballot_sync(0xffffffffu, !goes);
          n += stop ? __ffs(stop) - 1 : 32;
          if (stop) break;
        }
        const Block8 blk = block_of(p8, is_v, s0, h);
        const int old = at > 0 ? scale_exp(*blk.scale) : kScaleLo;
        float top = 0.f;
        unsigned live = 0;
        int c = 0;
        auto row = [&](int j) { return c * CAP + (j * TEAM + w) * GW + g; };
        for (; c * CAP < n; ++c) {
          live = values(p8, s, ln, a, n, hh, row, [&](int, float m) { top = fmaxf(top, m); });
        }
#pragma unroll
        for (int o = 16; o >= LPG; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        __syncthreads();  // the words below have been read for the run before
        if (lane == 0) s.top[0][w] = top;
        __syncthreads();
        const int e = max(old, scale_for(fmaxf(fmaxf(s.top[0][0], s.top[0][1]), fmaxf(s.top[0][2], s.top[0][3]))));
        if (threadIdx.x == 0) *blk.scale = (uint8_t)(e + 127);
        const bool again = n > CAP;
        for (c = 0; c * CAP < n; ++c) {
          if (again) live = values(p8, s, ln, a, n, hh, row, [](int, float) {});
#pragma unroll
          for (int j = 0; j < PASS; ++j)
            if ((live >> j & 1u) && ln.on) put(s, ln, blk.row0 + (int64_t)(at + row(j)) * blk.row, j, e);
        }
        if (at > 0 && e > old) rescale(p8, blk, at, n, e - old, threadIdx.x, kRope8Threads);
      }
    }
  }
};

template <int DT, int LPG, bool INTER, int TEAM, int R>
__global__ void __launch_bounds__(kRope8Threads, 4) rope_paged8_kernel(const RopePaged8Params p8, const Rope8Grid grid) {
  using K = Append8<DT, LPG, INTER, TEAM>;
  __shared__ typename K::Smem smem;
  pdl_prologue();
  const RopePagedParams& p = p8.r;
  const int l = (threadIdx.x & 31) % LPG;
  typename K::Lane ln;
  ln.l = l;
  const int lane = min(l, p.D / 16 - 1);
  ln.on = l == lane;
  ln.rot = lane < p.R / 16;
  lane_vectors<INTER>(p, lane, &ln.va, &ln.vb);
  if (blockIdx.x < (unsigned)grid.kv_blocks) {
    const int64_t unit = TEAM > 1 ? blockIdx.x : (int64_t)blockIdx.x * (kRope8Threads / 32) + threadIdx.x / 32;
    const int64_t win = unit / (2 * p.Hkv), t0 = win * grid.window;
    if (t0 >= p.T) return;
    const int hh = p.Hq + (int)(unit - win * (2 * p.Hkv));
    if (hh < p.Hq + p.Hkv) paged_freqs(p, lane, ln.rot, ln.fq);
    const int64_t end = min(p.T, t0 + grid.window);
    if constexpr (TEAM > 1) K::windows_of_team(p8, smem, ln, t0, end, hh);
    else K::window(p8, smem, ln, t0, end, hh);
    return;
  }
  constexpr int GW = 32 / LPG;
  const int64_t item = (int64_t)(blockIdx.x - grid.kv_blocks) * (kRope8Threads / 32) + threadIdx.x / 32;
  if (item >= p.T * p.ipt) return;
  const uint32_t tok = fast_div((uint32_t)item, p.ipt_magic, p.ipt_shift);
  const int64_t t = tok;
  const int first = (int)((uint32_t)item - tok * (uint32_t)p.ipt) * p.rpi, end = min(p.Hq, first + p.rpi);
  const int hh0 = first + (threadIdx.x & 31) / LPG;
  uint4 lo[R], hi[R];
#pragma unroll
  for (int j = 0; j < R; ++j) {  // groups past the item's end load its last row and drop it
    const char* src = paged_src(p, t, min(hh0 + j * GW, end - 1));
    lo[j] = ld16(src + ln.va * 2);
    hi[j] = ld16(src + ln.vb * 2);
  }
  const int32_t pos = p.pos[t];
  paged_freqs(p, lane, ln.rot, ln.fq);
  if (!pos_valid(pos)) {
    if ((threadIdx.x & 31) == 0) atomicOr(p.err, kErrPos);
    return;
  }
  RopeAngles an;
  paged_angles(p, pos, ln.fq, &an);
#pragma unroll
  for (int j = 0; j < R; ++j) {
    const int hh = hh0 + j * GW;
    float x[8], y[8];
    if (p.gamma_q) paged_row_math<DT, LPG, true, INTER>(p, lo[j], hi[j], p.gamma_q, an, ln.on, ln.rot, ln.va, ln.vb, x, y);
    else paged_row_math<DT, LPG, false, INTER>(p, lo[j], hi[j], nullptr, an, ln.on, ln.rot, ln.va, ln.vb, x, y);
    if (ln.on && hh < end) {
      char* dst = row_ptr(p.q_out, t, p.o_rs, 2) + (int64_t)hh * p.D * 2;
      st16(dst + ln.va * 2, pack<DT>(x));
      st16(dst + ln.vb * 2, pack<DT>(y));
    }
  }
}

template <int DT, int LPG, bool INTER>
void pick_vec(KernelEntry* out) {
  out->any_fn[0] = (const void*)rope_paged8_kernel<DT, LPG, INTER, 1, 1>;
  out->any_fn[1] = (const void*)rope_paged8_kernel<DT, LPG, INTER, 1, 4>;
  out->any_fn[2] = (const void*)rope_paged8_kernel<DT, LPG, INTER, 4, 1>;
  out->any_fn[3] = (const void*)rope_paged8_kernel<DT, LPG, INTER, 4, 4>;
}

}  // namespace

// The entry of a vector call; sets q's item split (the rule of rope_paged.cu: items of one head per lane group where
// they do not fill the GPU), the grid and its parts.
constexpr int64_t kRope8Small = 8;  // warps per SM
int rope_paged8_plan(RopePaged8Params* p8, Rope8Grid* grid, int32_t* threads, int64_t* blocks, int32_t sms) {
  RopePagedParams* p = &p8->r;
  const int lpg = p->D <= 64 ? 4 : p->D <= 128 ? 8 : 16, gw = 32 / lpg, rows = gw * (lpg == 4 ? 2 : 4);
  const bool team = p8->block.d > rows;
  constexpr int kWarps = kRope8Threads / 32;
  RopeSplit r = rope_split(p->Hq, gw, 1);
  if (p->T * r.ipt > 3 * (int64_t)sms) r = rope_split(p->Hq, gw, 4);
  p->ipt = r.ipt;
  p->rpi = r.rpi;
  p->ipt_magic = r.magic;
  p->ipt_shift = r.shift;
  // Tokens of a team's window: as many as a warp's rows; few tokens, whose runs may all be of one, in smaller windows for
  // more warps. 32 + 8 + 8 heads of 128 with q/k norm, windows of 4 / of 16 tokens, us: decode steps in blocks of 16, 64 of
  // them 4.4 / 7.3, 304 5.4 / 8.6, 512 7.5 / 9.5, 768 9.0 / 9.1, 1024 11.8 / 10.1, in blocks of 64 9.6 / 29.8, 19.6 / 31.7,
  // 32.6 / 35.1, 45.9 / 58.0, 59.5 / 65.6; a prompt of 304 in blocks of 16 7.5 / 10.6, of 64 7.0 / 7.0, 512 7.9 / 11.1 and
  // 8.6 / 6.7, 1024 9.4 / 11.3 and 12.8 / 8.7. The line (304 tokens of these heads) is where prompts in large blocks begin to
  // lose by small windows; steps would gain from them up to about 750.
  grid->window = p->T * 2 * p->Hkv <= 4 * kRope8Small * sms ? 4 : 16;
  const int64_t units = (p->T + grid->window - 1) / grid->window * 2 * p->Hkv;
  const int64_t kv = team ? units : (units + kWarps - 1) / kWarps, q = (p->T * r.ipt + kWarps - 1) / kWarps;
  grid->kv_blocks = (int32_t)kv;
  *threads = kRope8Threads;
  *blocks = kv + q;
  return (team ? 2 : 0) + (r.rpi > gw ? 1 : 0);
}

bool rope_paged8_kernel(int32_t dtype, int32_t variant, int32_t D, int32_t R, bool qknorm, bool inter,
                        KernelEntry* out, const char** why) {
  if (dtype != DT_BF16 && dtype != DT_FP16) { *why = "RoPE supports bf16 and fp16"; return false; }
  out->kind = KK_ROPE_PAGED8;
  if (variant != 1) {
    if (D % 16 != 0 || R % 16 != 0 || D < 32 || D > 256) {
      *why = "vector paged RoPE supports D in 32 .. 256 and R that are multiples of 16";
      return false;
    }
    out->vec = 8;
    auto vec = [&](auto dt) {
      constexpr int DT = decltype(dt)::value;
      if (D <= 64) inter ? pick_vec<DT, 4, true>(out) : pick_vec<DT, 4, false>(out);
      else if (D <= 128) inter ? pick_vec<DT, 8, true>(out) : pick_vec<DT, 8, false>(out);
      else inter ? pick_vec<DT, 16, true>(out) : pick_vec<DT, 16, false>(out);
    };
    if (dtype == DT_BF16) vec(std::integral_constant<int, DT_BF16>());
    else vec(std::integral_constant<int, DT_FP16>());
    out->fn = out->any_fn[0];
    return true;
  }
  out->vec = 1;
  auto pick = [&](auto dt) {
    constexpr int DT = decltype(dt)::value;
    return qknorm ? (inter ? (const void*)rope_paged8_generic_kernel<DT, true, true> : (const void*)rope_paged8_generic_kernel<DT, true, false>)
                  : (inter ? (const void*)rope_paged8_generic_kernel<DT, false, true> : (const void*)rope_paged8_generic_kernel<DT, false, false>);
  };
  out->fn = dtype == DT_BF16 ? pick(std::integral_constant<int, DT_BF16>()) : pick(std::integral_constant<int, DT_FP16>());
  return true;
}

}  // namespace trident
