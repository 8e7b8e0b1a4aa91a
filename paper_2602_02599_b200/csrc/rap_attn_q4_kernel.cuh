// Split-KV decode scan over a cache held in 4 bits (rap_decode_attn_q4): the copies, the work split and the merge around the
// per-warp arithmetic of rap_attn_q4_block.cuh.  Rows are 52 bytes where bf16 rows are 180.
//   * A tile (256 rows of K and of V, two bulk copies) is shared by the CTA's eight warps, 32 rows each; they take turns to
//     refill the stage of the tile before, once all are done with it (a ring per warp cost a quarter of all instructions).
//     Copies run on across units: batches of short sequences are chains of units, and a unit that one CTA scans alone is
//     written out directly.
//   * The balanced plan counts what a unit costs beside its tiles (Q4Plan).
// Every mbarrier wait is bounded: on timeout the CTA records RAP_ETIMEOUT and leaves.
#pragma once
#include "rap_attn_q4_block.cuh"

namespace {

constexpr int Q4_MAX_STG = 8;            // stages of one tile each
constexpr int Q4_OFF_MAIN = 896;         // barriers, merge scalars and flags below
constexpr int Q4_PAD = 64;               // the last row's fragment loads may reach a few words past it

// KSW, VSW: words per K / V row (odd); GC: heads per lane (1: up to four heads, 2: up to eight)
template <int KSW, int VSW, int GC>
struct Q4Cfg {
  static_assert(KSW % 2 == 1 && VSW % 2 == 1 && KSW <= 17 && VSW <= 17, "rows of up to 128 codes");
  using Engine = std::conditional_t<GC == 1, Q4Whole<KSW, VSW>, Q4Half<KSW, VSW>>;
  // Warps per CTA, two CTAs to an SM: eight of 128 registers, or six of 168 where the whole-number form has four groups of sums to
  // hold (with eight it spilled: 77 us for a batch of 16 with 16K rows of 128, with six 62).
  static constexpr int NW = GC == 1 && Engine::NGV == 4 ? 6 : 8;
  static constexpr int TILE = NW * Q4_BR;                             // rows per CTA tile
  static constexpr int CW = 32 * Engine::NGV;                         // channel slots of the reduction buffer
  static constexpr int MAIN_F = 32 * Engine::SUMS;                    // floats per warp: fp32 sums, then [4 GC][CW] for the merge
  static_assert(MAIN_F == 4 * GC * CW, "the two uses of it");
  static constexpr int STAGE_W = TILE * (KSW + VSW);                  // words per stage
  static constexpr int OFF_RING = Q4_OFF_MAIN + NW * MAIN_F * 4;
  static constexpr int FIT = (SMEM_BUDGET - OFF_RING - Q4_PAD) / (STAGE_W * 4);
  static constexpr int NSTG = FIT < Q4_MAX_STG ? FIT : Q4_MAX_STG;    // 3 for rows of 90, 2 for rows of 128
  static constexpr int SMEM = OFF_RING + NSTG * STAGE_W * 4 + Q4_PAD;
  static_assert(NSTG >= 2 && SMEM <= SMEM_BUDGET, "ring does not fit");
  static_assert(OFF_RING % 128 == 0 && STAGE_W % 32 == 0 && NW * MAIN_F >= RAP_MAX_GROUP * (RAP_MAX_SPLIT + 1), "merge weights fit");
};

struct Q4ScanParams {
  ScanParams s;
  int P, dv, G;
};

// The balanced split here: as in SkPlan, but a unit costs its tiles and Q4_UNIT more (its q, its merge), and where no unit has
// more than Q4_WHOLE tiles units are not split at all (a merge through global memory costs three or four tiles' time).  A
// unit's positions in the sequence that the CTAs share out evenly: Q4_UNIT empty ones, then its tiles; or one for all of them.
constexpr int Q4_UNIT = 2, Q4_WHOLE = 4;
struct Q4Plan : SkPlan {
  bool whole;
  int per, extra;              // T = per nc + extra
  // first position of CTA c, and the CTA that has position s (both as in SkPlan, floor(c T / nc), without 64-bit divisions: in
  // line they were a sixth of the kernel's code, and a short call's time is largely the fetching of code)
  __device__ __forceinline__ int first_of(int c) const { return c * per + (int)((unsigned)(c * extra) / (unsigned)nc); }
  __device__ __forceinline__ int cta_of(int s) const {
    const long long x = ((long long)s + 1) * nc - 1;
    int c = (int)((float)x / (float)T);      // a guess, at most a few off
    c = min(max(c, 0), nc - 1);
#pragma unroll 1
    while (c > 0 && first_of(c) > s) --c;
#pragma unroll 1
    while (c + 1 < nc && first_of(c + 1) <= s) ++c;
    return c;
  }
  __device__ __forceinline__ int positions(int tiles) const { return tiles == 0 ? 0 : whole ? 1 : tiles + Q4_UNIT; }
  __device__ __forceinline__ int empty() const { return whole ? 0 : Q4_UNIT; }
};
// The inclusive prefix of the positions of sequences 0..b goes to pref[0..B) (shared memory, room for `cap` ints; every thread
// of the CTA calls this); a batch too large for it is planned by every thread on its own (false).
__device__ __forceinline__ bool q4_plan(const ScanParams& p, int tile_rows, int* pref, int cap, Q4Plan* out) {
  const bool shared = p.B <= cap - 2;
  const int tid = threadIdx.x, lane = tid & 31;
  auto tiles = [&](int b) { return sk_tiles_of(p.seq_len, b, p.len_add, p.S_cap, tile_rows); };
  long long T = 0;
  int n_max = 0;
  if (!shared) {
#pragma unroll 1
    for (int b = 0; b < p.B; ++b) n_max = max(n_max, tiles(b));
    out->whole = n_max <= Q4_WHOLE;
#pragma unroll 1
    for (int b = 0; b < p.B; ++b) T += (long long)out->positions(tiles(b)) * p.Hkv;
  } else {
    if (tid < 32) {
#pragma unroll 1
      for (int b = lane; b < p.B; b += 32) n_max = max(n_max, tiles(b));
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) n_max = max(n_max, __shfl_xor_sync(0xffffffffu, n_max, o));
      out->whole = n_max <= Q4_WHOLE;
      int carry = 0;
#pragma unroll 1
      for (int base = 0; base < p.B; base += 32) {
        const int b = base + lane;
        int x = b < p.B ? out->positions(tiles(b)) * p.Hkv : 0;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int y = __shfl_up_sync(0xffffffffu, x, o);
          if (lane >= o) x += y;
        }
        if (b < p.B) pref[b] = carry + x;
        carry += __shfl_sync(0xffffffffu, x, 31);
      }
      if (lane == 0) {
        pref[cap - 2] = carry;
        pref[cap - 1] = n_max;
      }
    }
    __syncthreads();
    T = pref[cap - 2];
    n_max = pref[cap - 1];
    out->whole = n_max <= Q4_WHOLE;
  }
  out->T = (int)T;
  out->nc = out->per = out->extra = 0;
  if (T > 0) {
    int nc = min((int)gridDim.x, out->T);
    if (!out->whole) {         // at most RAP_MAX_SPLIT segments a unit: nc <= (RAP_MAX_SPLIT - 2) T / longest
      const unsigned longest = (unsigned)(n_max + Q4_UNIT), q = (unsigned)out->T / longest;
      if (q < 1024u) nc = min(nc, (int)((RAP_MAX_SPLIT - 2) * q + (RAP_MAX_SPLIT - 2) * ((unsigned)out->T - q * longest) / longest));
    }
    out->nc = max(1, nc);
    out->per = out->T / out->nc;
    out->extra = out->T - out->per * out->nc;
  }
  return shared;
}

template <int KSW, int VSW, int GC>
__global__ void __launch_bounds__(Q4Cfg<KSW, VSW, GC>::NW * 32, 2) attn_q4_kernel(const Q4ScanParams pp) {
  using C = Q4Cfg<KSW, VSW, GC>;
  const ScanParams& p = pp.s;
  constexpr int NW = C::NW, THREADS = NW * 32, ST = C::TILE, NSTG = C::NSTG;
  constexpr int CW = C::CW;
  extern __shared__ __align__(128) unsigned char q4_smem[];
  unsigned char* const smem = q4_smem;
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem);                        // [Q4_MAX_STG] a stage's copies have landed; [Q4_MAX_STG] its warps are done with it
  float* m_s = reinterpret_cast<float*>(smem + Q4_MAX_STG * 16);             // [NW][8] references of the warps
  float* l_s = m_s + NW * 8;                                                 // [NW][8] scaled row sums
  int* s_flag = reinterpret_cast<int*>(l_s + NW * 8);                        // time-out seen by any warp
  int* s_last = s_flag + 1;
  float* red = reinterpret_cast<float*>(smem + Q4_OFF_MAIN);                 // [NW][MAIN_F]: sums, merge buffer, merge weights
  static_assert(Q4_MAX_STG * 16 + NW * 64 + 8 <= Q4_OFF_MAIN, "barriers and merge scalars sit below");

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int gid = lane >> 2, tq = lane & 3;
  const int G = pp.G, DV = pp.dv;
  int b = 0, h = 0;
  Q4Plan plan;
  plan.T = 0; plan.nc = 0; plan.whole = false;
  int lo = 0, hi = 0, unit_start = 0;      // this CTA's positions, the current unit's first one
  if (p.balanced) {
    // the plan (reads the lengths only): computed by the first warp where the ring will be
    int* pref = reinterpret_cast<int*>(smem + C::OFF_RING);
    const bool shared_plan = q4_plan(p, ST, pref, NSTG * C::STAGE_W, &plan);
    // everything below reads what the previous kernel in the stream wrote, and writes what the next one may depend on
    pdl_wait();
    pdl_launch_dependents();
    if (blockIdx.x == 0) {   // sequences without any row are scanned by nobody: their output is zero
#pragma unroll 1
      for (int i = tid; i < p.other_units; i += THREADS) p.unit_cnt_other[i] = 0;   // counters a launch that gave up left behind
      if (tid == 0) *p.dyn_next_other = 0;          // and the piece counter a bf16 tensor-core launch before this one used
#pragma unroll 1
      for (int bb = 0; bb < p.B; ++bb) {
        const bool empty = shared_plan ? pref[bb] == (bb > 0 ? pref[bb - 1] : 0)
                                       : sk_tiles_of(p.seq_len, bb, p.len_add, p.S_cap, ST) == 0;
        if (empty)
#pragma unroll 1
          for (int i = tid; i < p.Hq * DV; i += THREADS) p.out[(size_t)bb * p.Hq * DV + i] = 0.f;
      }
    }
    if ((int)blockIdx.x >= plan.nc) return;
    lo = plan.first_of(blockIdx.x);
    hi = plan.first_of(blockIdx.x + 1);
    if (lo >= hi) return;
    int pb = 0;
    if (shared_plan) {       // the unit that holds position `lo`
      b = sk_seq_of(pref, p.B, lo);
      pb = b > 0 ? pref[b - 1] : 0;
    } else {
#pragma unroll 1
      for (b = 0; b < p.B; ++b) {
        const int nb = plan.positions(sk_tiles_of(p.seq_len, b, p.len_add, p.S_cap, ST)) * p.Hkv;
        if (lo < pb + nb) break;
        pb += nb;
      }
    }
    const int per = plan.positions(sk_tiles_of(p.seq_len, b, p.len_add, p.S_cap, ST));
    h = (lo - pb) / per;
    unit_start = pb + h * per;
  } else {
    pdl_wait();
    pdl_launch_dependents();
    b = blockIdx.z;
    h = blockIdx.y;
  }
  const uint32_t bar0 = smem_u32(bars);
  const uint32_t* ring = reinterpret_cast<const uint32_t*>(smem + C::OFF_RING);
  const uint32_t ring_u = smem_u32(ring);
  float* const my_main = red + warp * C::MAIN_F;                              // this warp's sums: [tile][lane][MV] while scanning
  if (tid == 0) {
    *s_flag = 0;
    for (int i = 0; i < Q4_MAX_STG; ++i) {
      mbar_init(bar0 + 8 * i, 1);
      mbar_init(bar0 + 8 * (Q4_MAX_STG + i), NW);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");      // the plan's stores, before copies land on them
  __syncthreads();

  typename C::Engine eng;
  eng.gid = gid; eng.tq = tq; eng.lane = lane;
  eng.at.place(ST, warp, gid, tq);
  int st = 0;                  // ring position of the next tile, running on across units
  uint32_t parity = 0;
  // With three stages or more a tile's stage is refilled when the next tile is done (the others have left it by then); with
  // two that would leave no time for the copy, so the warp whose turn it is waits for the others.
  constexpr int LAG = NSTG >= 3 ? 1 : 0;
  int turn = warp + LAG;       // tiles until this warp refills
  bool timed_out = false;

  // the segment being scanned: tiles [t_begin, t_begin + n_my) of unit (b, h), seg_tiles in all
  int len = 0, seg_tiles = 0, t_begin = 0, n_my = 0;
  auto length = [&](int seq) { return min(max(p.seq_len[seq] + p.len_add, 0), p.S_cap); };
  auto part = [&](int start, int tiles, int& first, int& count) {      // of the unit at position `start`, this CTA's tiles
    first = plan.whole ? 0 : max(0, lo - start - Q4_UNIT);
    count = (plan.whole ? tiles : min(tiles, max(0, hi - start - Q4_UNIT))) - first;
  };
  auto next_unit = [&](int& seq, int& head, int& start, int tiles) {   // (a further one exists where start < hi)
    start += plan.positions(tiles);
    if (++head == p.Hkv) {
      head = 0;
#pragma unroll 1
      do { ++seq; } while (seq < p.B - 1 && sk_tiles_of(p.seq_len, seq, p.len_add, p.S_cap, ST) == 0);
    }
  };
  auto find_segment = [&]() {          // the first unit from (b, h) on that has tiles for this CTA
#pragma unroll 1
    while (unit_start < hi) {
      len = length(b);
      seg_tiles = (len + ST - 1) / ST;
      part(unit_start, seg_tiles, t_begin, n_my);
      if (n_my > 0) return true;
      next_unit(b, h, unit_start, seg_tiles);
    }
    return false;
  };
  if (p.balanced) {
    if (!find_segment()) return;
  } else {
    len = length(b);
    seg_tiles = (len + ST - 1) / ST;
    const int tps = (seg_tiles + p.n_split - 1) / p.n_split;
    t_begin = min(seg_tiles, (int)blockIdx.x * tps);
    n_my = min(seg_tiles, t_begin + tps) - t_begin;
  }
  if (n_my <= 0) {             // (equal ranges only) nothing to scan: neutral partials
    float* base = p.ws + (((size_t)b * p.Hq + (size_t)h * G) * p.n_split + blockIdx.x) * (size_t)(DV + 2);
#pragma unroll 1
    for (int i = tid; i < G * (DV + 2); i += THREADS) {
      const int g = i / (DV + 2), c = i - g * (DV + 2);
      base[(size_t)g * p.n_split * (DV + 2) + c] = (c == DV) ? -INFINITY : 0.f;
    }
    return;
  }
  // Copies run ahead of the scan over the CTA's whole tile sequence, unit borders included: copy_ahead brings the tile that
  // lies k >= 0 places behind the current segment's first one (by one lane), if the CTA has it.
  bool begun = false;          // (test hook: only the very first tile goes without its copy)
  auto copy_ahead = [&](int k, int stg) {
    int ib = b, ih = h, ilen = len, it = t_begin + k;
    if (k >= n_my) {           // in a later unit (only in balanced mode)
      if (!p.balanced) return;
      int start = unit_start, tiles = seg_tiles, first = t_begin, count = n_my;
#pragma unroll 1
      do {
        k -= count;
        next_unit(ib, ih, start, tiles);
        if (start >= hi) return;
        ilen = length(ib);
        tiles = (ilen + ST - 1) / ST;
        part(start, tiles, first, count);
      } while (k >= count);
      it = first + k;
    }
    const int j0 = it * ST;
    const int rows = min(ST, ((ilen + 7) & ~7) - j0);        // rows a copy may touch: S_cap is a multiple of 8
    if (RAP_BOUNDS(j0 + rows - 1, p.S_cap, p.status, 0x402) && RAP_BOUNDS(rows - 1, ST, p.status, 0x404) &&
        RAP_BOUNDS(stg, NSTG, p.status, 0x403) && RAP_BOUNDS(ib, p.B, p.status, 0x401)) {
      const uint32_t kb = (uint32_t)rows * 4 * KSW, vb = (uint32_t)rows * 4 * VSW;     // multiples of 16: rows is a multiple of 8
      const uint32_t bar = bar0 + 8 * stg, dst = ring_u + 4 * stg * C::STAGE_W;
      const size_t row0 = ((size_t)ib * p.Hkv + ih) * (size_t)p.S_cap + j0;
      mbar_expect_tx(bar, kb + vb);
      if (!(p.dbg_skip_copy && blockIdx.x == 0 && !begun && stg == 0)) {
        bulk_g2s(dst, p.k + row0 * (4 * KSW), kb, bar);
        bulk_g2s(dst + 4 * ST * KSW, p.v + row0 * (4 * VSW), vb, bar);
      }
    }
  };
  if (tid == 0)
#pragma unroll 1
    for (int i = 0; i < NSTG; ++i) copy_ahead(i, i);
  begun = true;
  // q of a unit as it is stored: words 4 j + tq of the head on column gid
  constexpr int NGK = C::Engine::NGK;
  uint32_t w_q[NGK][4];
  auto load_q = [&]() {
    const bool on = C::Engine::q_on(gid, G);
    const uint32_t* qrow = p.q + ((size_t)b * p.Hq + (size_t)h * G + (on ? C::Engine::q_head(gid) : 0)) * pp.P;
#pragma unroll
    for (int j = 0; j < NGK; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int at = 4 * (4 * j + tq) + i;
        w_q[j][i] = (on && at < pp.P) ? qrow[at] : 0u;
      }
  };
  load_q();

  for (;;) {   // one pass per segment (a single one unless the mode is balanced)
    eng.begin(w_q, p.qscale);    // log2(e) / sqrt(D)
    int held = 0;                // tiles since the last flush, rounded down to turns
    int nrows = len - t_begin * ST - Q4_BR * warp;      // valid rows from this warp's block on
#pragma unroll 1
    for (int i = 0; i < n_my; ++i, nrows -= ST) {
      if (__any_sync(0xffffffffu, !mbar_test_wait(bar0 + 8 * st, parity)) &&
          !__all_sync(0xffffffffu, mbar_wait_slow(bar0 + 8 * st, parity, p.wait_limit))) {   // warp-uniform verdict
        timed_out = true;
        break;
      }
      const uint32_t* sw = ring + st * C::STAGE_W;
      bool in_ok = true;
#ifdef RAP_DEBUG_BOUNDS
      in_ok = __all_sync(0xffffffffu, RAP_BOUNDS((int)(sw - reinterpret_cast<const uint32_t*>(smem)) + eng.at.reach(), C::SMEM / 4, p.status, 0x405));
#endif
      if (in_ok && nrows > 0) eng.block(sw, nrows, my_main);
      // this warp is done with the stage (its loads have been used)
      __syncwarp();
      if (lane == 0) mbar_arrive(bar0 + 8 * (Q4_MAX_STG + st));
      if (turn-- == 0) {       // the warps take turns to refill
        turn = NW - 1;
        eng.settle();
        if ((held += NW) >= C::Engine::FLUSH) {
          eng.flush(my_main);
          held = 0;
        }
        const int old = LAG == 0 ? st : st == 0 ? NSTG - 1 : st - 1;
        if (!__all_sync(0xffffffffu, mbar_wait_bounded(bar0 + 8 * (Q4_MAX_STG + old), old > st ? parity ^ 1u : parity, p.wait_limit))) {
          timed_out = true;
          break;
        }
        if (lane == 0) copy_ahead(i - LAG + NSTG, old);
      }
      if (++st == NSTG) { st = 0; parity ^= 1u; }
    }

    // ---- merge the warps: common maximum per head, scaled sums ----
    eng.finish(my_main);
#pragma unroll
    for (int g = 0; g < GC; ++g)
#pragma unroll
      for (int d = 4; d < 32; d <<= 1) {
        eng.l_thr[g] += __shfl_xor_sync(0xffffffffu, eng.l_thr[g], d);
        eng.z_thr[g] += __shfl_xor_sync(0xffffffffu, eng.z_thr[g], d);
      }
    // row sums to [1, 2), and the references with them (whole numbers below 2^23: exact; logits beyond that are not right to a
    // place anyway and keep their reference): what a warp weighs in the merge is then in its reference alone
    float norm[GC];
#pragma unroll
    for (int g = 0; g < GC; ++g) {
      const int k = fabsf(eng.m_ref[g]) < 0x1p22f ? min(max(q4_exponent(eng.l_thr[g]), -126), 126) : 0;
      norm[g] = q4_pow2(-k);
      eng.m_ref[g] += (float)k;
    }
    if (timed_out && lane == 0) *s_flag = 1;
    if (gid == 0) {
#pragma unroll
      for (int g = 0; g < GC; ++g) m_s[warp * 8 + GC * tq + g] = eng.m_ref[g];
    }
    __syncthreads();
    if (*s_flag) {
      if (tid == 0) {
        atomicCAS(&p.status[0], 0, (int)RAP_ETIMEOUT);
        p.status[1] = (b * p.Hkv + h) * RAP_MAX_SPLIT + (int)(blockIdx.x % RAP_MAX_SPLIT);
      }
      // give copies still in flight a bounded chance to land before the shared memory is released
      if (tid == 0)
#pragma unroll 1
        for (int sg = 0; sg < NSTG; ++sg) {
          mbar_wait_bounded(bar0 + 8 * sg, 0, p.wait_limit);
          mbar_wait_bounded(bar0 + 8 * sg, 1, p.wait_limit);
        }
      __syncthreads();
      return;
    }
#pragma unroll
    for (int g = 0; g < GC; ++g) {
      const int head = GC * tq + g;
      float m_all = -INFINITY;
#pragma unroll
      for (int w = 0; w < NW; ++w) m_all = fmaxf(m_all, m_s[w * 8 + head]);
      const float d = eng.m_ref[g] - m_all;      // -inf or NaN: a warp without a block contributes nothing
      const float f = d >= -126.f ? norm[g] * q4_pow2((int)d) : 0.f;
      if (gid == 0) l_s[warp * 8 + head] = eng.l_thr[g] * f;
      if (head < G) eng.put(my_main + head * CW, g, f);
    }
    const int b0 = b, h0 = h, start0 = unit_start + plan.empty(), tiles0 = seg_tiles;      // this segment's place
    bool more = false;
    if (p.balanced) {          // the following unit; its q is on the way while this one is merged
      next_unit(b, h, unit_start, seg_tiles);
      more = find_segment();
      if (more) load_q();
    }
    __syncthreads();
    // the CTAs that share the unit (most often none but this one)
    int first = 0, nseg = p.balanced ? 1 : 0;
    if (p.balanced && !plan.whole && (start0 < lo || start0 + tiles0 > hi)) {
      first = plan.cta_of(start0);
      nseg = plan.cta_of(start0 + tiles0 - 1) - first + 1;
    }
    if (nseg == 1) {
      // the whole unit was scanned here: straight to the output
      const bool o_ok = RAP_BOUNDS(((size_t)b0 * p.Hq + (size_t)h0 * G + G) * DV - 1, (size_t)p.B * p.Hq * DV, p.status, 0x40c);
#pragma unroll 1
      for (int i = tid; i < G * DV && o_ok; i += THREADS) {
        const int g = i / DV, c = i - g * DV;
        float sum = 0.f, l = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
          sum += red[w * C::MAIN_F + g * CW + c];
          l += l_s[w * 8 + g];
        }
        p.out[((size_t)b0 * p.Hq + (size_t)h0 * G) * DV + i] = l != 0.f ? sum / l : 0.f;
      }
    } else {
      const size_t ws_head = (size_t)(p.balanced ? RAP_MAX_SPLIT : p.n_split) * (DV + 2);
      float* unit_ws = p.ws + ((size_t)b0 * p.Hq + (size_t)h0 * G) * ws_head;
      float* ws_base = unit_ws + (size_t)((int)blockIdx.x - first) * (DV + 2);
      const bool ws_ok = RAP_BOUNDS((ws_base - p.ws) + (long long)(G - 1) * ws_head + DV + 1, p.ws_floats, p.status, 0x409);
#pragma unroll 1
      for (int i = tid; i < G * DV && ws_ok; i += THREADS) {
        const int g = i / DV, c = i - g * DV;
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) sum += red[w * C::MAIN_F + g * CW + c];
        ws_base[g * ws_head + c] = sum;
      }
      if (tid < G && ws_ok) {
        float l = 0.f, mm = -INFINITY;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
          l += l_s[w * 8 + tid];
          mm = fmaxf(mm, m_s[w * 8 + tid]);
        }
        ws_base[tid * ws_head + DV] = mm;
        ws_base[tid * ws_head + DV + 1] = l;
      }
      if (!p.balanced) return;
      // ---- the CTA that delivers a unit's last partial merges them (no separate combine launch) ----
      __threadfence();           // this CTA's partials are visible before its arrival is counted
      __syncthreads();
      const int u = b0 * p.Hkv + h0;
      if (tid == 0) *s_last = RAP_BOUNDS(u, p.B * p.Hkv, p.status, 0x40a) && atomicAdd(&p.unit_cnt[u], 1) == nseg - 1;
      __syncthreads();
      if (*s_last) {
        __threadfence();
        const bool m_ok = RAP_BOUNDS((unit_ws - p.ws) + (long long)(G - 1) * ws_head + (long long)(nseg - 1) * (DV + 2) + DV + 1,
                                     p.ws_floats, p.status, 0x40b);
        float* wgt = red;        // [G][RAP_MAX_SPLIT] segment weights, then G reciprocals of the denominators
#pragma unroll 1
        for (int g = warp; g < G && m_ok; g += NW) {
          const float* gb = unit_ws + (size_t)g * ws_head;
          float mv[2], lv[2];
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const int sg = lane + 32 * k;
            lv[k] = sg < nseg ? __ldcg(gb + (size_t)sg * (DV + 2) + DV + 1) : 0.f;
            mv[k] = sg < nseg ? __ldcg(gb + (size_t)sg * (DV + 2) + DV) : -INFINITY;
          }
          float M = fmaxf(lv[0] != 0.f ? mv[0] : -INFINITY, lv[1] != 0.f ? mv[1] : -INFINITY);
#pragma unroll
          for (int d = 16; d > 0; d >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, d));
          float den = 0.f;
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const float wk = lv[k] != 0.f ? exp2f(mv[k] - M) : 0.f;      // (a NaN in a row sum is kept)
            wgt[g * RAP_MAX_SPLIT + lane + 32 * k] = wk;
            den += wk * lv[k];
          }
#pragma unroll
          for (int d = 16; d > 0; d >>= 1) den += __shfl_xor_sync(0xffffffffu, den, d);
          if (lane == 0) wgt[G * RAP_MAX_SPLIT + g] = den != 0.f ? 1.f / den : 0.f;
        }
        __syncthreads();
#pragma unroll 1
        for (int i = tid; i < G * DV && m_ok; i += THREADS) {
          const int g = i / DV, c = i - g * DV;
          const float* gb = unit_ws + (size_t)g * ws_head + c;
          float num = 0.f;
#pragma unroll 1
          for (int s0 = 0; s0 < nseg; s0 += 16) {      // sixteen loads in flight (four at a time: 1 us more at ten segments)
            float x[16];
#pragma unroll
            for (int k = 0; k < 16; ++k) x[k] = s0 + k < nseg ? __ldcg(gb + (size_t)(s0 + k) * (DV + 2)) : 0.f;
#pragma unroll
            for (int k = 0; k < 16; ++k) num = fmaf(wgt[g * RAP_MAX_SPLIT + s0 + k], x[k], num);
          }
          p.out[((size_t)b0 * p.Hq + (size_t)h0 * G) * DV + i] = num * wgt[G * RAP_MAX_SPLIT + g];
        }
        if (tid == 0) p.unit_cnt[u] = 0;   // ready for the next call on this context
      }
    }
    if (!more) break;
    __syncthreads();   // the reduction buffer and the merge scalars are reused by the next segment
  }   // segment loop
}

}  // namespace
