// One new token of every sequence over the rows that it sees: rap_decode_attn_window, and the sequences' own rows of
// rap_decode_attn_shared, for bf16 heads of 16 to 128 dims (2P) and 16 to 128 channels (d_v').
//
// Bound by HBM: a row of 2 (2P + d_v') bytes takes 2 G (2P + d_v') flops, so what matters is that copies never pause and that
// a launch ends soon.  The rows a unit (sequence, KV head) sees are at most three runs of consecutive cache rows (win_runs);
// each run is cut into blocks of 32 rows from a multiple of 8 on (8 rows start on a 16-byte boundary for every width), and
// all units' blocks form one sequence that the CTAs share evenly, whatever units they belong to.  Inside a CTA every warp is
// its own pipeline over every NW-th block: a ring of stages that it fills itself, no barrier until the unit ends.
//   * Rows of a multiple of 128 bytes come through tensor maps with the 128-byte swizzle, rows of another multiple of 16 are
//     copied 16 bytes a lane into rows padded so that fragment loads meet 32 banks; all others are contiguous bulk copies,
//     with the eight rows of a fragment spread so that they do.
//   * S^T = q K^T and O += P V are mma.sync m16n8k16 (M would be G <= 8 query heads: far below a tcgen05 tile, and no
//     descriptor describes rows of 180 bytes).  The 16 rows of A carry the softmax weights as three bf16 numbers, their
//     rounding and two remainders (24 bits together), instead of padding: up to four heads rows 0-3, 4-7 and 8-11 in ONE
//     instruction (q stands in rows 0-3 and again in 4-7, so every lane that needs a weight has computed it), up to eight
//     heads two of the three in the first instruction and the last in a second one.
//   * The running maximum is raised only when a logit exceeds it by more than 8 (in log2 units).
//   * A unit that several CTAs share leaves one partial (sums, maximum, weight) each; who delivers the last one joins them in
//     order, so a result does not depend on who that is.  The prefix of rap_decode_attn_shared comes as partials too.
// Measured (replayed from a graph; 1 to 3 us more a call made by itself): 32 sequences of up to 4100 rows, 8 KV heads, P = 45,
// d_v' = 90 (332 MB) in 56.5 us, 5.8 TB/s; one sequence in 11.4 us, which is latency: plan 2, first copy 2, three blocks a warp 2,
// arrival and join 3.
#pragma once
#include <cuda.h>

#include "rap_attn_common.cuh"
#include "rap_window_common.cuh"

namespace {

struct WsParams {
  const uint32_t* q;          // [B][Hq][P] bf16 pairs
  const unsigned char* k;     // [B][Hkv][S_cap][4 P bytes]
  const unsigned char* v;     // [B][Hkv][S_cap][2 dv bytes]
  const int32_t* seq_len;
  float* out;                 // [B][Hq][dv]
  WinPartials ws;
  long long ws_floats;        // size of the workspace from ws.pre on
  int32_t* unit_cnt;          // arrivals per unit, zero between calls
  int32_t* unit_cnt_other;    // the set of the launch before; cleared by this one
  int other_units;
  int32_t* status;
  int B, Hq, Hkv, G, P, dv, S_cap, n_sink, window, len_cap;
  float qscale;               // log2(e) / sqrt(D)
  int pad16;                  // 1: rows of a multiple of 16 bytes, copied into padded rows; 0: bulk copies
  int k_stride, v_stride;     // bytes between rows in shared memory
  int rs_log;                 // log2 of the row step between the columns of a fragment
  int stage_bytes, off_stage;
  int own;                    // blocks that a unit's end takes as long as
  int join_places;            // partials that the stages hold together
  uint32_t wait_limit;
  int dbg_skip_copy;          // test hook: the first unit's first block is armed and not copied
  int dbg_lost_bytes;         // test hook: a join waits for so many bytes more than it copies
  // shared prefixes (ws.n_pre > 0): what the plan of their splits is made of
  int n_groups, S_pre, sms;
  const int32_t* group_start;
  const int32_t* prefix_len;
};

__device__ __forceinline__ void ws_mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// one box of a 2-D tensor map (x = element column, y = row) into this CTA's shared memory; no multicast
__device__ __forceinline__ void ws_tma_2d(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
      "l"(map), "r"(x), "r"(y), "r"(bar)
      : "memory");
}
__device__ __forceinline__ float ws_ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t ws_pack(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint32_t ws_prmt(uint32_t a, uint32_t b, uint32_t sel) {
  uint32_t r;
  asm("prmt.b32 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(sel));
  return r;
}
__device__ __forceinline__ float ws_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float ws_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// The runs of a unit and their blocks of 32 rows; a unit without rows counts as one block, so that somebody writes its output.
struct WsUnit {
  WinRuns r;
  int a[3], nb[3], n;       // first row and number of blocks by run; blocks together (>= 1)
};
__device__ __forceinline__ WsUnit ws_unit(const WsParams& p, int b) {
  WsUnit u;
  u.r = win_runs(min(p.seq_len[b], p.len_cap), p.n_sink, p.window, p.S_cap);
  u.n = 0;
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    u.a[i] = u.r.lo[i] & ~7;
    u.nb[i] = u.r.n[i] > 0 ? (u.r.lo[i] + u.r.n[i] - u.a[i] + 31) >> 5 : 0;
    u.n += u.nb[i];
  }
  u.n = max(u.n, 1);
  return u;
}
__device__ __forceinline__ int ws_scan_add(int x, int lane) {      // inclusive prefix over the warp
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  return x;
}

// N: steps of 16 dims and blocks of 16 channels (the larger of the two); FOUR: up to four query heads a KV head; VODD: d_v' odd;
// NW: warps.  A short launch executes most of this once a CTA, so what it costs is fetching it: divisions by run-time numbers
// and 64-bit ones are kept out of the usual path.
constexpr int WS_STAGES = 2;
// LONG: for launches in which a warp may add up more than WS_LONG blocks of a unit.  The MMA cuts its sums where it adds them, it
// does not round them, which takes 1e-6 of a sum for every thousand rows (2.3e-6 where V has one sign), so here they leave the
// accumulators every WS_DRAIN blocks for the warp's part of the buffer that the warps' sums meet in, added there in fp32.  40
// sequences of 65,536 rows: 1.4e-5 -> 1.3e-6 of the output (3.7e-5 -> 1.6e-6).  Times within 4% of the other form's there;
// short launches would take 1 to 3 us more in it.
constexpr int WS_LONG = 64, WS_DRAIN = 32;
// TMA: rows of exactly 32 N bytes (K and V) through tensor maps, N = 4 or 8: panels of 32 rows x 128 bytes, the 16-byte chunk c
// of row r at chunk c ^ (r % 8)
template <int N, bool FOUR, bool VODD, int NW, bool TMA, bool LONG>
__global__ void __launch_bounds__(32 * NW, 2) win_scan_kernel(const WsParams p, const __grid_constant__ CUtensorMap map_k,
                                                              const __grid_constant__ CUtensorMap map_v) {
  static_assert(!TMA || N % 4 == 0, "whole panels");
  extern __shared__ __align__(128) unsigned char smem_raw[];
  unsigned char* smem = TMA ? smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u) : smem_raw;     // panels start on 1024 bytes
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem);                         // [NW][stages], at most 64 bytes; then the join's
  const uint32_t bar_join = smem_u32(smem) + 64;
  float* m_s = reinterpret_cast<float*>(smem + 128);                          // [4][8]
  float* l_s = m_s + 32;                                                      // [4][8]
  int* s_flag = reinterpret_cast<int*>(smem + 384);
  int* s_last = s_flag + 1;
  float* red = reinterpret_cast<float*>(smem + 512);                          // [NW][G][CW]; later the join's weights
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int gid = lane >> 2, tq = lane & 3;
  constexpr int NSTG = WS_STAGES, THREADS = NW * 32;
  const int G = p.G, P = p.P, dv = p.dv;

  if (tid == 0) {
    *s_flag = 0;
    for (int i = 0; i < NW * NSTG; ++i) mbar_init(smem_u32(bars) + 8 * i, p.pad16 ? 32 : 1);
    mbar_init(bar_join, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  // ---- the plan: every warp works it out from the lengths.  A unit counts p.own blocks more than it has ----
  int T = 0, n_max = 1, n_first = 0;
  for (int b0 = 0; b0 < p.B; b0 += 32) {
    const int n = b0 + lane < p.B ? ws_unit(p, b0 + lane).n + p.own : 0;
    if (b0 == 0) n_first = n;
    n_max = max(n_max, __reduce_max_sync(0xffffffffu, n));
    T += __reduce_add_sync(0xffffffffu, n);
  }
  T *= p.Hkv;
  const WinScanPlan plan = win_scan_plan(T, n_max, p.B * p.Hkv, (int)gridDim.x, p.own, p.ws.n_pre, p.pad16 != 0);
  const bool even = plan.even;
  const int nc = plan.nc, parts = plan.parts, share = plan.share, extra = plan.extra;
  if (blockIdx.x == 0)
    for (int i = tid; i < p.other_units; i += THREADS) p.unit_cnt_other[i] = 0;      // what a launch that gave up left behind
  if ((int)blockIdx.x >= nc) {
    if (p.ws.n_pre) pdl_wait();     // a launch is not over before the one that it overlaps
    return;
  }
  int cur = (int)blockIdx.x * share + min((int)blockIdx.x, extra);
  int hi = cur + share + ((int)blockIdx.x < extra ? 1 : 0);
  int b = 0, h, unit_start = 0;
  const int my_unit = even ? (int)blockIdx.x / parts : 0;
  if (even) {
    b = my_unit / p.Hkv;
  } else {
    for (int b0 = 0, carry = 0;; b0 += 32) {
      const int n = (b0 == 0 ? n_first : b0 + lane < p.B ? ws_unit(p, b0 + lane).n + p.own : 0) * p.Hkv;
      const int x = ws_scan_add(n, lane) + carry;
      const unsigned past = __ballot_sync(0xffffffffu, x > cur);
      if (past) {
        const int l = __ffs(past) - 1;
        b = b0 + l;
        unit_start = __shfl_sync(0xffffffffu, x - n, l);
        break;
      }
      carry = __shfl_sync(0xffffffffu, x, 31);
    }
  }
  WsUnit u = ws_unit(p, b);
  if (even) {
    const int part = (int)blockIdx.x - my_unit * parts;
    h = my_unit - b * p.Hkv;
    cur = p.own + (int)((long long)u.n * part / parts);
    hi = p.own + (int)((long long)u.n * (part + 1) / parts);
  } else {
    h = (cur - unit_start) / (u.n + p.own);
    unit_start += h * (u.n + p.own);
  }

  int pre_per = 1;
  if (p.ws.n_pre)
    pre_per = win_prefix_plan(p.group_start, p.prefix_len, p.n_groups, p.B, G, p.Hkv, p.S_pre, p.sms, p.ws.n_pre).per;
  const uint32_t bar0 = smem_u32(bars) + warp * NSTG * 8;
  unsigned char* wstage = smem + p.off_stage + (size_t)warp * NSTG * p.stage_bytes;
  const uint32_t wstage_u = smem_u32(wstage);
  // ---- fragment addresses inside a stage, in 32-bit words ----
  auto frag_row = [&](int t, int n) { return (n << p.rs_log) + (t & ((1 << p.rs_log) - 1)) + ((t >> p.rs_log) << (3 + p.rs_log)); };
  const int v_base = (32 * p.k_stride) >> 2;
  const int vpair = (p.v_stride << p.rs_log) >> 2;           // words between the two rows of a V register (an even row step where dv is odd)
  int koff[4], vofs[4];
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    koff[t] = ((frag_row(t, gid) * p.k_stride) >> 2) + tq;
    vofs[t] = v_base + ((frag_row(t, 2 * tq) * p.v_stride) >> 2) + gid;     // odd dv: rounded down for odd rows
  }
  int kx[8], vx[4][2];           // TMA: word of the lane in its row's chunk c; words of rows 2 tq + e in chunks of 16 channels
#pragma unroll
  for (int c = 0; c < 8; ++c) kx[c] = gid * 32 + ((c ^ gid) << 2) + tq;
#pragma unroll
  for (int cm = 0; cm < 4; ++cm)
#pragma unroll
    for (int e = 0; e < 2; ++e) vx[cm][e] = v_base + (2 * tq + e) * 32 + (((2 * cm + (gid >> 2)) ^ (2 * tq + e)) << 2) + (gid & 3);
  const int k_last = P - 8;                                   // the last steps are shifted back into the row
  const int c_last = VODD ? dv - 15 : dv - 16;                // so are the last blocks of channels (odd dv: one phantom channel)
  const int CW = c_last + 16;
  const int head = FOUR ? gid & 3 : gid;                      // the query head whose logits this lane holds
  const float cs = p.qscale;
  const int k_row = 4 * P, v_row = 2 * dv;                    // bytes in the cache

  __syncthreads();             // the barriers are initialised
  bool used = false;           // the ring has been read: copies into it come after those reads
  int st = 0;                  // ring position and phase of this warp, across units
  uint32_t parity = 0;
  bool timed_out = false, joined = false;
  uint32_t join_parity = 0;

  for (;;) {   // one pass per unit that this CTA touches
    const int t0 = max(cur - unit_start - p.own, 0);               // this CTA's blocks of the unit: [t0, t0 + n_my)
    const int n_my = min(u.n, hi - unit_start - p.own) - t0;
    if (n_my <= 0) break;                                           // its share ends in what the unit counts beyond its blocks
    const size_t unit = (size_t)b * p.Hkv + h;
    const unsigned char* kg = p.k + unit * (size_t)p.S_cap * (size_t)k_row;
    const unsigned char* vg = p.v + unit * (size_t)p.S_cap * (size_t)v_row;
    const bool empty = u.nb[0] + u.nb[1] + u.nb[2] == 0;
    const int n_blk = !empty && n_my > warp ? (int)((unsigned)(n_my - warp + NW - 1) / NW) : 0;
    int n_pre = 0;             // partials of the prefix, if the sequence has one
    if (p.ws.n_pre) {
      const int g = win_owner(p.group_start, p.n_groups, b);
      if (g < p.n_groups && p.group_start[g] <= b) n_pre = (win_group_tiles(p.prefix_len, g, p.S_pre) + pre_per - 1) / pre_per;
    }
    float* out = p.out + ((size_t)b * p.Hq + (size_t)h * G) * dv;
    if (empty && n_pre == 0) {
      for (int i = tid; i < G * dv; i += THREADS) out[i] = 0.f;
    } else {

    // first row of block i of this warp, and which of its 32 rows are seen
    auto block_at = [&](int i, int& row0, int& lo, int& hi_row) {
      int j = t0 + warp + i * NW, run = 0;
      if (j >= u.nb[0]) { j -= u.nb[0]; run = 1; }
      if (run == 1 && j >= u.nb[1]) { j -= u.nb[1]; run = 2; }
      const int a = run == 0 ? u.a[0] : run == 1 ? u.a[1] : u.a[2];
      const int l = run == 0 ? u.r.lo[0] : run == 1 ? u.r.lo[1] : u.r.lo[2];
      const int e = l + (run == 0 ? u.r.n[0] : run == 1 ? u.r.n[1] : u.r.n[2]);
      row0 = a + 32 * j;
      lo = max(0, l - row0);
      hi_row = min(32, e - row0);
    };
    auto issue_block = [&](int i, int stg) {
      int row0, lo, hi_row;
      block_at(i, row0, lo, hi_row);
      const int rows = (hi_row + 7) & ~7;                     // inside the cache: S_cap is a multiple of 8
      const uint32_t bar = bar0 + 8 * stg, dst = wstage_u + stg * p.stage_bytes;
      const bool ok = RAP_BOUNDS(row0, p.S_cap, p.status, 0x201) && RAP_BOUNDS(row0 + rows - 1, p.S_cap, p.status, 0x202) &&
                      RAP_BOUNDS(rows - 1, 32, p.status, 0x203) && RAP_BOUNDS(unit, (size_t)p.B * p.Hkv, p.status, 0x204);
      if (p.dbg_skip_copy && unit == 0 && t0 == 0 && warp == 0 && i == 0) {     // nothing is in flight for this stage when the CTA leaves
        if ((TMA || !p.pad16) && lane == 0) mbar_expect_tx(bar, 16);
        return;
      }
      const unsigned char* ks = kg + (size_t)row0 * k_row;
      const unsigned char* vs = vg + (size_t)row0 * v_row;
      if constexpr (TMA) {
        if (lane == 0) {         // whole boxes: rows of a neighbouring unit are masked, rows behind the tensor's end come as zeros
          if (used) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          mbar_expect_tx(bar, ok ? (uint32_t)(N * 1024 * 2) : 0u);
          const int y = (int)unit * p.S_cap + row0;
          if (ok) {
#pragma unroll
            for (int pn = 0; pn < N / 4; ++pn) ws_tma_2d(dst + pn * 4096, &map_k, 64 * pn, y, bar);
#pragma unroll
            for (int pn = 0; pn < N / 4; ++pn) ws_tma_2d(dst + N * 1024 + pn * 4096, &map_v, 64 * pn, y, bar);
          }
        }
      } else if (p.pad16) {
        const int c = lane & 15, kc = k_row >> 4, vc = v_row >> 4;
        for (int r = lane >> 4; r < rows && ok; r += 2) {
          if (c < kc)
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + r * p.k_stride + 16 * c), "l"(ks + (size_t)r * k_row + 16 * c) : "memory");
          if (c < vc)
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + 32 * p.k_stride + r * p.v_stride + 16 * c),
                         "l"(vs + (size_t)r * v_row + 16 * c) : "memory");
        }
        asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
      } else if (lane == 0) {
        if (used) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // earlier reads and zeros come first
        mbar_expect_tx(bar, ok ? (uint32_t)(rows * (k_row + v_row)) : 0u);
        if (ok) {
          bulk_g2s(dst, ks, (uint32_t)(rows * k_row), bar);
          bulk_g2s(dst + 32 * p.k_stride, vs, (uint32_t)(rows * v_row), bar);
        }
      }
    };
    static_assert(NSTG == 2, "one block ahead");
    if (n_blk > 0) issue_block(0, st);

    // ---- q as the A operand: words (8 ks + tq) and (8 ks + 4 + tq) of the lane's head; zero where a step overlaps the one before ----
    uint32_t qa[N][2];
    {
      const uint32_t* qrow = p.q + ((size_t)b * p.Hq + (size_t)h * G + (head < G ? head : 0)) * P;
#pragma unroll
      for (int ks = 0; ks < N; ++ks) {
        const int wb = min(8 * ks, k_last);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int w = wb + 4 * e + tq;
          qa[ks][e] = (head < G && w >= 8 * ks && RAP_BOUNDS(w, P, p.status, 0x205)) ? qrow[w] : 0u;
        }
      }
    }
    float o[N][2][4];
#pragma unroll
    for (int cb = 0; cb < N; ++cb)
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int r = 0; r < 4; ++r) o[cb][e][r] = 0.f;
    float m_ref = -INFINITY, l_thr = 0.f;
    float* red_w = red + (size_t)warp * G * CW;                  // this warp's sums [G][CW]
    float* rr = red_w + (size_t)(head < G ? head : 0) * CW;
    const bool holds = (FOUR ? gid < 4 : true) && head < G;     // this lane holds sums of its head
    // sum r (of two) of a block of channels over the three bf16 numbers of the weights.  Remainders of either sign times an
    // infinity of V would be NaN: the roundings' sum says what it is
    auto whole_sum = [&](const float (&oc)[4], int r) {
      float rest = oc[r + 2];
      if (FOUR) rest += __shfl_down_sync(0xffffffffu, oc[r], 16);
      const float t = oc[r] + rest;
      return t != t && fabsf(oc[r]) == INFINITY ? oc[r] : t;
    };

    for (int i = 0; i < n_blk; ++i) {
      if (i + 1 < n_blk) issue_block(i + 1, st ^ 1);
      if (!__all_sync(0xffffffffu, mbar_wait_bounded(bar0 + 8 * st, parity, p.wait_limit))) {
        timed_out = true;
        break;
      }
      int row0, lo, hi_row;
      block_at(i, row0, lo, hi_row);
      const uint32_t* w = reinterpret_cast<const uint32_t*>(wstage + (size_t)st * p.stage_bytes);
      const bool ragged = lo > 0 || hi_row < 32;
      if (ragged) {
        // rows that are not seen: their V is zero, so that the second product meets 0 * 0 there
        unsigned char* vz = wstage + (size_t)st * p.stage_bytes + 32 * p.k_stride;
        const int z0 = lo * p.v_stride, z1 = hi_row * p.v_stride, z2 = 32 * p.v_stride;     // bytes [0, z0) and [z1, z2)
        if constexpr (TMA) {     // a row is 128 bytes of every panel, whatever the swizzle
          for (int pn = 0; pn < N / 4; ++pn) {
            for (int i = 4 * lane; i < 128 * lo; i += 128) *reinterpret_cast<uint32_t*>(vz + pn * 4096 + i) = 0u;
            for (int i = 128 * hi_row + 4 * lane; i < 4096; i += 128) *reinterpret_cast<uint32_t*>(vz + pn * 4096 + i) = 0u;
          }
        } else if constexpr (VODD) {
          for (int i = 2 * lane; i < z0; i += 64) *reinterpret_cast<uint16_t*>(vz + i) = 0;
          for (int i = z1 + 2 * lane; i < z2; i += 64) *reinterpret_cast<uint16_t*>(vz + i) = 0;
        } else {
          for (int i = 4 * lane; i < z0; i += 128) *reinterpret_cast<uint32_t*>(vz + i) = 0u;
          for (int i = z1 + 4 * lane; i < z2; i += 128) *reinterpret_cast<uint32_t*>(vz + i) = 0u;
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
      }

      // ---- S^T = q K^T: four fragments of 8 rows ----
      float s[4][4];
#pragma unroll
      for (int t = 0; t < 4; ++t) s[t][0] = s[t][1] = s[t][2] = s[t][3] = 0.f;
#pragma unroll
      for (int ks = 0; ks < N; ++ks) {
        const int wb = min(8 * ks, k_last);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          uint32_t b0, b1;
          if constexpr (TMA) {
            b0 = w[kx[(2 * ks) % 8] + (ks / 4) * 1024 + 256 * t];
            b1 = w[kx[(2 * ks + 1) % 8] + (ks / 4) * 1024 + 256 * t];
          } else {
            b0 = w[koff[t] + wb];
            b1 = w[koff[t] + wb + 4];
          }
          ws_mma(s[t], qa[ks][0], 0u, qa[ks][1], 0u, b0, b1);
        }
      }

      // ---- softmax: lane (gid, tq) holds its head's logits of rows frag_row(t, 2 tq + e) ----
      float x[4][2];
      bool raise = false;
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int row = frag_row(t, 2 * tq + e);
          if (ragged && (row < lo || row >= hi_row)) s[t][e] = -INFINITY;
          x[t][e] = fmaf(s[t][e], cs, -m_ref);
          raise |= x[t][e] > 8.f;
        }
      if (__any_sync(0xffffffffu, raise || m_ref == -INFINITY)) {
        float mx = -INFINITY;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int e = 0; e < 2; ++e) mx = fmaxf(mx, s[t][e] * cs);
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
        const float m_new = fmaxf(m_ref, mx), ref = m_new == -INFINITY ? 0.f : m_new;
        const float alpha = ws_ex2(m_ref - ref);               // first block: 2^(-inf) = 0
        m_ref = m_new;
        l_thr *= alpha;
#pragma unroll
        for (int cb = 0; cb < N; ++cb)
#pragma unroll
          for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int r = 0; r < 4; ++r) o[cb][e][r] *= alpha;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int e = 0; e < 2; ++e) x[t][e] = fmaf(s[t][e], cs, -ref);
      }
      uint32_t p0[4], p1[4], p2[4];      // the weights of rows frag_row(t, 2 tq) and frag_row(t, 2 tq + 1): bf16 roundings, remainders, theirs
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        float a = ws_ex2(x[t][0]), c = ws_ex2(x[t][1]);
        l_thr += a + c;
        p0[t] = ws_pack(a, c);
        a -= ws_lo(p0[t]);
        c -= ws_hi(p0[t]);
        p1[t] = ws_pack(a, c);
        p2[t] = ws_pack(a - ws_lo(p1[t]), c - ws_hi(p1[t]));
        if (FOUR) {
          p0[t] = gid < 4 ? p0[t] : p1[t];
          p2[t] = gid < 4 ? p2[t] : 0u;
        }
      }

      // ---- O += P V: two steps of 16 rows (fragments 2 kb and 2 kb + 1), blocks of 16 channels ----
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        const uint32_t* v0 = w + vofs[2 * kb];
        const uint32_t* v1 = w + vofs[2 * kb + 1];
#pragma unroll
        for (int cb = 0; cb < N; ++cb) {
          const int cw = min(16 * cb, c_last) >> 1;
          uint32_t xa0, xb0, xa1, xb1;
          if constexpr (TMA) {
            xa0 = w[vx[cb % 4][0] + (cb / 4) * 1024 + 512 * kb];
            xb0 = w[vx[cb % 4][1] + (cb / 4) * 1024 + 512 * kb];
            xa1 = w[vx[cb % 4][0] + (cb / 4) * 1024 + 512 * kb + 256];
            xb1 = w[vx[cb % 4][1] + (cb / 4) * 1024 + 512 * kb + 256];
          } else {
            xa0 = v0[cw];
            xb0 = v0[cw + vpair];
            xa1 = v1[cw];
            xb1 = v1[cw + vpair];
          }
          const uint32_t be0 = ws_prmt(xa0, xb0, 0x5410u), bo0 = ws_prmt(xa0, xb0, 0x7632u);
          uint32_t be1, bo1;
          if constexpr (!VODD) {
            be1 = ws_prmt(xa1, xb1, 0x5410u);
            bo1 = ws_prmt(xa1, xb1, 0x7632u);
          } else {
            // odd rows of an odd dv: the aligned word holds channels (c - 1, c), the next one (c + 1, c + 2)
            const uint32_t ya1 = v1[cw + 1], yb1 = v1[cw + vpair + 1];
            be1 = ws_prmt(xa1, xb1, 0x7632u);
            bo1 = ws_prmt(ya1, yb1, 0x5410u);
          }
          if constexpr (FOUR) {
            ws_mma(o[cb][0], p0[2 * kb], p2[2 * kb], p0[2 * kb + 1], p2[2 * kb + 1], be0, be1);
            ws_mma(o[cb][1], p0[2 * kb], p2[2 * kb], p0[2 * kb + 1], p2[2 * kb + 1], bo0, bo1);
          } else {
            ws_mma(o[cb][0], p0[2 * kb], p1[2 * kb], p0[2 * kb + 1], p1[2 * kb + 1], be0, be1);
            ws_mma(o[cb][1], p0[2 * kb], p1[2 * kb], p0[2 * kb + 1], p1[2 * kb + 1], bo0, bo1);
            ws_mma(o[cb][0], 0u, p2[2 * kb], 0u, p2[2 * kb + 1], be0, be1);
            ws_mma(o[cb][1], 0u, p2[2 * kb], 0u, p2[2 * kb + 1], bo0, bo1);
          }
        }
      }
      __syncwarp();            // every lane is done with this stage before it is filled again
      used = true;
      if (++st == NSTG) { st = 0; parity ^= 1u; }

      if (LONG && (i % WS_DRAIN == WS_DRAIN - 1 || i + 1 == n_blk)) {      // rr and l_s, relative to m_s
        const bool more = i >= WS_DRAIN;
        const float m_old = more ? m_s[warp * 8 + gid] : m_ref, wt = m_old == m_ref ? 1.f : ws_ex2(m_old - m_ref);
        l_thr += __shfl_xor_sync(0xffffffffu, l_thr, 1);
        l_thr += __shfl_xor_sync(0xffffffffu, l_thr, 2);
        if (more) l_thr = fmaf(l_s[warp * 8 + gid], wt, l_thr);
        __syncwarp();
        if (tq == 0) {
          l_s[warp * 8 + gid] = l_thr;
          m_s[warp * 8 + gid] = m_ref;
        }
        l_thr = 0.f;
#pragma unroll
        for (int cb = 0; cb < N; ++cb) {
          const int c0 = min(16 * cb, c_last) + 4 * tq;        // four channels; those before 16 cb are the last block's too
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            const bool mine = holds && c0 + 2 * r >= 16 * cb;
            float2* at = reinterpret_cast<float2*>(rr + c0 + 2 * r);
            float2 x = make_float2(0.f, 0.f);
            if (mine && more) x = *at;
            x = make_float2(fmaf(x.x, wt, whole_sum(o[cb][0], r)), fmaf(x.y, wt, whole_sum(o[cb][1], r)));
            if (mine) *at = x;
          }
#pragma unroll
          for (int r = 0; r < 4; ++r) o[cb][0][r] = o[cb][1][r] = 0.f;
        }
        __syncwarp();
      }
    }

    // ---- the warps' sums together: common maximum per head ----
    if constexpr (LONG) {
      l_thr = n_blk > 0 ? l_s[warp * 8 + gid] : 0.f;
    } else {
      l_thr += __shfl_xor_sync(0xffffffffu, l_thr, 1);
      l_thr += __shfl_xor_sync(0xffffffffu, l_thr, 2);
    }
    if (timed_out && lane == 0) *s_flag = 1;
    if (tq == 0) m_s[warp * 8 + gid] = m_ref;
    __syncthreads();
    if (*s_flag) {
      if (tid == 0) win_report(p.status, RAP_ETIMEOUT, (int)unit);
      if (p.ws.n_pre) pdl_wait();
      // copies still in flight get a bounded chance to land before the shared memory is released
      if (lane == 0)
        for (int sg = 0; sg < NSTG; ++sg) {
          mbar_wait_bounded(bar0 + 8 * sg, 0, p.wait_limit);
          mbar_wait_bounded(bar0 + 8 * sg, 1, p.wait_limit);
        }
      __syncthreads();
      return;
    }
    float m_all = -INFINITY;
    for (int i = 0; i < NW; ++i) m_all = fmaxf(m_all, m_s[i * 8 + gid]);
    const float f = m_ref == -INFINITY ? 0.f : ws_ex2(m_ref - m_all);
    if (tq == 0) l_s[warp * 8 + gid] = l_thr * f;
    if constexpr (LONG) {
      for (int g = 0; g < G; ++g) {
        const float fg = __shfl_sync(0xffffffffu, f, 4 * g);
        for (int c = lane; c < CW; c += 32) red_w[g * CW + c] = n_blk > 0 ? red_w[g * CW + c] * fg : 0.f;
      }
    } else {
#pragma unroll
      for (int cb = 0; cb < N; ++cb) {
        const int c0 = min(16 * cb, c_last) + 4 * tq;
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float t = whole_sum(o[cb][e], r);
            if (holds) rr[c0 + 2 * r + e] = t * f;
          }
      }
    }
    __syncthreads();
    int my_seg, n_seg;             // this CTA's place among those that hold blocks of the unit, and how many they are
    if (even) {
      my_seg = u.n < parts ? t0 : (int)blockIdx.x - my_unit * parts;      // fewer blocks than CTAs: one each, the others none
      n_seg = min(u.n, parts);
    } else {
      const int first = plan.cta_of(unit_start + p.own);
      my_seg = (int)blockIdx.x - first;
      n_seg = plan.cta_of(unit_start + p.own + u.n - 1) - first + 1;
    }
    const bool alone = n_seg == 1 && n_pre == 0;
    const int dv4 = p.ws.dv4;
    const long long head0 = (long long)b * p.Hq + (long long)h * G;            // the unit's first query head
    const bool ws_ok = RAP_BOUNDS(my_seg, p.ws.slots, p.status, 0x206) &&
                       RAP_BOUNDS(reinterpret_cast<float*>(p.ws.own_pair(unit, my_seg) + G) - 1 - p.ws.pre, p.ws_floats, p.status, 0x207);
    for (int g = warp; g < G && ws_ok; g += NW) {
      float l = 0.f, mm = -INFINITY;
      for (int i = 0; i < NW; ++i) {
        l += l_s[i * 8 + g];
        mm = fmaxf(mm, m_s[i * 8 + g]);
      }
      const float inv = l != 0.f ? 1.f / l : 0.f;
      for (int c = lane; c < dv; c += 32) {
        float sum = 0.f;
        for (int i = 0; i < NW; ++i) sum += red[((size_t)i * G + g) * CW + c];
        if (alone) out[(size_t)g * dv + c] = sum * inv;
        else p.ws.own_sums(unit, my_seg)[g * dv4 + c] = sum;
      }
      if (!alone && lane == 0) p.ws.own_pair(unit, my_seg)[g] = make_float2(mm, l);
    }
    if (!alone) {
      // ---- who delivers a unit's last partial joins them, in order ----
      __syncthreads();
      if (tid == 0) {          // what the CTA has written is released with its arrival, what others have written acquired
        int before = n_seg - 1;
        if (n_seg > 1 && RAP_BOUNDS(unit, (size_t)p.B * p.Hkv, p.status, 0x208))
          asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], 1;" : "=r"(before) : "l"(&p.unit_cnt[unit]) : "memory");
        *s_last = before == n_seg - 1;
      }
      __syncthreads();
      if (*s_last) {
        if (p.ws.n_pre && !joined) pdl_wait();        // the prefix's partials come from the launch before
        joined = true;
        // The partials' sums come in as bulk copies, one round trip for all that fit the stages (all units' partials but the
        // largest): the prefix's split by split, the own ones in one run.  Their weights are worked out meanwhile.
        const int n = n_pre + n_seg, part = G * dv4;                 // n <= RAP_MAX_SPLIT by the plan
        float* sums = reinterpret_cast<float*>(smem + p.off_stage);
        float* wgt = red;                          // [G][RAP_MAX_SPLIT] weights over their sum
        auto fetch = [&](int s0, int m) {          // warp 0: partials [s0, s0 + m)
          if (lane == 0) {
            asm volatile("fence.proxy.async;" ::: "memory");        // the stages have been read; other CTAs' partials are acquired
            mbar_expect_tx(bar_join, (uint32_t)(m * part * 4 + p.dbg_lost_bytes));
          }
          __syncwarp();
          for (int s = s0 + lane; s < min(s0 + m, n_pre); s += 32)
            bulk_g2s(smem_u32(sums + (s - s0) * part), p.ws.pre_sums(head0, s), (uint32_t)(part * 4), bar_join);
          const int o0 = max(s0, n_pre), o1 = s0 + m;
          if (lane == 0 && o1 > o0)
            bulk_g2s(smem_u32(sums + (o0 - s0) * part), p.ws.own_sums(unit, o0 - n_pre), (uint32_t)((o1 - o0) * part * 4), bar_join);
        };
        int m = min(n, p.join_places);
        if (warp == 0) fetch(0, m);
        for (int g = warp; g < G; g += NW) {
          float mv[2], lv[2];
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const int sg = lane + 32 * k;
            const float2 x = sg < n_pre ? __ldcg(p.ws.pre_pair(head0 + g, sg)) : sg < n ? __ldcg(p.ws.own_pair(unit, sg - n_pre) + g) : make_float2(-INFINITY, 0.f);
            lv[k] = x.y;
            mv[k] = x.y != 0.f ? x.x : -INFINITY;
          }
          float M = fmaxf(mv[0], mv[1]);
#pragma unroll
          for (int s2 = 16; s2 > 0; s2 >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, s2));
          float den = 0.f;
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            mv[k] = lv[k] != 0.f ? exp2f(mv[k] - M) : 0.f;
            den += mv[k] * lv[k];
          }
#pragma unroll
          for (int s2 = 16; s2 > 0; s2 >>= 1) den += __shfl_xor_sync(0xffffffffu, den, s2);
          const float inv = den != 0.f ? 1.f / den : 0.f;
          wgt[g * RAP_MAX_SPLIT + lane] = mv[0] * inv;
          wgt[g * RAP_MAX_SPLIT + lane + 32] = mv[1] * inv;
        }
        constexpr int COLS = (8 * 32 + THREADS - 1) / THREADS;      // groups of four channels a thread has, at most
        float4 num[COLS];
#pragma unroll
        for (int k = 0; k < COLS; ++k) num[k] = make_float4(0.f, 0.f, 0.f, 0.f);
        bool got = true;
        for (int s0 = 0;;) {
          __syncthreads();
          got = __syncthreads_and(mbar_wait_bounded(bar_join, join_parity, p.wait_limit));
          if (!got) break;
          join_parity ^= 1u;
#pragma unroll
          for (int k = 0; k < COLS; ++k) {
            const int i = 4 * (tid + k * THREADS);
            if (i < part) {
              const float* wg = wgt + i / dv4 * RAP_MAX_SPLIT + s0;
              for (int s = 0; s < m; ++s) {
                const float4 v = *reinterpret_cast<const float4*>(sums + s * part + i);
                const float wk = wg[s];
                num[k].x = fmaf(wk, v.x, num[k].x);
                num[k].y = fmaf(wk, v.y, num[k].y);
                num[k].z = fmaf(wk, v.z, num[k].z);
                num[k].w = fmaf(wk, v.w, num[k].w);
              }
            }
          }
          s0 += m;
          if (s0 >= n) break;
          m = min(n - s0, p.join_places);
          __syncthreads();
          if (warp == 0) fetch(s0, m);
        }
        if (!got) {
          if (tid == 0) {
            win_report(p.status, RAP_ETIMEOUT, (int)unit);
            mbar_wait_bounded(bar_join, join_parity, p.wait_limit);      // copies still in flight: as above
          }
          if (p.ws.n_pre) pdl_wait();
          __syncthreads();
          return;
        }
#pragma unroll
        for (int k = 0; k < COLS; ++k) {
          const int i = 4 * (tid + k * THREADS);
          if (i < part) {
            const int g = i / dv4, c = i - g * dv4;
            float* og = out + (size_t)g * dv + c;
            og[0] = num[k].x;
            if (c + 1 < dv) og[1] = num[k].y;
            if (c + 2 < dv) og[2] = num[k].z;
            if (c + 3 < dv) og[3] = num[k].w;
          }
        }
        used = true;
        if (tid == 0) p.unit_cnt[unit] = 0;        // ready for the next call
      }
    }
    }
    // ---- the next unit, from its first block ----
    unit_start += u.n + p.own;
    cur = unit_start;
    if (cur >= hi) break;
    if (++h == p.Hkv) {
      h = 0;
      if (++b >= p.B) break;
      u = ws_unit(p, b);
    }
    __syncthreads();           // the sums and weights in shared memory have been read
  }
  if (p.ws.n_pre) pdl_wait();
}

// The form for G query heads a KV head, odd d_v' or not, rows through tensor maps or not, n steps of 16, nw warps
template <bool FOUR, bool VODD, bool LONG>
const void* scan_fn(int n, int nw) {
  switch (n * 8 + nw) {
    case 1 * 8 + 4: return (const void*)win_scan_kernel<1, FOUR, VODD, 4, false, LONG>;
    case 2 * 8 + 4: return (const void*)win_scan_kernel<2, FOUR, VODD, 4, false, LONG>;
    case 3 * 8 + 4: return (const void*)win_scan_kernel<3, FOUR, VODD, 4, false, LONG>;
    case 4 * 8 + 4: return (const void*)win_scan_kernel<4, FOUR, VODD, 4, false, LONG>;
    case 5 * 8 + 4: return (const void*)win_scan_kernel<5, FOUR, VODD, 4, false, LONG>;
    case 6 * 8 + 4: return (const void*)win_scan_kernel<6, FOUR, VODD, 4, false, LONG>;
    case 6 * 8 + 3: return (const void*)win_scan_kernel<6, FOUR, VODD, 3, false, LONG>;
    case 7 * 8 + 4: return (const void*)win_scan_kernel<7, FOUR, VODD, 4, false, LONG>;
    case 7 * 8 + 3: return (const void*)win_scan_kernel<7, FOUR, VODD, 3, false, LONG>;
    case 8 * 8 + 2: return (const void*)win_scan_kernel<8, FOUR, VODD, 2, false, LONG>;      // unpruned heads, seven or eight to a KV head
    case 8 * 8 + 3: return (const void*)win_scan_kernel<8, FOUR, VODD, 3, false, LONG>;
  }
  return nullptr;
}

template <bool FOUR, bool LONG>
const void* scan_tma_fn(int n) { return n == 4 ? (const void*)win_scan_kernel<4, FOUR, false, 4, true, LONG> : (const void*)win_scan_kernel<8, FOUR, false, 3, true, LONG>; }

template <bool LONG>
const void* scan_any(int G, bool vodd, bool tma, int n, int nw) {
  if (tma) return G <= 4 ? scan_tma_fn<true, LONG>(n) : scan_tma_fn<false, LONG>(n);
  if (G <= 4) return vodd ? scan_fn<true, true, LONG>(n, nw) : scan_fn<true, false, LONG>(n, nw);
  return vodd ? scan_fn<false, true, LONG>(n, nw) : scan_fn<false, false, LONG>(n, nw);
}

}  // namespace
