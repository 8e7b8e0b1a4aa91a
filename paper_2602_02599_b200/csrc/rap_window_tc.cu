// Attention of many queries over the same cache rows on tcgen05: rap_prefill_attn_window (the rows are a ragged block's new
// tokens) and the shared prefixes of rap_decode_attn_shared (the rows are the sequences of a group), for bf16 heads of up to
// 128 dims and channels.
//
// A CTA takes 256 rows of one (sequence or group, KV head) as two query tiles of 128, a row being a (token, query head) pair:
// the G query heads of a KV head sit side by side, so a block of 64 tokens with G = 4 fills both tiles, its rows see nearly the
// same window, and a staged K / V tile serves all of them.  It walks the 64-row key tiles that any of its rows sees: the sinks,
// then the window from the oldest visible position on (or one run from 0 where they meet).
//   S_X  = Q_X K^T   tcgen05.mma (M = 128, N = 64, K = 2P in steps of 16), accumulator in tensor memory, double buffered
//   P_X  = 2^(S - m) one thread per row: 64 logits in registers, masked only in tiles that reach an edge, lazy running maximum;
//                    every weight leaves as two bf16 numbers, its rounding and the remainder (17 bits: outputs are fp32 and one
//                    bf16 would put 1e-3 of error on them), which fill the 64 columns that the logits came from.  Measured
//                    against 64 bits 0.7e-6 ... 5.9e-6 of an output's size (7e-6 at 128 channels; 7.5e-6 and 1.1e-5
//                    where V is of one sign); a third bf16 number
//                    left 2.4e-6 ... 4.3e-6 on long rows (the sums in tensor memory are cut, not rounded, at every step, and it
//                    adds steps) and took 8 to 25% longer
//   O_X += P_X V     A = P from tensor memory: eight steps of 16, the roundings' four and the remainders' four over the same V
// Cache rows are not multiples of 16 bytes, so no tensor map describes them: six warps stage K and V with 4-byte cp.async
// into rings of four and five 128-byte-swizzled tiles (K as stored is the K-major operand, V as stored the N-major one).  Odd d_v'
// (HALF): every other row starts in the middle of a word, so V's words are copied as they lie and put in place when they have
// landed.  A rolling cache maps a position to its row; a tile is one run of rows, or two if it crosses the seam.
// A K / V tile of 23 KB takes (4 P + 8 d_v') 64 cycles of the tensor pipe per 128 rows and 64 x 128 / 16 of the exponential
// units: twice 576 and 512 cycles at P = 45.  Measured 2250 a tile: 8192 tokens at window 2048, 32 query heads, in 330 us replayed
// from a graph and 358 a call by itself (512 and 473 TFLOP/s of 2 (2P + d_v') a visible pair), the tensor pipe busy 43% of the
// time, the exponential units 39%, an issue slot 61%.  What bounds it is the softmax warps' stream of instructions (exponential, two conversions, two stores a logit) with the
// 4-byte copies beside it; four warps instead of two on a scheduler (half a row a thread) took 17% longer, remainders through
// shared memory 10%.  Few rows (prefixes of small groups, odd widths): the copies, 1300 to 2000 cycles a tile.
// Roles meet on mbarriers only; every wait is bounded and gives up early once another role has given up.
#include <math.h>

#include "rap_tc_common.cuh"
#include "rap_window_common.cuh"

namespace {

constexpr int WT_KT = 64;                              // keys per tile
constexpr int WT_THREADS = 512;                        // 8 softmax warps, 2 that issue MMAs, 6 that stage K and V
constexpr int WT_Q_BYTES = 2 * 128 * 128;              // [128 rows][<= 128 dims]: two 64-element atom columns
constexpr int WT_KV_BYTES = 2 * WT_KT * 128;           // [64 keys][<= 128 dims or channels]
constexpr int WT_TAIL = 320;                           // mbarriers, TMEM address, give-up flag
constexpr int WT_STAGES = 5, WT_K_STAGES = 4;           // V buffers and K buffers
constexpr int WT_DRAIN = 40;                           // tiles after which O leaves tensor memory
constexpr int WT_DRAIN_W = 32 * 17;                    // a softmax warp's buffer: 32 rows of 16 sums, on different banks
constexpr int WT_SMEM = 2 * WT_Q_BYTES + (WT_STAGES + WT_K_STAGES) * WT_KV_BYTES + 8 * WT_DRAIN_W * 4 + WT_TAIL;

struct WtParams {
  const __nv_bfloat16* q;      // [rows][Hq][P2]
  const __nv_bfloat16* k;      // [units][Hkv][S_cap][P2]
  const __nv_bfloat16* v;      // [units][Hkv][S_cap][dv]
  const int32_t* start;        // [units + 1]: first token (or sequence) of a unit in q
  const int32_t* len;          // [units]: length with the new tokens, or prefix length
  float* out;                  // [rows][Hq][dv]
  WinPartials ws;              // where a prefix's partials go
  int32_t* status;
  int units, rows, Hq, Hkv, G, P2, dv, S_cap, n_sink, window, sms;
  float qscale;                // log2(e) / sqrt(D)
};

__device__ __forceinline__ void wt_st8(uint32_t taddr, const uint32_t (&r)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(taddr), "r"(r[0]), "r"(r[1]),
               "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}

// The MMA-issuing warps run as whole warps and predicate each instruction on one elected lane: the descriptors then live in
// uniform registers.  A single lane's branch had every operand moved there one by one (a hundred cycles an MMA).
__device__ __forceinline__ uint32_t wt_elect() {
  uint32_t e;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(e));
  return e;
}
__device__ __forceinline__ void wt_mma_ss(uint32_t e, uint32_t tmem_d, uint32_t a_lo, uint32_t b_lo, uint32_t hi, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t.reg .b64 da, db;\n\t"
      "mov.b64 da, {%1, %3};\n\t"
      "mov.b64 db, {%2, %3};\n\t"
      "setp.ne.b32 p, %5, 0;\n\tsetp.ne.b32 q, %6, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %4, p;\n\t}" ::"r"(tmem_d),
      "r"(a_lo), "r"(b_lo), "r"(hi), "r"(idesc), "r"(acc), "r"(e)
      : "memory");
}
__device__ __forceinline__ void wt_mma_ts(uint32_t e, uint32_t tmem_d, uint32_t tmem_a, uint32_t b_lo, uint32_t hi, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t.reg .b64 db;\n\t"
      "mov.b64 db, {%2, %3};\n\t"
      "setp.ne.b32 p, %5, 0;\n\tsetp.ne.b32 q, %6, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %4, p;\n\t}" ::"r"(tmem_d),
      "r"(tmem_a), "r"(b_lo), "r"(hi), "r"(idesc), "r"(acc), "r"(e)
      : "memory");
}
// when the elected lane's MMAs complete (mma), or at once
__device__ __forceinline__ void wt_release(uint32_t e, uint32_t bar, bool mma) {
  if (mma)
    asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %1, 0;\n\t"
                 "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar), "r"(e) : "memory");
  else
    asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %1, 0;\n\t"
                 "@q mbarrier.arrive.shared::cta.b64 _, [%0];\n\t}" ::"r"(bar), "r"(e) : "memory");
}
__device__ __forceinline__ void wt_cp4(uint32_t dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ float wt_max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
// after the wait for loads: no arithmetic on what they return is moved ahead of it
template <int N>
__device__ __forceinline__ void wt_loaded(uint32_t* r) {
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+r"(r[i])::"memory");
}
__device__ __forceinline__ void wt_ld8(uint32_t taddr, uint32_t* r) {      // to be waited for
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(taddr)
               : "memory");
}
__device__ __forceinline__ void wt_ld16(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
        "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr)
      : "memory");
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
  wt_loaded<16>(r);
}

// DK = k-steps of Q K^T (ceil(2P / 16)); NVP = columns of the second MMA, a multiple of 16 from d_v' on.  LSUM: NVP > d_v', and
// column d_v' of every V tile holds the constant one, so that the row sums of the very weights that it multiplies come out of
// the second MMA (a fifth of the softmax threads' instructions otherwise).
// PREFIX: the rows are the sequences of group `unit`, all of which see all `len` rows of its cache, and the partials go to the
// workspace; otherwise the rows are new tokens of sequence `unit`.
template <int DK, int NVP, bool LSUM, bool HALF, bool PREFIX>
__global__ void __launch_bounds__(WT_THREADS, 1) win_tc_kernel(const WtParams p) {
  constexpr int NK = HALF ? 2 : 3, NV = 6 - NK;        // warps that stage K, and V (of odd width: twice the work)
  extern __shared__ unsigned char wt_raw[];
  unsigned char* smem = wt_raw + ((1024u - (pt_smem(wt_raw) & 1023u)) & 1023u);
  unsigned char* q_s = smem;                                   // Q_A, Q_B
  unsigned char* k_s = q_s + 2 * WT_Q_BYTES;                   // ring of K tiles
  unsigned char* v_s = k_s + WT_K_STAGES * WT_KV_BYTES;        // ring of V tiles (N-major)
  float* drain_s = reinterpret_cast<float*>(v_s + WT_STAGES * WT_KV_BYTES);
  unsigned char* tail = reinterpret_cast<unsigned char*>(drain_s + 8 * WT_DRAIN_W);
  const uint32_t bar_fk = pt_smem(tail), bar_ek = bar_fk + 8 * WT_STAGES, bar_fv = bar_ek + 8 * WT_STAGES,
                 bar_ev = bar_fv + 8 * WT_STAGES, bar_s = bar_ev + 8 * WT_STAGES /* [X][2] */, bar_p = bar_s + 32 /* [X][2] */,
                 bar_o = bar_p + 32 /* [X] */, bar_end = bar_o + 16 /* [X] */, bar_q = bar_end + 16 /* [X] */;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(tail + 32 * WT_STAGES + 112);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tail + 32 * WT_STAGES + 116);
  static_assert(32 * WT_STAGES + 120 <= WT_TAIL, "barriers and flags fit the tail");
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  const int G = p.G;
  if constexpr (PREFIX) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");   // the own rows' scan may start where SMs come free

  // ---- which unit, which of its rows, which KV head (and which split of a prefix): every warp walks the units, 256 rows a block ----
  int unit = -1, q0 = 0, h = blockIdx.y, split = 0, per = 0;
  if constexpr (PREFIX) per = win_prefix_plan(p.start, p.len, p.units, p.rows, G, p.Hkv, p.S_cap, p.sms, p.ws.n_pre).per;
  for (int u0 = 0, carry = 0; u0 < p.units; u0 += 32) {
    const int u = u0 + lane;
    int n = 0, n_split = 1;
    if (u < p.units) {
      n = (win_group_rows(p.start, u, p.rows, G) + 255) >> 8;
      if constexpr (PREFIX) n_split = (win_group_tiles(p.len, u, p.S_cap) + per - 1) / per * p.Hkv;
    }
    int x = n * n_split;
    const int mine = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += y;
    }
    const unsigned past = __ballot_sync(0xffffffffu, carry + x > (int)blockIdx.x);
    if (past) {
      const int l = __ffs(past) - 1;
      unit = u0 + l;
      int at = (int)blockIdx.x - carry - __shfl_sync(0xffffffffu, x - mine, l);
      if constexpr (PREFIX) {        // KV heads of a split side by side, then splits, then blocks of rows
        const int ns = __shfl_sync(0xffffffffu, n_split, l);
        q0 = at / ns * 256;
        at -= at / ns * ns;
        split = at / p.Hkv;
        h = at - split * p.Hkv;
      } else {
        q0 = at * 256;
      }
      break;
    }
    carry += __shfl_sync(0xffffffffu, x, 31);
  }
  if (unit < 0) return;                                        // fewer row blocks than CTAs
  const int first = min(max(p.start[unit], 0), p.rows);
  const int n_tok = min(max(p.start[unit + 1], first), p.rows) - first, n_rows = n_tok * G;

  // row r of the block is query head row_g of token row_t: rows in [0, 264) over G <= 8 by a 16-bit reciprocal, exact there
  const int t_base = q0 / G, t_rest = q0 - t_base * G, g_recip = (65536 + G - 1) / G;
  auto row_t = [&](int r) { return t_base + (((t_rest + r) * g_recip) >> 16); };

  const int kw = p.P2 >> 1;                          // 4-byte words per q / K row
  // (while the unit's numbers are on their way) K's pad dims are zero (Q's too, below; V's pad channels only reach accumulator
  // columns that nothing reads); LSUM: channel dv of all rows of every V buffer is one (odd dv: the producers write it with the
  // row's last word)
  for (int i = tid; i < WT_STAGES * WT_KT; i += WT_THREADS) {
    const int at = (i >> 6) * WT_KV_BYTES + (i & 63) * 128;
    for (int w = kw; w < 8 * DK && i < WT_K_STAGES * WT_KT; ++w) *reinterpret_cast<uint32_t*>(k_s + at + pt_swz2(4 * w, i & 7)) = 0u;
    if constexpr (LSUM) *reinterpret_cast<uint32_t*>(v_s + at + pt_swz2(4 * (p.dv >> 1), i & 7)) = p.dv & 1 ? 0x3f800000u : 0x3f80u;
  }

  // ---- the key tiles: n_st of sinks, then 64 rows each from position `base` on; nt[X] of them for query tile X ----
  const int len = PREFIX ? min(max(p.len[unit], 0), p.S_cap) : max(p.len[unit], 0);
  const int pos0 = len - n_tok;                                // position of the block's first token
  int n_st = 0, base = 0, jend, nt[2], pmin[2], pmax[2], t_first = 0;
#pragma unroll
  for (int X = 0; X < 2; ++X) {
    pmin[X] = pos0 + row_t(128 * X);
    pmax[X] = q0 + 128 * X < n_rows ? pos0 + row_t(min(n_rows - q0, 128 * X + 128) - 1) : -1;
  }
  if constexpr (PREFIX) {
    const int all = (len + WT_KT - 1) / WT_KT;
    t_first = split * per;
    jend = len;
#pragma unroll
    for (int X = 0; X < 2; ++X) nt[X] = q0 + 128 * X < n_rows ? min(all, t_first + per) - t_first : 0;
  } else {
    const int old = (int)max(0LL, (long long)pmin[0] - p.window + 1);            // the oldest position in a window
    if (old > p.n_sink) {
      n_st = (p.n_sink + WT_KT - 1) / WT_KT;
      base = old;
    }
    jend = max(pmax[0], pmax[1]) + 1;
#pragma unroll
    for (int X = 0; X < 2; ++X) nt[X] = pmax[X] >= 0 ? n_st + (pmax[X] - base) / WT_KT + 1 : 0;
  }
  const int n_max = max(nt[0], nt[1]);
  const __nv_bfloat16* kg = p.k + ((size_t)unit * p.Hkv + h) * (size_t)p.S_cap * p.P2;
  const __nv_bfloat16* vg = p.v + ((size_t)unit * p.Hkv + h) * (size_t)p.S_cap * p.dv;
  // first position of a tile, and the position behind its last one
  auto tile_at = [&](int tile, int& j0, int& j1) {
    if (PREFIX) {
      j0 = (t_first + tile) * WT_KT;
      j1 = jend;
    } else {
      j0 = tile < n_st ? tile * WT_KT : base + (tile - n_st) * WT_KT;
      j1 = tile < n_st ? p.n_sink : jend;
    }
  };

  if (tid == 0) {
    for (int i = 0; i < WT_STAGES; ++i) {
      pt_mbar_init(bar_fk + 8 * i, 32 * NK);
      pt_mbar_init(bar_ek + 8 * i, 2);               // both MMA-issuing lanes release a buffer
      pt_mbar_init(bar_fv + 8 * i, 32 * NV);
      pt_mbar_init(bar_ev + 8 * i, 2);
    }
    for (int i = 0; i < 4; ++i) {
      pt_mbar_init(bar_s + 8 * i, 1);
      pt_mbar_init(bar_p + 8 * i, 128);              // one barrier per S buffer: the softmax may be a tile ahead of who waits for it
    }
    for (int X = 0; X < 2; ++X) pt_mbar_init(bar_o + 8 * X, 1);
    pt_mbar_init(bar_end, 1);
    pt_mbar_init(bar_end + 8, 1);
    pt_mbar_init(bar_q, 128);
    pt_mbar_init(bar_q + 8, 128);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 8) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(pt_smem(tmem_slot)), "r"(512)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem_base = *tmem_slot;             // S_X(t): columns 128 X + 64 (t & 1); O_X: columns 256 + 128 X
  constexpr uint32_t IDESC_S = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(WT_KT >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
  constexpr uint32_t IDESC_O = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) | ((uint32_t)(NVP >> 3) << 17) |
                               ((uint32_t)(128 >> 4) << 24);
  auto wait = [&](uint32_t bar, uint32_t parity) -> bool {
    if (pt_test_wait(bar, parity)) return true;
    for (uint32_t i = 0; i < PT_WAIT_LIMIT; ++i) {
      if (pt_try_wait(bar, parity)) return true;
      if ((i & 15u) == 15u && *abort_flag) return false;
    }
    *abort_flag = (warp << 16) | (int)(bar - bar_fk) | 0x60000000;      // given up: which warp, on which barrier
    return false;
  };

  float l_run = 0.f, m_ref = -INFINITY;
  const int X = (warp >> 2) & 1;                     // softmax group = query tile
  const int row = (warp & 3) * 32 + lane;
  const uint32_t lane_off = (uint32_t)((warp & 3) * 32) << 16;
  const uint32_t tmem_o = tmem_base + 256 + 128 * X;
  // registers: two times 256 threads share the 512 x 128 that the block has (staging a prefix or
  // odd rows holds more addresses)
  static_assert(WT_THREADS == 512, "the split below is of 512 threads");
  if constexpr (PREFIX || HALF) {
    if (warp < 8) asm volatile("setmaxnreg.inc.sync.aligned.u32 152;");
    else asm volatile("setmaxnreg.dec.sync.aligned.u32 104;");
  } else {
    if (warp < 8) asm volatile("setmaxnreg.inc.sync.aligned.u32 168;");
    else asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
  }
  if (warp >= 10) {
    // ================= producers: NK warps stage K, NV warps V, eight tile rows at a time =================
    const bool is_v = warp >= 10 + NK;
    const int pw = warp - 10 - (is_v ? NK : 0), np = is_v ? NV : NK;
    const int rowlen = is_v ? p.dv : p.P2, rb = 2 * rowlen;
    const unsigned char* src0 = reinterpret_cast<const unsigned char*>(is_v ? vg : kg) + 4 * lane;
    unsigned char* ring = is_v ? v_s : k_s;
    const uint32_t bar_f = is_v ? bar_fv : bar_fk, bar_e = is_v ? bar_ev : bar_ek;
    const int words = (rowlen + 1) >> 1;
    const bool one = lane < words, two = lane + 32 < words;
    uint32_t swz[8];                                   // of the lane's first word in a tile row, by row % 8; its second one is 8 KB on
#pragma unroll
    for (int c = 0; c < 8; ++c) swz[c] = pt_swz2(4 * lane, c) + 128u * c;
    const int R = p.S_cap - p.n_sink;
    // the key of tile row i; V: keys k and k + 8 of sixteen lie side by side
    auto key_of = [&](int i) { return is_v ? (i & 48) + ((i & 15) >> 1) + 8 * (i & 1) : i; };
    // the rows of a tile are one run from row s0 on, or two if it crosses the seam of a rolling cache (false: more, the cache is
    // shorter than the tile)
    auto run_of = [&](int j0, int n, int& s0) {
      s0 = j0;
      if (PREFIX || j0 + n <= p.S_cap) return true;
      s0 = j0 >= p.n_sink ? p.n_sink + (j0 - p.n_sink) % R : j0;
      return s0 + n <= p.S_cap || n <= R;
    };
    // row of the tile's key r, then
    auto row_of = [&](int s0, int r) { return s0 + r - (!PREFIX && s0 + r >= p.S_cap ? R : 0); };
    // the first of this warp's groups of eight rows; they take turns, so that the odd group falls to each of them
    auto first_group = [&](int tile) { return is_v ? (pw + tile) % NV : (pw + tile) % NK; };
    // words as they lie in the cache, row by row; rows behind the tile's last are zeros and nothing is read for them
    auto copy_rows = [&](uint32_t du, int tile, int j0, int n, bool run, int s0) {
      // where the tile's first row lies, and where it would lie for the rows behind the seam
      const long long b0 = (long long)s0 * rb, b1 = (long long)(s0 - R) * rb;
      const unsigned char *run0 = src0 + (b0 & ~3LL), *run1 = src0 + (b1 & ~3LL);
      const int head0 = (int)(b0 & 3), head1 = (int)(b1 & 3);
#pragma unroll 1
      for (int g = first_group(tile); g < WT_KT / 8; g += np) {
        const uint32_t dg = du + g * 1024;
        if (HALF && n == WT_KT && s0 + n <= p.S_cap && RAP_BOUNDS(s0 + n - 1, p.S_cap, p.status, 0x302)) {      // no predicates
#pragma unroll
          for (int c = 0; c < 8; ++c) {
            const unsigned char* src = run0 + ((head0 + key_of(8 * g + c) * rb) & ~3);
            if (one) wt_cp4(dg + swz[c], src);
            if (two) wt_cp4(dg + swz[c] + 8192, src + 128);
          }
        } else if (run) {
#pragma unroll
          for (int c = 0; c < 8; ++c) {
            const int r = key_of(8 * g + c), bytes = r < n && RAP_BOUNDS(row_of(s0, r), p.S_cap, p.status, 0x302) ? 4 : 0;
            const bool seam = !PREFIX && bytes && s0 + r >= p.S_cap;
            const unsigned char* src = (seam ? run1 : run0) + (bytes ? ((seam ? head1 : head0) + r * rb) & ~3 : 0);
            if (one) pt_cp4(dg + swz[c], src, bytes);
            if (two) pt_cp4(dg + swz[c] + 8192, src + 128, bytes);
          }
        } else {
#pragma unroll 1
          for (int c = 0; c < 8; ++c) {
            const int r = key_of(8 * g + c), sl = r < n ? win_slot(j0 + r, p.n_sink, p.S_cap) : 0;
            const unsigned char* src = src0 + (((size_t)sl * (size_t)rb) & ~(size_t)3);
            const int bytes = r < n && RAP_BOUNDS(sl, p.S_cap, p.status, 0x303) ? 4 : 0;
            const uint32_t d = dg + 128u * c + pt_swz2(4 * lane, c);
            if (one) pt_cp4(d, src, bytes);
            if (two) pt_cp4(d + 8192, src + 128, bytes);
          }
        }
      }
    };
    // A prefix's rows come from HBM, once: what a launch keeps on its way with 4-byte copies alone is a third of what HBM takes
    // (2200 cycles a tile), so their lines are asked into L2 some tiles ahead, a tile's as one bulk request of whole 16-byte
    // units (a cache's end is one: S_cap is a multiple of 8).
    constexpr int L2_AHEAD = 12;
    auto prefetch = [&](int tile) {
      if (!PREFIX || pw != 0 || lane != 0 || tile >= n_max) return;
      int j0, j1;
      tile_at(tile, j0, j1);
      const size_t b0 = (size_t)j0 * (size_t)rb & ~(size_t)15, b1 = ((size_t)min(j0 + WT_KT, j1) * (size_t)rb + 15) & ~(size_t)15;
      if (!RAP_BOUNDS(b1 - 1, (size_t)p.S_cap * (size_t)rb, p.status, 0x30a)) return;
      asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(src0 + b0), "r"((uint32_t)(b1 - b0)) : "memory");
    };
#pragma unroll 1
    for (int t = 0; t < L2_AHEAD; ++t) prefetch(t);
    if (HALF && is_v) {
      // Rows of an odd number of half words: every other one starts in the middle of a word.  The words that hold a row are
      // copied as they lie, AHEAD tiles ahead; once they have landed, a lane that copied a word of such a row puts its half and
      // the half from the lane behind in its place (no lane reads what another one copied).
      constexpr int AHEAD = 3;                         // below WT_STAGES - 1: the tile before the oldest unfinished one is never waited for
      int stg = 0, use = 0, fix = 0;
      uint32_t keep[2], ones[2];                       // LSUM: the high half of a row's last word is the constant one
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const bool last = LSUM && lane + 32 * i == words - 1;
        keep[i] = last ? 0xffffu : ~0u;
        ones[i] = last ? 0x3f800000u : 0u;
      }
      for (int step = 0; step < n_max + AHEAD; ++step) {
        if (step < n_max) {
          int j0, j1, s0;
          tile_at(step, j0, j1);
          if (use > 0 && !__all_sync(0xffffffffu, wait(bar_e + 8 * stg, (use - 1) & 1))) break;
          const int n = min(WT_KT, j1 - j0);
          const bool run = run_of(j0, n, s0);
          prefetch(step + L2_AHEAD);
          copy_rows(pt_smem(ring + stg * WT_KV_BYTES), step, j0, n, run, s0);
          if (++stg == WT_STAGES) { stg = 0; ++use; }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        if (step < AHEAD) continue;
        asm volatile("cp.async.wait_group %0;" ::"n"(AHEAD) : "memory");
        int j0, j1, s0;
        tile_at(step - AHEAD, j0, j1);
        const int n = min(WT_KT, j1 - j0);
        const bool run = run_of(j0, n, s0);
        unsigned char* vt = ring + fix * WT_KV_BYTES;
        // (without a branch on the row's parity: eight rows' loads, shuffles and stores then overlap)
        auto place = [&](uint32_t* w0, int odd) {
          uint32_t v0 = w0[0], v1 = w0[2048];
          const uint32_t n0 = __shfl_sync(0xffffffffu, v0, (lane + 1) & 31), n1 = __shfl_sync(0xffffffffu, v1, (lane + 1) & 31);
          v0 = __funnelshift_r(v0, lane == 31 ? n1 : n0, odd * 16);
          v1 = __funnelshift_r(v1, n1, odd * 16);
          v0 = (v0 & keep[0]) | ones[0];
          v1 = (v1 & keep[1]) | ones[1];
          if (one) w0[0] = v0;
          if (two) w0[2048] = v1;
        };
#pragma unroll 1
        for (int g = first_group(step - AHEAD); g < WT_KT / 8; g += np) {
          if (run) {
#pragma unroll
            for (int c = 0; c < 8; ++c) place(reinterpret_cast<uint32_t*>(vt + g * 1024 + swz[c]), row_of(s0, key_of(8 * g + c)) & 1);
          } else {
#pragma unroll 1
            for (int c = 0; c < 8; ++c)
              place(reinterpret_cast<uint32_t*>(vt + g * 1024 + 128 * c + pt_swz2(4 * lane, c)), win_slot(j0 + min(key_of(8 * g + c), n - 1), p.n_sink, p.S_cap) & 1);
          }
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar_f + 8 * fix) : "memory");
        if (++fix == WT_STAGES) fix = 0;
      }
    } else {
      int stg = 0, use = 0;
      for (int tile = 0; tile < n_max; ++tile) {
        int j0, j1, s0;
        tile_at(tile, j0, j1);
        if (use > 0 && !wait(bar_e + 8 * stg, (use - 1) & 1)) break;
        const uint32_t du = pt_smem(ring + stg * WT_KV_BYTES);
        const int n = min(WT_KT, j1 - j0);
        const bool run = run_of(j0, n, s0);
        prefetch(tile + L2_AHEAD);
        if (!RAP_BOUNDS(n - 1, WT_KT, p.status, 0x304) || !RAP_BOUNDS(run ? s0 : 0, p.S_cap, p.status, 0x305) ||
            !RAP_BOUNDS(run ? row_of(s0, n - 1) : 0, p.S_cap, p.status, 0x306))
          break;
        if (n == WT_KT && s0 + n <= p.S_cap) {
          // a full tile in one run: no predicates, running pointers (V: from key k to k + 8 and back to k + 1)
          const long long even = is_v ? 8LL * rb : rb, odd = is_v ? -7LL * rb : rb;
#pragma unroll 1
          for (int g = first_group(tile); g < WT_KT / 8; g += np) {
            const unsigned char* a = src0 + (size_t)(s0 + key_of(8 * g)) * (size_t)rb;
            const uint32_t dg = du + g * 1024;
#pragma unroll
            for (int c = 0; c < 8; ++c) {
              if (one) wt_cp4(dg + swz[c], a);
              if (two) wt_cp4(dg + swz[c] + 8192, a + 128);
              a += (c & 1) ? odd : even;
            }
          }
        } else {
          copy_rows(du, tile, j0, n, run, s0);
        }
        // the arrival is triggered by the completion of this thread's copies: go on to the next tile
        asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar_f + 8 * stg) : "memory");
        if (++stg == (is_v ? WT_STAGES : WT_K_STAGES)) { stg = 0; ++use; }
      }
    }
    // copies that nobody waited for (a role gave up) have landed before the shared memory is used for the output
    asm volatile("cp.async.wait_all;" ::: "memory");
  } else if (warp >= 8) {
    // ================= MMA issue: warp 8 for query tile A, warp 9 for query tile B =================
    // A buffer of the rings is free when both warps have committed past it; a warp whose tile needs no more keys keeps
    // arriving in step (after the buffer was filled), so the phases stay aligned.
    if (n_max > 0) {
      const int Y = warp - 8, n_y = Y ? nt[1] : nt[0];
      const uint32_t e = wt_elect();
      const uint32_t tmem_sy = tmem_base + 128u * (uint32_t)Y, tmem_oy = tmem_base + 256u + 128u * (uint32_t)Y;
      constexpr uint32_t DESC_HI = (1024u >> 4) | (1u << 14) | (2u << 29);
      constexpr uint32_t BUF16 = (uint32_t)WT_KV_BYTES >> 4;
      const uint32_t q_lo = (((pt_smem(q_s) + (uint32_t)Y * WT_Q_BYTES) & 0x3FFFFu) >> 4) | (1u << 16);
      const uint32_t k_lo0 = ((pt_smem(k_s) & 0x3FFFFu) >> 4) | (1u << 16);
      const uint32_t v_lo0 = ((pt_smem(v_s) & 0x3FFFFu) >> 4) | ((8192u >> 4) << 16);
      auto wait_all = [&](uint32_t bar, uint32_t parity) { return __all_sync(0xffffffffu, wait(bar, parity)) != 0; };
      auto issue_s = [&](uint32_t kbuf, uint32_t sbuf) {     // S into buffer sbuf from K buffer kbuf
        const uint32_t kb = k_lo0 + kbuf * BUF16, td = tmem_sy + 64u * sbuf;
#pragma unroll
        for (int ks = 0; ks < DK; ++ks)
          wt_mma_ss(e, td, q_lo + (uint32_t)(((ks >> 2) * 16384 + (ks & 3) * 32) >> 4),
                    kb + (uint32_t)(((ks >> 2) * 8192 + (ks & 3) * 32) >> 4), DESC_HI, IDESC_S, ks > 0 ? 1u : 0u);
        wt_release(e, bar_s + 8 * (2 * Y + sbuf), true);
      };
      bool ok = (n_y == 0 || wait_all(bar_q + 8 * Y, 0)) && wait_all(bar_fk, 0);
      if (ok) {
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        if (n_y > 0) issue_s(0, 0);
        wt_release(e, bar_ek, n_y > 0);
      }
      uint32_t kbuf = 1, kpar = 0;       // ring position and phase of K tile + 1
      uint32_t vbuf = 0, vpar = 0;       // of V tile
      for (int tile = 0; ok && tile < n_max; ++tile) {
        const uint32_t sb = (uint32_t)tile & 1u;
        if (tile + 1 < n_max) {
          if (!wait_all(bar_fk + 8 * kbuf, kpar)) { ok = false; break; }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          if (tile + 1 < n_y) issue_s(kbuf, sb ^ 1u);
          wt_release(e, bar_ek + 8 * kbuf, tile + 1 < n_y);
          if (++kbuf == WT_K_STAGES) { kbuf = 0; kpar ^= 1u; }
        }
        if (!wait_all(bar_fv + 8 * vbuf, vpar)) { ok = false; break; }
        if (tile < n_y) {
          if (!wait_all(bar_p + 8 * (2 * Y + sb), (uint32_t)(tile >> 1) & 1u)) { ok = false; break; }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          const uint32_t vb = v_lo0 + vbuf * BUF16, ta = tmem_sy + 64u * sb;
#pragma unroll
          for (int ks = 0; ks < WT_KT / 8; ++ks)    // sixteen keys' roundings (eight columns), then their remainders, over the same V
            wt_mma_ts(e, tmem_oy, ta + 8u * (uint32_t)ks, vb + (uint32_t)((ks >> 1) * 2048 >> 4), DESC_HI, IDESC_O,
                      (tile % WT_DRAIN > 0 || ks > 0) ? 1u : 0u);
          wt_release(e, bar_o + 8 * Y, true);
        }
        wt_release(e, bar_ev + 8 * vbuf, tile < n_y);
        if (++vbuf == WT_STAGES) { vbuf = 0; vpar ^= 1u; }
      }
      // every MMA issued above has completed before tensor memory is released, also when a role has given up
      wt_release(e, bar_end + 8 * Y, true);
      for (uint32_t i = 0; i < PT_WAIT_LIMIT && !__all_sync(0xffffffffu, pt_try_wait(bar_end + 8 * Y, 0)); ++i) {}
    }
    __syncwarp();
  } else {
    // ================= softmax group X: one thread per row of query tile X =================
    const int n = q0 + 128 * X + row;
    const int pos = n < n_rows ? pos0 + row_t(128 * X + row) : -1;
    const bool active = q0 + 128 * X + (warp & 3) * 32 < n_rows;       // some row of this warp is one
    const int n_my = X ? nt[1] : nt[0], p_min = X ? pmin[1] : pmin[0], p_max = X ? pmax[1] : pmax[0];
    bool rows_ok = true;
    if (n_my > 0) {
      // Q_X: a warp stages its 32 rows, all in flight at once; rows behind the block's last and pad dims are zeros
      const uint32_t* qsrc = reinterpret_cast<const uint32_t*>(p.q) + ((size_t)(first + t_base) * p.Hq + (size_t)h * G) * kw + lane;
      unsigned char* qd = q_s + X * WT_Q_BYTES + (warp & 3) * 32 * 128 + ((lane & 3) << 2);
      uint32_t qv[32][2];
#pragma unroll
      for (int u = 0; u < 32; ++u) {
        const int rr = 128 * X + (warp & 3) * 32 + u, t = row_t(rr) - t_base;
        const bool ok = q0 + rr < n_rows && RAP_BOUNDS(first + t_base + t, p.rows, p.status, 0x307);
        const uint32_t* src = qsrc + ((size_t)t * p.Hq + (t_rest + rr - t * G)) * kw;
        qv[u][0] = ok && lane < kw ? __ldg(src) : 0u;
        qv[u][1] = ok && lane + 32 < kw ? __ldg(src + 32) : 0u;
      }
#pragma unroll
      for (int u = 0; u < 32; ++u) {
        unsigned char* d = qd + u * 128 + (((lane >> 2) ^ (u & 7)) << 4);
        if (lane < 8 * DK) *reinterpret_cast<uint32_t*>(d) = qv[u][0];
        if (lane + 32 < 8 * DK) *reinterpret_cast<uint32_t*>(d + 128 * 128) = qv[u][1];
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar_q + 8 * X) : "memory");
    }
    // a row of this query tile: its head's place behind that of the block's first token; where that one's sums go
    auto head_of = [&](int r) { const int t = row_t(128 * X + r); return (t - t_base) * p.Hq + (q0 + 128 * X + r - t * G); };
    auto first_dst = [&]() {
      const long long head0 = (long long)(first + t_base) * p.Hq + (long long)h * G;
      return PREFIX ? p.ws.pre_sums(head0, split) : p.out + head0 * p.dv;
    };
    // Sums in tensor memory are cut at every step, which takes 2e-6 of them per 1024 rows (the row sum's part of it cancels where
    // that comes from there too): every 2560 rows they are added to what the output (or the partial) holds, relative to the
    // maximum m_acc, and begin again (12,000 rows: errors of 3e-5 without, 4e-6 to 7e-6 with it, at 10 to 20% of the time there)
    float l_acc = 0.f, m_acc = -INFINITY;
    auto drained_weight = [&]() { return m_acc == m_ref ? 1.f : pt_ex2(m_acc - m_ref); };
    int tile = 0;
    for (int t_new = 0; t_new < n_my && rows_ok; t_new += WT_DRAIN) {
      const int t_end = min(n_my, t_new + WT_DRAIN);
#pragma unroll 1
      for (; tile < t_end; ++tile) {
        int j0, j1;
        tile_at(tile, j0, j1);
        const uint32_t trow = tmem_base + 128u * (uint32_t)X + 64u * (uint32_t)(tile & 1) + lane_off;
        if (!__all_sync(0xffffffffu, wait(bar_s + 8 * (2 * X + (tile & 1)), (tile >> 1) & 1))) { rows_ok = false; break; }
        if (active) {
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          // nothing of the tile is hidden from any row of this query tile
          // (differences: positions end at 2^31 - 2)
          const bool whole = PREFIX ? j1 - j0 >= WT_KT
                                    : tile >= n_st && p_min - j0 >= WT_KT - 1 && p_max - j0 < p.window && j1 - j0 >= WT_KT;
          if (!whole) {
            // the few tiles at an edge: hidden logits become -infinity (weight 0) where they are, so that the tiles' common path
            // knows no mask.  Seen are columns [0, c1), without those behind the sinks and before the window
            const int c1 = PREFIX ? j1 - j0 : min(j1, pos + 1) - j0;
            const int c_win = PREFIX ? 0 : (int)max(0LL, (long long)pos - p.window + 1 - j0), c_sink = PREFIX ? 0 : p.n_sink - j0;
            auto below = [](int c) { return c <= 0 ? 0ull : c >= 64 ? ~0ull : (1ull << c) - 1; };
            const uint64_t seen = below(c1) & (~below(c_win) | below(c_sink));
#pragma unroll 1
            for (int c = 0; c < 64; c += 16) {
              uint32_t e[16];
              wt_ld16(trow + c, e);
              const uint32_t bits = (uint32_t)(seen >> c);
#pragma unroll
              for (int j = 0; j < 16; ++j)
                if (!(bits & (1u << j))) e[j] = 0xff800000u;
              wt_st8(trow + c, *reinterpret_cast<uint32_t(*)[8]>(e));
              wt_st8(trow + c + 8, *reinterpret_cast<uint32_t(*)[8]>(e + 8));
            }
            asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
          }
          uint32_t r[64];
          pt_ld32_nowait(trow, *reinterpret_cast<uint32_t(*)[32]>(r));
          pt_ld32_nowait(trow + 32, *reinterpret_cast<uint32_t(*)[32]>(r + 32));
          asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
          wt_loaded<64>(r);
          float mx4[4];
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            mx4[c] = __uint_as_float(r[16 * c]);
#pragma unroll
            for (int j = 1; j < 15; j += 2) mx4[c] = wt_max3(mx4[c], __uint_as_float(r[16 * c + j]), __uint_as_float(r[16 * c + j + 1]));
            mx4[c] = fmaxf(mx4[c], __uint_as_float(r[16 * c + 15]));
          }
          const float mx = fmaxf(wt_max3(mx4[0], mx4[1], mx4[2]), mx4[3]) * p.qscale;
          float alpha = 1.f;
          if (mx > m_ref + 8.f) {          // lazy reference maximum: weights stay <= 2^8
            alpha = pt_ex2(m_ref - mx);
            m_ref = mx;
            l_run *= alpha;
          }
          const float nm = m_ref == -INFINITY ? 0.f : -m_ref;
          if (tile > t_new && __any_sync(0xffffffffu, alpha != 1.f)) {
            // rare: rescale this warp's accumulator rows in tensor memory, once the previous tile's update is in
            if (!__all_sync(0xffffffffu, wait(bar_o + 8 * X, (tile - 1) & 1))) { rows_ok = false; break; }
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll 1
            for (int c0 = 0; c0 < NVP; c0 += 16) {
              uint32_t oc[16];
              wt_ld16(tmem_o + lane_off + c0, oc);
#pragma unroll
              for (int j = 0; j < 16; ++j) oc[j] = __float_as_uint(__uint_as_float(oc[j]) * alpha);
              wt_st8(tmem_o + lane_off + c0, *reinterpret_cast<uint32_t(*)[8]>(oc));
              wt_st8(tmem_o + lane_off + c0 + 8, *reinterpret_cast<uint32_t(*)[8]>(oc + 8));
            }
          }
          // p = rounding + remainder.  Columns k and k + 8 of sixteen make a pair: its roundings replace column k, its remainders
          // column k + 8, so the registers that the logits came in leave again as whole blocks (a store of eight columns each cost
          // a third of the kernel's time), and the V rows of sixteen keys are staged in that order
          float ls[2] = {0.f, 0.f};
#pragma unroll
          for (int g16 = 0; g16 < 64; g16 += 16)
#pragma unroll
            for (int k = g16; k < g16 + 8; ++k) {
              const float p0 = pt_ex2(fmaf(__uint_as_float(r[k]), p.qscale, nm)), p1 = pt_ex2(fmaf(__uint_as_float(r[k + 8]), p.qscale, nm));
              if constexpr (!LSUM) {
                ls[0] += p0;
                ls[1] += p1;
              }
              const __nv_bfloat162 v2 = __floats2bfloat162_rn(p0, p1);
              const uint32_t hi = *reinterpret_cast<const uint32_t*>(&v2);
              uint64_t p2, h2, x2;
              float x0, x1;
              asm("mov.b64 %0, {%1, %2};" : "=l"(p2) : "f"(p0), "f"(p1));
              asm("mov.b64 %0, {%1, %2};" : "=l"(h2) : "r"(hi << 16), "r"(hi & 0xffff0000u));
              asm("sub.rn.f32x2 %0, %1, %2;" : "=l"(x2) : "l"(p2), "l"(h2));
              asm("mov.b64 {%0, %1}, %2;" : "=f"(x0), "=f"(x1) : "l"(x2));
              const __nv_bfloat162 w2 = __floats2bfloat162_rn(x0, x1);
              r[k] = hi;
              r[k + 8] = *reinterpret_cast<const uint32_t*>(&w2);
            }
          // over the columns that the logits came from; the next S into this buffer is issued after the MMA that reads these
          pt_st32(trow, *reinterpret_cast<uint32_t(*)[32]>(r));
          pt_st32(trow + 32, *reinterpret_cast<uint32_t(*)[32]>(r + 32));
          if constexpr (!LSUM) l_run += ls[0] + ls[1];
          asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
          asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        }
        asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar_p + 8 * (2 * X + (tile & 1))) : "memory");
      }
      if (rows_ok && tile < n_my && active) {
        // (the next S was issued behind the product before the last one: once it is there, only the last one's phase can be open)
        if (!__all_sync(0xffffffffu, wait(bar_s + 8 * (2 * X + (tile & 1)), (tile >> 1) & 1) && wait(bar_o + 8 * X, (tile - 1) & 1))) { rows_ok = false; break; }
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const float w = drained_weight();
        const bool drained = tile > WT_DRAIN;
        // sixteen columns at a time through shared memory, so that they leave as pieces of rows; where no maximum has moved since
        // the last time nothing is read back
        const bool same = __all_sync(0xffffffffu, w == 1.f);
        const int my_head = head_of(row), r_n = n_rows - q0 - 128 * X - (warp & 3) * 32, cc = lane & 15;
        float* buf = drain_s + (warp & 7) * WT_DRAIN_W;
        const bool in = RAP_BOUNDS(split, PREFIX ? p.ws.n_pre : 1, p.status, 0x30c);
#pragma unroll 1
        for (int c0 = 0; c0 < p.dv; c0 += 16) {
          uint32_t oc[16];
          wt_ld16(tmem_o + lane_off + c0, oc);
          __syncwarp();
#pragma unroll
          for (int c = 0; c < 16; ++c) buf[lane * 17 + c] = __uint_as_float(oc[c]);
          __syncwarp();
          float* dst0 = first_dst() + c0 + cc;
#pragma unroll 4
          for (int r2 = 0; r2 < 32; r2 += 2) {
            const int r = r2 + (lane >> 4);
            float* dst = dst0 + (long long)__shfl_sync(0xffffffffu, my_head, r) * (PREFIX ? p.ws.dv4 : p.dv);
            const float wr = __shfl_sync(0xffffffffu, w, r), x = buf[r * 17 + cc];
            if (r >= r_n || c0 + cc >= p.dv || !in || !RAP_BOUNDS(first + row_t(128 * X + (warp & 3) * 32 + r), p.rows, p.status, 0x30d)) continue;
            if (!drained) *dst = x;
            else if (same) asm volatile("red.relaxed.gpu.global.add.f32 [%0], %1;" ::"l"(dst), "f"(x) : "memory");
            else *dst = x + __ldcg(dst) * wr;
          }
        }
        if constexpr (LSUM) l_acc = l_acc * w + __uint_as_float(pt_ld1(tmem_o + lane_off + (uint32_t)p.dv));
        m_acc = m_ref;
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
      }
    }
    // ---- the output.  A thread owns a row in tensor memory, but a row of the output is contiguous in global memory: a warp
    // passes its 32 rows through its part of Q_X's tiles, CC columns at a time (rows of CC + 1 floats hit 32 banks), and they
    // leave as pieces of whole rows.  Every MMA of the query tile is done when bar_end says so.
    if (rows_ok && n_my > 0) rows_ok = __all_sync(0xffffffffu, wait(bar_end + 8 * X, 0));
    if (rows_ok && active) {
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      constexpr int CC = NVP == 128 ? 32 : NVP / 2;
      static_assert(CC % 8 == 0 && 4 * 32 * (CC + 1) * 4 <= WT_Q_BYTES, "four warps' rows fit the tile");
      float* o_s = reinterpret_cast<float*>(q_s + X * WT_Q_BYTES) + (warp & 3) * 32 * (CC + 1);
      const bool drained = n_my > WT_DRAIN;
      const float w = drained ? drained_weight() : 0.f;
      const int my_head = head_of((warp & 3) * 32 + lane);
      if (LSUM && n_my > 0) l_run = __uint_as_float(pt_ld1(tmem_o + lane_off + (uint32_t)p.dv)) + l_acc * w;
      const float f = PREFIX ? 1.f : l_run != 0.f ? 1.f / l_run : 0.f;
      const int r_first = 128 * X + (warp & 3) * 32, r_n = min(32, n_rows - q0 - r_first);
      if (PREFIX && lane < r_n) {
        *p.ws.pre_pair((long long)(first + t_base) * p.Hq + (long long)h * G + my_head, split) = make_float2(m_ref, l_run);
      }
#pragma unroll 1
      for (int c0 = 0; c0 < p.dv; c0 += CC) {
        uint32_t oc[CC];
        if (n_my > 0) {
#pragma unroll
          for (int c = 0; c < CC; c += 8) wt_ld8(tmem_o + lane_off + c0 + c, oc + c);
          asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
          wt_loaded<CC>(oc);
        }
        const bool some = n_my > 0 && l_run != 0.f;              // nothing seen: zeros
        __syncwarp();
#pragma unroll
        for (int c = 0; c < CC; ++c) o_s[lane * (CC + 1) + c] = some ? __uint_as_float(oc[c]) * f : 0.f;
        __syncwarp();
        const int n_c = min(CC, p.dv - c0);
        float* dst0 = first_dst() + c0 + lane;
        const int dst_row = PREFIX ? p.ws.dv4 : p.dv;
        if (drained) {
#pragma unroll 1
          for (int r = 0; r < r_n; r += 8) {
            float old[8][2];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
              const float* src = dst0 + (long long)__shfl_sync(0xffffffffu, my_head, r + u) * dst_row;
              old[u][0] = r + u < r_n && lane < n_c ? __ldcg(src) : 0.f;
              old[u][1] = r + u < r_n && lane + 32 < n_c ? __ldcg(src + 32) : 0.f;
            }
#pragma unroll
            for (int u = 0; u < 8; ++u) {
              const float wr = __shfl_sync(0xffffffffu, w * f, r + u);
              if (lane < n_c) o_s[(r + u) * (CC + 1) + lane] += old[u][0] * wr;
              if (lane + 32 < n_c) o_s[(r + u) * (CC + 1) + lane + 32] += old[u][1] * wr;
            }
          }
        }
#pragma unroll 4
        for (int r = 0; r < r_n; ++r) {
          if (!RAP_BOUNDS(first + row_t(r_first + r), p.rows, p.status, 0x308) || !RAP_BOUNDS(split, PREFIX ? p.ws.n_pre : 1, p.status, 0x309)) break;
          float* dst = dst0 + (long long)__shfl_sync(0xffffffffu, my_head, r) * dst_row;
          if (lane < n_c) dst[0] = o_s[r * (CC + 1) + lane];
          if (lane + 32 < n_c) dst[32] = o_s[r * (CC + 1) + lane + 32];
        }
      }
      asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    }
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (*abort_flag != 0 && tid == 0) win_report(p.status, RAP_ETIMEOUT, *abort_flag);
  if (warp == 8) {
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(512) : "memory");
  }
}

template <int DK, int NVP, bool LSUM, bool HALF, bool PREFIX>
rap_status launch_as(rap_ctx* ctx, const WtParams& p, int blocks, cudaStream_t st) {
  const int smem = WT_SMEM + 1024;
  RAP_CUDA_TRY(ctx, rap_raise_smem(ctx, win_tc_kernel<DK, NVP, LSUM, HALF, PREFIX>, smem));
  const dim3 grid(blocks, PREFIX ? 1 : p.Hkv);
  win_tc_kernel<DK, NVP, LSUM, HALF, PREFIX><<<grid, WT_THREADS, smem, st>>>(p);
  ctx->launches++;
  RAP_CUDA_TRY(ctx, cudaGetLastError());
  return RAP_OK;
}
template <int DK, int NVP, bool LSUM, bool PREFIX>
rap_status launch_wt(rap_ctx* ctx, const WtParams& p, int blocks, cudaStream_t st) {
  if constexpr (LSUM)
    if (p.dv & 1) return launch_as<DK, NVP, LSUM, true, PREFIX>(ctx, p, blocks, st);
  return launch_as<DK, NVP, LSUM, false, PREFIX>(ctx, p, blocks, st);     // 128 channels, the one width without LSUM, is even
}
template <bool PREFIX>
rap_status launch_any(rap_ctx* ctx, const WtParams& p, int blocks, cudaStream_t st) {
  // the steps and columns that the head needs, in four sizes; 128 channels leave no column for the row sums
  const int dk = (p.P2 + 15) / 16, nv = p.dv + 1;
  if (dk <= 4 && nv <= 80) return launch_wt<4, 80, true, PREFIX>(ctx, p, blocks, st);
  if (dk <= 6 && nv <= 96) return launch_wt<6, 96, true, PREFIX>(ctx, p, blocks, st);
  if (dk <= 7 && nv <= 112) return launch_wt<7, 112, true, PREFIX>(ctx, p, blocks, st);
  if (nv <= 128) return launch_wt<8, 128, true, PREFIX>(ctx, p, blocks, st);
  return launch_wt<8, 128, false, PREFIX>(ctx, p, blocks, st);
}

WtParams base_params(rap_ctx* ctx, const rap_win_args& a) {
  WtParams p = {};
  p.q = (const __nv_bfloat16*)a.q; p.out = a.out; p.status = ctx->d_status;
  p.rows = a.T; p.Hq = a.Hq; p.Hkv = a.Hkv; p.G = a.Hq / a.Hkv; p.P2 = a.P2; p.dv = a.dv;
  p.qscale = (float)(1.4426950408889634 / sqrt((double)a.head_dim));
  p.sms = ctx->sm_count;
  return p;
}

}  // namespace

bool rap_win_tc_takes(const rap_win_args& a) {
  return a.dtype == RAP_BF16 && a.P2 <= 128 && a.dv <= 128 && a.Hkv <= 65535 && (long long)a.T * (a.Hq / a.Hkv) < (1LL << 31) - 256;
}

rap_status rap_launch_win_tc(rap_ctx* ctx, const rap_win_args& a, cudaStream_t st) {
  WtParams p = base_params(ctx, a);
  p.k = (const __nv_bfloat16*)a.k; p.v = (const __nv_bfloat16*)a.v; p.start = a.row_start; p.len = a.seq_len; p.units = a.B;
  p.S_cap = a.S_cap; p.n_sink = a.n_sink; p.window = a.window;
  // row blocks of 256: as many as T rows can make, one more for each sequence that may begin a block
  const int seqs = a.B < a.T ? a.B : a.T;
  const int blocks = (int)((long long)a.T * p.G / 256) + seqs;
  return launch_any<false>(ctx, p, blocks, st);
}

// The prefixes' partials of rap_decode_attn_shared, *n_pre of them for each query head (0: the prefixes are empty)
rap_status rap_launch_win_prefix(rap_ctx* ctx, const rap_win_args& a, int* n_pre, cudaStream_t st) {
  *n_pre = 0;
  if (a.h_prefix_max == 0) return RAP_OK;
  WtParams p = base_params(ctx, a);
  p.k = (const __nv_bfloat16*)a.kp; p.v = (const __nv_bfloat16*)a.vp; p.start = a.group_start; p.len = a.prefix_len; p.units = a.n_groups;
  p.S_cap = a.S_pre; p.n_sink = 0; p.window = 0x7fffffff;
  // the device makes the plan (win_prefix_plan); here only how many CTAs it can come to
  const long long tiles = (a.h_prefix_max + WT_KT - 1) / WT_KT, groups = a.n_groups < a.B ? a.n_groups : a.B;
  const long long pieces = (long long)a.Hkv * (groups > 1 ? (long long)a.B * p.G / 256 + groups : ((long long)a.B * p.G + 255) / 256);
  const long long blocks = 2 * pieces <= ctx->sm_count ? ctx->sm_count : 4LL * ctx->sm_count + pieces;
  if (blocks > 0x7fffffffLL) return RAP_ESHAPE;
  *n_pre = (int)(tiles < WIN_MAX_PRE ? tiles : WIN_MAX_PRE);
  p.ws = win_partials(ctx->d_attn_ws, (long long)a.B * a.Hq, p.G, a.dv, *n_pre);
  return launch_any<true>(ctx, p, (int)blocks, st);
}
