// Split-KV decode scan over a cache held in 4 bits (rap_decode_attn_q4).  Same work plan, per-warp copy pipelines, lazy
// online softmax and fused merge as the other tensor-core scans; rows are 52 bytes where bf16 rows are 180, so the issue
// slots per row -- above all those of the integer pipe, which unpacks -- are what the design is about (mma.sync m16n8k16,
// fp16 in, fp32 accumulate):
//   * The cache is the A operand (16 rows, or 16 channels, on M), the query heads the B operand (8 columns): half the
//     padding of the other way round.
//   * A nibble under no exponent bits is an fp16 subnormal (c 2^-22 in bits 2..5, c 2^-18 in bits 6..9), so an operand
//     register of two codes is ONE mask of a shifted word: no exponent constant, no conversion, no offset to subtract.
//     Which code sits on which k-slot is free as long as both operands agree; on the K side the factor of 16 between the
//     two positions goes into q (exactly).  Row strides are compile-time constants, so every fragment load is one
//     instruction.
//   * S = K q: q enters in fp16, scaled per head by a power of two into fp16's range (a bf16 number keeps all its bits
//     down to 2^-28 of the head's largest).  A logit is s_K (sum q c - 7.5 sum q) + z_K sum q; the 7.5 sum q is the
//     initial value of the accumulator, the row's step and middle are applied to the accumulators in fp32.  Up to four
//     heads sit on the even columns, so that every lane ends up with one head of four rows and no logit twice.
//   * O += V p: the row's step goes into its weight, which enters as two fp16 numbers: its upper 8 bits and the rest
//     (19 bits together).  Up to four heads they are two columns of one MMA, beyond that two MMAs.  The tensor core aligns
//     the 16 products of a step by their exponents and cuts them off below, and a subnormal operand brings its leading
//     zeros along: hence the short first part, and all V codes in the highest position (output off by 7e-6 from bits 0..3,
//     9e-7 from bits 4..7).  The softmax reference is not the largest logit but the one that makes the largest weight,
//     its step included, 4 .. 8 (raised when one passes 2^15), so that steps of any magnitude stay inside fp16; a power of
//     two in every weight drops out of the quotient.  The middles are summed apart, in fp32.
//   * The codes 0..15 are 7.5 off centre, and a tensor core's running sum, which is cut off rather than rounded, must not
//     carry an offset that grows with the row: of every two rows that share an operand register the second enters with its
//     codes complemented (15 - c, the same mask operation) and its weight negated, so the offsets alternate in sign (output
//     off by 3e-4 at 32K rows without it).  What is left of them is 7.5 times the sum of the signed weights, which one MMA
//     against ones keeps along.  Every Q4_FLUSH blocks the accumulators move into fp32 sums in shared memory, which keeps
//     the cut-off of a long row's running sum below 1e-6 as well.
//   * Weights leave the first MMA with rows on M and enter the second with rows on K: one 8x8 transpose per 8 rows.
//   * Block row of tile row i (0..7) of half-tile t is 4 i + t: rows of an odd number of words then start on eight
//     banks, four apart, and all fragment and scale loads are free of conflicts.
//   * A tile (256 rows of K and of V, two bulk copies) is shared by the CTA's eight warps, 32 rows each; they take turns to
//     refill the stage of the tile before, once all are done with it (a ring per warp cost a quarter of all instructions).
//     Copies run on across units: batches of short sequences are chains of units, and a unit that one CTA scans alone is
//     written out directly.
// Rows past the end of a sequence get weight, step and middle zero by selection; their bytes may be anything.
// Every mbarrier wait is bounded: on timeout the CTA records RAP_ETIMEOUT and leaves.
#pragma once
#include <type_traits>

#include "rap_attn_common.cuh"
#include "rap_q4_common.cuh"

namespace {

constexpr float Q4_WEIGHT_MAX = 32768.f; // a weight (step included) above this raises the reference of its head
constexpr int Q4_BR = 32;                // rows per warp block
constexpr int Q4_MAX_STG = 8;            // stages of one tile each
constexpr int Q4_FLUSH = 16;             // blocks between two moves of the accumulators into shared memory
constexpr int Q4_OFF_MAIN = 896;         // barriers, merge scalars and flags below
constexpr int Q4_PAD = 64;               // the last row's fragment loads may reach one word past it

// KSW, VSW: words per K / V row (odd); GC: heads per lane (1: up to four heads, the two parts of a weight on neighbouring
// columns; 2: up to eight heads)
template <int KSW, int VSW, int GC>
struct Q4Cfg {
  static_assert(KSW % 2 == 1 && VSW % 2 == 1 && KSW <= 17 && VSW <= 17, "rows of up to 128 codes");
  static constexpr int NGK = (KSW + 2) / 4, NGV = (VSW + 2) / 4;      // groups of 4 words: 32 dims / channels
  static constexpr int NW = 8;                                    // warps per CTA (ten, at 96 registers, measured 8% slower)
  static constexpr int TILE = NW * Q4_BR;                             // rows per CTA tile
  static constexpr int NT = 2 * NGV;                                  // tiles of 16 channels
  static constexpr int CW = 32 * NGV;                                 // channel slots of the reduction buffer
  static constexpr int MAIN_F = 4 * GC * CW;                          // floats per warp: fp32 sums, then [4 GC][CW] for the merge
  static constexpr int STAGE_W = TILE * (KSW + VSW);               // words per stage
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

__device__ __forceinline__ void q4_mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// the same with other accumulators to start from
__device__ __forceinline__ void q4_mma_from(float (&d)[4], const float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                            uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %11, %12, %13};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(c[0]), "f"(c[1]), "f"(c[2]), "f"(c[3]));
}
// a value the compiler takes for unknown, so that it stays in its register instead of being made anew at every use
template <bool KEEP>
__device__ __forceinline__ uint32_t q4_keep(uint32_t x) {
  if constexpr (!KEEP) return x;
  uint32_t r;
  asm volatile("mov.b32 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}
__device__ __forceinline__ float q4_ex2(float x) {      // 2^x, one instruction; 2^(-inf) = 0
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t q4_pack(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ float q4_low(uint32_t h2) {
  float r;
  asm("{.reg .b16 l, h; mov.b32 {l, h}, %1; cvt.f32.f16 %0, l;}" : "=f"(r) : "r"(h2));
  return r;
}
__device__ __forceinline__ float q4_high(uint32_t h2) {
  float r;
  asm("{.reg .b16 l, h; mov.b32 {l, h}, %1; cvt.f32.f16 %0, h;}" : "=f"(r) : "r"(h2));
  return r;
}
__device__ __forceinline__ uint32_t q4_transpose(uint32_t x) {      // an 8x8 tile of 16-bit numbers across the warp
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}
__device__ __forceinline__ float q4_pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }      // -126 <= e <= 127
__device__ __forceinline__ int q4_exponent(float x) { return (int)((__float_as_uint(x) >> 23) & 255u) - 127; }
// two codes with the second row's complemented, (y ^ flip) & MASK with flip in a register: one instruction, where two
// immediates would make two
template <uint32_t MASK>
__device__ __forceinline__ uint32_t q4_pair(uint32_t y, uint32_t flip) {
  uint32_t r;
  asm("lop3.b32 %0, %1, %2, %3, 0x28;" : "=r"(r) : "r"(y), "r"(flip), "n"(MASK));
  return r;
}
__device__ __forceinline__ uint32_t q4_mul2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

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
    while (c > 0 && first_of(c) > s) --c;
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
  constexpr int NGK = C::NGK, NGV = C::NGV, NT = C::NT, CW = C::CW, MV = 2 * GC;      // MV: sums per lane and tile
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
      for (int i = tid; i < p.B * p.Hkv; i += THREADS) p.unit_cnt_other[i] = 0;   // counters a launch that gave up left behind
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

  // Fragment addressing inside a stage (words).  K: half-tile t, tile row gid: block row 4 gid + t, word 4 j + tq of group
  // j.  V: k-slots 2 tq, 2 tq + 1 of half-tile t: block rows 8 tq + t and 8 tq + 4 + t.
  const int k_blk = Q4_BR * warp * KSW, v_blk = C::TILE * KSW + Q4_BR * warp * VSW;      // this warp's block of a tile
  const int k_at = k_blk + 4 * gid * KSW + tq;
  const int v_at = v_blk + 8 * tq * VSW + gid;
  const int vh_at = 2 * (v_blk + 8 * tq * VSW) + 8 * (NGV - 1) + gid;     // half words: the last, odd group of 32
  const int ksz_at = k_blk + 4 * gid * KSW + KSW - 1, vsz_at = v_blk + 4 * gid * VSW + VSW - 1;
  const uint32_t row_sign = (gid & 1) ? 0x80000000u : 0u;      // rows 4 gid + t of odd gid are the second of their pair
  constexpr uint32_t LO = 0x000f000fu, HI = 0x00f000f0u, up = 0x64006400u;      // up: 2^10 twice
  const uint32_t flip0 = q4_keep<true>(0x000f0000u), flip4 = q4_keep<true>(0x00f00000u);
  constexpr bool KEEP = false;
  const uint32_t one0 = q4_keep<KEEP>(0x3c003c00u), one1 = q4_keep<KEEP>(0x3c003c00u), one2 = q4_keep<KEEP>(0x3c003c00u),
                 one3 = q4_keep<KEEP>(0x3c003c00u);
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
  // q of a unit as it is stored: column gid is head gid / 2 on even columns (GC = 1) or head gid (GC = 2), else zeros
  uint32_t w_q[NGK][4];
  auto load_q = [&]() {
    const int col_head = GC == 1 ? gid >> 1 : gid;
    const bool on = col_head < G && (GC == 2 || (gid & 1) == 0);
    const uint32_t* qrow = p.q + ((size_t)b * p.Hq + (size_t)h * G + (on ? col_head : 0)) * pp.P;
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
    // ---- q as the B operand.  Of word w = 4 j + tq of a row: k-slots 2 tq, 2 tq + 1 and 2 tq + 8, 2 tq + 9 hold dims 8 w + (0, 4) and (2, 6) in one
    // step, (1, 5) and (3, 7) in the next; a code counts 2^-24, 2^-22 and 2^-20, 2^-18 there, which q makes up for. ----
    uint32_t qa[NGK][2], qb[NGK][2];
    float off[4], f_q[GC], zq[GC], m_ref[GC], l_thr[GC], z_thr[GC];
    {
      float top = 0.f, sum = 0.f;
#pragma unroll
      for (int j = 0; j < NGK; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float x0 = __uint_as_float(w_q[j][i] << 16), x1 = __uint_as_float(w_q[j][i] & 0xffff0000u);
          top = fmaxf(top, fmaxf(fabsf(x0), fabsf(x1)));
          sum += x0 + x1;
        }
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
      const int e = min(max(8 - q4_exponent(top), -100), 120);        // the largest |q| 2^e lies in [2^8, 2^9)
      const float sc = q4_pow2(e);
      float seen = 0.f;            // sum of q 2^e as the MMAs see it
#pragma unroll
      for (int j = 0; j < NGK; ++j) {
        float x[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x[2 * i] = __uint_as_float(w_q[j][i] << 16) * sc;
          x[2 * i + 1] = __uint_as_float(w_q[j][i] & 0xffff0000u) * sc;
        }
        qa[j][0] = q4_pack(64.f * x[0], 64.f * x[4]);
        qa[j][1] = q4_pack(16.f * x[2], 16.f * x[6]);
        qb[j][0] = q4_pack(4.f * x[1], 4.f * x[5]);
        qb[j][1] = q4_pack(x[3], x[7]);
        seen += 0.015625f * (q4_low(qa[j][0]) + q4_high(qa[j][0])) + 0.0625f * (q4_low(qa[j][1]) + q4_high(qa[j][1])) +
                0.25f * (q4_low(qb[j][0]) + q4_high(qb[j][0])) + (q4_low(qb[j][1]) + q4_high(qb[j][1]));
      }
      seen += __shfl_xor_sync(0xffffffffu, seen, 1);
      seen += __shfl_xor_sync(0xffffffffu, seen, 2);
      sum += __shfl_xor_sync(0xffffffffu, sum, 1);
      sum += __shfl_xor_sync(0xffffffffu, sum, 2);
      // what the accumulator columns 2 tq, 2 tq + 1 need, from the lanes that hold those columns of q
      const float cs = p.qscale;   // log2(e) / sqrt(D)
      const float off_c = -7.5f * 0x1p-18f * seen, f_c = cs * q4_pow2(18 - e), z_c = cs * sum;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        off[i] = __shfl_sync(0xffffffffu, off_c, 4 * (2 * tq + i));
        off[2 + i] = __uint_as_float(q4_keep<KEEP>(__float_as_uint(off[i])));
      }
#pragma unroll
      for (int i = 0; i < GC; ++i) {
        f_q[i] = __shfl_sync(0xffffffffu, f_c, 4 * (2 * tq + i));
        zq[i] = __shfl_sync(0xffffffffu, z_c, 4 * (2 * tq + i));
        m_ref[i] = -INFINITY;
        l_thr[i] = z_thr[i] = 0.f;
      }
    }
    float o[NT][4], dsum[4];
#pragma unroll
    for (int t = 0; t < NT; ++t) o[t][0] = o[t][1] = o[t][2] = o[t][3] = 0.f;
    dsum[0] = dsum[1] = dsum[2] = dsum[3] = 0.f;
    bool have_main = false;      // the sums in shared memory hold something
    // the accumulators, less 7.5 per summed (signed) weight, plus what shared memory holds of them; channel rows gid (r = 0)
    // and gid + 8 (1) of tile t, in units of 2^-14 and 2^-20.  GC = 1: both columns belong to one head.
    auto total = [&](int t, int r, int g) {
      const float unit = r ? -7.5f * 0x1p-20f : -7.5f * 0x1p-14f;
      float v = GC == 1 ? fmaf(unit, dsum[0], o[t][2 * r]) + fmaf(unit, dsum[1], o[t][2 * r + 1]) : fmaf(unit, dsum[g], o[t][2 * r + g]);
      if (have_main) v += my_main[(t * 32 + lane) * MV + r * GC + g];
      return v;
    };

    // one block of 32 rows; TAIL: some of them (4 gid + t >= nrows) lie past the end
    auto block = [&](auto tail, const uint32_t* __restrict__ sw, int nrows, bool first) {
      constexpr bool TAIL = decltype(tail)::value;
      // ---- S = K q: two tiles of 16 rows, two steps of 16 dims per group ----
      float s[2][4];
#pragma unroll
      for (int mt = 0; mt < 2; ++mt) {
#pragma unroll
        for (int j = 0; j < NGK; ++j) {
          const uint32_t x0 = sw[k_at + 2 * mt * KSW + 4 * j], x1 = sw[k_at + (2 * mt + 1) * KSW + 4 * j];
          const uint32_t h0 = x0 >> 6, h1 = x1 >> 6;
          const uint32_t a0 = x0 & 0x000f000fu, a1 = x1 & 0x000f000fu, a2 = h0 & 0x003c003cu, a3 = h1 & 0x003c003cu;
          if (j == 0) q4_mma_from(s[mt], off, a0, a1, a2, a3, qa[j][0], qa[j][1]);
          else q4_mma(s[mt], a0, a1, a2, a3, qa[j][0], qa[j][1]);
          q4_mma(s[mt], x0 & 0x00f000f0u, x1 & 0x00f000f0u, h0 & 0x03c003c0u, h1 & 0x03c003c0u, qb[j][0], qb[j][1]);
        }
      }
      // ---- logits in base 2 less the reference maximum; weights times the (scaled, signed) V steps ----
      uint32_t ksz[4], vsz[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        ksz[t] = sw[ksz_at + t * KSW];
        vsz[t] = sw[vsz_at + t * VSW];
        if (TAIL && 4 * gid + t >= nrows) ksz[t] = vsz[t] = 0u;
      }
      float e[4][GC], w[4][GC];
      for (bool raised = false;; raised = true) {
        float big = 0.f;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const float ks = q4_step(ksz[t]), kz = q4_middle(ksz[t]);
          const float vs = __uint_as_float(vsz[t] * 65536u + row_sign);      // the step, negated on the second row of a pair
#pragma unroll
          for (int g = 0; g < GC; ++g) {
            float x = fmaf(ks * f_q[g], s[t >> 1][2 * (t & 1) + g], fmaf(kz, zq[g], -m_ref[g]));
            if (TAIL && 4 * gid + t >= nrows) x = -INFINITY;
            e[t][g] = q4_ex2(x);
            w[t][g] = e[t][g] * vs;
            big = q4_max(big, fabsf(w[t][g]));
          }
        }
        if (raised || !__any_sync(0xffffffffu, first || !(big <= Q4_WEIGHT_MAX))) break;
        // raise the references so that the block's largest weight (its step included) becomes 4 .. 8
#pragma unroll
        for (int g = 0; g < GC; ++g) {
          float x[4], mx = -3e38f, most = 0.f;
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            x[t] = fmaf(q4_step(ksz[t]) * f_q[g], s[t >> 1][2 * (t & 1) + g], q4_middle(ksz[t]) * zq[g]);
            if (TAIL && 4 * gid + t >= nrows) x[t] = -INFINITY;
            mx = fmaxf(mx, x[t]);
          }
#pragma unroll
          for (int d = 4; d < 32; d <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
#pragma unroll
          for (int t = 0; t < 4; ++t) most = fmaxf(most, q4_ex2(x[t] - mx) * q4_step(vsz[t]));
#pragma unroll
          for (int d = 4; d < 32; d <<= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, d));
          const float m_new = fmaxf(m_ref[g], mx + (most > 0.f ? (float)min(max(q4_exponent(most) - 2, -80), 100) : 0.f));
          const float alpha = q4_ex2(m_ref[g] - m_new);          // first block: 2^(-inf) = 0
          m_ref[g] = m_new;
          l_thr[g] *= alpha;
          z_thr[g] *= alpha;
          constexpr int c = GC == 1 ? 2 : 1;                     // columns of this head
#pragma unroll
          for (int t = 0; t < NT; ++t) {
#pragma unroll
            for (int i = 0; i < c; ++i) {
              o[t][g + i] *= alpha;
              o[t][2 + g + i] *= alpha;
            }
            if (have_main) {
              my_main[(t * 32 + lane) * MV + g] *= alpha;
              my_main[(t * 32 + lane) * MV + GC + g] *= alpha;
            }
          }
#pragma unroll
          for (int i = 0; i < c; ++i) dsum[g + i] *= alpha;
        }
      }
      // ---- row sums; the weights as fp16 pairs, turned into the B operand ----
      uint32_t pb[4], pl[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const float vz = q4_middle(vsz[t]);
        float top[GC], rest[GC];
#pragma unroll
        for (int g = 0; g < GC; ++g) {
          l_thr[g] += e[t][g];
          z_thr[g] = fmaf(e[t][g], vz, z_thr[g]);
          top[g] = __uint_as_float(__float_as_uint(w[t][g]) & 0xffff0000u);
          rest[g] = w[t][g] - top[g];
        }
        if constexpr (GC == 1) {
          pb[t] = q4_transpose(q4_pack(top[0], rest[0]));
          pl[t] = 0u;
        } else {
          pb[t] = q4_transpose(q4_pack(top[0], top[GC - 1]));
          pl[t] = q4_transpose(q4_pack(rest[0], rest[GC - 1]));
        }
      }
      // ---- O += V p: two steps of 16 rows, tiles of 16 channels ----
#pragma unroll
      for (int mt = 0; mt < 2; ++mt) {
        const uint32_t b0 = pb[2 * mt], b1 = pb[2 * mt + 1];
        [[maybe_unused]] const uint32_t c0 = pl[2 * mt], c1 = pl[2 * mt + 1];
        // four channels of 16 rows: y holds k-slots 2 tq, 2 tq + 1, z those + 8; codes 0 .. 3 go to rows gid and
        // gid + 8 of two tiles
        auto tiles = [&](float (&acc0)[4], float (&acc1)[4], uint32_t y, uint32_t z) {
          const uint32_t a0 = q4_mul2(q4_pair<LO>(y, flip0), up), a1 = q4_pair<HI>(y, flip4);
          const uint32_t a2 = q4_mul2(q4_pair<LO>(z, flip0), up), a3 = q4_pair<HI>(z, flip4);
          q4_mma(acc0, a0, a1, a2, a3, b0, b1);
          if constexpr (GC == 2) q4_mma(acc0, a0, a1, a2, a3, c0, c1);
          y >>= 8;
          z >>= 8;
          const uint32_t d0 = q4_mul2(q4_pair<LO>(y, flip0), up), d1 = q4_pair<HI>(y, flip4);
          const uint32_t d2 = q4_mul2(q4_pair<LO>(z, flip0), up), d3 = q4_pair<HI>(z, flip4);
          q4_mma(acc1, d0, d1, d2, d3, b0, b1);
          if constexpr (GC == 2) q4_mma(acc1, d0, d1, d2, d3, c0, c1);
        };
        q4_mma(dsum, one0, one1, one2, one3, b0, b1);
        if constexpr (GC == 2) q4_mma(dsum, one0, one1, one2, one3, c0, c1);
        const uint32_t* v0 = sw + v_at + 2 * mt * VSW;
#pragma unroll
        for (int u = 0; u < NGV / 2; ++u) {      // 64 channels: word 8 u + gid holds channels 64 u + 8 gid ..
          const uint32_t xa = v0[8 * u], xb = v0[8 * u + 4 * VSW], xc = v0[8 * u + VSW], xd = v0[8 * u + 5 * VSW];
          const uint32_t ya = __byte_perm(xa, xb, 0x5410), yb = __byte_perm(xa, xb, 0x7632);
          const uint32_t za = __byte_perm(xc, xd, 0x5410), zb = __byte_perm(xc, xd, 0x7632);
          tiles(o[4 * u], o[4 * u + 1], ya, za);
          tiles(o[4 * u + 2], o[4 * u + 3], yb, zb);
        }
        if constexpr (NGV % 2 == 1) {            // the last 32 channels: half word 8 (NGV - 1) + gid holds channels + 4 gid ..
          const uint16_t* vh = reinterpret_cast<const uint16_t*>(sw) + vh_at + 4 * mt * VSW;
          const uint32_t y = __byte_perm(vh[0], vh[8 * VSW], 0x5410), z = __byte_perm(vh[2 * VSW], vh[10 * VSW], 0x5410);
          tiles(o[NT - 2], o[NT - 1], y, z);
        }
      }
    };

    bool fresh = true;           // no row of this segment so far
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
      const int at = (int)(sw - reinterpret_cast<const uint32_t*>(smem));      // the largest offsets this lane reads
      in_ok = __all_sync(0xffffffffu, RAP_BOUNDS(at + k_at + 3 * KSW + 4 * NGK - 4, C::SMEM / 4, p.status, 0x406) &&
                                          RAP_BOUNDS(at + v_at + 7 * VSW + (NGV > 1 ? 8 * (NGV / 2 - 1) : 0), C::SMEM / 4, p.status, 0x405) &&
                                          RAP_BOUNDS(2 * at + vh_at + 14 * VSW, C::SMEM / 2, p.status, 0x407) &&
                                          RAP_BOUNDS(at + vsz_at + 3 * VSW, C::SMEM / 4, p.status, 0x408));
#endif
      if (in_ok && nrows > 0) {
        if (nrows >= Q4_BR) block(std::false_type{}, sw, nrows, fresh);
        else block(std::true_type{}, sw, nrows, fresh);
        fresh = false;
      }
      if ((i & (Q4_FLUSH - 1)) == Q4_FLUSH - 1) {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
          for (int r = 0; r < MV; ++r) my_main[(t * 32 + lane) * MV + r] = total(t, r / GC, r % GC);
          o[t][0] = o[t][1] = o[t][2] = o[t][3] = 0.f;
        }
        dsum[0] = dsum[1] = dsum[2] = dsum[3] = 0.f;
        have_main = true;
      }
      // this warp is done with the stage (its loads have been used)
      __syncwarp();
      if (lane == 0) mbar_arrive(bar0 + 8 * (Q4_MAX_STG + st));
      if (turn-- == 0) {       // the warps take turns to refill
        turn = NW - 1;
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
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      float v[MV];
#pragma unroll
      for (int r = 0; r < MV; ++r) v[r] = total(t, r / GC, r % GC);
#pragma unroll
      for (int r = 0; r < MV; ++r) o[t][r] = v[r];
    }
#pragma unroll
    for (int g = 0; g < GC; ++g)
#pragma unroll
      for (int d = 4; d < 32; d <<= 1) {
        l_thr[g] += __shfl_xor_sync(0xffffffffu, l_thr[g], d);
        z_thr[g] += __shfl_xor_sync(0xffffffffu, z_thr[g], d);
      }
    if (timed_out && lane == 0) *s_flag = 1;
    if (gid == 0) {
#pragma unroll
      for (int g = 0; g < GC; ++g) m_s[warp * 8 + GC * tq + g] = m_ref[g];
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
      const float f = m_ref[g] == -INFINITY ? 0.f : q4_ex2(m_ref[g] - m_all);   // a warp without a block contributes nothing
      if (gid == 0) l_s[warp * 8 + head] = l_thr[g] * f;
      if (head < G) {
        float* rr = my_main + head * CW;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          const bool wide = t < 4 * (NGV / 2);
          const int c = wide ? 64 * (t / 4) + 8 * gid + 2 * (t % 4) : 32 * (NGV - 1) + 4 * gid + 2 * (t % 2);
          rr[c] = fmaf(o[t][g], 0x1p14f, z_thr[g]) * f;
          rr[c + 1] = fmaf(o[t][GC + g], 0x1p20f, z_thr[g]) * f;
        }
      }
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
          for (int sg = 0; sg < nseg; ++sg) num += wgt[g * RAP_MAX_SPLIT + sg] * __ldcg(gb + (size_t)sg * (DV + 2));
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
