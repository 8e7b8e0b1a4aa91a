// What a warp does with 32 rows of a 4-bit cache (the scan around it: rap_attn_q4_kernel.cuh).  Two forms, by the number of
// query heads that share a KV head.  In both a lane owns rows 4 gid + t (t = 0 .. 3) of the block; K rows are the A operand of
// S = K q, V channels that of O += V p, the heads sit on the eight columns of B: half the padding of the other way round.
// Block row of tile row i of half-tile t is 4 i + t: rows of an odd number of words then start on eight banks, four apart, and
// all loads are free of conflicts.  Row strides are compile-time constants, so every load is one instruction.
//
// What bounds both is not the tensor cores (a third busy) but instruction issue and above all the integer pipe, which takes two
// cycles an instruction: at HBM speed a 32-row block of 90-wide rows has 480 cycles.
//
// Q4Whole, up to four heads: whole-number arithmetic (mma.sync m16n8k32, u8 x s8 and u8 x u8, s32 accumulate).  A stored byte is
// b = c + 16 c' for two neighbouring codes, and goes into the MMA as it is; one mask of a word gives the four c.  Hence
//   * logits: 16 (q c + q' c') = q' b + (16 q - q') c.  q is a whole number of 22 bits (scaled per head by a power of two), its two
//     coefficients four signed bytes each; digits 0 and 2 of a head sit on neighbouring columns of one MMA, 1 and 3 of another.
//     The offset -7.5 sum q is the accumulators' initial value.  Every product and sum is exact.
//   * outputs: sum p c from the masked bytes, sum p c' = (sum p b - sum p c) / 16.  A row's weight, its V step included, is a whole
//     number of 32 bits whose four bytes are the digits: the register of a lane's weight is already the pair of 16-bit columns
//     that the transpose wants.  The reference of the softmax makes the block's largest weight 2^27 .. 2^29 and is raised when
//     one passes 2^32.  Sums are exact, 7.5 sum p comes off in whole numbers too.  A weight's fraction (2^-27 of the largest, or
//     less) is cut at a point that moves by the golden section from block to block, so that equal weights far below the largest --
//     100,000 of 2^-26 beside one of 1 -- are right in the sum (rounded to nearest they were off together, by a quarter).
// A word of eight codes costs one mask on the K side and three byte permutes or masks on the V side, where fp16 operands cost
// five and eight (measured on 32 heads, 8 KV heads, 32K rows, batch 32: 158 us against 167).
//
// Q4Half, five to eight heads: the whole-number form would need twice the accumulators, 96 registers for rows of 90; on six warps of
// 168 registers it took 117 us for five heads over 4 sequences of up to 100K rows, this form 84.  fp16 in,
// fp32 accumulate (m16n8k16):
//   * A nibble under no exponent bits is an fp16 subnormal, so an operand register of two codes is one mask of a shifted word.
//     Which code sits on which k-slot is free as long as both operands agree; on the K side the factors between the positions go
//     into q (exactly), which is scaled per head by a power of two into fp16's range.
//   * A weight enters as two fp16 numbers, its upper 8 bits and the rest (19 bits together).  The tensor core aligns the products
//     of a step by their exponents and cuts them off below, and a subnormal operand brings its leading zeros along: hence the
//     short first part, and V codes of bits 0..3 scaled up (output off by 7e-6 from bits 0..3, 9e-7 from bits 4..7).
//   * The running sum is cut off rather than rounded, so it must not carry the codes' offset of 7.5, which grows with the row: of
//     every two rows that share an operand register the second enters with its codes complemented (15 - c, the same mask
//     operation) and its weight negated (off by 3e-4 at 32K rows without it).  What is left is 7.5 times the sum of the signed
//     weights, which one MMA against ones keeps along.  Every FLUSH blocks the accumulators move into fp32 sums in shared memory.
//   * The reference makes the largest weight 2^9 .. 2^11 (fp16 ends 33 places below that), raised when one passes 2^15.
// The middles are summed apart in fp32; a power of two in every weight drops out of the quotient.  Rows past the end get weight,
// step and middle zero by selection (TAIL); their bytes may be anything.
//
// In both the reference is bounded by the sums of exponentials and of exponentials times middle too, not by the weights alone: rows
// without a step (constant rows) weigh nothing, however far their logits lie above the reference.  A block in which a lane's sums pass
// 2^104 raises it so that they fall below 2^103, which leaves 2^25 rows room in fp32.  (Up to four heads the bound costs nothing
// that can be measured, from five on 3%: 82 us became 84.)
// It only ever rises, so a block without a step sets it as low as those sums allow, 97 places below its largest logit: any block with
// steps that counts beside it then finds its weights too large, not too small.  References are whole numbers, and scaling from one to
// another is exact: two may lie 200 places apart where their rows count alike (zero rows beside V of 1e20).  For the same reason every
// warp's sums are scaled before the merge so that its row sum lies in [1, 2).
#pragma once
#include <type_traits>

#include "rap_attn_common.cuh"
#include "rap_q4_common.cuh"

namespace {

constexpr int Q4_BR = 32;                // rows per warp block
constexpr float Q4_SUM_MAX = 0x1p104f;   // of a lane's exponentials and of their products with the middles, in a block
constexpr int Q4_SUM_TOP = 97;           // exponent that a raise leaves the largest of either

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
__device__ __forceinline__ uint32_t q4_keep(uint32_t x) {
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
// 2^d of a whole number d <= 0; 0 below 2^-149, for -inf and for a NaN
__device__ __forceinline__ float q4_down(float d) {
  return d >= -149.f ? __uint_as_float(d >= -126.f ? (uint32_t)((int)d + 127) << 23 : 1u << ((int)d + 149)) : 0.f;
}
// Scales a row sum and a middles' sum by 2^d; returns the factor for the sums of weights.  (Where 2^d is no fp32 number no sum of
// weights counts any longer beside the new block's, but sums of exponentials may: in two factors.)
__device__ __forceinline__ float q4_lower(float d, float& l, float& z) {
  const float f = q4_down(d);
  if (f == 0.f && d >= -252.f) {
    const float rest = q4_down(d + 126.f);
    l = l * 0x1p-126f * rest;
    z = z * 0x1p-126f * rest;
  } else {
    l *= f;
    z *= f;
  }
  return f;
}
// How far above a row's logit the reference has to lie, given the row's last word: so that the weight times the step stays below
// 2^(want + 2), and the sums below Q4_SUM_TOP.  From the exponents alone, since the row may weigh nothing beside another one (its 2^x
// relative to the largest underflows) and yet be the one whose step matters.  (A step or a middle of 0 counts as 2^-127.)
__device__ __forceinline__ float q4_lift(uint32_t sz, int want) {
  const int step = (int)((sz >> 7) & 255u) - 127, middle = (int)((sz >> 23) & 255u) - 127;
  return (float)max(step - want, max(middle, 0) - Q4_SUM_TOP);
}
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
// whole-number MMAs: codes (u8) by digits of q (s8) or of a weight (u8)
__device__ __forceinline__ void q4_imma_from(int (&d)[4], const int (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                             uint32_t b1) {
  asm("mma.sync.aligned.m16n8k32.row.col.s32.u8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %11, %12, %13};"
      : "=r"(d[0]), "=r"(d[1]), "=r"(d[2]), "=r"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "r"(c[0]), "r"(c[1]), "r"(c[2]), "r"(c[3]));
}
__device__ __forceinline__ void q4_imma_from(int (&d)[4], const int (&c)[4], uint32_t a0, uint32_t a1, uint32_t b0) {
  asm("mma.sync.aligned.m16n8k16.row.col.s32.u8.s8.s32 {%0, %1, %2, %3}, {%4, %5}, {%6}, {%7, %8, %9, %10};"
      : "=r"(d[0]), "=r"(d[1]), "=r"(d[2]), "=r"(d[3])
      : "r"(a0), "r"(a1), "r"(b0), "r"(c[0]), "r"(c[1]), "r"(c[2]), "r"(c[3]));
}
__device__ __forceinline__ void q4_imma_u(int (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k32.row.col.s32.u8.u8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Where a lane reads: words from the start of a tile's stage.  K: half-tile t, tile row gid, word 4 j + tq of group j.  V: k-slots of
// a lane are block rows 8 tq + t and 8 tq + 4 + t.
template <int KSW, int VSW>
struct Q4At {
  static constexpr int NGK = (KSW + 2) / 4, NGV = (VSW + 2) / 4;      // groups of 4 words: 32 dims / channels
  int k, v, vh, ksz, vsz;
  __device__ __forceinline__ void place(int tile_rows, int warp, int gid, int tq) {
    const int k_blk = Q4_BR * warp * KSW, v_blk = tile_rows * KSW + Q4_BR * warp * VSW;
    k = k_blk + 4 * gid * KSW + tq;
    v = v_blk + 8 * tq * VSW + gid;                                   // word 8 u + gid of a row: channels 64 u + 8 gid ..
    vh = 2 * (v_blk + 8 * tq * VSW) + 8 * (NGV - 1) + gid;            // half words: the last, odd group of 32
    ksz = k_blk + 4 * gid * KSW + KSW - 1;                            // steps and middles
    vsz = v_blk + 4 * gid * VSW + VSW - 1;
  }
  // the largest offsets that a lane reads, in words (index checks of the bounds-checking build)
  __device__ __forceinline__ int reach() const {
    return max(max(k + 3 * KSW + 4 * NGK - 4, vsz + 3 * VSW), max(v + 7 * VSW + (NGV > 1 ? 8 * (NGV / 2 - 1) : 0), (vh + 14 * VSW) / 2));
  }
};

// ---- up to four heads ----------------------------------------------------------------------------------------------------
template <int KSW, int VSW>
struct Q4Whole {
  using At = Q4At<KSW, VSW>;
  static constexpr int NGK = At::NGK, NGV = At::NGV, HPL = 1;         // heads per lane
  static constexpr int SUMS = 4 * NGV;                                // fp32 sums per lane: 4 channels of each of NGV tiles
  static constexpr int FLUSH = 512;                                   // blocks: 255 * 255 * 32 * 512 < 2^31
  static constexpr uint32_t LOW = 0x0f0f0f0fu;
  static constexpr float LIMIT = 4294967040.f;                        // rounds to less than 2^32
  int gid, tq, lane;
  At at;
  uint32_t qd[NGK][4];         // B operands of word group j: digits (0 | 2) and (1 | 3) of the bytes' coefficient, then of the codes'
  int off[4], zero[4];         // -120 sum q as 2^16 off[1] + off[0], on both tile halves
  int acc[NGV][2][2][4];       // [tile][bytes, codes][digits 0 and 2, 1 and 3][row gid: two columns, row gid + 8: two columns]
  uint32_t s_even, s_odd;      // sums of the weights' digits: column gid, this lane's rows
  float f_q, zq, m_ref[1], l_thr[1], z_thr[1], l_part, z_part;      // l, z: sums of the weights, and with the middles; see settle
  float limit;                 // of a weight: above it the reference is raised; 0: flush at the next block
  float point;                 // where a weight's fraction is cut: up from 1 - point on
  bool have, dirty;            // shared memory / the accumulators hold something

  __device__ __forceinline__ static int q_head(int gid) { return gid >> 1; }
  __device__ __forceinline__ static bool q_on(int gid, int G) { return (gid >> 1) < G; }

  __device__ __forceinline__ void begin(const uint32_t (&w)[NGK][4], float cs) {
    float top = 0.f, sum = 0.f;
#pragma unroll
    for (int j = 0; j < NGK; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float x0 = __uint_as_float(w[j][i] << 16), x1 = __uint_as_float(w[j][i] & 0xffff0000u);
        top = fmaxf(top, fmaxf(fabsf(x0), fabsf(x1)));
        sum += x0 + x1;
      }
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
    const int e = min(21 - q4_exponent(top), 120);                    // the largest |q| 2^e lies in [2^21, 2^22)
    const float sc = q4_pow2(e);
    int total = 0;
    const uint32_t mine = (gid & 1) ? 0x7362u : 0x5140u;              // this column's two digits of four, of two numbers
#pragma unroll
    for (int j = 0; j < NGK; ++j) {
      uint32_t x[2][4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int qe = __float2int_rn(__uint_as_float(w[j][i] << 16) * sc), qo = __float2int_rn(__uint_as_float(w[j][i] & 0xffff0000u) * sc);
        total += qe + qo;
        // balanced digits -128 .. 127 of a number: the bytes of (x + 0x80808080) less 128 each
        x[0][i] = (uint32_t)qo + 0x80808080u;
        x[1][i] = (uint32_t)(16 * qe - qo) + 0x80808080u;
      }
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const uint32_t y = __byte_perm(x[k][0], x[k][1], mine), z = __byte_perm(x[k][2], x[k][3], mine);
        qd[j][2 * k] = __byte_perm(y, z, 0x5410) ^ 0x80808080u;
        qd[j][2 * k + 1] = __byte_perm(y, z, 0x7632) ^ 0x80808080u;
      }
    }
#pragma unroll
    for (int o = 1; o < 4; o <<= 1) {
      total += __shfl_xor_sync(0xffffffffu, total, o);
      sum += __shfl_xor_sync(0xffffffffu, sum, o);
    }
    sum = fmaf(top, 0.f, sum);                                        // an infinity in q makes its head's outputs NaN
    const long long offset = -120LL * total;                          // |total| < 2^29
    const int high = (int)((offset + 32768) >> 16), low = (int)(offset - ((long long)high << 16));
    const int from = 8 * tq;                                          // a lane that holds this lane's head
    off[0] = off[2] = __shfl_sync(0xffffffffu, low, from);
    off[1] = off[3] = __shfl_sync(0xffffffffu, high, from);
    f_q = __shfl_sync(0xffffffffu, cs * q4_pow2(-4 - e), from);
    zq = __shfl_sync(0xffffffffu, cs * sum, from);
    zero[0] = zero[1] = zero[2] = zero[3] = 0;
    m_ref[0] = -INFINITY;
    l_thr[0] = z_thr[0] = l_part = z_part = 0.f;
    clear();
    have = dirty = false;
    limit = LIMIT;
    point = 0.125f * gid;
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int t = 0; t < NGV; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[t][i >> 3][(i >> 2) & 1][i & 3] = 0;
    s_even = s_odd = 0u;
  }
  // the accumulators as numbers, 7.5 per summed weight taken off, plus what shared memory holds; channels 0 .. 3 of tile t
  __device__ __forceinline__ void total(float* sums, float (&v)[NGV][4]) {
    uint32_t e = s_even, o = s_odd;
#pragma unroll
    for (int d = 1; d < 4; d <<= 1) {
      e += __shfl_xor_sync(0xffffffffu, e, d);
      o += __shfl_xor_sync(0xffffffffu, o, d);
    }
    const int s[4] = {(int)__shfl_sync(0xffffffffu, e, 8 * tq), (int)__shfl_sync(0xffffffffu, o, 8 * tq),
                      (int)__shfl_sync(0xffffffffu, e, 8 * tq + 4), (int)__shfl_sync(0xffffffffu, o, 8 * tq + 4)};
#pragma unroll
    for (int t = 0; t < NGV; ++t) {
      float4 was = make_float4(0.f, 0.f, 0.f, 0.f);
      if (have) was = reinterpret_cast<const float4*>(sums)[t * 32 + lane];
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        float x = 0.f, y = 0.f;
#pragma unroll
        for (int d = 3; d >= 0; --d) {
          const int b = acc[t][0][d & 1][2 * r + (d >> 1)], c = acc[t][1][d & 1][2 * r + (d >> 1)];
          x = fmaf(x, 256.f, (float)(2 * c - 15 * s[d]));
          y = fmaf(y, 256.f, (float)(b - c - 120 * s[d]));
        }
        v[t][2 * r] = fmaf(x, 0.5f, r ? was.z : was.x);
        v[t][2 * r + 1] = fmaf(y, 0.0625f, r ? was.w : was.y);
      }
    }
  }
  // the sums of the last blocks to those of all (called every few blocks: fewer additions to a number that one large weight has
  // made large)
  __device__ __forceinline__ void settle() {
    l_thr[0] += l_part;
    z_thr[0] += z_part;
    l_part = z_part = 0.f;
  }
  __device__ __forceinline__ void flush(float*) { limit = 0.f; }      // (done by the next block: one copy of the code)

  struct Rows {                // of the lane's four rows
    float s[4], w[4], big;                                            // 16 sum q (c - 7.5), weights times V step, their maximum
    float l, z;                                                       // sums of the weights, and with the middles
    uint32_t ksz[4], vsz[4];
  };
  template <bool TAIL>
  __device__ __forceinline__ void weigh(const uint32_t* __restrict__ sw, int nrows, Rows& r) {
    // ---- logits: two tiles of 16 rows, 64 dims a step ----
#pragma unroll
    for (int mt = 0; mt < 2; ++mt) {
      const uint32_t* x = sw + at.k + 2 * mt * KSW;
      int even[4], odd[4];
#pragma unroll
      for (int j = 0; j < NGK; j += 2) {
        const int (&from_e)[4] = j == 0 ? off : even;
        const int (&from_o)[4] = j == 0 ? zero : odd;
        const uint32_t a0 = x[4 * j], a1 = x[KSW + 4 * j];
        if (j + 1 < NGK) {
          const uint32_t a2 = x[4 * j + 4], a3 = x[KSW + 4 * j + 4];
          const uint32_t c0 = a0 & LOW, c1 = a1 & LOW, c2 = a2 & LOW, c3 = a3 & LOW;
          const int k = j + 1 < NGK ? j + 1 : j;
          q4_imma_from(even, from_e, a0, a1, a2, a3, qd[j][0], qd[k][0]);
          q4_imma_from(odd, from_o, a0, a1, a2, a3, qd[j][1], qd[k][1]);
          q4_imma_from(even, even, c0, c1, c2, c3, qd[j][2], qd[k][2]);
          q4_imma_from(odd, odd, c0, c1, c2, c3, qd[j][3], qd[k][3]);
        } else {
          const uint32_t c0 = a0 & LOW, c1 = a1 & LOW;
          q4_imma_from(even, from_e, a0, a1, qd[j][0]);
          q4_imma_from(odd, from_o, a0, a1, qd[j][1]);
          q4_imma_from(even, even, c0, c1, qd[j][2]);
          q4_imma_from(odd, odd, c0, c1, qd[j][3]);
        }
      }
#pragma unroll
      for (int i = 0; i < 2; ++i)      // digits 3 .. 0
        r.s[2 * mt + i] = fmaf((float)(odd[2 * i + 1] * 256 + even[2 * i + 1]), 65536.f, (float)(odd[2 * i] * 256 + even[2 * i]));
    }
    // ---- weights ----
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      r.ksz[t] = sw[at.ksz + t * KSW];
      r.vsz[t] = sw[at.vsz + t * VSW];
      if (TAIL && 4 * gid + t >= nrows) r.ksz[t] = r.vsz[t] = 0u;
    }
    weights(r, TAIL ? nrows : Q4_BR);
  }
  __device__ __forceinline__ void weights(Rows& r, int nrows) {
    r.big = 0.f;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      float x = fmaf(q4_step(r.ksz[t]) * f_q, r.s[t], fmaf(q4_middle(r.ksz[t]), zq, -m_ref[0]));
      if (4 * gid + t >= nrows) x = -INFINITY;
      const float e = q4_ex2(x);
      r.w[t] = e * q4_step(r.vsz[t]);
      r.big = q4_max(r.big, r.w[t]);
      r.l = t ? r.l + e : e;
      r.z = t ? fmaf(e, q4_middle(r.vsz[t]), r.z) : e * q4_middle(r.vsz[t]);
    }
  }
  // raise the reference so that the block's largest weight (its step included) becomes 2^27 .. 2^29, or as far as the sums ask
  // for; what is summed so far moves to shared memory, scaled
  __device__ __forceinline__ void raise(Rows& r, int nrows, float* sums) {
    float top = -3e38f;
#pragma unroll
    for (int t = 0; t < 4; ++t)
      if (4 * gid + t < nrows)
        top = fmaxf(top, fmaf(q4_step(r.ksz[t]) * f_q, r.s[t], q4_middle(r.ksz[t]) * zq) + q4_lift(r.vsz[t], 27));
#pragma unroll
    for (int d = 4; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
    const float m_old = m_ref[0], m_new = fmaxf(m_old, floorf(top));
    m_ref[0] = m_new;
    settle();
    const float alpha = q4_lower(m_old - m_new, l_thr[0], z_thr[0]);      // first block: 2^(-inf) = 0
    if (dirty) {
      float v[NGV][4];
      total(sums, v);
#pragma unroll
      for (int t = 0; t < NGV; ++t)
        reinterpret_cast<float4*>(sums)[t * 32 + lane] = make_float4(v[t][0] * alpha, v[t][1] * alpha, v[t][2] * alpha, v[t][3] * alpha);
      clear();
      have = true;
      dirty = false;
    }
    limit = LIMIT;
    weights(r, nrows);
  }

  __device__ __forceinline__ void block(const uint32_t* __restrict__ sw, int nrows, float* sums) {
    Rows r;
    if (nrows >= Q4_BR) weigh<false>(sw, nrows, r);
    else weigh<true>(sw, nrows, r);
    // (a first block's reference is -inf)
    if (__any_sync(0xffffffffu, !(r.big < limit) || !(r.l + fabsf(r.z) < Q4_SUM_MAX))) raise(r, nrows, sums);
    // ---- row sums; the weights' digits, turned into the B operand: k-slots 4 tq .. are rows 8 tq + t, 8 tq + 4 + t of t = 0, 1 (2, 3) ----
    l_part += r.l;
    z_part += r.z;
    uint32_t p[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) p[t] = q4_transpose(__float2uint_rz(r.w[t] + point));
    point += 0.618034f;
    if (point >= 1.f) point -= 1.f;
    const uint32_t e0 = __byte_perm(p[0], p[1], 0x6420), e1 = __byte_perm(p[2], p[3], 0x6420);
    const uint32_t o0 = __byte_perm(p[0], p[1], 0x7531), o1 = __byte_perm(p[2], p[3], 0x7531);
    s_even = __dp4a(e0, 0x01010101u, __dp4a(e1, 0x01010101u, s_even));
    s_odd = __dp4a(o0, 0x01010101u, __dp4a(o1, 0x01010101u, s_odd));
    dirty = true;
    // ---- sums of the bytes and of their lower codes ----
    auto tile = [&](int (&c)[2][2][4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3) {
      q4_imma_u(c[0][0], a0, a1, a2, a3, e0, e1);
      q4_imma_u(c[0][1], a0, a1, a2, a3, o0, o1);
      const uint32_t d0 = a0 & LOW, d1 = a1 & LOW, d2 = a2 & LOW, d3 = a3 & LOW;
      q4_imma_u(c[1][0], d0, d1, d2, d3, e0, e1);
      q4_imma_u(c[1][1], d0, d1, d2, d3, o0, o1);
    };
    const uint32_t* v0 = sw + at.v;
#pragma unroll
    for (int u = 0; u < NGV / 2; ++u) {        // 64 channels: four bytes of a word, transposed over four rows
      uint32_t b[2][4];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const uint32_t* y = v0 + 8 * u + 2 * k * VSW;
        const uint32_t xa = y[0], xb = y[4 * VSW], xc = y[VSW], xd = y[5 * VSW];
        const uint32_t f = __byte_perm(xa, xb, 0x5140), g = __byte_perm(xa, xb, 0x7362);
        const uint32_t h = __byte_perm(xc, xd, 0x5140), i = __byte_perm(xc, xd, 0x7362);
        b[k][0] = __byte_perm(f, h, 0x5410);
        b[k][1] = __byte_perm(f, h, 0x7632);
        b[k][2] = __byte_perm(g, i, 0x5410);
        b[k][3] = __byte_perm(g, i, 0x7632);
      }
      tile(acc[2 * u], b[0][0], b[0][1], b[1][0], b[1][1]);
      tile(acc[2 * u + 1], b[0][2], b[0][3], b[1][2], b[1][3]);
    }
    if constexpr (NGV % 2 == 1) {              // the last 32: two bytes of a half word
      const uint16_t* vh = reinterpret_cast<const uint16_t*>(sw) + at.vh;
      uint32_t b[2][2];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const uint16_t* y = vh + 4 * k * VSW;
        const uint32_t f = __byte_perm(y[0], y[8 * VSW], 0x5140), g = __byte_perm(y[2 * VSW], y[10 * VSW], 0x5140);
        b[k][0] = __byte_perm(f, g, 0x5410);
        b[k][1] = __byte_perm(f, g, 0x7632);
      }
      tile(acc[NGV - 1], b[0][0], b[0][1], b[1][0], b[1][1]);
    }
  }

  // scaled sums of head g of this lane to the merge buffer (which may lie where `sums` does)
  float out[NGV][4];
  __device__ __forceinline__ void finish(float* sums) {
    settle();
    total(sums, out);
  }
  __device__ __forceinline__ void put(float* rr, int, float f) const {
#pragma unroll
    for (int t = 0; t < NGV; ++t) {
      const int c = t < 2 * (NGV / 2) ? 64 * (t / 2) + 8 * gid + 4 * (t % 2) : 32 * (NGV - 1) + 4 * gid;
#pragma unroll
      for (int i = 0; i < 4; ++i) rr[c + i] = (out[t][i] + z_thr[0]) * f;
    }
  }
};

// ---- five to eight heads -----------------------------------------------------------------------------------------------------
template <int KSW, int VSW>
struct Q4Half {
  using At = Q4At<KSW, VSW>;
  static constexpr int NGK = At::NGK, NGV = At::NGV, HPL = 2;
  static constexpr int NT = 2 * NGV;                                  // tiles of 16 channels
  static constexpr int SUMS = 4 * NT;
  static constexpr int FLUSH = 16;
  static constexpr float WEIGHT_MAX = 32768.f;
  static constexpr uint32_t LO = 0x000f000fu, HI = 0x00f000f0u, UP = 0x64006400u;      // UP: 2^10 twice
  int gid, tq, lane;
  At at;
  uint32_t qa[NGK][2], qb[NGK][2];
  float off[4], f_q[2], zq[2], m_ref[2], l_thr[2], z_thr[2];
  q4_f2 l_part, z_part;        // sums of the last blocks, both heads
  float o[NT][4], dsum[4];     // columns 2 tq, 2 tq + 1 are this lane's heads
  uint32_t flip0, flip4, row_sign;
  bool have;

  __device__ __forceinline__ static int q_head(int gid) { return gid; }
  __device__ __forceinline__ static bool q_on(int gid, int G) { return gid < G; }

  // Of word w = 4 j + tq of a row: k-slots 2 tq, 2 tq + 1 and 2 tq + 8, 2 tq + 9 hold dims 8 w + (0, 4) and (2, 6) in one step,
  // (1, 5) and (3, 7) in the next; a code counts 2^-24, 2^-22 and 2^-20, 2^-18 there, which q makes up for.
  __device__ __forceinline__ void begin(const uint32_t (&w)[NGK][4], float cs) {
    float top = 0.f, sum = 0.f;
#pragma unroll
    for (int j = 0; j < NGK; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float x0 = __uint_as_float(w[j][i] << 16), x1 = __uint_as_float(w[j][i] & 0xffff0000u);
        top = fmaxf(top, fmaxf(fabsf(x0), fabsf(x1)));
        sum += x0 + x1;
      }
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
    const int e = min(max(8 - q4_exponent(top), -109), 120);          // the largest |q| 2^e lies in [2^8, 2^9)
    const float sc = q4_pow2(e);
    float seen = 0.f;            // sum of q 2^e as the MMAs see it
#pragma unroll
    for (int j = 0; j < NGK; ++j) {
      float x[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[j][i] << 16) * sc;
        x[2 * i + 1] = __uint_as_float(w[j][i] & 0xffff0000u) * sc;
      }
      qa[j][0] = q4_pack(64.f * x[0], 64.f * x[4]);
      qa[j][1] = q4_pack(16.f * x[2], 16.f * x[6]);
      qb[j][0] = q4_pack(4.f * x[1], 4.f * x[5]);
      qb[j][1] = q4_pack(x[3], x[7]);
      seen += 0.015625f * (q4_low(qa[j][0]) + q4_high(qa[j][0])) + 0.0625f * (q4_low(qa[j][1]) + q4_high(qa[j][1])) +
              0.25f * (q4_low(qb[j][0]) + q4_high(qb[j][0])) + (q4_low(qb[j][1]) + q4_high(qb[j][1]));
    }
#pragma unroll
    for (int d = 1; d < 4; d <<= 1) {
      seen += __shfl_xor_sync(0xffffffffu, seen, d);
      sum += __shfl_xor_sync(0xffffffffu, sum, d);
    }
    sum = fmaf(top, 0.f, sum);   // an infinity in q makes its head's outputs NaN
    // what the accumulator columns 2 tq, 2 tq + 1 need, from the lanes that hold those columns of q
    const float off_c = -7.5f * 0x1p-18f * seen, f_c = cs * q4_pow2(18 - e), z_c = cs * sum;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      off[i] = off[2 + i] = __shfl_sync(0xffffffffu, off_c, 4 * (2 * tq + i));
      f_q[i] = __shfl_sync(0xffffffffu, f_c, 4 * (2 * tq + i));
      zq[i] = __shfl_sync(0xffffffffu, z_c, 4 * (2 * tq + i));
      m_ref[i] = -INFINITY;
      l_thr[i] = z_thr[i] = 0.f;
    }
    l_part = z_part = 0ull;
    flip0 = q4_keep(0x000f0000u);
    flip4 = q4_keep(0x00f00000u);
    row_sign = (gid & 1) ? 0x80000000u : 0u;      // rows 4 gid + t of odd gid are the second of their pair
    clear();
    have = false;
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int t = 0; t < NT; ++t) o[t][0] = o[t][1] = o[t][2] = o[t][3] = 0.f;
    dsum[0] = dsum[1] = dsum[2] = dsum[3] = 0.f;
  }
  // the accumulators, less 7.5 per summed (signed) weight, plus what shared memory holds: channel rows gid (heads 2 tq, 2 tq + 1) and
  // gid + 8 of tile t, in units of 2^-14 and 2^-20
  __device__ __forceinline__ void total(float* sums) {
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      float4 was = make_float4(0.f, 0.f, 0.f, 0.f);
      if (have) was = reinterpret_cast<const float4*>(sums)[t * 32 + lane];
      o[t][0] = fmaf(-7.5f * 0x1p-14f, dsum[0], o[t][0]) + was.x;
      o[t][1] = fmaf(-7.5f * 0x1p-14f, dsum[1], o[t][1]) + was.y;
      o[t][2] = fmaf(-7.5f * 0x1p-20f, dsum[0], o[t][2]) + was.z;
      o[t][3] = fmaf(-7.5f * 0x1p-20f, dsum[1], o[t][3]) + was.w;
    }
  }
  __device__ __forceinline__ void settle() {
    float a, b;
    q4_apart(l_part, a, b);
    l_thr[0] += a;
    l_thr[1] += b;
    q4_apart(z_part, a, b);
    z_thr[0] += a;
    z_thr[1] += b;
    l_part = z_part = 0ull;
  }
  __device__ __forceinline__ void flush(float* sums) {
    total(sums);
#pragma unroll
    for (int t = 0; t < NT; ++t) reinterpret_cast<float4*>(sums)[t * 32 + lane] = make_float4(o[t][0], o[t][1], o[t][2], o[t][3]);
    clear();
    have = true;
  }

  struct Rows {                // of the lane's four rows, each for two heads
    float s[2][4], w[4][2], big;
    q4_f2 l, z;                // sums of the weights, and with the middles
    uint32_t ksz[4], vsz[4];
  };
  template <bool TAIL>
  __device__ __forceinline__ void weigh(const uint32_t* __restrict__ sw, int nrows, Rows& r) {
    // ---- S = K q: two tiles of 16 rows, two steps of 16 dims per group ----
#pragma unroll
    for (int mt = 0; mt < 2; ++mt) {
#pragma unroll
      for (int j = 0; j < NGK; ++j) {
        const uint32_t x0 = sw[at.k + 2 * mt * KSW + 4 * j], x1 = sw[at.k + (2 * mt + 1) * KSW + 4 * j];
        const uint32_t h0 = x0 >> 6, h1 = x1 >> 6;
        const uint32_t a0 = x0 & 0x000f000fu, a1 = x1 & 0x000f000fu, a2 = h0 & 0x003c003cu, a3 = h1 & 0x003c003cu;
        if (j == 0) q4_mma_from(r.s[mt], off, a0, a1, a2, a3, qa[j][0], qa[j][1]);
        else q4_mma(r.s[mt], a0, a1, a2, a3, qa[j][0], qa[j][1]);
        q4_mma(r.s[mt], x0 & 0x00f000f0u, x1 & 0x00f000f0u, h0 & 0x03c003c0u, h1 & 0x03c003c0u, qb[j][0], qb[j][1]);
      }
    }
    // ---- weights ----
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      r.ksz[t] = sw[at.ksz + t * KSW];
      r.vsz[t] = sw[at.vsz + t * VSW];
      if (TAIL && 4 * gid + t >= nrows) r.ksz[t] = r.vsz[t] = 0u;
    }
    weights(r, TAIL ? nrows : Q4_BR);
  }
  __device__ __forceinline__ void weights(Rows& r, int nrows) {
    r.big = 0.f;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const float ks = q4_step(r.ksz[t]), kz = q4_middle(r.ksz[t]);
      const float vs = __uint_as_float(r.vsz[t] * 65536u + row_sign);      // the step, negated on the second row of a pair
      float x[2];                // (both heads in one instruction each)
      q4_apart(q4_fma(q4_mul(q4_two(ks, ks), q4_two(f_q[0], f_q[1])), q4_two(r.s[t >> 1][2 * (t & 1)], r.s[t >> 1][2 * (t & 1) + 1]),
                      q4_fma(q4_two(kz, kz), q4_two(zq[0], zq[1]), q4_two(-m_ref[0], -m_ref[1]))), x[0], x[1]);
#pragma unroll
      for (int g = 0; g < 2; ++g) x[g] = q4_ex2(4 * gid + t < nrows ? x[g] : -INFINITY);
      const q4_f2 e = q4_two(x[0], x[1]);
      const float vz = q4_middle(r.vsz[t]);
      q4_apart(q4_mul(e, q4_two(vs, vs)), r.w[t][0], r.w[t][1]);
      r.big = q4_max3(r.big, fabsf(r.w[t][0]), fabsf(r.w[t][1]));
      r.l = t ? q4_add(r.l, e) : e;
      r.z = t ? q4_fma(e, q4_two(vz, vz), r.z) : q4_mul(e, q4_two(vz, vz));
    }
  }
  // of a lane's sums
  __device__ __forceinline__ static float sum_size(const Rows& r) {
    float a, b, c, d;
    q4_apart(r.l, a, b);
    q4_apart(r.z, c, d);
    return (a + b) + (fabsf(c) + fabsf(d));
  }
  // raise the references so that the block's largest weight (its step included) becomes 2^9 .. 2^11, or as far as the sums ask for
  __device__ __forceinline__ void raise(Rows& r, int nrows, float* sums) {
    settle();
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      float top = -3e38f;
#pragma unroll
      for (int t = 0; t < 4; ++t)
        if (4 * gid + t < nrows)
          top = fmaxf(top, fmaf(q4_step(r.ksz[t]) * f_q[g], r.s[t >> 1][2 * (t & 1) + g], q4_middle(r.ksz[t]) * zq[g]) + q4_lift(r.vsz[t], 9));
#pragma unroll
      for (int d = 4; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
      const float m_old = m_ref[g], m_new = fmaxf(m_old, floorf(top));
      m_ref[g] = m_new;
      const float alpha = q4_lower(m_old - m_new, l_thr[g], z_thr[g]);      // first block: 2^(-inf) = 0
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        o[t][g] *= alpha;
        o[t][2 + g] *= alpha;
        if (have) {
          sums[(t * 32 + lane) * 4 + g] *= alpha;
          sums[(t * 32 + lane) * 4 + 2 + g] *= alpha;
        }
      }
      dsum[g] *= alpha;
    }
    weights(r, nrows);
  }

  __device__ __forceinline__ void block(const uint32_t* __restrict__ sw, int nrows, float* sums) {
    Rows r;
    if (nrows >= Q4_BR) weigh<false>(sw, nrows, r);
    else weigh<true>(sw, nrows, r);
    // (a first block's references are -inf)
    if (__any_sync(0xffffffffu, !(r.big <= WEIGHT_MAX) || !(sum_size(r) < Q4_SUM_MAX))) raise(r, nrows, sums);
    // ---- row sums; the weights as fp16 pairs, turned into the B operand ----
    l_part = q4_add(l_part, r.l);
    z_part = q4_add(z_part, r.z);
    uint32_t pb[4], pl[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      float top[2], rest[2];
#pragma unroll
      for (int g = 0; g < 2; ++g) top[g] = __uint_as_float(__float_as_uint(r.w[t][g]) & 0xffff0000u);
      q4_apart(q4_fma(q4_two(top[0], top[1]), q4_two(-1.f, -1.f), q4_two(r.w[t][0], r.w[t][1])), rest[0], rest[1]);
      pb[t] = q4_transpose(q4_pack(top[0], top[1]));
      pl[t] = q4_transpose(q4_pack(rest[0], rest[1]));
    }
    // ---- O += V p: two steps of 16 rows, tiles of 16 channels ----
#pragma unroll
    for (int mt = 0; mt < 2; ++mt) {
      const uint32_t b0 = pb[2 * mt], b1 = pb[2 * mt + 1], c0 = pl[2 * mt], c1 = pl[2 * mt + 1];
      // four channels of 16 rows: y holds k-slots 2 tq, 2 tq + 1, z those + 8; codes 0 .. 3 go to rows gid and gid + 8 of two tiles
      auto tiles = [&](float (&acc0)[4], float (&acc1)[4], uint32_t y, uint32_t z) {
        const uint32_t a0 = q4_mul2(q4_pair<LO>(y, flip0), UP), a1 = q4_pair<HI>(y, flip4);
        const uint32_t a2 = q4_mul2(q4_pair<LO>(z, flip0), UP), a3 = q4_pair<HI>(z, flip4);
        q4_mma(acc0, a0, a1, a2, a3, b0, b1);
        q4_mma(acc0, a0, a1, a2, a3, c0, c1);
        y >>= 8;
        z >>= 8;
        const uint32_t d0 = q4_mul2(q4_pair<LO>(y, flip0), UP), d1 = q4_pair<HI>(y, flip4);
        const uint32_t d2 = q4_mul2(q4_pair<LO>(z, flip0), UP), d3 = q4_pair<HI>(z, flip4);
        q4_mma(acc1, d0, d1, d2, d3, b0, b1);
        q4_mma(acc1, d0, d1, d2, d3, c0, c1);
      };
      constexpr uint32_t ones = 0x3c003c00u;
      q4_mma(dsum, ones, ones, ones, ones, b0, b1);
      q4_mma(dsum, ones, ones, ones, ones, c0, c1);
      const uint32_t* v0 = sw + at.v + 2 * mt * VSW;
#pragma unroll
      for (int u = 0; u < NGV / 2; ++u) {
        const uint32_t xa = v0[8 * u], xb = v0[8 * u + 4 * VSW], xc = v0[8 * u + VSW], xd = v0[8 * u + 5 * VSW];
        tiles(o[4 * u], o[4 * u + 1], __byte_perm(xa, xb, 0x5410), __byte_perm(xc, xd, 0x5410));
        tiles(o[4 * u + 2], o[4 * u + 3], __byte_perm(xa, xb, 0x7632), __byte_perm(xc, xd, 0x7632));
      }
      if constexpr (NGV % 2 == 1) {
        const uint16_t* vh = reinterpret_cast<const uint16_t*>(sw) + at.vh + 4 * mt * VSW;
        tiles(o[NT - 2], o[NT - 1], __byte_perm(vh[0], vh[8 * VSW], 0x5410), __byte_perm(vh[2 * VSW], vh[10 * VSW], 0x5410));
      }
    }
  }

  __device__ __forceinline__ void finish(float* sums) {
    settle();
    total(sums);
  }
  __device__ __forceinline__ void put(float* rr, int g, float f) const {
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int c = t < 4 * (NGV / 2) ? 64 * (t / 4) + 8 * gid + 2 * (t % 4) : 32 * (NGV - 1) + 4 * gid + 2 * (t % 2);
      rr[c] = fmaf(o[t][g], 0x1p14f, z_thr[g]) * f;
      rr[c + 1] = fmaf(o[t][2 + g], 0x1p20f, z_thr[g]) * f;
    }
  }
};

}  // namespace
