// The 4-bit row format, shared by everything that writes or reads it.  A row x of W numbers keeps codes c_i in 0..15, a
// step s and a middle z (both bf16):
//     z = bf16(hi / 2 + lo / 2),   s = bf16(max(hi - z, z - lo) / 7.5),   c_i = rint((x_i - z) (1 / s) + 7.5),
//     x_i ~ z + s (c_i - 7.5),
// hi and lo being the row's extremes, every step decided in fp32 (round half to even, no contraction).  The middle is
// rounded first and the step taken from it, so the codes stay inside 0..15 without clipping: |x - z| <= 7.5 s (1 + 2^-8).
// A step below the smallest normal number counts as zero (codes 8, the row reads back as z); a row with a NaN, an
// infinity or a range beyond fp32 has no such form and is held as NaN (step and middle NaN, codes 8).
// Layout: an odd number of 32-bit words, so that rows staged back to back in shared memory start on different banks; byte
// i holds code 2i (low half) and 2i + 1 (high half), then zeros, and the last word is s (low half) and z (high half).
#pragma once
#include <math.h>

#include "rap_internal.h"

namespace {

constexpr int Q4_MAX_WIDTH = 256;      // one lane of a warp per word of eight codes

__host__ __device__ constexpr int q4_row_words(int W) { return (((W + 1) / 2 + 4 + 3) / 4) | 1; }

__device__ __forceinline__ float q4_ld(const float* p) { return *p; }
__device__ __forceinline__ float q4_ld(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void q4_st(float* p, float v) { *p = v; }
__device__ __forceinline__ void q4_st(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

// maximum and minimum that keep a NaN (fmaxf drops it)
__device__ __forceinline__ float q4_max(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float q4_min(float a, float b) {
  float r;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

__device__ __forceinline__ float q4_max3(float a, float b, float c) {
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ float q4_min3(float a, float b, float c) {
  float r;
  asm("min.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

struct Q4Row {
  float z, r;            // middle; 1 / step (0 where the step is)
  uint32_t sz;           // the row's last word
  bool bad;              // not representable
};
__device__ __forceinline__ Q4Row q4_decide(float hi, float lo) {
  Q4Row q;
  q.z = __bfloat162float(__float2bfloat16_rn(__fadd_rn(__fmul_rn(hi, 0.5f), __fmul_rn(lo, 0.5f))));
  const float reach = q4_max(__fsub_rn(hi, q.z), __fsub_rn(q.z, lo));
  // reach / 7.5, correctly rounded: the fp64 product is 2^-52 off the quotient, and 2 reach / 15 lies at least a thirtieth of
  // an fp32 step from any rounding border (15 times a border is an odd multiple of its last place, which no fp32 number is)
  float s = __bfloat162float(__float2bfloat16_rn((float)((double)reach * (1.0 / 7.5))));
  q.bad = !(s < INFINITY);
  if (s < 1.17549435e-38f) s = 0.f;
  q.r = s > 0.f ? __frcp_rn(s) : 0.f;
  q.sz = q.bad ? 0x7fff7fffu : (__float_as_uint(q.z) & 0xffff0000u) | (__float_as_uint(s) >> 16);      // bf16 numbers: exact
  return q;
}
// code of x: adding 1.5 * 2^23 rounds to an integer (half to even) and leaves it in the low mantissa bits
__device__ __forceinline__ uint32_t q4_code(float x, const Q4Row& q) {
  const float t = __fadd_rn(__fmul_rn(__fsub_rn(x, q.z), q.r), 7.5f);
  return q.bad ? 8u : __float_as_uint(__fadd_rn(t, 12582912.0f)) & 15u;
}
// two fp32 numbers in one instruction (each rounded as by itself): half the issue slots
typedef unsigned long long q4_f2;
__device__ __forceinline__ q4_f2 q4_two(float a, float b) {
  q4_f2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void q4_apart(q4_f2 x, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(x)); }
__device__ __forceinline__ q4_f2 q4_add(q4_f2 a, q4_f2 b) {
  q4_f2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ q4_f2 q4_mul(q4_f2 a, q4_f2 b) {
  q4_f2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ q4_f2 q4_fma(q4_f2 a, q4_f2 b, q4_f2 c) {
  q4_f2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
// a word of eight codes: with 1.5 2^23 added a place is 0x4b400000 + code as an integer, and the eight sum up as digits
__device__ __forceinline__ uint32_t q4_word(const float (&x)[8], const Q4Row& q) {
  uint32_t word = 0u - 0x4b400000u * 0x11111111u;
  const q4_f2 z = q4_two(-q.z, -q.z), r = q4_two(q.r, q.r), half = q4_two(7.5f, 7.5f), magic = q4_two(12582912.0f, 12582912.0f);
  const q4_f2 one = q4_two(1.f, 1.f);      // (a sum behind a product of this width is contracted into one rounding; a fused one is not)
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    float a, b;
    q4_apart(q4_add(q4_fma(q4_mul(q4_add(q4_two(x[i], x[i + 1]), z), r), one, half), magic), a, b);
    word += __float_as_uint(a) << (4 * i);
    word += __float_as_uint(b) << (4 * i + 4);
  }
  return q.bad ? 0x88888888u : word;
}
__device__ __forceinline__ float q4_step(uint32_t sz) { return __uint_as_float(sz << 16); }
__device__ __forceinline__ float q4_middle(uint32_t sz) { return __uint_as_float(sz & 0xffff0000u); }

}  // namespace
