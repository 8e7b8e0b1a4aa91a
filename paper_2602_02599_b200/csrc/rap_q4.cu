// The cache held in 4 bits (format: rap_q4_common.cuh): conversion of rows and of a layer's cache in both directions, the
// RoPE / append epilogue that quantises new K and V rows straight from their fp32 values, and the launch side of the split-KV
// attention over a 4-bit cache: the tensor-core scan (rap_attn_q4_kernel.cuh) for bf16 q~ and rows of up to 128 numbers,
// a shape-generic kernel behind it.
#include "rap_attn_q4_kernel.cuh"

rap_status rap_launch_proj_tc(rap_ctx* ctx, const rap_proj_args& a, int* ksplit_out, cudaStream_t st);
rap_status rap_launch_proj_generic(rap_ctx* ctx, const rap_proj_args& a, cudaStream_t st);

namespace {

__device__ __forceinline__ void q4_st2(float* p, float a, float b) { *reinterpret_cast<float2*>(p) = make_float2(a, b); }
__device__ __forceinline__ void q4_st2(__nv_bfloat16* p, float a, float b) {
  *reinterpret_cast<__nv_bfloat162*>(p) = __floats2bfloat162_rn(a, b);
}
__device__ __forceinline__ float warp_max_nan(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = q4_max(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}
__device__ __forceinline__ float warp_min_nan(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = q4_min(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}

// ---- rows to 4 bits and back ----------------------------------------------------------------------------------------
// Both directions are bound by the bytes they move (W e + row bytes per row each way).  R rows are one contiguous range on
// either side: a bulk copy brings them into shared memory, four threads work on each row from there (word k of a row belongs
// to thread k mod 4), a bulk copy takes the result out.  Row lengths of any parity are an affair of the shared memory alone.
// The CTAs walk over the chunks with the grid's stride, the next chunk's copy in flight under the current one's arithmetic
// and the last one's way out under both.  Odd bytes at the end (a bulk copy moves multiples of 16) go by plain loads and
// stores, so nothing behind the last row is touched.
constexpr int Q4R_STAGE = 18 * 1024;     // most bytes of a chunk's fp32 / bf16 rows; R is a multiple of 8, at most 64

int q4_rows_per_cta(int W, int elem) {
  int r = 64;
  while (r > 8 && r * W * elem > Q4R_STAGE) r /= 2;
  return r;
}
struct Q4Chunk {
  const unsigned char* src;
  unsigned char* dst;
  int in_bytes, out_bytes, rows, W;
  bool is_v;
};
// bytes of an input / output buffer that holds n (the loads of a row's last word may reach 32 past it)
__host__ __device__ constexpr int q4_buffer(int n) { return (n + 47) / 16 * 16; }
constexpr int Q4R_HEAD = 128;            // the two barriers
constexpr int Q4R_THREADS = 128;         // 32 rows at a time

// `total` chunks over the grid: chunk(c) says where chunk c lies, body(chunk, in, out) works from one buffer into the other
template <typename Chunk, typename Body>
__device__ __forceinline__ void q4_rows_pipeline(unsigned char* smem, int in_cap, int out_cap, long long total, int32_t* status,
                                                 Chunk chunk, Body body) {
  long long c = blockIdx.x;
  if (c >= total) return;
  const uint32_t bars = smem_u32(smem);
  unsigned char* const in0 = smem + Q4R_HEAD;
  unsigned char* const out0 = in0 + 2 * in_cap;
  if (threadIdx.x == 0) {
    mbar_init(bars, 1);
    mbar_init(bars + 8, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();
  auto bring = [&](const Q4Chunk& k, int buf) {
    const int bulk = k.in_bytes & ~15;
    unsigned char* to = in0 + buf * in_cap;
    if (threadIdx.x == 0) {
      mbar_expect_tx(bars + 8 * buf, bulk);
      if (bulk) bulk_g2s(smem_u32(to), k.src, bulk, bars + 8 * buf);
    }
    for (int i = bulk + threadIdx.x; i < k.in_bytes; i += blockDim.x) to[i] = k.src[i];
  };
  Q4Chunk now = chunk(c);
  bring(now, 0);
  int buf = 0;
  uint32_t parity = 0;
  for (;;) {
    const bool more = c + gridDim.x < total;
    Q4Chunk next = now;
    if (more) {
      next = chunk(c + gridDim.x);
      bring(next, buf ^ 1);            // (everyone left that buffer before the last barrier below)
    }
    // the copy has landed, and the store that read this output buffer two chunks ago is done with it
    const bool here = mbar_wait_bounded(bars + 8 * buf, parity);
    if (threadIdx.x == 0) asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
    if (!__syncthreads_and(here)) {    // one verdict for the CTA
      if (threadIdx.x == 0) {
        atomicCAS(&status[0], 0, (int)RAP_ETIMEOUT);
        status[1] = (int)blockIdx.x;
        if (more) mbar_wait_bounded(bars + 8 * (buf ^ 1), buf ? parity ^ 1u : parity);      // a copy in flight may still land
      }
      break;
    }
    unsigned char* out = out0 + buf * out_cap;
    body(now, in0 + buf * in_cap, out);
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncthreads();
    const int bulk = now.out_bytes & ~15;
    if (threadIdx.x == 0) {
      if (bulk)
        asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(now.dst), "r"(smem_u32(out)), "r"(bulk) : "memory");
      asm volatile("cp.async.bulk.commit_group;" ::: "memory");
    }
    for (int i = bulk + threadIdx.x; i < now.out_bytes; i += blockDim.x) now.dst[i] = out[i];
    if (!more) break;
    c += gridDim.x;
    now = next;
    parity ^= (uint32_t)buf;           // both buffers have been used once more
    buf ^= 1;
  }
  if (threadIdx.x == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");     // shared memory may go
}

// How rows lie in shared memory: on words, on half words (bf16 rows of odd length), or on 16 bytes (lengths that are multiples
// of 8; those of 64 and 128, where all rows start on one bank, are eight times as slow word by word)
enum Q4Rows { Q4_WORDS, Q4_HALVES, Q4_VECTORS };

// eight numbers of a row in shared memory, from element `at` on, of which the first n count (the others become the first one),
// and the row's extremes so far
template <Q4Rows HOW, bool PART>
__device__ __forceinline__ void q4_eight(const float* base, int at, int n, float (&v)[8], float& hi, float& lo) {
  if constexpr (HOW == Q4_VECTORS) {
    const float4 a = *reinterpret_cast<const float4*>(base + at), b = *reinterpret_cast<const float4*>(base + at + 4);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = base[at + i];
  }
  if constexpr (PART && HOW != Q4_VECTORS) {
#pragma unroll
    for (int i = 1; i < 8; ++i) v[i] = i < n ? v[i] : v[0];
  }
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    hi = q4_max3(hi, v[i], v[i + 1]);
    lo = q4_min3(lo, v[i], v[i + 1]);
  }
}
template <Q4Rows HOW, bool PART>
__device__ __forceinline__ void q4_eight(const __nv_bfloat16* base, int at, int n, float (&v)[8], float& hi, float& lo) {
  // rows of odd length may start on a half word: five words, shifted into place
  constexpr bool ODD = HOW == Q4_HALVES;
  const uint32_t* w = reinterpret_cast<const uint32_t*>(base) + (at >> 1);
  uint32_t y[4];
  if constexpr (HOW == Q4_VECTORS) {
    const uint4 a = *reinterpret_cast<const uint4*>(w);
    y[0] = a.x; y[1] = a.y; y[2] = a.z; y[3] = a.w;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = w[i];
  }
  if constexpr (ODD) {
    const uint32_t sh = (at & 1) * 16, last = w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = __funnelshift_r(y[i], i < 3 ? y[i + 1] : last, sh);
  }
  if constexpr (PART && HOW != Q4_VECTORS) {
    const uint32_t twice = __byte_perm(y[0], 0, 0x1010);
    if constexpr (ODD) y[0] = n > 1 ? y[0] : twice;
#pragma unroll
    for (int i = 1; i < 4; ++i) {
      if constexpr (ODD) y[i] = 2 * i + 1 < n ? y[i] : 2 * i < n ? __byte_perm(y[i], y[0], 0x5410) : twice;
      else y[i] = 2 * i < n ? y[i] : twice;
    }
  }
  __nv_bfloat162 a = *reinterpret_cast<__nv_bfloat162*>(&y[0]), b = a;
#pragma unroll
  for (int i = 1; i < 4; ++i) {
    const __nv_bfloat162 c = *reinterpret_cast<__nv_bfloat162*>(&y[i]);
    a = __hmax2_nan(a, c);
    b = __hmin2_nan(b, c);
  }
  hi = q4_max3(hi, __low2float(a), __high2float(a));
  lo = q4_min3(lo, __low2float(b), __high2float(b));
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(y[i] << 16);
    v[2 * i + 1] = __uint_as_float(y[i] & 0xffff0000u);
  }
}

// WPT = ceil(W / 32): words of codes per thread, four threads a row, so only a thread's last word can be short (or past the
// end: it then works on the row's first numbers again and stores nothing).
// What bounds the conversion is instruction issue next to the bytes: 513 instructions for 8 rows of 90 took 70 us for a
// million rows, hence no branches, extremes of bf16 pairs, and digits summed by one multiply-add each.
template <typename T, int WPT, Q4Rows HOW>
__device__ __forceinline__ void quantize_chunk(const T* x, uint32_t* out, int rows, int W, int nw) {
  const int q = threadIdx.x & 3;
  const int last = 8 * (q + 4 * (WPT - 1)), left = W - last;           // this thread's last word: elements from `last` on
  const uint32_t mask = left >= 8 ? 0xffffffffu : left > 0 ? (1u << (4 * left)) - 1u : 0u;
  const bool store_last = q + 4 * (WPT - 1) < nw - 1;
  for (int row = threadIdx.x >> 2; row < ((rows + 7) & ~7); row += Q4R_THREADS / 4) {      // (whole warps: the shuffles)
    const int at0 = min(row, rows - 1) * W + 8 * q;
    float v[WPT][8];
    float hi = -INFINITY, lo = INFINITY;
#pragma unroll
    for (int k = 0; k < WPT - 1; ++k) q4_eight<HOW, false>(x, at0 + 32 * k, 8, v[k], hi, lo);
    q4_eight<HOW, true>(x, left > 0 ? at0 + 32 * (WPT - 1) : at0 - 8 * q, left > 0 ? left : 1, v[WPT - 1], hi, lo);
#pragma unroll
    for (int o = 1; o < 4; o <<= 1) {
      hi = q4_max(hi, __shfl_xor_sync(0xffffffffu, hi, o));
      lo = q4_min(lo, __shfl_xor_sync(0xffffffffu, lo, o));
    }
    const Q4Row r = q4_decide(hi, lo);
    if (row < rows) {
      uint32_t* o = out + row * nw;
#pragma unroll
      for (int k = 0; k < WPT - 1; ++k) o[q + 4 * k] = q4_word(v[k], r);
      const uint32_t word = q4_word(v[WPT - 1], r) & mask;
      if (store_last) o[q + 4 * (WPT - 1)] = word;
      if (q == 0) o[nw - 1] = r.sz;
    }
  }
}

template <typename T, int WPT, Q4Rows HOW>
__global__ void __launch_bounds__(Q4R_THREADS) quantize_rows_q4_kernel(const T* __restrict__ src, uint32_t* __restrict__ dst,
                                                               long long n_rows, int W, int R, int32_t* __restrict__ status) {
  extern __shared__ __align__(128) unsigned char q4_rows_smem[];
  const int nw = q4_row_words(W), row_bytes = W * (int)sizeof(T);
  auto chunk = [&](long long c) {
    const int rows = (int)min((long long)R, n_rows - c * R);
    return Q4Chunk{reinterpret_cast<const unsigned char*>(src + c * R * W), reinterpret_cast<unsigned char*>(dst + c * R * nw),
                   rows * row_bytes, rows * nw * 4, rows, W, false};
  };
  q4_rows_pipeline(q4_rows_smem, q4_buffer(R * row_bytes), q4_buffer(R * nw * 4), (n_rows + R - 1) / R, status, chunk,
                   [&](const Q4Chunk& k, const unsigned char* in, unsigned char* to) {
                     quantize_chunk<T, WPT, HOW>(reinterpret_cast<const T*>(in), reinterpret_cast<uint32_t*>(to), k.rows, W, nw);
                   });
}

// eight numbers to a row in shared memory, from element `at` on; PART: the first n of them (a row's last word)
template <Q4Rows HOW, bool PART>
__device__ __forceinline__ void q4_put8(float* base, int at, const float (&v)[8], int n) {
  if constexpr (HOW == Q4_VECTORS) {
    *reinterpret_cast<float4*>(base + at) = make_float4(v[0], v[1], v[2], v[3]);
    *reinterpret_cast<float4*>(base + at + 4) = make_float4(v[4], v[5], v[6], v[7]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (!PART || i < n) base[at + i] = v[i];
  }
}
template <Q4Rows HOW, bool PART>
__device__ __forceinline__ void q4_put8(__nv_bfloat16* base, int at, const float (&v)[8], int n) {
  uint32_t y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
    y[i] = *reinterpret_cast<const uint32_t*>(&h);
  }
  if constexpr (HOW == Q4_VECTORS) {
    *reinterpret_cast<uint4*>(base + at) = make_uint4(y[0], y[1], y[2], y[3]);
  } else if constexpr (HOW == Q4_WORDS) {      // (rows of even length: n is even)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (!PART || 2 * i < n) *reinterpret_cast<uint32_t*>(base + at + 2 * i) = y[i];
  } else if constexpr (PART) {
    unsigned short* u = reinterpret_cast<unsigned short*>(base) + at;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) u[i] = (unsigned short)(y[i >> 1] >> (16 * (i & 1)));
  } else {      // rows of odd length may start on a half word: three whole words and two halves, the same stores for either start
    const bool odd = at & 1;
    uint32_t* w = reinterpret_cast<uint32_t*>(base + at + odd);
    unsigned short* u = reinterpret_cast<unsigned short*>(base) + at;
#pragma unroll
    for (int i = 0; i < 3; ++i) w[i] = odd ? __funnelshift_r(y[i], y[i + 1], 16) : y[i];
    u[odd ? 0 : 6] = (unsigned short)(odd ? y[0] : y[3]);
    u[7] = (unsigned short)(y[3] >> 16);
  }
}
// The numbers of a word: a code in bits 4 i .. (i = 1 .. 4) under the exponent of 2^23 is 2^23 + c 16^i; less 2^23 + 7.5 16^i it
// is (c - 7.5) 16^i exactly, and the step takes the 16^-i along (exactly too: 2^-126 - 7 - 16 is the last bit there is): one
// mask, one addition, one fused multiply-add a number.  Codes 0 and 5 to 7 come into place by a shift.
// Rows that may start on a half word: all words but the last go without tests (with them 8 rows of 115 took 643 instructions, 700,000
// 74 us; without 41).  Rows on words: the tests are few, and a separate last word would be a pass
// more (read-back of 16 sequences of up to 8K rows of 90: 12.3 us against 14.2).
template <typename T, Q4Rows HOW>
__device__ __forceinline__ void dequantize_chunk(const uint32_t* in, T* out, int rows, int W) {
  const int nw = q4_row_words(W), q = threadIdx.x & 3;
  uint32_t base;                 // 0x4b000000 in a register: mask and exponent in one instruction
  asm volatile("mov.b32 %0, 0x4b000000;" : "=r"(base));
  for (int row = threadIdx.x >> 2; row < rows; row += Q4R_THREADS / 4) {
    const uint32_t sz = in[row * nw + nw - 1];
    const float z = q4_middle(sz);
    float s[5];
    s[0] = q4_step(sz);
#pragma unroll
    for (int i = 1; i < 5; ++i) s[i] = s[i - 1] * 0.0625f;
    auto number = [&](uint32_t w, int i) {       // the code in bits 4 i ..
      uint32_t bits;
      asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(bits) : "r"(w), "r"(15u << (4 * i)), "r"(base));
      const float one = (float)(1u << (4 * i));
      return fmaf(s[i], __uint_as_float(bits) - (8388608.f + 7.5f * one), z);
    };
    auto eight = [&](int e0, auto part) {
      const uint32_t word = in[row * nw + (e0 >> 3)], up = word << 4, down = word >> 8;
      const float v[8] = {number(up, 1), number(word, 1), number(word, 2), number(word, 3), number(word, 4), number(down, 3),
                          number(down, 4), number(word >> 12, 4)};
      q4_put8<HOW, decltype(part)::value>(out, row * W + e0, v, W - e0);
    };
    int e0 = 8 * q;
    if constexpr (HOW == Q4_WORDS) {
#pragma unroll 4
      for (; e0 < W; e0 += 32) eight(e0, std::true_type{});
    } else {
#pragma unroll 4
      for (; e0 + 8 <= W; e0 += 32) eight(e0, std::false_type{});
      if (HOW == Q4_HALVES && e0 < W) eight(e0, std::true_type{});
    }
  }
}

template <typename T, Q4Rows HOW>
__global__ void __launch_bounds__(Q4R_THREADS) dequantize_rows_q4_kernel(const uint32_t* __restrict__ src, T* __restrict__ dst,
                                                                 long long n_rows, int W, int R, int32_t* __restrict__ status) {
  extern __shared__ __align__(128) unsigned char q4_rows_smem[];
  const int nw = q4_row_words(W), row_bytes = W * (int)sizeof(T);
  auto chunk = [&](long long c) {
    const int rows = (int)min((long long)R, n_rows - c * R);
    return Q4Chunk{reinterpret_cast<const unsigned char*>(src + c * R * nw), reinterpret_cast<unsigned char*>(dst + c * R * W),
                   rows * nw * 4, rows * row_bytes, rows, W, false};
  };
  q4_rows_pipeline(q4_rows_smem, q4_buffer(R * nw * 4), q4_buffer(R * row_bytes), (n_rows + R - 1) / R, status, chunk,
                   [&](const Q4Chunk& k, const unsigned char* in, unsigned char* to) {
                     dequantize_chunk<T, HOW>(reinterpret_cast<const uint32_t*>(in), reinterpret_cast<T*>(to), k.rows, W);
                   });
}

// A layer's K rows and V rows up to every sequence's length.  The chunks of R rows that exist -- per sequence
// (K or V) x KV head x rows -- form one sequence (a grid over all positions spent 15 us on CTAs without rows in a batch of
// unlike lengths); a CTA finds its chunks in the prefix of the sequences' chunk counts, which it makes first.
constexpr int Q4R_SEQS = 1024;           // sequences per launch
constexpr int Q4R_PLAN = ((Q4R_SEQS + 2) * 4 + 127) / 128 * 128;      // bytes of the prefix, in front of the barriers
template <typename T, Q4Rows HOW_K, Q4Rows HOW_V>
__global__ void __launch_bounds__(Q4R_THREADS)
read_cache_q4_kernel(const uint32_t* __restrict__ k4, const uint32_t* __restrict__ v4, T* __restrict__ k, T* __restrict__ v,
                     const int32_t* __restrict__ seq_len, int B, int Hkv, int S_cap, int P2, int dv, int len_max, int R,
                     int32_t* __restrict__ status) {
  extern __shared__ __align__(128) unsigned char q4_rows_smem[];
  int* const pref = reinterpret_cast<int*>(q4_rows_smem);
  SkPlan plan;
  sk_plan_shared(seq_len, B, 2 * Hkv, 0, len_max, R, (int)gridDim.x, pref, Q4R_SEQS + 2, &plan);
  auto chunk = [&](long long c) {
    const int b = sk_seq_of(pref, B, (int)c);
    const int len = min(max(seq_len[b], 0), len_max), per = (len + R - 1) / R;
    const int at = (int)c - (b ? pref[b - 1] : 0), unit = at / per, pos = (at - unit * per) * R, rows = min(len - pos, R);
    const bool is_v = unit >= Hkv;
    const size_t row = ((size_t)b * Hkv + unit - (is_v ? Hkv : 0)) * S_cap + pos;
    const int W = is_v ? dv : P2, nw = q4_row_words(W);
    return Q4Chunk{reinterpret_cast<const unsigned char*>((is_v ? v4 : k4) + row * nw),
                   reinterpret_cast<unsigned char*>((is_v ? v : k) + row * W), rows * nw * 4, rows * W * (int)sizeof(T), rows, W, is_v};
  };
  const int wide = max(P2, dv);
  q4_rows_pipeline(q4_rows_smem + Q4R_PLAN, q4_buffer(R * q4_row_words(wide) * 4), q4_buffer(R * wide * (int)sizeof(T)), plan.T, status, chunk,
                   [&](const Q4Chunk& c, const unsigned char* in, unsigned char* to) {
                     if (c.is_v) dequantize_chunk<T, HOW_V>(reinterpret_cast<const uint32_t*>(in), reinterpret_cast<T*>(to), c.rows, c.W);
                     else dequantize_chunk<T, HOW_K>(reinterpret_cast<const uint32_t*>(in), reinterpret_cast<T*>(to), c.rows, c.W);
                   });
}

// RoPE / append epilogue with quantisation.  One CTA per (row t, KV head h), one warp per item: the G query heads of h
// (rotated, rounded to the storage dtype, written to q_out as in the unquantised path), its key head (rotated, quantised,
// appended) and its value head (quantised, appended).  All of them rotate by the same angles, so the sines and cosines are
// taken once per CTA (one warp per item on its own: 34 us for 512 rows of the 8B-shaped layer, this: 12.2).
// A code is a step function of the rotated number, so an error of an fp32 place moves one now and then by a whole step, and the
// rotation of the key head is fixed to the bit: sines and cosines of the fp64 angle in fp64, rounded to fp32, then products and
// sums rounded one by one.  (With the query heads' fp32 sines two or three codes of 370,000 were another one.)  The fp64 pair is
// taken before the GEMM is awaited: by itself the kernel takes 12.2 us for 512 rows where it took 10.6, behind the GEMM and with
// the read-backs 39.4 either way (43.4 with the pair behind the wait).
// A lane owns KP pairs of neighbouring numbers, that is whole bytes of a quantised row; P <= 128 and d_v' <= 256, so KP <= 4.
// y holds `ksplit` partial results, each [T][n_out].
template <typename T, int KP, bool BIAS>
__global__ void __launch_bounds__(32 * (RAP_MAX_GROUP + 2))
rope_append_q4_kernel(const float* __restrict__ y, int ksplit, const T* __restrict__ bias, const int32_t* __restrict__ seq_id,
                      const int32_t* __restrict__ pos, const int32_t* __restrict__ slot, const double* __restrict__ inv_freq,
                      T* __restrict__ q_out, uint32_t* __restrict__ k4, uint32_t* __restrict__ v4, int Trows, int Hq, int Hkv,
                      int P2, int dv, int half_dim, int B_cache, int S_cap, int32_t* __restrict__ status) {
  __shared__ float2 turn[256];                   // (cosine, sine) of every pair: P for the query heads, P for the key head
  const int t = blockIdx.x, h = blockIdx.y;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int P = P2 >> 1, G = Hq / Hkv;
  const int n_out = (Hq + Hkv) * P2 + Hkv * dv;
  const int p = pos[t];
  for (int c = threadIdx.x; c < 2 * P; c += blockDim.x) {
    // fp64 angle and reduction to [-pi, pi] (off by 2^-50 at most); for the query heads fp32 sine and cosine of the reduced
    // angle (as in the unquantised path)
    const double ang = (double)p * inv_freq[h * half_dim + (c < P ? c : c - P)];
    const double turns = rint(ang * 0.15915494309189535);
    const double red = fma(-turns, 2.4492935982947064e-16, fma(-turns, 6.283185307179586, ang));
    if (c < P) {
      float sf, cf;
      sincosf((float)red, &sf, &cf);
      turn[c] = make_float2(cf, sf);
    } else {
      double sd, cd;
      sincospi(red * 0.3183098861837907, &sd, &cd);      // (sincos itself has a branch for far angles: 72 bytes of stack)
      turn[c] = make_float2((float)cd, (float)sd);
    }
  }
  // launched behind the GEMM with programmatic serialization: the GEMM's results (and, through the GEMM, the end of the scan before
  // it) are awaited here.  What is read above, positions and frequencies, no kernel of such a chain writes.
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int sq = seq_id ? seq_id[t] : t;
  const int sl = slot ? slot[t] : p;
  const bool row_ok = (sq >= 0 && sq < B_cache && sl >= 0 && sl < S_cap);
  if (!row_ok && h == 0 && threadIdx.x == 0) {
    atomicCAS(&status[0], 0, (int)RAP_ECAPACITY);
    status[1] = t;
  }
  const bool is_q = warp < G, is_v = warp > G;
  // columns of Y: q heads, then k heads (2P each), then v heads
  const int col0 = is_v ? (Hq + Hkv) * P2 + h * dv : (is_q ? h * G + warp : Hq + h) * P2;
  const int W = is_v ? dv : P2;
  const size_t split_stride = (size_t)Trows * n_out;
  const float* yr = y + (size_t)t * n_out + col0;
  float a[KP], b[KP];
#pragma unroll
  for (int k = 0; k < KP; ++k) {
    const int c = 2 * (lane + 32 * k);
    a[k] = c < W ? yr[c] : 0.f;
    b[k] = c + 1 < W ? yr[c + 1] : 0.f;
  }
  for (int s = 1; s < ksplit; ++s) {                                   // the sums in split order
    yr += split_stride;
#pragma unroll
    for (int k = 0; k < KP; ++k) {
      const int c = 2 * (lane + 32 * k);
      a[k] += c < W ? yr[c] : 0.f;
      b[k] += c + 1 < W ? yr[c + 1] : 0.f;
    }
  }
  if constexpr (BIAS) {
#pragma unroll
    for (int k = 0; k < KP; ++k) {
      const int c = 2 * (lane + 32 * k);
      if (c < W) a[k] += q4_ld(bias + col0 + c);
      if (c + 1 < W) b[k] += q4_ld(bias + col0 + c + 1);
    }
  }
  __syncthreads();
  if (!is_v) {
#pragma unroll
    for (int k = 0; k < KP; ++k) {
      const int i = lane + 32 * k;
      if (i < P) {
        const float2 cs = turn[is_q ? i : P + i];
        const float x0 = a[k], x1 = b[k];
        const float c0 = __fmul_rn(x0, cs.x), c1 = __fmul_rn(x1, cs.x);
        a[k] = is_q ? fmaf(-x1, cs.y, c0) : __fsub_rn(c0, __fmul_rn(x1, cs.y));      // q~: the same roundings as the unquantised kernels
        b[k] = is_q ? fmaf(x0, cs.y, c1) : __fadd_rn(__fmul_rn(x0, cs.y), c1);
      }
    }
  }
  if (is_q) {
    T* dst = q_out + ((size_t)t * Hq + h * G + warp) * P2;
#pragma unroll
    for (int k = 0; k < KP; ++k) {
      const int i = lane + 32 * k;
      if (i < P) {
        q4_st2(dst + 2 * i, a[k], b[k]);
      }
    }
    return;
  }
  if (!row_ok) return;
  float hi = -INFINITY, lo = INFINITY;
#pragma unroll
  for (int k = 0; k < KP; ++k) {
    const int c = 2 * (lane + 32 * k);
    if (c < W) { hi = q4_max(hi, a[k]); lo = q4_min(lo, a[k]); }
    if (c + 1 < W) { hi = q4_max(hi, b[k]); lo = q4_min(lo, b[k]); }
  }
  const Q4Row q = q4_decide(warp_max_nan(hi), warp_min_nan(lo));
  const int nw = q4_row_words(W);
  uint32_t* row = (is_v ? v4 : k4) + (((size_t)sq * Hkv + h) * S_cap + sl) * (size_t)nw;
  unsigned char* bytes = reinterpret_cast<unsigned char*>(row);
#pragma unroll
  for (int k = 0; k < KP; ++k) {
    const int i = lane + 32 * k, c = 2 * i;
    if (c < W) bytes[i] = (unsigned char)(q4_code(a[k], q) | (c + 1 < W ? q4_code(b[k], q) << 4 : 0u));
    else if (i < 4 * (nw - 1)) bytes[i] = 0;      // (4 (nw - 1) <= 32 KP)
  }
  if (lane == 0) row[nw - 1] = q.sz;
}

// ---- shape-generic split-KV attention over a 4-bit cache: fp32 q~, rows wider than 128, and the cross-check ----------
constexpr int Q4G_TILE = 64;
constexpr int Q4G_THREADS = 256;

template <typename T>
__global__ void __launch_bounds__(Q4G_THREADS)
attn_q4_generic_kernel(const T* __restrict__ q, const unsigned char* __restrict__ k4, const unsigned char* __restrict__ v4,
                       const int32_t* __restrict__ seq_len, int len_add, int Hq, int Hkv, int P2, int dv, int S_cap,
                       float qscale, int n_split, float* __restrict__ ws) {
  extern __shared__ float smem[];
  const int G = Hq / Hkv;
  const int kb_row = 4 * q4_row_words(P2), vb_row = 4 * q4_row_words(dv);
  float* q_s = smem;                      // [G][P2] scaled by log2(e) / sqrt(D)
  float* s_s = q_s + G * P2;              // [G][TILE] logits, then weights
  float* qsum_s = s_s + G * Q4G_TILE;     // [G] sums of the scaled q
  float* alpha_s = qsum_s + G;            // [G]
  const int split = blockIdx.x, h = blockIdx.y, b = blockIdx.z;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int len = min(max(seq_len[b] + len_add, 0), S_cap);
  const int n_tiles = (len + Q4G_TILE - 1) / Q4G_TILE;
  const int tps = (n_tiles + n_split - 1) / n_split;
  const int tile_begin = split * tps, tile_end = min(n_tiles, tile_begin + tps);
  for (int i = tid; i < G * P2; i += Q4G_THREADS) q_s[i] = q4_ld(q + ((size_t)b * Hq + h * G) * P2 + i) * qscale;
  __syncthreads();
  if (warp < G) {
    float sum = 0.f;
    for (int d = lane; d < P2; d += 32) sum += q_s[warp * P2 + d];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) qsum_s[warp] = sum;
  }
  const unsigned char* kb = k4 + ((size_t)b * Hkv + h) * (size_t)S_cap * kb_row;
  const unsigned char* vb = v4 + ((size_t)b * Hkv + h) * (size_t)S_cap * vb_row;
  float m_run = -INFINITY, l_run = 0.f;
  float acc[RAP_MAX_GROUP];
#pragma unroll
  for (int g = 0; g < RAP_MAX_GROUP; ++g) acc[g] = 0.f;
  __syncthreads();
  for (int tile = tile_begin; tile < tile_end; ++tile) {
    const int j0 = tile * Q4G_TILE;
    const int nj = min(Q4G_TILE, len - j0);
    for (int j = warp; j < nj; j += Q4G_THREADS / 32) {
      const unsigned char* kr = kb + (size_t)(j0 + j) * kb_row;
      float part[RAP_MAX_GROUP];
#pragma unroll
      for (int g = 0; g < RAP_MAX_GROUP; ++g) part[g] = 0.f;
      for (int c = lane; c < P2 / 2; c += 32) {
        const uint32_t byte = kr[c];
        const float c0 = (float)(byte & 15u) - 7.5f, c1 = (float)(byte >> 4) - 7.5f;
#pragma unroll
        for (int g = 0; g < RAP_MAX_GROUP; ++g)
          if (g < G) part[g] = fmaf(c1, q_s[g * P2 + 2 * c + 1], fmaf(c0, q_s[g * P2 + 2 * c], part[g]));
      }
      const uint32_t sz = *reinterpret_cast<const uint32_t*>(kr + kb_row - 4);
#pragma unroll
      for (int g = 0; g < RAP_MAX_GROUP; ++g) {
        if (g < G) {
          float v = part[g];
#pragma unroll
          for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
          if (lane == 0) s_s[g * Q4G_TILE + j] = fmaf(q4_step(sz), v, q4_middle(sz) * qsum_s[g]);
        }
      }
    }
    __syncthreads();
    if (warp < G) {
      const int g = warp;
      float mx = -INFINITY;
      for (int j = lane; j < nj; j += 32) mx = fmaxf(mx, s_s[g * Q4G_TILE + j]);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
      const float m_new = fmaxf(m_run, mx);
      float sum = 0.f;
      for (int j = lane; j < nj; j += 32) {
        const float pw = exp2f(s_s[g * Q4G_TILE + j] - m_new);
        s_s[g * Q4G_TILE + j] = pw;
        sum += pw;
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
      const float alpha = exp2f(m_run - m_new);
      l_run = l_run * alpha + sum;
      m_run = m_new;
      if (lane == 0) alpha_s[g] = alpha;
    }
    __syncthreads();
    if (tid < dv) {
#pragma unroll
      for (int g = 0; g < RAP_MAX_GROUP; ++g)
        if (g < G) acc[g] *= alpha_s[g];
      for (int j = 0; j < nj; ++j) {
        const unsigned char* vr = vb + (size_t)(j0 + j) * vb_row;
        const uint32_t sz = *reinterpret_cast<const uint32_t*>(vr + vb_row - 4);
        const float vv = fmaf(q4_step(sz), (float)((vr[tid >> 1] >> (4 * (tid & 1))) & 15u) - 7.5f, q4_middle(sz));
#pragma unroll
        for (int g = 0; g < RAP_MAX_GROUP; ++g)
          if (g < G) acc[g] = fmaf(s_s[g * Q4G_TILE + j], vv, acc[g]);
      }
    }
    __syncthreads();
  }
#pragma unroll
  for (int g = 0; g < RAP_MAX_GROUP; ++g) {
    if (g < G) {
      float* dst = ws + (((size_t)b * Hq + h * G + g) * n_split + split) * (size_t)(dv + 2);
      if (tid < dv) dst[tid] = acc[g];
      if (warp == g && lane == 0) {
        dst[dv] = m_run;
        dst[dv + 1] = l_run;
      }
    }
  }
}

// out[b][g][c] = sum_s 2^(m_s - M) acc_s[c] / sum_s 2^(m_s - M) l_s; an empty split has l = 0 (a NaN in l is kept)
__global__ void attn_q4_combine_kernel(const float* __restrict__ ws, int n_split, int dv, float* __restrict__ out) {
  const size_t bg = blockIdx.x;
  const float* base = ws + bg * n_split * (size_t)(dv + 2);
  float M = -INFINITY;
  for (int s = 0; s < n_split; ++s)
    if (base[(size_t)s * (dv + 2) + dv + 1] != 0.f) M = fmaxf(M, base[(size_t)s * (dv + 2) + dv]);
  float den = 0.f;
  for (int s = 0; s < n_split; ++s) {
    const float l = base[(size_t)s * (dv + 2) + dv + 1];
    if (l != 0.f) den += exp2f(base[(size_t)s * (dv + 2) + dv] - M) * l;
  }
  for (int c = threadIdx.x; c < dv; c += blockDim.x) {
    float num = 0.f;
    for (int s = 0; s < n_split; ++s) {
      const float l = base[(size_t)s * (dv + 2) + dv + 1];
      if (l != 0.f) num += exp2f(base[(size_t)s * (dv + 2) + dv] - M) * base[(size_t)s * (dv + 2) + c];
    }
    out[bg * dv + c] = den != 0.f ? num / den : 0.f;
  }
}

}  // namespace

namespace {
// rows per chunk, shared memory (all of it dynamic; `plan` bytes beside barriers and buffers) and CTAs of a launch over
// `chunks(R)` chunks
struct Q4RowsLaunch { int R, smem; unsigned grid; };
template <typename Chunks>
Q4RowsLaunch q4_rows_launch(rap_ctx* ctx, int W, int elem, int plan, Chunks chunks) {
  Q4RowsLaunch l;
  auto bytes = [&](int R) { return plan + Q4R_HEAD + 2 * (q4_buffer(R * W * elem) + q4_buffer(R * 4 * q4_row_words(W))); };
  l.R = q4_rows_per_cta(W, elem);
  // what a launch may take without asking for more (the plan beside 64 bf16 rows of 138 to 144 numbers is over it)
  while (l.R > 8 && bytes(l.R) > 48 * 1024) l.R /= 2;
  while (l.R > 16 && chunks(l.R) < 2 * ctx->sm_count) l.R /= 2;      // small calls: shorter chunks on more SMs
  l.smem = bytes(l.R);
  int fit = (220 * 1024) / (l.smem + 1024);      // CTAs an SM holds, by shared memory and by threads
  if (fit > 2048 / Q4R_THREADS) fit = 2048 / Q4R_THREADS;
  const long long n = chunks(l.R), most = (long long)fit * ctx->sm_count;
  l.grid = (unsigned)(n < most ? n : most);
  return l;
}
}  // namespace

template <typename T>
static rap_status launch_quantize(rap_ctx* ctx, long long n_rows, int W, const void* src, void* dst, cudaStream_t st) {
  const Q4RowsLaunch l = q4_rows_launch(ctx, W, (int)sizeof(T), 0, [&](int R) { return (n_rows + R - 1) / R; });
  auto go = [&](auto kernel) { kernel<<<l.grid, Q4R_THREADS, l.smem, st>>>((const T*)src, (uint32_t*)dst, n_rows, W, l.R, ctx->d_status); };
  auto pick = [&](auto how) {
    constexpr Q4Rows HOW = decltype(how)::value;
    switch ((W + 31) / 32) {
      case 1: go(quantize_rows_q4_kernel<T, 1, HOW>); break;
      case 2: go(quantize_rows_q4_kernel<T, 2, HOW>); break;
      case 3: go(quantize_rows_q4_kernel<T, 3, HOW>); break;
      case 4: go(quantize_rows_q4_kernel<T, 4, HOW>); break;
      case 5: go(quantize_rows_q4_kernel<T, 5, HOW>); break;
      case 6: go(quantize_rows_q4_kernel<T, 6, HOW>); break;
      case 7: go(quantize_rows_q4_kernel<T, 7, HOW>); break;
      default: go(quantize_rows_q4_kernel<T, 8, HOW>);
    }
  };
  if (W % 8 == 0) pick(std::integral_constant<Q4Rows, Q4_VECTORS>{});
  else if (sizeof(T) == 2 && W % 2) pick(std::integral_constant<Q4Rows, Q4_HALVES>{});
  else pick(std::integral_constant<Q4Rows, Q4_WORDS>{});
  ctx->launches++;
  RAP_CUDA_TRY(ctx, cudaGetLastError());
  return RAP_OK;
}

rap_status rap_launch_quantize_rows_q4(rap_ctx* ctx, int32_t dtype_in, long long n_rows, int W, const void* src, void* dst,
                                       cudaStream_t st) {
  return dtype_in == RAP_F32 ? launch_quantize<float>(ctx, n_rows, W, src, dst, st)
                             : launch_quantize<__nv_bfloat16>(ctx, n_rows, W, src, dst, st);
}

template <typename T>
static rap_status launch_dequantize(rap_ctx* ctx, long long n_rows, int W, const void* src, void* dst, cudaStream_t st) {
  const Q4RowsLaunch l = q4_rows_launch(ctx, W, (int)sizeof(T), 0, [&](int R) { return (n_rows + R - 1) / R; });
  auto go = [&](auto kernel) {
    kernel<<<l.grid, Q4R_THREADS, l.smem, st>>>((const uint32_t*)src, (T*)dst, n_rows, W, l.R, ctx->d_status);
  };
  if (W % 8 == 0) go(dequantize_rows_q4_kernel<T, Q4_VECTORS>);
  else if (sizeof(T) == 2 && W % 2) go(dequantize_rows_q4_kernel<T, Q4_HALVES>);
  else go(dequantize_rows_q4_kernel<T, Q4_WORDS>);
  ctx->launches++;
  RAP_CUDA_TRY(ctx, cudaGetLastError());
  return RAP_OK;
}

rap_status rap_launch_dequantize_rows_q4(rap_ctx* ctx, int32_t dtype_out, long long n_rows, int W, const void* src, void* dst,
                                         cudaStream_t st) {
  return dtype_out == RAP_F32 ? launch_dequantize<float>(ctx, n_rows, W, src, dst, st)
                              : launch_dequantize<__nv_bfloat16>(ctx, n_rows, W, src, dst, st);
}

template <typename T>
static rap_status launch_read_cache(rap_ctx* ctx, int B, int Hkv, int S_cap, int P2, int dv, const uint32_t* k4, const uint32_t* v4,
                                    const int32_t* seq_len, int len_max, T* k, T* v, cudaStream_t st) {
  const Q4RowsLaunch l = q4_rows_launch(ctx, P2 > dv ? P2 : dv, (int)sizeof(T), Q4R_PLAN,
                                        [&](int R) { return 2LL * B * Hkv * ((len_max + R - 1) / R); });
  if (2LL * B * Hkv * ((len_max + l.R - 1) / l.R) > 0x7fffffffLL) return RAP_ESHAPE;
  auto go = [&](auto kernel) {
    kernel<<<l.grid, Q4R_THREADS, l.smem, st>>>(k4, v4, k, v, seq_len, B, Hkv, S_cap, P2, dv, len_max, l.R, ctx->d_status);
  };
  auto pick = [&](auto k_how) {      // (K rows are of even length)
    constexpr Q4Rows HOW_K = decltype(k_how)::value;
    if (dv % 8 == 0) go(read_cache_q4_kernel<T, HOW_K, Q4_VECTORS>);
    else if (sizeof(T) == 2 && dv % 2) go(read_cache_q4_kernel<T, HOW_K, Q4_HALVES>);
    else go(read_cache_q4_kernel<T, HOW_K, Q4_WORDS>);
  };
  if (P2 % 8 == 0) pick(std::integral_constant<Q4Rows, Q4_VECTORS>{});
  else pick(std::integral_constant<Q4Rows, Q4_WORDS>{});
  ctx->launches++;
  RAP_CUDA_TRY(ctx, cudaGetLastError());
  return RAP_OK;
}

rap_status rap_launch_read_cache_q4(rap_ctx* ctx, int dtype, int B, int Hkv, int S_cap, int P2, int dv, const void* k4, const void* v4,
                                    const int32_t* seq_len, int len_max, void* k, void* v, cudaStream_t st) {
  for (int b = 0; b < B; b += Q4R_SEQS) {      // (one launch unless the batch is enormous)
    const int n = B - b < Q4R_SEQS ? B - b : Q4R_SEQS;
    const size_t row = (size_t)b * Hkv * S_cap;
    const uint32_t* ks = (const uint32_t*)k4 + row * q4_row_words(P2);
    const uint32_t* vs = (const uint32_t*)v4 + row * q4_row_words(dv);
    const rap_status s =
        dtype == RAP_F32 ? launch_read_cache(ctx, n, Hkv, S_cap, P2, dv, ks, vs, seq_len + b, len_max, (float*)k + row * P2,
                                             (float*)v + row * dv, st)
                         : launch_read_cache(ctx, n, Hkv, S_cap, P2, dv, ks, vs, seq_len + b, len_max, (__nv_bfloat16*)k + row * P2,
                                             (__nv_bfloat16*)v + row * dv, st);
    if (s != RAP_OK) return s;
  }
  return RAP_OK;
}

template <typename T>
static cudaError_t launch_rope_append(const cudaLaunchConfig_t& cfg, rap_ctx* ctx, const rap_proj_args& a, int ksplit) {
  auto go = [&](auto kernel) {
    return cudaLaunchKernelEx(&cfg, kernel, (const float*)ctx->d_proj_ws, ksplit, (const T*)a.bias, a.seq_id, a.pos, a.slot, a.inv_freq,
                              (T*)a.q_out, (uint32_t*)a.k_cache, (uint32_t*)a.v_cache, a.T, a.Hq, a.Hkv, a.P2, a.dv, a.half_dim,
                              a.B_cache, a.S_cap, ctx->d_status);
  };
  auto pick = [&](auto bias) {
    constexpr bool BIAS = decltype(bias)::value;
    const int kp = ((a.P2 > a.dv ? a.P2 : a.dv) + 63) / 64;
    return kp == 1 ? go(rope_append_q4_kernel<T, 1, BIAS>) : kp == 2 ? go(rope_append_q4_kernel<T, 2, BIAS>)
                                                                     : go(rope_append_q4_kernel<T, 4, BIAS>);
  };
  return a.bias ? pick(std::true_type{}) : pick(std::false_type{});
}

// a.k_cache / a.v_cache are the quantised caches of this layer
rap_status rap_launch_qkv_rope_append_q4(rap_ctx* ctx, const rap_proj_args& a, cudaStream_t st) {
  int ksplit = 1;
  rap_status s = RAP_EUNSUPPORTED;
  if (a.dtype == RAP_BF16) s = rap_launch_proj_tc(ctx, a, &ksplit, st);
  if (s == RAP_EUNSUPPORTED) {
    ksplit = 1;
    s = rap_launch_proj_generic(ctx, a, st);
  }
  if (s != RAP_OK) return s;
  if (a.Hkv > 65535) return RAP_ESHAPE;
  // launched behind the library's own GEMM with programmatic serialization, so that its launch overlaps the GEMM's tail (the
  // CUDA-core GEMM never triggers early, which makes the attribute a no-op there)
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)a.T, (unsigned)a.Hkv, 1);
  cfg.blockDim = dim3(32 * (a.Hq / a.Hkv + 2), 1, 1);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  const cudaError_t err = a.dtype == RAP_F32 ? launch_rope_append<float>(cfg, ctx, a, ksplit) : launch_rope_append<__nv_bfloat16>(cfg, ctx, a, ksplit);
  RAP_CUDA_TRY(ctx, err);
  ctx->launches++;
  return RAP_OK;
}

// bf16 q~, rows of up to 128 numbers, any group size: one launch (balanced split) or scan and combine (explicit n_split)
static rap_status launch_attn_q4_scan(rap_ctx* ctx, const rap_attn_args& a, cudaStream_t st) {
  const int G = a.Hq / a.Hkv;
  const rap_q4_entry* e = rap_q4_find(q4_row_words(a.P2), q4_row_words(a.dv), G <= 4 ? 1 : 2);
  if (!e) return RAP_EUNSUPPORTED;
  Q4ScanParams p;
  p.s = rap_fill_scan_params(ctx, a, a.n_split);
  p.P = a.P2 / 2; p.dv = a.dv; p.G = G;
  if (!p.s.balanced && (a.B > 65535 || a.Hkv > 65535)) return RAP_ESHAPE;
  if (ctx->dbg_arm_timeout) {     // test hook: one stage is armed without a copy and polled a few thousand times only
    p.s.wait_limit = 4096;
    p.s.dbg_skip_copy = 1;
    ctx->dbg_arm_timeout = 0;
  }
  RAP_CUDA_TRY(ctx, rap_raise_smem(ctx, e->fn, e->smem));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = p.s.balanced ? dim3(2 * ctx->sm_count) : dim3(p.s.n_split, a.Hkv, a.B);
  cfg.blockDim = dim3(e->threads);
  cfg.dynamicSmemBytes = (size_t)e->smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = a.pdl ? 1 : 0;      // the kernel waits for its predecessor before it reads q~ or a cache row
  void* args[] = {&p};
  RAP_CUDA_TRY(ctx, cudaLaunchKernelExC(&cfg, e->fn, args));
  ctx->launches++;
  if (p.s.balanced) return RAP_OK;
  attn_q4_combine_kernel<<<a.B * a.Hq, 128, 0, st>>>(ctx->d_attn_ws, p.s.n_split, a.dv, a.out);
  ctx->launches++;
  RAP_CUDA_TRY(ctx, cudaGetLastError());
  return RAP_OK;
}

// a.k / a.v are the quantised caches; a.q has the storage dtype
rap_status rap_launch_attn_q4(rap_ctx* ctx, const rap_attn_args& a, cudaStream_t st) {
  if (a.dtype == RAP_BF16 && a.P2 <= 128 && a.dv <= 128 && ctx->attn_variant != 1) return launch_attn_q4_scan(ctx, a, st);
  if (a.B > 65535 || a.Hkv > 65535) return RAP_ESHAPE;
  const int G = a.Hq / a.Hkv;
  int n_split = a.n_split;
  if (n_split <= 0) {      // a few CTAs per SM, splits of at least four tiles
    const int n_tiles = (a.h_len_max + Q4G_TILE - 1) / Q4G_TILE;
    n_split = (8 * ctx->sm_count + a.B * a.Hkv - 1) / (a.B * a.Hkv);
    if (n_split > n_tiles / 4) n_split = n_tiles / 4;
    if (n_split > RAP_MAX_SPLIT) n_split = RAP_MAX_SPLIT;
    if (n_split < 1) n_split = 1;
  }
  const float qscale = (float)(1.4426950408889634 / sqrt((double)a.head_dim));
  const size_t smem = (size_t)(G * a.P2 + G * Q4G_TILE + 2 * G) * sizeof(float);
  dim3 grid(n_split, a.Hkv, a.B);
  if (a.dtype == RAP_F32)
    attn_q4_generic_kernel<float><<<grid, Q4G_THREADS, smem, st>>>((const float*)a.q, (const unsigned char*)a.k,
                                                                   (const unsigned char*)a.v, a.seq_len, a.len_add, a.Hq, a.Hkv,
                                                                   a.P2, a.dv, a.S_cap, qscale, n_split, ctx->d_attn_ws);
  else
    attn_q4_generic_kernel<__nv_bfloat16><<<grid, Q4G_THREADS, smem, st>>>(
        (const __nv_bfloat16*)a.q, (const unsigned char*)a.k, (const unsigned char*)a.v, a.seq_len, a.len_add, a.Hq, a.Hkv, a.P2,
        a.dv, a.S_cap, qscale, n_split, ctx->d_attn_ws);
  ctx->launches++;
  RAP_CUDA_TRY(ctx, cudaGetLastError());
  attn_q4_combine_kernel<<<a.B * a.Hq, 128, 0, st>>>(ctx->d_attn_ws, n_split, a.dv, a.out);
  ctx->launches++;
  RAP_CUDA_TRY(ctx, cudaGetLastError());
  return RAP_OK;
}
