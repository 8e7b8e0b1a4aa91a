// The cache held in 4 bits (format: rap_q4_common.cuh): conversion of rows and of a layer's cache in both directions, the
// RoPE / append epilogue that quantises new K and V rows straight from their fp32 values, and the launch side of the split-KV
// attention over a 4-bit cache: the tensor-core scan (rap_attn_q4_kernel.cuh) for bf16 q~ and rows of up to 128 numbers,
// a shape-generic kernel behind it.
#include "rap_attn_q4_kernel.cuh"

rap_status rap_launch_proj_tc(rap_ctx* ctx, const rap_proj_args& a, int* ksplit_out, cudaStream_t st);
rap_status rap_launch_proj_generic(rap_ctx* ctx, const rap_proj_args& a, cudaStream_t st);

namespace {

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
// Both directions are bound by the bytes they move (W e + row bytes per row each way).  A CTA takes R rows, whose bytes are
// one contiguous range on either side: one bulk copy brings them into shared memory, four threads work on each row from
// there (word k of a row belongs to thread k mod 4), one bulk copy takes the result out.  Row lengths of any parity are an
// affair of the shared memory alone, and eight or more CTAs per SM keep enough bytes in flight.  The last rows' odd bytes
// (a bulk copy moves multiples of 16) go by plain loads and stores.
constexpr int Q4R_STAGE = 18 * 1024;     // target for a CTA's fp32 / bf16 rows; R is a multiple of 8, at most 64

int q4_rows_per_cta(int W, int elem) {
  int r = 64;
  while (r > 8 && r * W * elem > Q4R_STAGE) r /= 2;
  return r;
}
int q4_rows_smem(int W, int elem, int R) { return 16 + (R * W * elem + 31) / 16 * 16 + R * 4 * q4_row_words(W); }

// bytes [0, n) of a 16-byte aligned global range into shared memory; every thread of the CTA calls it.  false: the wait ran out
__device__ __forceinline__ bool q4_bring(unsigned char* dst, const unsigned char* src, int n, uint32_t bar, uint32_t parity, bool again,
                                         int32_t* status) {
  const int bulk = n & ~15;
  if (threadIdx.x == 0) {
    if (!again) {
      mbar_init(bar, 1);
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    mbar_expect_tx(bar, bulk);
    if (bulk) bulk_g2s(smem_u32(dst), src, bulk, bar);
  }
  for (int i = bulk + threadIdx.x; i < n; i += blockDim.x) dst[i] = src[i];
  __syncthreads();
  if (__syncthreads_and(mbar_wait_bounded(bar, parity))) return true;      // one verdict for the CTA
  if (threadIdx.x == 0) {
    atomicCAS(&status[0], 0, (int)RAP_ETIMEOUT);
    status[1] = (int)blockIdx.x;
  }
  return false;
}
// the way out: every thread has written its part of src (shared)
__device__ __forceinline__ void q4_take(unsigned char* dst, const unsigned char* src, int n) {
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  __syncthreads();
  const int bulk = n & ~15;
  if (threadIdx.x == 0 && bulk) {
    asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(dst), "r"(smem_u32(src)), "r"(bulk) : "memory");
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
  }
  for (int i = bulk + threadIdx.x; i < n; i += blockDim.x) dst[i] = src[i];
  if (threadIdx.x == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");     // shared memory is free after this
}

// eight numbers of a row in shared memory, from element `at` on, and the row's extremes so far
template <bool ODD>
__device__ __forceinline__ void q4_eight(const float* base, int at, float (&v)[8], float& hi, float& lo) {
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = base[at + i];
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    hi = q4_max3(hi, v[i], v[i + 1]);
    lo = q4_min3(lo, v[i], v[i + 1]);
  }
}
template <bool ODD>
__device__ __forceinline__ void q4_eight(const __nv_bfloat16* base, int at, float (&v)[8], float& hi, float& lo) {
  // rows of odd length may start on a half word: five words, shifted into place
  const uint32_t* w = reinterpret_cast<const uint32_t*>(base) + (at >> 1);
  uint32_t y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) y[i] = w[i];
  if constexpr (ODD) {
    const uint32_t sh = (at & 1) * 16, last = w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = __funnelshift_r(y[i], i < 3 ? y[i + 1] : last, sh);
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

// WPT: words of codes per thread, four threads a row; ODD: rows of an odd number of bf16 numbers
template <typename T, int WPT, bool ODD>
__global__ void __launch_bounds__(256) quantize_rows_q4_kernel(const T* __restrict__ src, uint32_t* __restrict__ dst,
                                                               long long n_rows, int W, int R, int32_t* __restrict__ status) {
  extern __shared__ __align__(128) unsigned char q4_rows_smem_buf[];
  const int nw = q4_row_words(W);
  unsigned char* in = q4_rows_smem_buf + 16;
  uint32_t* out = reinterpret_cast<uint32_t*>(in + (R * W * (int)sizeof(T) + 31) / 16 * 16);
  const long long row0 = (long long)blockIdx.x * R;
  const int rows = (int)min((long long)R, n_rows - row0);
  if (!q4_bring(in, reinterpret_cast<const unsigned char*>(src + row0 * W), rows * W * (int)sizeof(T), smem_u32(q4_rows_smem_buf), 0, false, status))
    return;
  const int row = threadIdx.x >> 2, q = threadIdx.x & 3;
  // (threads past the last row work on the first one's numbers and store nothing: the shuffles below want whole warps)
  const int at0 = (row < rows ? row : 0) * W;
  const T* x = reinterpret_cast<const T*>(in);
  float v[WPT][8];
  float hi = q4_ld(x + at0), lo = hi;
#pragma unroll
  for (int k = 0; k < WPT; ++k) {
    const int e0 = 8 * (q + 4 * k);
    if (e0 + 8 <= W) {
      q4_eight<ODD>(x, at0 + e0, v[k], hi, lo);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        v[k][i] = q4_ld(x + at0 + (e0 + i < W ? e0 + i : 0));      // past the end: a number of the row, masked below
        hi = q4_max(hi, v[k][i]);
        lo = q4_min(lo, v[k][i]);
      }
    }
  }
#pragma unroll
  for (int o = 1; o < 4; o <<= 1) {
    hi = q4_max(hi, __shfl_xor_sync(0xffffffffu, hi, o));
    lo = q4_min(lo, __shfl_xor_sync(0xffffffffu, lo, o));
  }
  const Q4Row r = q4_decide(hi, lo);
  if (row < rows) {
#pragma unroll
    for (int k = 0; k < WPT; ++k) {
      const int w = q + 4 * k, left = W - 8 * w;       // codes this word holds, at most 8
      if (w < nw - 1) {      // (nw - 1 <= 4 WPT: the padding word is among them)
        uint32_t word = q4_word(v[k], r);
        if (left < 8) word &= left > 0 ? (1u << (4 * left)) - 1u : 0u;
        out[row * nw + w] = word;
      }
    }
    if (q == 0) out[row * nw + nw - 1] = r.sz;
  }
  q4_take(reinterpret_cast<unsigned char*>(dst + row0 * nw), reinterpret_cast<const unsigned char*>(out), rows * nw * 4);
}

__device__ __forceinline__ void q4_put8(float* base, int at, const float (&v)[8], int n) {
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i < n) base[at + i] = v[i];
}
__device__ __forceinline__ void q4_put8(__nv_bfloat16* base, int at, const float (&v)[8], int n) {
  if ((at & 1) == 0 && n >= 8) {
    uint32_t* w = reinterpret_cast<uint32_t*>(base + at);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 y = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&y);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) base[at + i] = __float2bfloat16_rn(v[i]);
  }
}
// `rows` packed rows at src -> numbers at dst, by one CTA.  A CTA may call it again: *turn counts the calls, false: a wait ran out
template <typename T>
__device__ __forceinline__ bool q4_rows_back(const uint32_t* src, T* dst, int rows, int W, int R, int32_t* status, uint32_t* turn) {
  extern __shared__ __align__(128) unsigned char q4_rows_smem_buf[];
  const int nw = q4_row_words(W);
  unsigned char* out = q4_rows_smem_buf + 16;
  unsigned char* in = out + (R * W * (int)sizeof(T) + 31) / 16 * 16;
  if (!q4_bring(in, reinterpret_cast<const unsigned char*>(src), rows * nw * 4, smem_u32(q4_rows_smem_buf), *turn & 1u, *turn > 0, status))
    return false;
  ++*turn;
  const uint32_t* words = reinterpret_cast<const uint32_t*>(in);
  const int row = threadIdx.x >> 2, q = threadIdx.x & 3;
  if (row < rows) {
    const uint32_t sz = words[row * nw + nw - 1];
    const float s = q4_step(sz), z = q4_middle(sz);
    for (int e0 = 8 * q; e0 < W; e0 += 32) {
      const uint32_t word = words[row * nw + (e0 >> 3)];
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        // the code under the exponent of 2^22 (a last place of 1/2), less 2^22 + 7.5
        const uint32_t bits = 0x4a800000u | ((i == 0 ? word << 1 : word >> (4 * i - 1)) & 0x1eu);
        v[i] = fmaf(s, __uint_as_float(bits) - 4194311.5f, z);
      }
      q4_put8(reinterpret_cast<T*>(out), row * W + e0, v, W - e0);
    }
  }
  q4_take(reinterpret_cast<unsigned char*>(dst), out, rows * W * (int)sizeof(T));
  return true;
}

template <typename T>
__global__ void __launch_bounds__(256) dequantize_rows_q4_kernel(const uint32_t* __restrict__ src, T* __restrict__ dst,
                                                                 long long n_rows, int W, int R, int32_t* __restrict__ status) {
  const long long row0 = (long long)blockIdx.x * R;
  uint32_t turn = 0;
  q4_rows_back(src + row0 * q4_row_words(W), dst + row0 * W, (int)min((long long)R, n_rows - row0), W, R, status, &turn);
}

// A layer's K rows and V rows up to every sequence's length.  The chunks of R rows that exist -- per sequence
// (K or V) x KV head x rows -- form one sequence that the CTAs walk through with the grid's stride (a grid over all
// positions spent 15 us on CTAs without rows in a batch of unlike lengths).
template <typename T>
__global__ void __launch_bounds__(256)
read_cache_q4_kernel(const uint32_t* __restrict__ k4, const uint32_t* __restrict__ v4, T* __restrict__ k, T* __restrict__ v,
                     const int32_t* __restrict__ seq_len, int B, int Hkv, int S_cap, int P2, int dv, int len_max, int R,
                     int32_t* __restrict__ status) {
  long long before = 0;        // chunks of the sequences before b
  uint32_t turn = 0;
  int b = 0, len = min(min(seq_len[0], S_cap), len_max), chunks = max(len + R - 1, 0) / R;
  for (long long c = blockIdx.x;; c += gridDim.x) {
    while (c - before >= 2LL * Hkv * chunks) {
      before += 2LL * Hkv * chunks;
      if (++b >= B) return;
      len = min(min(seq_len[b], S_cap), len_max);
      chunks = max(len + R - 1, 0) / R;
    }
    const int unit = (int)((c - before) / chunks), pos = (int)((c - before) - (long long)unit * chunks) * R;
    const bool is_v = unit >= Hkv;
    const size_t row = ((size_t)b * Hkv + unit - (is_v ? Hkv : 0)) * S_cap + pos;
    const int W = is_v ? dv : P2;
    if (!q4_rows_back((is_v ? v4 : k4) + row * q4_row_words(W), (is_v ? v : k) + row * W, min(len - pos, R), W, R, status, &turn)) return;
  }
}

// RoPE / append epilogue with quantisation.  One CTA per (row t, KV head h), one warp per item: the G query heads of h
// (rotated, rounded to the storage dtype, written to q_out as in the unquantised path), its key head (rotated in fp32,
// quantised, appended) and its value head (quantised, appended).  All of them rotate by the same angles, so the sines and
// cosines -- fp64 angle and reduction -- are taken once per CTA (one warp per item on its own: 34 us for 512 rows of the
// 8B-shaped layer, this: 11).  A lane owns pairs of neighbouring numbers, that is whole bytes of a quantised row: P <= 128,
// d_v' <= 256, so at most four.  y holds `ksplit` partial results, each [T][n_out].
template <typename T>
__global__ void __launch_bounds__(32 * (RAP_MAX_GROUP + 2))
rope_append_q4_kernel(const float* __restrict__ y, int ksplit, const T* __restrict__ bias, const int32_t* __restrict__ seq_id,
                      const int32_t* __restrict__ pos, const int32_t* __restrict__ slot, const double* __restrict__ inv_freq,
                      T* __restrict__ q_out, uint32_t* __restrict__ k4, uint32_t* __restrict__ v4, int Trows, int Hq, int Hkv,
                      int P2, int dv, int half_dim, int B_cache, int S_cap, int32_t* __restrict__ status) {
  // launched behind the GEMM with programmatic serialization inside a decode step: nothing above this line touches
  // memory; the GEMM's results (and, through the GEMM, the end of the scan before it) are awaited here
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  __shared__ float2 turn[128];                                         // (cosine, sine) of every pair
  const int t = blockIdx.x / Hkv, h = blockIdx.x - t * Hkv;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int P = P2 >> 1, G = Hq / Hkv;
  const int n_out = (Hq + Hkv) * P2 + Hkv * dv;
  const int p = pos[t];
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
  float a[4], b[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    a[k] = b[k] = 0.f;
    if (64 * k < W) {
      const int c = 2 * (lane + 32 * k);
#pragma unroll 4
      for (int s = 0; s < ksplit; ++s) {                               // the sums in split order
        a[k] += c < W ? yr[s * split_stride + c] : 0.f;
        b[k] += c + 1 < W ? yr[s * split_stride + c + 1] : 0.f;
      }
      if (bias && c < W) a[k] += q4_ld(bias + col0 + c);
      if (bias && c + 1 < W) b[k] += q4_ld(bias + col0 + c + 1);
    }
  }
  for (int c = threadIdx.x; c < P; c += blockDim.x) {
    // fp64 angle and reduction to [-pi, pi], fp32 sine and cosine of the reduced angle (as in the unquantised path)
    const double ang = (double)p * inv_freq[h * half_dim + c];
    const double turns = rint(ang * 0.15915494309189535);
    const double red = fma(-turns, 2.4492935982947064e-16, fma(-turns, 6.283185307179586, ang));
    float sf, cf;
    sincosf((float)red, &sf, &cf);
    turn[c] = make_float2(cf, sf);
  }
  __syncthreads();
  if (!is_v) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int i = lane + 32 * k;
      if (i < P) {
        const float2 cs = turn[i];
        const float x0 = a[k], x1 = b[k];
        a[k] = fmaf(-x1, cs.y, __fmul_rn(x0, cs.x));          // the same roundings as the unquantised kernels
        b[k] = fmaf(x0, cs.y, __fmul_rn(x1, cs.x));
      }
    }
  }
  if (is_q) {
    T* dst = q_out + ((size_t)t * Hq + h * G + warp) * P2;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int i = lane + 32 * k;
      if (i < P) {
        q4_st(dst + 2 * i, a[k]);
        q4_st(dst + 2 * i + 1, b[k]);
      }
    }
    return;
  }
  if (!row_ok) return;
  float hi = -INFINITY, lo = INFINITY;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int c = 2 * (lane + 32 * k);
    if (c < W) { hi = q4_max(hi, a[k]); lo = q4_min(lo, a[k]); }
    if (c + 1 < W) { hi = q4_max(hi, b[k]); lo = q4_min(lo, b[k]); }
  }
  const Q4Row q = q4_decide(warp_max_nan(hi), warp_min_nan(lo));
  const int nw = q4_row_words(W);
  uint32_t* row = (is_v ? v4 : k4) + (((size_t)sq * Hkv + h) * S_cap + sl) * (size_t)nw;
  unsigned char* bytes = reinterpret_cast<unsigned char*>(row);
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int i = lane + 32 * k, c = 2 * i;
    if (c < W) bytes[i] = (unsigned char)(q4_code(a[k], q) | (c + 1 < W ? q4_code(b[k], q) << 4 : 0u));
    else if (i < 4 * (nw - 1)) bytes[i] = 0;
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

template <typename T>
static rap_status launch_quantize(rap_ctx* ctx, long long n_rows, int W, const void* src, void* dst, cudaStream_t st) {
  const int R = q4_rows_per_cta(W, (int)sizeof(T)), smem = q4_rows_smem(W, (int)sizeof(T), R);
  const unsigned blocks = (unsigned)((n_rows + R - 1) / R);
  auto go = [&](auto kernel) { kernel<<<blocks, 4 * R, smem, st>>>((const T*)src, (uint32_t*)dst, n_rows, W, R, ctx->d_status); };
  auto pick = [&](auto odd) {
    constexpr bool ODD = decltype(odd)::value;
    switch ((W + 31) / 32) {
      case 1: go(quantize_rows_q4_kernel<T, 1, ODD>); break;
      case 2: go(quantize_rows_q4_kernel<T, 2, ODD>); break;
      case 3: go(quantize_rows_q4_kernel<T, 3, ODD>); break;
      case 4: go(quantize_rows_q4_kernel<T, 4, ODD>); break;
      default: go(quantize_rows_q4_kernel<T, 8, ODD>);
    }
  };
  if constexpr (sizeof(T) == 2) {
    if (W & 1) pick(std::true_type{});
    else pick(std::false_type{});
  } else {
    pick(std::false_type{});
  }
  ctx->launches++;
  RAP_CUDA_TRY(ctx, cudaGetLastError());
  return RAP_OK;
}

rap_status rap_launch_quantize_rows_q4(rap_ctx* ctx, int32_t dtype_in, long long n_rows, int W, const void* src, void* dst,
                                       cudaStream_t st) {
  return dtype_in == RAP_F32 ? launch_quantize<float>(ctx, n_rows, W, src, dst, st)
                             : launch_quantize<__nv_bfloat16>(ctx, n_rows, W, src, dst, st);
}

rap_status rap_launch_dequantize_rows_q4(rap_ctx* ctx, int32_t dtype_out, long long n_rows, int W, const void* src, void* dst,
                                         cudaStream_t st) {
  const int e = rap_elem_bytes(dtype_out), R = q4_rows_per_cta(W, e), smem = q4_rows_smem(W, e, R);
  const unsigned blocks = (unsigned)((n_rows + R - 1) / R);
  if (dtype_out == RAP_F32)
    dequantize_rows_q4_kernel<float><<<blocks, 4 * R, smem, st>>>((const uint32_t*)src, (float*)dst, n_rows, W, R, ctx->d_status);
  else
    dequantize_rows_q4_kernel<__nv_bfloat16><<<blocks, 4 * R, smem, st>>>((const uint32_t*)src, (__nv_bfloat16*)dst, n_rows, W, R,
                                                                          ctx->d_status);
  ctx->launches++;
  RAP_CUDA_TRY(ctx, cudaGetLastError());
  return RAP_OK;
}

rap_status rap_launch_read_cache_q4(rap_ctx* ctx, int dtype, int B, int Hkv, int S_cap, int P2, int dv, const void* k4, const void* v4,
                                    const int32_t* seq_len, int len_max, void* k, void* v, cudaStream_t st) {
  const int W = P2 > dv ? P2 : dv, e = rap_elem_bytes(dtype), R = q4_rows_per_cta(W, e), smem = q4_rows_smem(W, e, R);
  const long long chunks = 2LL * B * Hkv * ((len_max + R - 1) / R), most = 8LL * ctx->sm_count;      // eight CTAs fit an SM
  const unsigned grid = (unsigned)(chunks < most ? chunks : most);
  if (dtype == RAP_F32)
    read_cache_q4_kernel<float><<<grid, 4 * R, smem, st>>>((const uint32_t*)k4, (const uint32_t*)v4, (float*)k, (float*)v, seq_len, B,
                                                           Hkv, S_cap, P2, dv, len_max, R, ctx->d_status);
  else
    read_cache_q4_kernel<__nv_bfloat16><<<grid, 4 * R, smem, st>>>((const uint32_t*)k4, (const uint32_t*)v4, (__nv_bfloat16*)k,
                                                                   (__nv_bfloat16*)v, seq_len, B, Hkv, S_cap, P2, dv, len_max, R,
                                                                   ctx->d_status);
  ctx->launches++;
  RAP_CUDA_TRY(ctx, cudaGetLastError());
  return RAP_OK;
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
  if ((long long)a.T * a.Hkv > 0x7fffffffLL) return RAP_ESHAPE;
  // inside a decode step (a.pdl): launched behind the tcgen05 GEMM with programmatic serialization, so that its launch
  // overlaps the GEMM's tail (the CUDA-core GEMM never triggers early, which makes the attribute a no-op there)
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(a.T * a.Hkv), 1, 1);
  cfg.blockDim = dim3(32 * (a.Hq / a.Hkv + 2), 1, 1);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = a.pdl ? 1 : 0;
  const float* y = ctx->d_proj_ws;
  uint32_t* k4 = (uint32_t*)a.k_cache;
  uint32_t* v4 = (uint32_t*)a.v_cache;
  if (a.dtype == RAP_F32)
    RAP_CUDA_TRY(ctx, cudaLaunchKernelEx(&cfg, rope_append_q4_kernel<float>, y, ksplit, (const float*)a.bias, a.seq_id, a.pos,
                                         a.slot, a.inv_freq, (float*)a.q_out, k4, v4, a.T, a.Hq, a.Hkv, a.P2, a.dv, a.half_dim,
                                         a.B_cache, a.S_cap, ctx->d_status));
  else
    RAP_CUDA_TRY(ctx, cudaLaunchKernelEx(&cfg, rope_append_q4_kernel<__nv_bfloat16>, y, ksplit, (const __nv_bfloat16*)a.bias,
                                         a.seq_id, a.pos, a.slot, a.inv_freq, (__nv_bfloat16*)a.q_out, k4, v4, a.T, a.Hq, a.Hkv,
                                         a.P2, a.dv, a.half_dim, a.B_cache, a.S_cap, ctx->d_status));
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
