// Attention with a sliding window and sinks (one new token of every sequence, ragged blocks of new tokens), attention over a
// prefix that a group of sequences shares, and the slot maps of ragged batches: launch side, the kernel for every shape and
// type, and the slot-map kernel.  The kernels for bf16 heads of up to 128 dims are in rap_window_scan.cu (one token) and
// rap_window_tc.cu (blocks, shared prefixes).
#include <math.h>

#include "rap_window_common.cuh"

namespace {

constexpr int WG_THREADS = 256;   // >= largest d_v' (head_dim <= 256)
constexpr int WG_TILE = 64;       // cache rows per tile

template <typename T> __device__ __forceinline__ float wg_ld(const T* p);
template <> __device__ __forceinline__ float wg_ld<float>(const float* p) { return *p; }
template <> __device__ __forceinline__ float wg_ld<__nv_bfloat16>(const __nv_bfloat16* p) { return __bfloat162float(*p); }

// Any 2P, d_v' <= 256, G <= 8, fp32 or bf16.  CTA (row, KV head, split): the G query heads of one token over its share of the
// rows that the token sees -- the shared prefix's first, then its own -- tile by tile with a running maximum and sum, all in
// fp32.  Eight lanes compute a row's logits; a thread owns a channel of the output for every n_grp-th row of the tile (256 /
// channels, a power of two), and the groups' sums are added at the end.  Bound by latency at the sizes that fp32 stacks have: a
// tile's loads are all on their way at once (8 sequences of 260 rows, fp32, two KV heads: 12.3 us; 28.7 with a load at a time).  One split writes the output; several leave (accumulators, maximum, sum) for
// win_combine_kernel, which is launched under the scan's tail.
template <typename T>
__global__ void __launch_bounds__(WG_THREADS) win_generic_kernel(const rap_win_args a, float qscale, int n_split, float* __restrict__ ws) {
  extern __shared__ float wg_smem[];
  const int G = a.Hq / a.Hkv, P2 = a.P2, dv = a.dv;
  float* q_s = wg_smem;                    // [G][P2], scaled by log2(e) / sqrt(D)
  float* s_s = q_s + G * P2;               // [G][WG_TILE]
  float* alpha_s = s_s + G * WG_TILE;      // [G]
  float* l_s = alpha_s + G;                // [G]
  float* red = l_s + G;                    // [n_grp - 1][dv] of one head
  const int row = blockIdx.x, h = blockIdx.y, split = blockIdx.z;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

  int b = row, len;
  if (a.row_start) {
    if (row >= a.row_start[a.B]) return;                        // behind the last sequence: left as it was
    b = win_owner(a.row_start, a.B, row);
    if (b >= a.B) return;
    len = a.seq_len[b] - (a.row_start[b + 1] - row) + 1;       // positions up to this token's own
  } else {
    len = a.seq_len[b];
  }
  if (a.n_groups) len = min(len, a.S_cap);
  const WinRuns w = win_runs(len, a.n_sink, a.window, a.S_cap);
  int pre = 0;
  const T *kp = nullptr, *vp = nullptr;
  if (a.n_groups) {
    const int g = win_owner(a.group_start, a.n_groups, b);
    if (g < a.n_groups && a.group_start[g] <= b) {
      pre = min(max(a.prefix_len[g], 0), a.S_pre);
      kp = (const T*)a.kp + ((size_t)g * a.Hkv + h) * (size_t)a.S_pre * P2;
      vp = (const T*)a.vp + ((size_t)g * a.Hkv + h) * (size_t)a.S_pre * dv;
    }
  }
  const T* kc = (const T*)a.k + ((size_t)b * a.Hkv + h) * (size_t)a.S_cap * P2;
  const T* vc = (const T*)a.v + ((size_t)b * a.Hkv + h) * (size_t)a.S_cap * dv;
  const int e0 = w.n[0], e1 = e0 + w.n[1], own = e1 + w.n[2];
  const long long total = (long long)pre + own;
  auto cache_row = [&](int j) { return j < e0 ? w.lo[0] + j : j < e1 ? w.lo[1] + j - e0 : w.lo[2] + j - e1; };
  const long long per = ((total + n_split - 1) / n_split + WG_TILE - 1) / WG_TILE * WG_TILE;
  const long long v0 = min(total, split * per), v1 = min(total, v0 + per);

  for (int i = tid; i < G * P2; i += WG_THREADS)
    q_s[i] = wg_ld<T>((const T*)a.q + ((size_t)row * a.Hq + h * G) * P2 + i) * qscale;
  // V: thread (grp, ch)
  const int w_log = dv <= 32 ? 5 : dv <= 64 ? 6 : dv <= 128 ? 7 : 8, n_grp = WG_THREADS >> w_log;
  const int ch = tid & ((1 << w_log) - 1), grp = tid >> w_log;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  float m_run = -INFINITY, l_run = 0.f;    // warp g < G, the same in every lane
  float acc[RAP_MAX_GROUP];
#pragma unroll
  for (int g = 0; g < RAP_MAX_GROUP; ++g) acc[g] = 0.f;
  __syncthreads();

  for (long long j0 = v0; j0 < v1; j0 += WG_TILE) {
    const int nj = (int)min((long long)WG_TILE, v1 - j0);
#pragma unroll 2
    for (int j = tid >> 3; j < WG_TILE; j += WG_THREADS / 8) {
      const int l8 = lane & 7;
      const long long v = j0 + min(j, nj - 1);
      const T* kr = v < pre ? kp + (size_t)v * P2 : kc + (size_t)cache_row((int)(v - pre)) * P2;
      float part[RAP_MAX_GROUP];
#pragma unroll
      for (int g = 0; g < RAP_MAX_GROUP; ++g) part[g] = 0.f;
#pragma unroll 4
      for (int d = l8; d < P2; d += 8) {
        const float kv = wg_ld<T>(kr + d);
#pragma unroll
        for (int g = 0; g < RAP_MAX_GROUP; ++g)
          if (g < G) part[g] = fmaf(kv, q_s[g * P2 + d], part[g]);
      }
#pragma unroll
      for (int g = 0; g < RAP_MAX_GROUP; ++g) {
        if (g < G) {
          float s = part[g];
#pragma unroll
          for (int o = 4; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
          if (l8 == 0) s_s[g * WG_TILE + j] = s;
        }
      }
    }
    __syncthreads();
    if (warp < G) {       // running maximum and sum: warp g owns head g
      const int g = warp;
      float mx = -INFINITY;
      for (int j = lane; j < nj; j += 32) mx = fmaxf(mx, s_s[g * WG_TILE + j]);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
      const float m_new = fmaxf(m_run, mx), ref = m_new == -INFINITY ? 0.f : m_new;
      float sum = 0.f;
      for (int j = lane; j < nj; j += 32) {
        const float p = exp2f(s_s[g * WG_TILE + j] - ref);
        s_s[g * WG_TILE + j] = p;
        sum += p;
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
      const float alpha = exp2f(m_run - ref);      // first tile: 2^(-inf) = 0
      l_run = l_run * alpha + sum;
      m_run = m_new;
      if (lane == 0) alpha_s[g] = alpha;
    }
    __syncthreads();
    if (ch < dv) {
#pragma unroll
      for (int g = 0; g < RAP_MAX_GROUP; ++g)
        if (g < G) acc[g] *= alpha_s[g];
#pragma unroll 4
      for (int j = grp; j < nj; j += n_grp) {
        const long long v = j0 + j;
        const float vv = wg_ld<T>((v < pre ? vp + (size_t)v * dv : vc + (size_t)cache_row((int)(v - pre)) * dv) + ch);
#pragma unroll
        for (int g = 0; g < RAP_MAX_GROUP; ++g)
          if (g < G) acc[g] = fmaf(s_s[g * WG_TILE + j], vv, acc[g]);
      }
    }
    __syncthreads();
  }
  if (n_grp > 1) {       // the groups' sums, one head at a time
#pragma unroll
    for (int g = 0; g < RAP_MAX_GROUP; ++g) {
      if (g < G) {
        if (grp > 0 && ch < dv) red[(grp - 1) * dv + ch] = acc[g];
        __syncthreads();
        if (grp == 0 && ch < dv)
          for (int i = 1; i < n_grp; ++i) acc[g] += red[(i - 1) * dv + ch];
        __syncthreads();
      }
    }
  }
  if (n_split == 1) {
    if (warp < G && lane == 0) l_s[warp] = l_run;
    __syncthreads();
#pragma unroll
    for (int g = 0; g < RAP_MAX_GROUP; ++g)
      if (g < G && tid < dv) a.out[((size_t)row * a.Hq + h * G + g) * dv + tid] = l_s[g] != 0.f ? acc[g] / l_s[g] : 0.f;
    return;
  }
#pragma unroll
  for (int g = 0; g < RAP_MAX_GROUP; ++g) {
    if (g < G) {
      float* dst = ws + (((size_t)row * a.Hq + h * G + g) * n_split + split) * (size_t)(dv + 2);
      if (tid < dv) dst[tid] = acc[g];
      if (warp == g && lane == 0) {
        dst[dv] = m_run;
        dst[dv + 1] = l_run;
      }
    }
  }
}

// out = sum_s 2^(m_s - M) acc_s / sum_s 2^(m_s - M) l_s over the splits of one query head (an empty split has l = 0)
__global__ void __launch_bounds__(128) win_combine_kernel(const float* __restrict__ ws, int n_split, int dv, float* __restrict__ out) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const float* base = ws + (size_t)blockIdx.x * n_split * (size_t)(dv + 2);
  float M = -INFINITY, den = 0.f;
  for (int s = 0; s < n_split; ++s)
    if (base[(size_t)s * (dv + 2) + dv + 1] != 0.f) M = fmaxf(M, base[(size_t)s * (dv + 2) + dv]);
  for (int s = 0; s < n_split; ++s) {
    const float l = base[(size_t)s * (dv + 2) + dv + 1];
    if (l != 0.f) den += exp2f(base[(size_t)s * (dv + 2) + dv] - M) * l;
  }
  for (int c = threadIdx.x; c < dv; c += blockDim.x) {
    float num = 0.f;
    for (int s = 0; s < n_split; ++s)
      if (base[(size_t)s * (dv + 2) + dv + 1] != 0.f) num += exp2f(base[(size_t)s * (dv + 2) + dv] - M) * base[(size_t)s * (dv + 2) + c];
    out[(size_t)blockIdx.x * dv + c] = den != 0.f ? num / den : 0.f;
  }
}

rap_status launch_generic(rap_ctx* ctx, const rap_win_args& a, cudaStream_t st) {
  if (a.Hkv > 65535) return RAP_ESHAPE;      // grid.y
  const int G = a.Hq / a.Hkv;
  int n_split = 1;
  if (!a.row_start) {   // one token a sequence: split the rows until the SMs are busy, a tile at least in each
    const long long rows = (a.n_groups ? (long long)a.h_prefix_max + a.h_len_max : 0) +
                           (a.n_groups ? 0 : (long long)(a.h_len_max < a.window ? a.h_len_max : a.window) + a.n_sink);
    const long long tiles = (rows + WG_TILE - 1) / WG_TILE, units = (long long)a.T * a.Hkv;
    long long ns = (8LL * ctx->sm_count + units - 1) / units;
    ns = ns > tiles ? tiles : ns;
    n_split = (int)(ns > RAP_MAX_SPLIT ? RAP_MAX_SPLIT : ns < 1 ? 1 : ns);
  }
  const float qscale = (float)(1.4426950408889634 / sqrt((double)a.head_dim));
  const size_t smem = (size_t)(G * a.P2 + G * WG_TILE + 2 * G + WG_THREADS) * sizeof(float);
  const dim3 grid(a.T, a.Hkv, n_split);
  if (a.dtype == RAP_F32) win_generic_kernel<float><<<grid, WG_THREADS, smem, st>>>(a, qscale, n_split, ctx->d_attn_ws);
  else win_generic_kernel<__nv_bfloat16><<<grid, WG_THREADS, smem, st>>>(a, qscale, n_split, ctx->d_attn_ws);
  ctx->launches++;
  RAP_CUDA_TRY(ctx, cudaGetLastError());
  if (n_split > 1) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(a.T * a.Hq);
    cfg.blockDim = dim3(128);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    RAP_CUDA_TRY(ctx, cudaLaunchKernelEx(&cfg, win_combine_kernel, (const float*)ctx->d_attn_ws, n_split, a.dv, a.out));
    ctx->launches++;
    RAP_CUDA_TRY(ctx, cudaGetLastError());
  }
  return RAP_OK;
}

// ---- slot maps ----------------------------------------------------------------------------------------------------------------
// Every CTA walks all sequences, SL_THREADS at a time: a block-wide prefix sum of the new tokens gives their first rows, and
// the CTA's share of the rows finds its sequence by bisection in that piece.  Bound by a launch and a few dependent loads: 12
// bytes a row are written.  Lengths that are advanced in place are written by the CTA that comes last (a counter, zero again
// afterwards), when all have read them.
constexpr int SL_THREADS = 512;
__global__ void __launch_bounds__(SL_THREADS) build_slots_kernel(int B, const int32_t* seq_len, const int32_t* __restrict__ new_len,
                                                                 const int32_t* __restrict__ pos_base, int T, int n_sink, int S_cap,
                                                                 int32_t* __restrict__ row_start, int32_t* __restrict__ seq_id,
                                                                 int32_t* __restrict__ pos, int32_t* __restrict__ slot, int32_t* len_out,
                                                                 int32_t* ticket, int32_t* status) {
  __shared__ long long start_s[SL_THREADS + 1];
  __shared__ int past_s[SL_THREADS], base_s[SL_THREADS];
  __shared__ long long warp_s[SL_THREADS / 32];
  __shared__ int last_s;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const long long per = ((long long)T + gridDim.x - 1) / gridDim.x;
  const long long r0 = per * blockIdx.x, r1 = min((long long)T, r0 + per);
  const bool first_cta = blockIdx.x == 0;
  long long carry = 0;
  for (int b0 = 0; b0 < B; b0 += SL_THREADS) {
    const int b = b0 + tid, nb = min(SL_THREADS, B - b0);
    int past = 0, fresh = 0, base = 0;
    if (b < B) {
      past = seq_len[b];
      fresh = new_len[b];
      if (pos_base) base = pos_base[b];
      if (first_cta && (past < 0 || fresh < 0 || base < 0)) win_report(status, RAP_EINVAL, b);
      past = max(past, 0);
      fresh = max(fresh, 0);
      base = max(base, 0);
      if (first_cta && (long long)past + fresh > 0x7fffffffLL) win_report(status, RAP_EINVAL, b);
    }
    long long x = fresh;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long y = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += y;
    }
    if (lane == 31) warp_s[warp] = x;
    __syncthreads();
    if (warp == 0) {
      long long v = lane < SL_THREADS / 32 ? warp_s[lane] : 0;
#pragma unroll
      for (int o = 1; o < SL_THREADS / 32; o <<= 1) {
        const long long y = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += y;
      }
      if (lane < SL_THREADS / 32) warp_s[lane] = v;
    }
    __syncthreads();
    const long long end = carry + x + (warp > 0 ? warp_s[warp - 1] : 0);      // rows up to and including this sequence
    start_s[tid + 1] = end;
    if (tid == 0) start_s[0] = carry;
    past_s[tid] = past;
    base_s[tid] = base;
    __syncthreads();
    if (first_cta && b < B) {
      row_start[b + 1] = (int32_t)min(end, (long long)T);
      if (len_out && len_out != seq_len) len_out[b] = (int32_t)min((long long)past + fresh, 0x7fffffffLL);
      if (end > T) win_report(status, RAP_ECAPACITY, b);
      const long long rolled = (long long)past + fresh - max(past, n_sink);     // new tokens behind the sinks
      if (rolled > S_cap - n_sink) win_report(status, RAP_ECAPACITY, b);
    }
    const long long lo = max(r0, carry), hi = min(r1, start_s[nb]);
    for (long long r = lo + tid; r < hi; r += SL_THREADS) {
      int s = 0, e = nb - 1;                       // smallest s with start_s[s + 1] > r
      while (s < e) {
        const int mid = (s + e) >> 1;
        if (start_s[mid + 1] > r) e = mid; else s = mid + 1;
      }
      const long long p = past_s[s] + (r - start_s[s]), q = p + base_s[s];
      if (q > 0x7fffffffLL) {
        win_report(status, RAP_EINVAL, b0 + s);
        continue;
      }
      const long long n_end = past_s[s] + (start_s[s + 1] - start_s[s]);
      const bool taken = p >= n_sink && p + (S_cap - n_sink) < n_end;           // a later new token takes this row
      seq_id[r] = b0 + s;
      pos[r] = (int32_t)q;
      slot[r] = taken ? -1 : win_slot((int)p, n_sink, S_cap);
    }
    carry = start_s[nb];
    __syncthreads();
  }
  if (first_cta && tid == 0) row_start[0] = 0;
  if (!len_out || len_out != seq_len) return;
  if (tid == 0) {
    last_s = 1;
    if (gridDim.x > 1) {
      __threadfence();                             // this CTA's reads of the lengths are done (barrier above)
      last_s = atomicAdd(ticket, 1) == (int)gridDim.x - 1;
      if (last_s) *ticket = 0;
    }
  }
  __syncthreads();
  if (last_s)
    for (int b = tid; b < B; b += SL_THREADS)
      len_out[b] = (int32_t)min((long long)max(seq_len[b], 0) + max(new_len[b], 0), 0x7fffffffLL);
}

}  // namespace

rap_status rap_launch_build_slots(rap_ctx* ctx, int B, const int32_t* seq_len, const int32_t* new_len, const int32_t* pos_base, int T,
                                  int n_sink, int S_cap, int32_t* row_start, int32_t* seq_id, int32_t* pos, int32_t* slot,
                                  int32_t* len_out, cudaStream_t st) {
  // two rows a thread: more CTAs read the lengths again, fewer write longer (9400 rows of 64 sequences: 5.2 us with 2048 rows a
  // CTA and a counter, 3.4 as it is)
  const int ctas = (int)(((long long)T + 1023) / 1024);
  const int grid = ctas < 1 ? 1 : ctas > 2 * ctx->sm_count ? 2 * ctx->sm_count : ctas;
  int32_t* ticket = ctx->d_win_cnt + 2 * (size_t)ctx->desc.max_batch * ctx->desc.n_kv_heads;
  build_slots_kernel<<<grid, SL_THREADS, 0, st>>>(B, seq_len, new_len, pos_base, T, n_sink, S_cap, row_start, seq_id, pos, slot, len_out,
                                                  ticket, ctx->d_status);
  ctx->launches++;
  RAP_CUDA_TRY(ctx, cudaGetLastError());
  return RAP_OK;
}

rap_status rap_launch_decode_window(rap_ctx* ctx, const rap_win_args& a, cudaStream_t st) {
  return rap_win_scan_takes(a) ? rap_launch_win_scan(ctx, a, 0, st) : launch_generic(ctx, a, st);
}
rap_status rap_launch_prefill_window(rap_ctx* ctx, const rap_win_args& a, cudaStream_t st) {
  return rap_win_tc_takes(a) ? rap_launch_win_tc(ctx, a, st) : launch_generic(ctx, a, st);
}
rap_status rap_launch_decode_shared(rap_ctx* ctx, const rap_win_args& a, cudaStream_t st) {
  if (!rap_win_tc_takes(a) || !rap_win_scan_takes(a)) return launch_generic(ctx, a, st);
  int n_pre = 0;
  const rap_status s = rap_launch_win_prefix(ctx, a, &n_pre, st);
  return s == RAP_OK ? rap_launch_win_scan(ctx, a, n_pre, st) : s;
}
