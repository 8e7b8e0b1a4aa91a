// Launch side of win_scan_kernel (rap_window_scan_kernel.cuh).
#include "rap_window_scan_kernel.cuh"

const void* rap_win_scan_long_fn(int G, bool vodd, bool tma, int n, int nw);      // rap_window_scan_long.cu

namespace {

// About how many blocks of a unit one warp can get, from what the host knows: every unit as long as the bounds allow
long long most_blocks(const WsParams& p, const rap_win_args& a, int n_pre, int grid, int nw) {
  const long long rows = a.n_groups ? a.h_len_max : (long long)(a.h_len_max < a.window ? a.h_len_max : a.window) + a.n_sink;
  const long long n = (rows + 31) / 32 + 3, units = (long long)a.B * a.Hkv;      // a run begins and ends inside a block
  const long long share = units < grid ? n / (grid / units) : n;                  // by units of a size ...
  const long long least = n / (RAP_MAX_SPLIT - n_pre - 3);                        // ... and for all partials to have places
  const long long cta = (share > least ? share : least) + 2;
  return ((cta < n ? cta : n) + nw - 1) / nw;
}

// what a unit's end takes, in blocks of half a microsecond: 3 us, or 10 with a prefix's splits to join
int unit_end(int n_pre) { return n_pre ? 20 : 6; }

}  // namespace

rap_status rap_debug_window_plan(int32_t sm_count, int32_t B, int32_t n_kv_heads, const int32_t* h_blocks, int32_t n_pre, int32_t padded,
                                 int32_t* most, int32_t* places) {
  if (!h_blocks || !most || !places || sm_count < 1 || B < 1 || n_kv_heads < 1 || n_pre < 0 || n_pre > WIN_MAX_PRE) return RAP_EINVAL;
  const int own = unit_end(n_pre);
  long long T = 0;
  int n_max = 1;
  for (int b = 0; b < B; ++b) {
    if (h_blocks[b] < 1 || h_blocks[b] > (1 << 26)) return RAP_EINVAL;      // 2^31 rows
    T += (long long)(h_blocks[b] + own) * n_kv_heads;
    if (h_blocks[b] + own > n_max) n_max = h_blocks[b] + own;
  }
  if (T > 0x7fffffffLL) return RAP_EINVAL;
  const WinScanPlan plan = win_scan_plan((int)T, n_max, B * n_kv_heads, 2 * sm_count, own, n_pre, padded != 0);
  *most = 0;
  *places = RAP_MAX_SPLIT - n_pre;
  for (int b = 0, start = 0; b < B; ++b)
    for (int h = 0; h < n_kv_heads; ++h, start += h_blocks[b] + own) {
      const int first = plan.cta_of(start + own), last = plan.cta_of(start + own + h_blocks[b] - 1);
      const int n = plan.even ? (h_blocks[b] < plan.parts ? h_blocks[b] : plan.parts) : last - first + 1;
      if (n > *most) *most = n;
    }
  return RAP_OK;
}

bool rap_win_scan_takes(const rap_win_args& a) {
  return a.dtype == RAP_BF16 && a.P2 >= 16 && a.P2 <= 128 && a.dv >= 16 && a.dv <= 128;
}

// n_pre: the most partials of a shared prefix that the launch before leaves for a head (0: none)
rap_status rap_launch_win_scan(rap_ctx* ctx, const rap_win_args& a, int n_pre, cudaStream_t st) {
  WsParams p = {};
  p.q = (const uint32_t*)a.q; p.k = (const unsigned char*)a.k; p.v = (const unsigned char*)a.v; p.seq_len = a.seq_len;
  p.out = a.out; p.ws = win_partials(ctx->d_attn_ws, (long long)a.B * a.Hq, a.Hq / a.Hkv, a.dv, n_pre); p.ws_floats = (long long)(ctx->attn_ws_bytes / sizeof(float)); p.status = ctx->d_status;
  p.B = a.B; p.Hq = a.Hq; p.Hkv = a.Hkv; p.G = a.Hq / a.Hkv; p.P = a.P2 / 2; p.dv = a.dv; p.S_cap = a.S_cap;
  p.n_sink = a.n_sink; p.window = a.window; p.len_cap = a.n_groups ? a.S_cap : 0x7fffffff;
  p.qscale = (float)(1.4426950408889634 / sqrt((double)a.head_dim));
  p.n_groups = a.n_groups; p.group_start = a.group_start; p.prefix_len = a.prefix_len; p.S_pre = a.S_pre; p.sms = ctx->sm_count;
  p.wait_limit = WAIT_LIMIT;
  p.own = unit_end(n_pre);
  if (ctx->dbg_arm_timeout) {        // test hook (rap_debug_arm_wait_timeout)
    p.wait_limit = 4096;
    p.dbg_skip_copy = 1;
    ctx->dbg_arm_timeout = 0;
  }
  if (ctx->dbg_arm_join) {           // test hook (rap_debug_arm_join_timeout)
    p.wait_limit = 4096;
    p.dbg_lost_bytes = 16;
    ctx->dbg_arm_join = 0;
  }
  {   // two sets of counters take turns; each launch clears the one its predecessor used
    const size_t n_units = (size_t)ctx->desc.max_batch * ctx->desc.n_kv_heads;
    const uint32_t set = ctx->win_epoch++ & 1u;
    if (a.B * a.Hkv > ctx->win_units) ctx->win_units = a.B * a.Hkv;
    p.other_units = ctx->win_units;
    p.unit_cnt = ctx->d_win_cnt + set * n_units;
    p.unit_cnt_other = ctx->d_win_cnt + (set ^ 1u) * n_units;
  }
  const int k_row = 2 * a.P2, v_row = 2 * a.dv;
  const bool vodd = (a.dv & 1) != 0;
  const long long cache_rows = (long long)a.B * a.Hkv * a.S_cap;
  const bool tma = k_row == v_row && (k_row == 128 || k_row == 256) && cache_rows < (1LL << 31);       // rows are the maps' y
  p.pad16 = (!tma && k_row % 16 == 0 && v_row % 16 == 0) ? 1 : 0;
  if (p.pad16) {
    // 16 bytes more where a row is an even number of 16-byte units: then eight rows start on different banks
    p.k_stride = k_row + (k_row % 32 == 0 ? 16 : 0);
    p.v_stride = v_row + (v_row % 32 == 0 ? 16 : 0);
    p.rs_log = 0;
  } else {
    p.k_stride = k_row;
    p.v_stride = v_row;
    // the eight rows of a fragment 4, 2 or 1 apart: P words a row times the step = 4 * odd puts them on different banks; odd
    // d_v' wants the two rows of a register to be of one parity
    p.rs_log = (p.P & 1) ? 2 : (p.P & 2) ? 1 : vodd ? 1 : 0;      // (tensor maps: rows 0-7 of a fragment in order)
  }
  p.stage_bytes = tma ? 32 * (p.k_stride + p.v_stride) : (32 * (p.k_stride + p.v_stride) + 16 + 127) / 128 * 128;
  const int cw = (vodd ? a.dv + 1 : a.dv);
  // two CTAs an SM; four warps with two stages each where they fit (up to 13 KB a stage), else three
  const int nk = (p.P + 7) / 8, nv = (a.dv + 15) / 16, n = nk > nv ? nk : nv;
  int nw = n == 8 ? 3 : 4, smem = 0;
  for (;; --nw) {
    const int red = nw * p.G * cw * 4, join = p.G * RAP_MAX_SPLIT * 4;
    const int unit = tma ? 1024 : 128;
    p.off_stage = (512 + (red > join ? red : join) + unit - 1) / unit * unit;
    smem = p.off_stage + nw * WS_STAGES * p.stage_bytes + (tma ? 1024 : 0);
    p.join_places = nw * WS_STAGES * p.stage_bytes / (4 * p.G * p.ws.dv4);      // partials that fit the stages
    if (smem <= SMEM_BUDGET || nw == 2) break;
  }
  const bool sums_long = most_blocks(p, a, n_pre, 2 * ctx->sm_count, nw) > WS_LONG;
  const void* fn = sums_long ? rap_win_scan_long_fn(p.G, vodd, tma, n, nw) : scan_any<false>(p.G, vodd, tma, n, nw);
  alignas(64) unsigned char map_k[128] = {0}, map_v[128] = {0};      // CUtensorMap images (the other forms ignore them)
  if (tma) {
    if (!rap_tensor_map_bf16(ctx, map_k, a.k, (uint64_t)cache_rows, (uint64_t)a.P2, 32) ||
        !rap_tensor_map_bf16(ctx, map_v, a.v, (uint64_t)cache_rows, (uint64_t)a.dv, 32))
      return RAP_EUNSUPPORTED;
  }
  if (!fn || smem > SMEM_BUDGET) return RAP_EUNSUPPORTED;
  RAP_CUDA_TRY(ctx, rap_raise_smem(ctx, fn, SMEM_BUDGET));
  void* args[] = {&p, map_k, map_v};
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(2 * ctx->sm_count);
  cfg.blockDim = dim3(32 * nw);
  cfg.dynamicSmemBytes = (size_t)smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = n_pre ? 1 : 0;      // behind the prefix's launch: it scans the sequences' own rows meanwhile and waits for it before joining
  RAP_CUDA_TRY(ctx, cudaLaunchKernelExC(&cfg, fn, args));
  ctx->launches++;
  RAP_CUDA_TRY(ctx, cudaGetLastError());
  return RAP_OK;
}
