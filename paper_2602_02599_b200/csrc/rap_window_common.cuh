// Which cache rows a query sees: a window, a few first positions that stay visible (sinks), whole or rolling caches.
#pragma once
#include "rap_internal.h"

namespace {

// Rows of one cache that a single query sees, as at most three runs of consecutive rows: the sinks, and the window behind
// them, which a rolling cache may wrap once.  Position p lies in row p for p < n_sink, else n_sink + (p - n_sink) mod R with
// R = S_cap - n_sink >= 1, so for any length every row is inside the cache.
struct WinRuns {
  int lo[3], n[3];
};
__device__ __forceinline__ WinRuns win_runs(int len, int n_sink, int window, int S_cap) {
  WinRuns w;
  len = max(len, 0);
  const int R = S_cap - n_sink;
  w.lo[0] = 0;
  w.n[0] = min(n_sink, len);
  const int n = min(len - max(n_sink, len - window), R);       // positions [len - n, len) behind the sinks
  w.lo[1] = n_sink;
  w.n[1] = w.lo[2] = w.n[2] = 0;
  if (n > 0) {
    const int a = len <= S_cap ? len - n : n_sink + (len - n - n_sink) % R;
    w.lo[1] = a;
    w.n[1] = min(n, S_cap - a);
    w.lo[2] = n_sink;
    w.n[2] = n - w.n[1];
    if (a == w.n[0]) {                                          // the window begins right behind the sinks: one run
      w.lo[1] = 0;
      w.n[1] += w.n[0];
      w.n[0] = 0;
    }
  }
  return w;
}
__device__ __forceinline__ int win_slot(int pos, int n_sink, int S_cap) { return pos < n_sink ? pos : n_sink + (pos - n_sink) % (S_cap - n_sink); }

// first b in [0, n) whose range [start[b], start[b + 1]) ends behind r, or n: the sequence of row r, the group of sequence r
__device__ __forceinline__ int win_owner(const int32_t* start, int n, int r) {
  int lo = 0, hi = n;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (start[mid + 1] > r) hi = mid; else lo = mid + 1;
  }
  return lo;
}

// Partials in the context's workspace: d_v' sums (dv4: a multiple of four), and (maximum, weight) pairs apart from them.  The
// own rows' lie by unit (sequence, KV head): RAP_MAX_SPLIT - n_pre places, each of the unit's G query heads.  A shared prefix's
// lie ahead of them split by split over all heads, n_pre times (a CTA writes one split of 256 neighbouring rows).  The sums of
// one place or split of a unit are one run of G * dv4 floats.
struct WinPartials {
  float* pre;          // [n_pre][heads][dv4], then [n_pre][heads][2]
  float* own;          // [units][slots][G][dv4], then [units][slots][G][2]
  long long heads;     // B * H_q
  int dv4, n_pre, slots, G;
  __device__ __forceinline__ float* pre_sums(long long head, int s) const { return pre + (s * heads + head) * dv4; }
  __device__ __forceinline__ float2* pre_pair(long long head, int s) const { return reinterpret_cast<float2*>(pre + n_pre * heads * dv4) + s * heads + head; }
  __device__ __forceinline__ float* own_sums(long long unit, int s) const { return own + (unit * slots + s) * (long long)(G * dv4); }
  __device__ __forceinline__ float2* own_pair(long long unit, int s) const { return reinterpret_cast<float2*>(own + heads * slots * dv4) + (unit * slots + s) * G; }
};
static inline WinPartials win_partials(float* ws, long long heads, int G, int dv, int n_pre) {
  WinPartials w;
  w.heads = heads; w.G = G; w.dv4 = (dv + 3) & ~3; w.n_pre = n_pre; w.slots = RAP_MAX_SPLIT - n_pre;
  w.pre = ws;
  w.own = ws + ((n_pre * heads * (w.dv4 + 2) + 3) & ~3LL);      // 16-byte aligned
  return w;
}

// How the prefixes' tiles of 64 rows are shared by the SMs: a (group, 256 rows, KV head) of n tiles takes ceil(n / per) CTAs,
// `per` tiles each.  With fewer such pieces than half the SMs one wave of CTAs holds everything (sum of ceil(n / per) <= all
// tiles / per + pieces); with more, four waves' worth of at least 16 tiles even out what the pieces differ by.  Every warp
// that calls it gets the same answer.
constexpr int WIN_MAX_PRE = 40;      // most splits of a prefix: the own rows keep RAP_MAX_SPLIT - 40 places
struct WinPrefixPlan {
  int per;             // tiles of a split
};
__device__ __forceinline__ int win_group_rows(const int32_t* start, int g, int B, int G) {
  const int s0 = min(max(start[g], 0), B), s1 = min(max(start[g + 1], s0), B);
  return (s1 - s0) * G;
}
__device__ __forceinline__ int win_group_tiles(const int32_t* len, int g, int S_cap) { return (min(max(len[g], 0), S_cap) + 63) >> 6; }
__device__ __forceinline__ WinPrefixPlan win_prefix_plan(const int32_t* start, const int32_t* len, int n_groups, int B, int G, int Hkv, int S_cap,
                                                         int sms, int n_pre) {
  const int lane = threadIdx.x & 31;
  int pieces = 0, most = 0;
  long long all = 0;
  for (int g0 = 0; g0 < n_groups; g0 += 32) {
    const int g = g0 + lane;
    int blocks = 0, tiles = 0;
    if (g < n_groups) {
      tiles = win_group_tiles(len, g, S_cap);
      blocks = tiles ? (win_group_rows(start, g, B, G) + 255) >> 8 : 0;
    }
    pieces += __reduce_add_sync(0xffffffffu, blocks);
    most = max(most, __reduce_max_sync(0xffffffffu, blocks ? tiles : 0));
    // tiles * blocks < 2^31 in a lane: a cache's rows and a batch's rows fit a GPU together
    const int lo = (tiles * blocks) & 0xffff, hi = (tiles * blocks) >> 16;
    all += __reduce_add_sync(0xffffffffu, lo) + ((long long)__reduce_add_sync(0xffffffffu, hi) << 16);
  }
  pieces *= Hkv;
  all *= Hkv;
  WinPrefixPlan pl;
  long long per = 2 * pieces <= sms ? (all + sms - pieces - 1) / (sms - pieces) : max(16LL, (all + 4 * sms - 1) / (4 * sms));
  per = max(per, (long long)(most + n_pre - 1) / n_pre);
  pl.per = (int)max(1LL, min(per, 0x7fffffffLL));
  return pl;
}

// How the one-token scan shares its blocks of 32 rows among the CTAs.  A unit (sequence, KV head) counts `own` blocks more than
// the n that it has, ahead of them; T is the sum over all units, n_max the largest unit's count.  CTAs that hold blocks of a unit
// leave a partial each, and there are RAP_MAX_SPLIT - n_pre places for them behind a shared prefix's, so the plan keeps every
// unit on at most that many CTAs: with `share` blocks or more in each, n consecutive blocks touch at most (n - 2) / share + 2.
// The host runs the same code (rap_debug_window_plan).
struct WinScanPlan {
  int nc;                // CTAs that have work
  int parts;             // even: CTAs of each unit
  int share, extra;      // otherwise: blocks of a CTA; the first `extra` CTAs have one more
  bool even;
  __host__ __device__ __forceinline__ int cta_of(int tile) const {      // whose share holds this block
    const int mark = extra * (share + 1);
    return tile < mark ? tile / (share + 1) : extra + (tile - mark) / share;
  }
};
__host__ __device__ __forceinline__ WinScanPlan win_scan_plan(int T, int n_max, int units, int grid, int own, int n_pre, bool padded) {
  WinScanPlan pl;
  const int places = RAP_MAX_SPLIT - n_pre;
  // every CTA has a block for each of its warps, and enough for the longest unit's partials to have a place
  const int least = n_max - own > 2 ? (n_max - own - 2) / (places - 1) + 1 : 1;      // (n - 2) / least <= places - 2
  int nc = (T + 3) >> 2;
  nc = nc < grid ? nc : grid;
  if (T / nc < least) nc = T / least;
  // Units of about the same size (within a fifth of the largest): the same number of CTAs for each, so that no CTA ends two of
  // them, if that leaves at most a quarter of the CTA slots empty -- HBM is as busy with those missing (32 sequences of 4096
  // rows 65.9 -> 61.8 us; not with padded rows, which keep the SMs busier: 66 -> 71 us there).  Four blocks a CTA, as above.
  int most_parts = (n_max - own) >> 2;
  most_parts = most_parts < 1 ? 1 : most_parts < places - 2 ? most_parts : places - 2;
  int parts = grid / units;
  pl.even = parts >= 1 && !padded && (long long)n_max * units <= (long long)T + T / 5 && (parts > most_parts || units * parts * 4 >= grid * 3);
  pl.parts = parts < most_parts ? parts : most_parts;
  pl.nc = pl.even ? units * pl.parts : nc;
  pl.share = T / pl.nc;
  pl.extra = T - pl.share * pl.nc;
  return pl;
}

__device__ __forceinline__ void win_report(int32_t* status, int code, int detail) {
  if (atomicCAS(&status[0], 0, code) == 0) status[1] = detail;
}

}  // namespace
