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

// Partials of a query head in the context's workspace: RAP_MAX_SPLIT rows of d_v' sums (a multiple of four), then as many
// (maximum, weight) pairs
__host__ __device__ __forceinline__ size_t win_partial_floats(int dv) { return (size_t)RAP_MAX_SPLIT * (((dv + 3) & ~3) + 2); }

__device__ __forceinline__ void win_report(int32_t* status, int code, int detail) {
  if (atomicCAS(&status[0], 0, code) == 0) status[1] = detail;
}

}  // namespace
