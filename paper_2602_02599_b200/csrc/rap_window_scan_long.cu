// The forms of win_scan_kernel for launches in which a warp may add up many blocks of a unit (LONG).
#include "rap_window_scan_kernel.cuh"

const void* rap_win_scan_long_fn(int G, bool vodd, bool tma, int n, int nw) { return scan_any<true>(G, vodd, tma, n, nw); }
