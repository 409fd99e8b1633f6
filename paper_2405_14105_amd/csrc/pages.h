// Windows, rows and pages of a step, as the kernels of rotate.hip and pages.hip
// look them up.  Whatever the caller's arrays hold, what comes out stays within
// the buffers.
#pragma once

#include "scan.h"

namespace dsi {

// rows [r0, r1) of window b, within the step's
__device__ __forceinline__ void window_rows(const PageArgs& p, int rows, int b, int& r0, int& r1) {
  r0 = min(max(p.row0[b], 0), rows);
  r1 = min(max(p.row0[b + 1], r0), rows);
}
__device__ __forceinline__ long long window_positions(const PageArgs& p) { return (long long)p.max_pages * p.bpp * 32; }

__device__ __forceinline__ int wave_scan_incl(int v) {
  dpp_steps([&](auto s) { v += dpp_from<decltype(s)::ctrl, decltype(s)::rows>(0, v); });
  return v;
}
__device__ __forceinline__ int wave_total(int v) { return __builtin_amdgcn_readlane(wave_scan_incl(v), 63); }

// The window that holds item t, windows contributing count(b) items each, and
// the item's number within it; -1 if there are not that many.  Every lane of
// the wave calls it with the same t.
template <typename F>
__device__ __forceinline__ int find_item(int n_windows, int t, F&& count, int& rest) {
  const int lane = threadIdx.x & 63;
  for (int b0 = 0; b0 < n_windows; b0 += 64) {
    const int c = b0 + lane < n_windows ? count(b0 + lane) : 0;
    const int incl = wave_scan_incl(c);
    const unsigned long long over = __ballot(incl > t);
    if (over) {
      const int l = __ffsll((long long)over) - 1;
      rest = t - __builtin_amdgcn_readlane(incl - c, l);
      return b0 + l;
    }
    t -= __builtin_amdgcn_readlane(incl, 63);
  }
  return -1;
}
// the window of row r, or -1
__device__ __forceinline__ int window_of_row(const PageArgs& p, int rows, int r) {
  const int lane = threadIdx.x & 63;
  for (int b0 = 0; b0 < p.n_windows; b0 += 64) {
    bool in = false;
    if (b0 + lane < p.n_windows) {
      int r0, r1;
      window_rows(p, rows, b0 + lane, r0, r1);
      in = r >= r0 && r < r1;
    }
    const unsigned long long m = __ballot(in);
    if (m) return b0 + __ffsll((long long)m) - 1;
  }
  return -1;
}
// the pool's index of the block that holds a window's positions [32 kb, 32 kb + 32)
// of a KV head, or -1 without a page
__device__ __forceinline__ long long block_of(const PageArgs& p, int b, int kvh, int kb) {
  const int e = kb / p.bpp;
  if (e < 0 || e >= p.max_pages) return -1;
  const int page = p.table[(size_t)b * p.max_pages + e];
  if (page < 0 || page >= p.n_pages) return -1;
  return ((long long)page * p.nkv + kvh) * p.bpp + (kb - e * p.bpp);
}

}  // namespace dsi
