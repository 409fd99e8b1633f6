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
// the wave calls it with the same t.  More than 64 windows: four a lane,
// whose loads are in flight together.
template <typename F>
__device__ __forceinline__ int find_item(int n_windows, int t, F&& count, int& rest) {
  const int lane = threadIdx.x & 63;
  if (n_windows <= 64) {
    const int c = lane < n_windows ? count(lane) : 0, incl = wave_scan_incl(c);
    const unsigned long long over = __ballot(incl > t);
    const int l = __ffsll((long long)over) - 1;
    if (over) rest = t - __builtin_amdgcn_readlane(incl - c, l);
    return l;
  }
  for (int b0 = 0; b0 < n_windows; b0 += 256) {
    int c[4], sum = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int b = b0 + lane * 4 + i, n = count(min(b, n_windows - 1));
      c[i] = b < n_windows ? n : 0;
      sum += c[i];
    }
    const int incl = wave_scan_incl(sum);
    const unsigned long long over = __ballot(incl > t);
    if (over) {
      const int l = __ffsll((long long)over) - 1;
      rest = t - __builtin_amdgcn_readlane(incl - sum, l);
      int b = b0 + l * 4;
#pragma unroll
      for (int i = 0; i < 3; ++i) {
        const int n = __builtin_amdgcn_readlane(c[i], l);
        if (b != b0 + l * 4 + i || rest < n) continue;
        rest -= n;
        ++b;
      }
      return b;
    }
    t -= __builtin_amdgcn_readlane(incl, 63);
  }
  return -1;
}
// the window of row r, or -1: the last of 64 runs of windows that begins no later,
// and its windows
__device__ __forceinline__ int window_of_row(const PageArgs& p, int rows, int r) {
  const int lane = threadIdx.x & 63, n = p.n_windows, run = (n + 63) >> 6;
  int b0 = 0;
  if (run > 1) {
    const unsigned long long m = __ballot(lane * run < n && p.row0[min(lane * run, n)] <= r);
    if (!m) return -1;
    b0 = (63 - __clzll((long long)m)) * run;
  }
  const int b = b0 + lane;
  bool in = false;
  if (lane < (run > 1 ? run : 64) && b < n) {
    int r0, r1;
    window_rows(p, rows, b, r0, r1);
    in = r >= r0 && r < r1;
  }
  const unsigned long long m = __ballot(in);
  return m ? b0 + __ffsll((long long)m) - 1 : -1;
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
