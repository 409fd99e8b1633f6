// Head norms and the position rotation of a step's queries and keys, and the
// way of keys and values into a cache in pages.
//
//   y = x / sqrt(mean(x^2) + eps) * gain  (optional, per head)
//   (a', b') = g (a cos t - b sin t, b cos t + a sin t),  t = p f_j
//
// Bound by reading and writing the rows once.  A lane holds VEC turned pairs of
// one head in two 16-byte pieces (half style: VEC entries at j and VEC at j +
// dim/2; pairs: 2 VEC entries in a row), 64 / LPH heads a wave at a time, so the
// sines of a row are made once a wave and serve all heads that it works on.
// Angles: p f is formed in fp64 in turns and reduced there; what is left, at
// most half a turn, is rounded to fp32 (2^-24 of it) and goes to sincospi.
// Rows, strides or a dim that 16-byte pieces do not fit take VEC = 1.
// Values of a page lie [dim][32 positions]: 32 positions of a head are turned
// over in LDS so that full runs of 8 positions leave as 16 bytes; a step of one
// row writes 2 bytes into each dim's run, as the layout has it.
#include <algorithm>

#include "pages.h"

namespace dsi {

namespace {

constexpr int kRotWaves = 4;

template <typename T, int VEC>
__device__ __forceinline__ void load_piece(const T* p, float (&v)[VEC]) {
  if constexpr (VEC == 1) {
    if constexpr (sizeof(T) == 2) v[0] = bf_bits2f(*p);
    else v[0] = *p;
  } else {
    const u32x4 x = *(const u32x4*)p;
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(x[i] << 16);
        v[2 * i + 1] = __uint_as_float(x[i] & 0xFFFF0000u);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(x[i]);
    }
  }
}
// VEC entries of a type known at run time; 16-byte aligned runs where VEC > 1
template <int VEC>
__device__ __forceinline__ void store_piece(void* base, size_t at, bool bf16, const float (&v)[VEC]) {
  if constexpr (VEC == 1) {
    if (bf16) ((uint16_t*)base)[at] = f2bf_bits(v[0]);
    else ((float*)base)[at] = v[0];
  } else if (bf16) {
    uint32_t w[VEC / 2];
#pragma unroll
    for (int i = 0; i < VEC / 2; ++i) w[i] = f2bf_pair(v[2 * i], v[2 * i + 1]);
    if constexpr (VEC == 8) *(u32x4*)((uint16_t*)base + at) = u32x4{w[0], w[1], w[2], w[3]};
    else *(uint2*)((uint16_t*)base + at) = uint2{w[0], w[1]};
  } else {
#pragma unroll
    for (int i = 0; i < VEC / 4; ++i)
      *(f32x4*)((float*)base + at + 4 * i) = f32x4{v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]};
  }
}

// values of one block of 32 positions and KV head
template <typename T, int VEC>
__device__ __forceinline__ void append_values(const RotateArgs& a, uint32_t (&tile)[32][129], int item) {
  const PageArgs& p = a.pg;
  const int kvh = item % p.nkv;
  int in = 0;
  const int b = find_item(p.n_windows, item / p.nkv, [&](int w) {
    int r0, r1;
    window_rows(p, a.rows, w, r0, r1);
    const long long at = p.len[w];
    // blocks that the rows touch; none of a window that cannot hold its first row
    return r1 > r0 && at >= 0 && at < window_positions(p) ? (int)((at + (r1 - r0) - 1) / 32 - at / 32) + 1 : 0;
  }, in);
  if (b < 0) return;
  int r0, r1;
  window_rows(p, a.rows, b, r0, r1);
  const int len = p.len[b];
  const int kb = len / 32 + in;
  const long long blk = block_of(p, b, kvh, kb);
  if (blk < 0) return;
  // positions [lo, hi) of the block are the step's
  const int lo = max(len - kb * 32, 0), hi = (int)min(32ll, (long long)len + (r1 - r0) - (long long)kb * 32);
  const int first = r0 + kb * 32 - len;   // the row of the block's position 0
  const T* src = (const T*)a.v + (size_t)kvh * a.hd;
  const int ppr = a.hd / VEC;             // pieces per row
  for (int i = threadIdx.x + lo * ppr; i < hi * ppr; i += kRotWaves * 64) {
    const int pos = i / ppr, d = (i - pos * ppr) * VEC;
    float v[VEC];
    load_piece<T, VEC>(src + (size_t)(first + pos) * a.ldv + d, v);
#pragma unroll
    for (int e = 0; e < VEC; ++e) tile[pos][d + e] = p.kvb ? (uint32_t)f2bf_bits(v[e]) : __float_as_uint(v[e]);
  }
  __syncthreads();
  const size_t base = (size_t)blk * 32 * a.hd;
  for (int i = threadIdx.x; i < 4 * a.hd; i += kRotWaves * 64) {
    const int d = i >> 2, g = (i & 3) * 8;
    if (g >= hi || g + 8 <= lo) continue;
    const size_t at = base + (size_t)d * 32 + g;
    uint32_t x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = tile[g + e][d];
    if (g >= lo && g + 8 <= hi) {
      if (p.kvb) {
        *(u32x4*)((uint16_t*)p.v + at) = u32x4{x[0] | x[1] << 16, x[2] | x[3] << 16, x[4] | x[5] << 16, x[6] | x[7] << 16};
      } else {
        *(u32x4*)((uint32_t*)p.v + at) = u32x4{x[0], x[1], x[2], x[3]};
        *(u32x4*)((uint32_t*)p.v + at + 4) = u32x4{x[4], x[5], x[6], x[7]};
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (g + e < lo || g + e >= hi) continue;
        if (p.kvb) ((uint16_t*)p.v)[at + e] = (uint16_t)x[e];
        else ((uint32_t*)p.v)[at + e] = x[e];
      }
    }
  }
}

template <typename T, int VEC>
__global__ __launch_bounds__(kRotWaves * 64) void k_rotate(RotateArgs a) {
  __shared__ uint32_t tile[32][129];
  if ((int)blockIdx.x >= a.row_blocks) {
    append_values<T, VEC>(a, tile, (int)blockIdx.x - a.row_blocks);
    return;
  }
  const int lane = threadIdx.x & 63;
  const long long wave = (long long)blockIdx.x * kRotWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = (int)(wave / a.wpr), part = (int)(wave - (long long)r * a.wpr);
  if (r >= a.rows) return;
  const PageArgs& p = a.pg;
  // the row's position, and where its keys go
  int pos = a.pos && a.dim ? a.pos[r] : 0;
  long long page_row = -1;   // block of KV head 0
  int slot = 0;
  if (p.n_windows) {
    const int b = window_of_row(p, a.rows, r);
    if (b < 0) return;
    const long long at = (long long)p.len[b] + (r - min(max(p.row0[b], 0), a.rows));
    if (!a.pos) pos = (int)at;
    if (p.len[b] >= 0 && at < window_positions(p)) {
      page_row = block_of(p, b, 0, (int)(at >> 5));
      slot = (int)(at & 31);
    }
  }
  const int units = a.hd / (2 * VEC);
  int lph = 1;               // lanes per head: units, rounded up to a power of two
  while (lph < units) lph *= 2;
  const int u = lane & (lph - 1), hpp = 64 / lph;
  const bool live = u < units;
  // where the lane's two pieces lie in a head, and the pairs they make
  const int turned = a.dim / (2 * VEC);     // units of whole turned pairs (half style)
  int pa, pb;
  if (a.style || u >= turned) pa = u * 2 * VEC, pb = pa + VEC;
  else pa = u * VEC, pb = a.dim / 2 + u * VEC;
  float cs[VEC], sn[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) {
    const int j = u * VEC + e;
    cs[e] = 1.f;
    sn[e] = 0.f;
    if (live && j < a.dim / 2) {
      const double t = (double)pos * a.freq[j] * 0.15915494309189533577;   // turns
      sincospif(2.f * (float)(t - rint(t)), &sn[e], &cs[e]);
      cs[e] *= a.gain;
      sn[e] *= a.gain;
    }
  }
  const int heads = a.nq + a.nk;
  const int p0 = part * a.ppw, p1 = min(p0 + a.ppw, a.passes);
  for (int ps = p0; ps < p1; ++ps) {
    const int h = ps * hpp + lane / lph;
    const bool on = live && h < heads, isq = h < a.nq;
    const int hh = isq ? h : h - a.nq;
    float x[VEC], y[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) x[e] = y[e] = 0.f;
    if (on) {
      const T* src = (isq ? (const T*)a.q + (size_t)r * a.ldq : (const T*)a.k + (size_t)r * a.ldk) + (size_t)hh * a.hd;
      load_piece<T, VEC>(src + pa, x);
      load_piece<T, VEC>(src + pb, y);
    }
    if (a.gq || a.gk) {
      float s = 0.f;
#pragma unroll
      for (int e = 0; e < VEC; ++e) s = fmaf(x[e], x[e], fmaf(y[e], y[e], s));
      for (int o = 1; o < lph; o *= 2) s += __shfl_xor(s, o);
      const float* g = isq ? a.gq : a.gk;
      if (on && g) {
        const float f = 1.f / sqrtf(s / (float)a.hd + a.eps);
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          x[e] = x[e] * f * g[pa + e];
          y[e] = y[e] * f * g[pb + e];
        }
      }
    }
    if (!on) continue;
    if (!a.style) {
      if (u < turned) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const float l = x[e], m = y[e];
          x[e] = l * cs[e] - m * sn[e];
          y[e] = m * cs[e] + l * sn[e];
        }
      }
    } else {
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        if (u * VEC + e >= a.dim / 2) continue;
        // entries 2e, 2e + 1 of x and y after each other (one of each where VEC is 1)
        float& l = VEC == 1 ? x[0] : 2 * e < VEC ? x[2 * e % VEC] : y[2 * e % VEC];
        float& m = VEC == 1 ? y[0] : 2 * e < VEC ? x[(2 * e + 1) % VEC] : y[(2 * e + 1) % VEC];
        const float l0 = l, m0 = m;
        l = l0 * cs[e] - m0 * sn[e];
        m = m0 * cs[e] + l0 * sn[e];
      }
    }
    if (isq || !p.n_windows) {
      void* dst = isq ? a.qo : a.ko;
      const size_t at = (size_t)r * (isq ? a.ldqo : a.ldko) + (size_t)hh * a.hd;
      store_piece<VEC>(dst, at + pa, a.bf16, x);
      store_piece<VEC>(dst, at + pb, a.bf16, y);
    } else if (page_row >= 0) {
      const size_t base = (size_t)(page_row + (long long)hh * p.bpp) * 32 * a.hd + slot * 32;
      store_piece<VEC>(p.k, base + (size_t)(pa >> 5) * 1024 + (pa & 31), p.kvb, x);
      store_piece<VEC>(p.k, base + (size_t)(pb >> 5) * 1024 + (pb & 31), p.kvb, y);
    }
  }
}

template <typename T, int VEC>
hipError_t launch(RotateArgs a, hipStream_t s) {
  int lph = 1;
  while (lph < a.hd / (2 * VEC)) lph *= 2;
  const int heads = a.nq + a.nk, hpp = 64 / lph;
  a.passes = (heads + hpp - 1) / hpp;
  // a row's waves share nothing: one pass each until the rows alone fill the card
  const long long waves = (long long)a.rows * a.passes;
  a.ppw = (int)std::min((long long)a.passes, std::max(1ll, waves / 8192));
  a.wpr = (a.passes + a.ppw - 1) / a.ppw;
  a.row_blocks = heads ? (int)(((long long)a.rows * a.wpr + kRotWaves - 1) / kRotWaves) : 0;
  long long values = 0;
  if (a.pg.n_windows) {
    // blocks that the windows' rows touch, at most: 1 + (r - 1) / 32 rounded up of r rows
    const int n = std::min(a.pg.n_windows, a.rows);
    values = (long long)a.pg.nkv * std::min((long long)a.rows, 2ll * n + (a.rows - n) / 32);
  }
  if (a.row_blocks + values < 1) return hipSuccess;
  hipLaunchKernelGGL((k_rotate<T, VEC>), dim3((unsigned)(a.row_blocks + values)), dim3(kRotWaves * 64), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rotate(RotateArgs a, bool wide, hipStream_t s) {
  if (a.bf16) return wide ? launch<uint16_t, 8>(a, s) : launch<uint16_t, 1>(a, s);
  return wide ? launch<float, 4>(a, s) : launch<float, 1>(a, s);
}

}  // namespace dsi
