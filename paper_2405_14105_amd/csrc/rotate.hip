// Head norms and the position rotation of a step's queries and keys, and the
// way of keys and values into a cache in pages.
//
//   y = x / sqrt(mean(x^2) + eps) * gain  (optional, per head)
//   (a', b') = g (a cos t - b sin t, b cos t + a sin t),  t = p f_j
//
// Bound by reading and writing the rows once.  A wave takes a row, or some of its
// heads where there are few rows.  A lane holds VEC turned pairs of one head in two
// 16-byte pieces (half style: VEC entries from j and VEC from j + dim/2 on; pairs: 2
// VEC entries in a row), 64 / LPH heads a wave at a time, the next two groups of them
// on their way meanwhile; what is not turned lies in further lanes, 2 VEC entries
// each.  Loads and stores of 16 bytes need no more than the type's alignment; where a
// dim fills no whole pieces the last ones overlap.
// A row's sines are made once a wave, one pair a lane, and the lanes read those of
// their pairs from LDS.  p f is formed in fp64 in turns and reduced there; what is
// left, at most half a turn, goes to sincospi in fp32, and what that leaves of it turns
// the result on: sines near zero keep their digits.
// 2048 rows of 8B: fp32 (84 MB) 13.6 us, 6.2 TB/s; bf16 (42 MB) 12, with norms 14, where
// vector instructions are issued in 69 % of the busy cycles and a lane's sines go
// through scratch (68 bytes a lane, 17 of the 38 MB written): four waves a SIMD leave
// 128 registers, 139 are needed.  Three waves without scratch are no faster: 12, with
// norms 15.6, 1026 rows of 13B 21.2 instead of 19.4.  A workgroup
// for a row, its sines made by one wave: 14 and 16.  8 bytes a piece for bf16: 11.7
// and 16.  Rows of a dim that fills no whole pieces, entry by entry: 23 us instead of 14.
// Values of a page lie [dim][32 positions]: 32 positions of a head are turned
// over in LDS so that full runs of 8 positions leave as 16 bytes; a step of one
// row writes 2 bytes into each dim's run, as the layout has it.  1024 windows of one row
// (8B) take 57 us, most of it such blocks.  By the waves that take the rows' keys it
// is 34, but the registers that this needs cost every call: 1026 rows of 13B 21.6 us
// instead of 19, 42 rows of 8B 4.85 instead of 4.6.
#include <algorithm>

#include "pages.h"

namespace dsi {

namespace {

constexpr int kRotWaves = 4;
constexpr int kRotPairs = 64;   // of a head, at most
constexpr int kRotFull = 4096;  // waves that rows are spread over, head by head, where they are few

// 16 bytes with the type's alignment
template <typename T>
struct Piece;
template <>
struct Piece<float> {
  static constexpr int N = 4;
  typedef uint32_t vec __attribute__((ext_vector_type(4), aligned(4)));
};
template <>
struct Piece<uint16_t> {
  static constexpr int N = 8;
  typedef uint32_t vec __attribute__((ext_vector_type(4), aligned(2)));
};
// n of a piece's N entries (the others 0), as bits
template <typename T>
__device__ __forceinline__ u32x4 load_piece(const T* p, int n) {
  constexpr int N = Piece<T>::N;
  if (n >= N) return *(const typename Piece<T>::vec*)p;
  u32x4 x = u32x4{0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (i < n) {
      if constexpr (sizeof(T) == 2) x[i >> 1] |= (uint32_t)p[i] << (16 * (i & 1));
      else x[i] = __float_as_uint(p[i]);
    }
  return x;
}
template <typename T>
__device__ __forceinline__ void floats_of(const u32x4& x, float (&v)[Piece<T>::N]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 2) {
      v[2 * i] = __uint_as_float(x[i] << 16);
      v[2 * i + 1] = __uint_as_float(x[i] & 0xFFFF0000u);
    } else {
      v[i] = __uint_as_float(x[i]);
    }
  }
}
template <int N>
__device__ __forceinline__ void scale_by(float (&v)[N], float f, const float* g, int n) {
#pragma unroll
  for (int i = 0; i < N; i += 4) {
    float x[4];
    floats_of<float>(load_piece<float>(g + i, n - i), x);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[i + e] = v[i + e] * f * x[e];
  }
}
// n of N entries to `at` of an array whose type is known at run time
template <int N>
__device__ __forceinline__ void store_piece(void* base, size_t at, bool bf16, int n, const float (&v)[N]) {
  if (n < N) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (i >= n) continue;
      if (bf16) ((uint16_t*)base)[at + i] = f2bf_bits(v[i]);
      else ((float*)base)[at + i] = v[i];
    }
  } else if (bf16) {
    uint32_t w[N / 2];
#pragma unroll
    for (int i = 0; i < N / 2; ++i) w[i] = f2bf_pair(v[2 * i], v[2 * i + 1]);
    typedef uint32_t two __attribute__((ext_vector_type(2), aligned(2)));
    uint16_t* d = (uint16_t*)base + at;
    if constexpr (N == 8) *(Piece<uint16_t>::vec*)d = u32x4{w[0], w[1], w[2], w[3]};
    else *(two*)d = two{w[0], w[1]};
  } else {
    float* d = (float*)base + at;
#pragma unroll
    for (int i = 0; i < N / 4; ++i)
      *(Piece<float>::vec*)(d + 4 * i) = u32x4{__float_as_uint(v[4 * i]), __float_as_uint(v[4 * i + 1]), __float_as_uint(v[4 * i + 2]), __float_as_uint(v[4 * i + 3])};
  }
}
// the same into a block of keys, [hd/32][32 positions][32]; `at` is the position's
// entry of dim 0, d the piece's first dim
template <int N>
__device__ __forceinline__ void store_key(void* base, size_t at, int d, bool bf16, int n, const float (&v)[N]) {
  if ((d & 31) + N <= 32) {
    store_piece<N>(base, at + (size_t)(d >> 5) * 1024 + (d & 31), bf16, n, v);
    return;
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {   // over two of the layout's runs of 32 dims
    const size_t to = at + (size_t)((d + i) >> 5) * 1024 + ((d + i) & 31);
    if (i >= n) continue;
    if (bf16) ((uint16_t*)base)[to] = f2bf_bits(v[i]);
    else ((float*)base)[to] = v[i];
  }
}

// the sum over groups of n lanes (a power of two), for all of them: lanes of a row of
// 16 meet by DPP patterns, of which the mirrors do where a half's lanes are alike
__device__ __forceinline__ float sum_of_group(float s, int n) {
  if (n > 1) s += dpp_from<0xB1, 0xF>(s, s);
  if (n > 2) s += dpp_from<0x4E, 0xF>(s, s);
  if (n > 4) s += dpp_from<0x141, 0xF>(s, s);
  if (n > 8) s += dpp_from<0x140, 0xF>(s, s);
  if (n > 16) s += __shfl_xor(s, 16);
  if (n > 32) s += __shfl_xor(s, 32);
  return s;
}

// values of one block of 32 positions and KV head
template <typename T>
__device__ __forceinline__ void append_values(const RotateArgs& a, uint32_t (&tile)[32][129], int item) {
  constexpr int N = Piece<T>::N;
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
  const int ppr = a.hd / N;               // pieces per row
  for (int i = threadIdx.x + lo * ppr; i < hi * ppr; i += kRotWaves * 64) {
    const int pos = i / ppr, d = (i - pos * ppr) * N;
    float v[N];
    floats_of<T>(load_piece<T>(src + (size_t)(first + pos) * a.ldv + d, N), v);
#pragma unroll
    for (int e = 0; e < N; ++e) tile[pos][d + e] = p.kvb ? (uint32_t)f2bf_bits(v[e]) : __float_as_uint(v[e]);
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

template <typename T>
__global__ __launch_bounds__(kRotWaves * 64, 4) void k_rotate(RotateArgs a) {
  constexpr int VEC = Piece<T>::N;
  __shared__ union {
    uint32_t tile[32][129];
    float2 turn[kRotWaves][kRotPairs];
  } sh;
  if ((int)blockIdx.x >= a.row_blocks) {
    append_values<T>(a, sh.tile, (int)blockIdx.x - a.row_blocks);
    return;
  }
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const long long wave = (long long)blockIdx.x * kRotWaves + w;
  const int r = (int)(wave / a.parts), part = (int)(wave - (long long)r * a.parts);
  if (r >= a.rows) return;
  const PageArgs& p = a.pg;
  // where the lane's two pieces lie in a head.  A last unit that would not be whole
  // starts earlier: its first dupx and dupy entries are another lane's too, which
  // makes the same of them.  na and nb are less than VEC only where a head has no
  // more pairs, or no more of what is not turned.
  const int pairs = a.dim / 2, turned = (pairs + VEC - 1) / VEC;   // units with pairs
  const int u = lane & (a.lph - 1), hpp = 64 / a.lph;
  int pa, pb, na = VEC, nb = VEC, j0 = 0, over;
  if (u < turned) {
    j0 = max(min(u * VEC, pairs - VEC), 0);
    over = u * VEC - j0;
    const int n = min(VEC, pairs - j0);
    if (a.style) {
      pa = 2 * j0, pb = pa + VEC, na = min(VEC, 2 * n), nb = max(0, 2 * n - VEC);
      over *= 2;
    } else {
      pa = j0, pb = pairs + j0, na = nb = n;
    }
  } else {
    const int at = a.dim + (u - turned) * 2 * VEC, rest = a.hd - a.dim;
    pa = rest >= 2 * VEC ? min(at, a.hd - 2 * VEC) : a.dim;
    pb = rest >= VEC ? min(pa + VEC, a.hd - VEC) : a.hd;
    na = at < a.hd ? min(VEC, rest) : 0;
    nb = at < a.hd && rest > VEC ? VEC : 0;
    over = at - pa + (pa + VEC - pb);
  }
  const bool split = u < turned && !a.style;   // both pieces overlap alike
  const int dupx = split ? over : u < turned || a.hd - a.dim >= 2 * VEC ? min(over, VEC) : 0;
  const int dupy = split ? over : u < turned || a.hd - a.dim >= 2 * VEC ? max(0, over - VEC) : over;
  const int heads = a.nq + a.nk;
  // the wave's groups of hpp heads
  const int p0 = part * a.passes / a.parts, p1 = (part + 1) * a.passes / a.parts;
  struct Raw {
    u32x4 a, b;
  };
  auto load = [&](int ps) {
    const int h = ps * hpp + lane / a.lph;
    Raw x{u32x4{0, 0, 0, 0}, u32x4{0, 0, 0, 0}};
    if (ps >= p1 || na <= 0 || h >= heads) return x;
    const T* src = h < a.nq ? (const T*)a.q + (size_t)r * a.ldq + (size_t)h * a.hd : (const T*)a.k + (size_t)r * a.ldk + (size_t)(h - a.nq) * a.hd;
    x.a = load_piece<T>(src + pa, na);
    x.b = load_piece<T>(src + pb, nb);
    return x;
  };
  Raw x0 = load(p0), x1 = load(p0 + 1);
  // the row's position, and where its keys go
  int pos = a.pos && a.dim ? a.pos[r] : 0, slot = 0;
  long long block = -1;   // of KV head 0
  if (p.n_windows) {
    const int b = window_of_row(p, a.rows, r);
    if (b < 0) return;
    const long long at = (long long)p.len[b] + (r - min(max(p.row0[b], 0), a.rows));
    if (!a.pos) pos = (int)at;
    if (p.len[b] >= 0 && at < window_positions(p)) {
      block = block_of(p, b, 0, (int)(at >> 5));
      slot = (int)(at & 31);
    }
  }
  if (lane < pairs) {
    double t = (double)pos * a.freq[lane] * 0.15915494309189533577;   // turns
    t -= rint(t);
    const float near = (float)t, rest = (float)((t - near) * 6.283185307179586477);
    float s, c;
    sincospif(2.f * near, &s, &c);
    sh.turn[w][lane] = make_float2((c - rest * s) * a.gain, (s + rest * c) * a.gain);
  }
  // the wave's own: the LDS takes a wave's accesses in their order
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  float cs[VEC], sn[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) {
    const float2 v = sh.turn[w][min(j0 + e, kRotPairs - 1)];
    cs[e] = v.x;
    sn[e] = v.y;
  }
  for (int ps = p0; ps < p1; ++ps) {
    const Raw raw = x0;
    x0 = x1;
    x1 = load(ps + 2);
    const int h = ps * hpp + lane / a.lph;
    const bool on = na > 0 && h < heads, isq = h < a.nq;
    const int hh = isq ? h : h - a.nq;
    float x[VEC], y[VEC];
    floats_of<T>(raw.a, x);
    floats_of<T>(raw.b, y);
    if (a.gq || a.gk) {
      float s = 0.f;
#pragma unroll
      for (int e = 0; e < VEC; ++e) s += (e >= dupx ? x[e] * x[e] : 0.f) + (e >= dupy ? y[e] * y[e] : 0.f);
      s = sum_of_group(s, a.lph);
      const float* g = isq ? a.gq : a.gk;
      if (on && g) {
        const float f = 1.f / sqrtf(s / (float)a.hd + a.eps);
        scale_by<VEC>(x, f, g + pa, na);
        scale_by<VEC>(y, f, g + pb, nb);
      }
    }
    if (!on) continue;
    if (u < turned) {
      if (!a.style) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const float l = x[e], m = y[e];
          x[e] = l * cs[e] - m * sn[e];
          y[e] = m * cs[e] + l * sn[e];
        }
      } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          // entries 2e and 2e + 1 of x and y after each other
          float& l = 2 * e < VEC ? x[2 * e % VEC] : y[2 * e % VEC];
          float& m = 2 * e < VEC ? x[(2 * e + 1) % VEC] : y[(2 * e + 1) % VEC];
          const float l0 = l, m0 = m;
          l = l0 * cs[e] - m0 * sn[e];
          m = m0 * cs[e] + l0 * sn[e];
        }
      }
    }
    if (isq || !p.n_windows) {
      void* dst = isq ? a.qo : a.ko;
      const size_t at = (size_t)r * (isq ? a.ldqo : a.ldko) + (size_t)hh * a.hd;
      store_piece<VEC>(dst, at + pa, a.bf16, na, x);
      store_piece<VEC>(dst, at + pb, a.bf16, nb, y);
    } else if (block >= 0) {
      const size_t base = (size_t)(block + (long long)hh * p.bpp) * 32 * a.hd + slot * 32;
      store_key<VEC>(p.k, base, pa, p.kvb, na, x);
      store_key<VEC>(p.k, base, pb, p.kvb, nb, y);
    }
  }
}

template <typename T>
hipError_t launch(RotateArgs a, hipStream_t s) {
  constexpr int VEC = Piece<T>::N;
  const int units = (a.dim / 2 + VEC - 1) / VEC + (a.hd - a.dim + 2 * VEC - 1) / (2 * VEC);
  a.lph = 1;
  while (a.lph < units) a.lph *= 2;
  const int heads = a.nq + a.nk, hpp = 64 / a.lph;
  a.passes = (heads + hpp - 1) / hpp;
  // waves of a row: one, or while the rows are few one for each group of heads
  a.parts = (int)std::max(1ll, std::min((long long)a.passes, (long long)kRotFull / a.rows));
  a.row_blocks = heads ? (int)(((long long)a.rows * a.parts + kRotWaves - 1) / kRotWaves) : 0;
  long long values = 0;
  if (a.pg.n_windows) {
    // blocks that the windows' rows touch, at most: 1 + (r - 1) / 32 rounded up of r rows
    const int n = std::min(a.pg.n_windows, a.rows);
    values = (long long)a.pg.nkv * std::min((long long)a.rows, 2ll * n + (a.rows - n) / 32);
  }
  if (a.row_blocks + values < 1) return hipSuccess;
  if (a.row_blocks + values > kMaxStepBlocks) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL((k_rotate<T>), dim3((unsigned)(a.row_blocks + values)), dim3(kRotWaves * 64), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rotate(RotateArgs a, hipStream_t s) { return a.bf16 ? launch<uint16_t>(a, s) : launch<float>(a, s); }

}  // namespace dsi
