// Attention of a step's rows over their windows' pages.
//
//   o = sum_j p_j v_j / sum_j p_j,  p_j = e^{scale q k_j - m},  m the maximum
//
// Rows and the heads that share a KV head are numbered together (query x = row
// * G + head of the group), so that tiles of queries are full whatever the
// group; a tile's keys are cut into chunks, an item is one chunk of one tile and
// KV head.  Lengths are the device's: every workgroup works out the cut itself
// from the windows' lengths and rows, so that items are about equally long and
// about `target` in number whatever the windows are.
// S^T = K Q^T and O^T = V^T P^T in 32 x 32 x 16 MFMAs: the rows of the K operand
// are taken in an order in which a lane's scores are already its fragments of
// P^T, and a block's layout is such that every operand is 16 contiguous bytes.
// Parts of a tile are joined by a second launch.
#include <algorithm>

#include "pages.h"

namespace dsi {

namespace {

typedef __attribute__((__vector_size__(16 * sizeof(float)))) float f32x16;

constexpr int kUnit = 128;        // keys of a unit: a block of 32 for each of a workgroup's waves

__device__ __forceinline__ f32x16 zero16() {
  return f32x16{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
}
__device__ __forceinline__ f32x16 mfma32(const u32x4& a, const u32x4& b, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(a), as_bf16x8(b), c, 0, 0, 0);
}
__device__ __forceinline__ float max_over_32(float x) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ __forceinline__ float sum_over_32(float x) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}

// ------------------------------------------------------------------ the cut

struct Cut {
  int r0, R, len;       // the window's rows
  bool bad;             // its rows do not fit: NaN
  int tiles, units, chunks;
};
__device__ __forceinline__ Cut cut_of(const PageAttnArgs& a, int b, int per) {
  Cut c;
  int r1;
  window_rows(a.pg, a.rows, b, c.r0, r1);
  c.R = r1 - c.r0;
  c.len = a.pg.len[b];
  const int G = a.nq / a.pg.nkv;
  const long long queries = (long long)c.R * G;
  c.tiles = queries >= a.qlo && queries <= a.qhi ? (int)((queries + a.tile - 1) / a.tile) : 0;
  c.bad = c.len < 0 || (long long)c.len + c.R > window_positions(a.pg);
  if (c.bad) c.len = 0;
  long long span = c.bad ? 0 : (long long)c.len + c.R;
  if (a.reach) span = min(span, (long long)a.reach + (a.tile + G - 2) / G) + 31;   // a tile's rows, from a block's first position on
  c.units = max(1, (int)((span + kUnit - 1) / kUnit));
  c.chunks = per ? (c.units + per - 1) / per : 1;
  return c;
}
// units of an item: few enough that the call has about `target` of them.  Every
// lane of every wave gets the same.
__device__ __forceinline__ int units_per_item(const PageAttnArgs& a) {
  const int lane = threadIdx.x & 63;
  double work = 0.0;
  for (int b = lane; b < a.pg.n_windows; b += 64) {
    const Cut c = cut_of(a, b, 0);
    work += (double)c.tiles * c.units;
  }
  work = wave_sum(work) * a.pg.nkv;
  return (int)fmin(fmax(ceil(work / a.target), (double)a.least), 1e9);
}
// One item, or one tile that is cut into several
struct Item {
  Cut c;
  int b, tile, chunk;
  int slot;             // of the tile's chunk 0, for tiles of several chunks
};
template <bool JOIN>
__device__ __forceinline__ bool find(const PageAttnArgs& a, int per, int t, Item& it) {
  const int lane = threadIdx.x & 63;
  int slots = 0;
  for (int b0 = 0; b0 < a.pg.n_windows; b0 += 64) {
    const Cut c = b0 + lane < a.pg.n_windows ? cut_of(a, b0 + lane, per) : Cut{0, 0, 0, false, 0, 0, 0};
    const int items = c.tiles * c.chunks, split = c.chunks > 1 ? items : 0;
    const int n = JOIN ? (c.chunks > 1 ? c.tiles : 0) : items;
    const int incl = wave_scan_incl(n), sincl = wave_scan_incl(split);
    const unsigned long long over = __ballot(incl > t);
    if (over) {
      const int l = __ffsll((long long)over) - 1;
      const int in = t - __builtin_amdgcn_readlane(incl - n, l);
      slots += __builtin_amdgcn_readlane(sincl - split, l);
      it.b = b0 + l;
      it.c = cut_of(a, it.b, per);
      it.tile = JOIN ? in : in / it.c.chunks;
      it.chunk = JOIN ? 0 : in - it.tile * it.c.chunks;
      it.slot = slots + it.tile * it.c.chunks;
      return true;
    }
    t -= __builtin_amdgcn_readlane(incl, 63);
    slots += __builtin_amdgcn_readlane(sincl, 63);
  }
  return false;
}
// positions [lo, hi) that a tile's rows see, lo the first of its block
__device__ __forceinline__ void tile_span(const PageAttnArgs& a, const Item& it, int G, int& first, int& last, int& lo, int& hi) {
  first = it.c.len + it.tile * a.tile / G;                                        // position of the first row
  last = it.c.len + min(it.c.R - 1, ((it.tile + 1) * a.tile - 1) / G);            // and of the last
  lo = a.reach ? max(0, first - a.reach + 1) & ~31 : 0;
  hi = last + 1;
}

// ------------------------------------------------------------------ few rows

// the parts of an fp32 number in bf16
template <int N>
__device__ __forceinline__ void split_parts(const float (&v)[8], u32x4 (&p)[N]) {
  float rest[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) rest[e] = v[e];
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      p[i][e] = f2bf_pair(rest[2 * e], rest[2 * e + 1]);
      if (i + 1 < N) {
        rest[2 * e] -= __uint_as_float(p[i][e] << 16);
        rest[2 * e + 1] -= __uint_as_float(p[i][e] & 0xFFFF0000u);
      }
    }
}

// A lane's eight entries of an operand
template <bool KVB>
struct Frag {
  u32x4 p[KVB ? 1 : 2];
};
template <bool KVB>
__device__ __forceinline__ Frag<KVB> load_frag(const void* base, size_t at) {
  return *(const Frag<KVB>*)((const char*)base + at * (KVB ? 2 : 4));
}
__device__ __forceinline__ float f32_of(const Frag<false>& f, int e) { return __uint_as_float(f.p[e >> 2][e & 3]); }
template <bool KVB>
__device__ __forceinline__ Frag<KVB> nan_frag() {
  Frag<KVB> f;
#pragma unroll
  for (int i = 0; i < (KVB ? 1 : 2); ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) f.p[i][e] = KVB ? 0x7FC07FC0u : 0x7FC00000u;
  return f;
}
// Splits a value fragment into what is finite and, as ones, what is not; true
// if there is anything of the second in the wave
__device__ __forceinline__ bool part_finite(Frag<true>& f, Frag<true>& ind) {
  uint32_t any = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint32_t x = f.p[0][e];
    const bool lo = (x & 0x7F80u) == 0x7F80u, hi = (x & 0x7F800000u) == 0x7F800000u;
    f.p[0][e] = (lo ? 0u : x & 0xFFFFu) | (hi ? 0u : x & 0xFFFF0000u);
    ind.p[0][e] = (lo ? 0x3F80u : 0u) | (hi ? 0x3F800000u : 0u);
    any |= ind.p[0][e];
  }
  return __ballot(any != 0) != 0;
}
__device__ __forceinline__ bool part_finite(Frag<false>& f, Frag<false>& ind) {
  uint32_t any = 0;
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const bool not_finite = (f.p[i][e] & 0x7F800000u) == 0x7F800000u;
      ind.p[i][e] = not_finite ? 0x3F800000u : 0u;
      f.p[i][e] = not_finite ? 0u : f.p[i][e];
      any |= ind.p[i][e];
    }
  return __ballot(any != 0) != 0;
}

// One item: the waves take the chunk's blocks of 32 keys in turn, each with a
// maximum, a sum and outputs of its own for all of the tile's queries, and meet
// in LDS at the end.  A block's keys and values go from memory to registers, the
// next block's while this one's are worked on; queries lie in LDS in fragment
// order.  Bound by reading the pages.
// QT: bf16 parts of a query (1: bf16 queries), PT: of a probability; fp32 caches
// take fp32 MFMAs and neither.
template <bool KVB, int HD, bool QB, int NQ>
__global__ __launch_bounds__(256) void k_page_few(PageAttnArgs a) {
  constexpr int QT = KVB ? (QB ? 1 : 3) : 1, PT = KVB ? (QB ? 2 : 3) : 1;
  constexpr int DS = HD / 16, DT = HD / 32;
  constexpr int kQ = NQ * QT * DS * 64 * (KVB ? 1 : 2);   // 16-byte pieces of the queries
  constexpr int kO = 4 * HD * 32 / 4;                      // and of the waves' outputs
  __shared__ u32x4 sm[kQ > kO ? kQ : kO];
  __shared__ float wm[4][NQ * 32], wl[4][NQ * 32];
  const int lane = threadIdx.x & 63, q32 = lane & 31, hh = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kvh = blockIdx.x % a.pg.nkv;
  const int per = units_per_item(a);
  Item it;
  if (!find<false>(a, per, blockIdx.x / a.pg.nkv, it)) return;
  const int G = a.nq / a.pg.nkv, NX = it.c.R * G;
  int first, last, lo, hi;
  tile_span(a, it, G, first, last, lo, hi);
  const long long u0 = (long long)it.chunk * per;
  const int kb0 = (int)min((long long)(lo >> 5) + u0 * 4, (long long)(1 << 30));
  const int kb1 = (int)min((long long)kb0 + (long long)per * 4, (long long)((hi + 31) >> 5));
  // the row, head and position of query n of the tile
  auto query = [&](int n, int& row, int& head, int& pos) {
    const int x = min(it.tile * a.tile + n, NX - 1);
    const int i = x / G;
    row = it.c.r0 + i;
    head = kvh * G + (x - i * G);
    pos = it.c.len + i;
    return it.tile * a.tile + n < NX;
  };
  if (it.c.bad) {
    for (int n = w; n < NQ * 32; n += 4) {
      int row, head, pos;
      if (!query(n, row, head, pos)) continue;
      for (int d = lane; d < HD; d += 64) {
        const size_t at = (size_t)row * a.ldo + (size_t)head * HD + d;
        if constexpr (QB) ((uint16_t*)a.out)[at] = 0x7FC0;
        else ((float*)a.out)[at] = NAN;
      }
    }
    return;
  }
  int pos[NQ], from[NQ];
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    int row, head;
    query(n * 32 + q32, row, head, pos[n]);
    from[n] = a.reach ? pos[n] - a.reach + 1 : 0;
  }
  // queries into LDS: piece (n, part, ds): lane (query q32, dims ds * 16 + 8 hh ..)
  for (int f = w; f < NQ * DS; f += 4) {
    const int n = f / DS, ds = f % DS;
    int row, head, ps;
    query(n * 32 + q32, row, head, ps);
    const size_t at = (size_t)row * a.ldq + (size_t)head * HD + ds * 16 + hh * 8;
    if constexpr (QB && KVB) {
      sm[(n * DS + ds) * 64 + lane] = *(const u32x4*)((const uint16_t*)a.q + at);
    } else {
      float v[8];
      if constexpr (QB) {
        const u32x4 x = *(const u32x4*)((const uint16_t*)a.q + at);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          v[2 * e] = __uint_as_float(x[e] << 16);
          v[2 * e + 1] = __uint_as_float(x[e] & 0xFFFF0000u);
        }
      } else {
        const f32x4 x = *(const f32x4*)((const float*)a.q + at), y = *(const f32x4*)((const float*)a.q + at + 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = x[e], v[4 + e] = y[e];
      }
      if constexpr (KVB) {
        u32x4 p[3];
        split_parts<3>(v, p);
#pragma unroll
        for (int i = 0; i < 3; ++i) sm[((n * 3 + i) * DS + ds) * 64 + lane] = p[i];
      } else {
        u32x4* d = sm + ((n * DS + ds) * 64 + lane) * 2;
        d[0] = u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
        d[1] = u32x4{__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7])};
      }
    }
  }

  // the key of an operand row, in the order that leaves P^T in place
  const int key = 16 * (q32 >> 4) + 8 * ((q32 >> 2) & 1) + 4 * ((q32 >> 3) & 1) + (q32 & 3);
  Frag<KVB> kf[DS], vf[DT][2];
  auto load_k = [&](int blk) {
#pragma unroll
    for (int ds = 0; ds < DS; ++ds)
      kf[ds] = blk < 0 ? nan_frag<KVB>()
                       : load_frag<KVB>(a.pg.k, (size_t)blk * (32 * HD) + (ds >> 1) * 1024 + key * 32 + (ds & 1) * 16 + hh * 8);
  };
  auto load_v = [&](int blk) {
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
      for (int s = 0; s < 2; ++s)
        vf[t][s] = blk < 0 ? nan_frag<KVB>() : load_frag<KVB>(a.pg.v, (size_t)blk * (32 * HD) + (t * 32 + q32) * 32 + s * 16 + hh * 8);
  };
  // blocks of this wave: kb0 + w + 4 i; lane l knows the pool's block of i = 64 g + l
  int mine = -1;
  auto look = [&](int i0) {
    const int kb = kb0 + w + 4 * (i0 + lane);
    mine = kb < kb1 ? (int)block_of(a.pg, it.b, kvh, kb) : -1;
  };
  const int nb = kb1 > kb0 + w ? (kb1 - kb0 - w + 3) / 4 : 0;
  float m[NQ], l[NQ];
  f32x16 o[NQ][DT];
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    m[n] = -INFINITY;
    l[n] = 0.f;
#pragma unroll
    for (int t = 0; t < DT; ++t) o[n][t] = zero16();
  }
  if (nb) {
    look(0);
    const int blk = __builtin_amdgcn_readlane(mine, 0);
    load_k(blk);
    load_v(blk);
  }
  __syncthreads();
  for (int i = 0; i < nb; ++i) {
    const int p0 = (kb0 + w + 4 * i) * 32;
    const bool full = p0 + 31 <= first && (!a.reach || p0 > last - a.reach);
    int next = -1;
    if (i + 1 < nb) {
      if (((i + 1) & 63) == 0) look(i + 1);
      next = __builtin_amdgcn_readlane(mine, (i + 1) & 63);
    }
    f32x16 s[NQ];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      s[n] = zero16();
#pragma unroll
      for (int ds = 0; ds < DS; ++ds) {
        if constexpr (KVB) {
#pragma unroll
          for (int p = 0; p < QT; ++p) s[n] = mfma32(kf[ds].p[0], sm[((n * QT + p) * DS + ds) * 64 + lane], s[n]);
        } else {
          const Frag<false> qf = *(const Frag<false>*)&sm[((n * DS + ds) * 64 + lane) * 2];
#pragma unroll
          for (int e = 0; e < 8; ++e) s[n] = __builtin_amdgcn_mfma_f32_32x32x2f32(f32_of(kf[ds], e), f32_of(qf, e), s[n], 0, 0, 0);
        }
      }
    }
    if (i + 1 < nb) load_k(next);
    // lane: keys p0 + 16 (r / 8) + 8 hh + r % 8 of query q32
    float alpha[NQ];
    bool moved = false;
    uint32_t vis[NQ];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      vis[n] = 0xFFFFu;
      if (!full) {
        vis[n] = 0;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int kp = p0 + 16 * (r >> 3) + 8 * hh + (r & 7);
          const bool in = kp <= pos[n] && kp >= from[n];
          vis[n] |= in ? 1u << r : 0u;
          s[n][r] = in ? s[n][r] : -INFINITY;
        }
      }
      float mx = s[n][0];
#pragma unroll
      for (int r = 1; r < 16; ++r) mx = fmaxf(mx, s[n][r]);
      const float mnew = fmaxf(m[n], max_over_32(mx) * a.scale2);
      const float base = mnew == -INFINITY ? 0.f : mnew;
      alpha[n] = __builtin_amdgcn_exp2f(m[n] - base);
      moved |= mnew != m[n];
      float sum = 0.f;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[n][r] = __builtin_amdgcn_exp2f(fmaf(s[n][r], a.scale2, -base));
        sum += s[n][r];
      }
      l[n] = l[n] * alpha[n] + sum;
      m[n] = mnew;
    }
    if (__ballot(moved)) {
#pragma unroll
      for (int n = 0; n < NQ; ++n)
#pragma unroll
        for (int t = 0; t < DT; ++t) o[n][t] *= alpha[n];
    }
    u32x4 pf[NQ][2][PT];
    if constexpr (KVB) {
#pragma unroll
      for (int n = 0; n < NQ; ++n)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float v[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = s[n][8 * h + e];
          split_parts<PT>(v, pf[n][h]);
        }
    }
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        // values that only some rows see, or none: what is not finite among
        // them reaches no other row's sum
        Frag<KVB> ind;
        if (!full && part_finite(vf[t][h], ind)) {
#pragma unroll
          for (int n = 0; n < NQ; ++n) {
            f32x16 c = zero16();
            if constexpr (KVB) {
              u32x4 one;
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const uint32_t two = vis[n] >> (8 * h + 2 * e);
                one[e] = (two & 1 ? 0x3F80u : 0u) | (two & 2 ? 0x3F800000u : 0u);
              }
              c = mfma32(ind.p[0], one, c);
            } else {
#pragma unroll
              for (int e = 0; e < 8; ++e)
                c = __builtin_amdgcn_mfma_f32_32x32x2f32(f32_of(ind, e), vis[n] >> (8 * h + e) & 1 ? 1.f : 0.f, c, 0, 0, 0);
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) o[n][t][r] = c[r] > 0.f ? NAN : o[n][t][r];
          }
        }
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
          if constexpr (KVB) {
#pragma unroll
            for (int p = 0; p < PT; ++p) o[n][t] = mfma32(vf[t][h].p[0], pf[n][h][p], o[n][t]);
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) o[n][t] = __builtin_amdgcn_mfma_f32_32x32x2f32(f32_of(vf[t][h], e), s[n][8 * h + e], o[n][t], 0, 0, 0);
          }
        }
      }
    if (i + 1 < nb) load_v(next);
  }

  // the waves meet: maxima and sums, then the outputs, 32 queries at a time
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    l[n] = sum_over_32(l[n]);
    if (hh == 0) {
      wm[w][n * 32 + q32] = m[n];
      wl[w][n * 32 + q32] = l[n];
    }
  }
  float* const so = (float*)sm;
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    __syncthreads();   // queries, or the outputs before, are no longer read
    float M = -INFINITY;
#pragma unroll
    for (int i = 0; i < 4; ++i) M = fmaxf(M, wm[i][n * 32 + q32]);
    const float base = M == -INFINITY ? 0.f : M;
    float L = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) L += wl[i][n * 32 + q32] * __builtin_amdgcn_exp2f(wm[i][n * 32 + q32] - base);
    const float f = __builtin_amdgcn_exp2f(m[n] - base);
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int d = t * 32 + 8 * (r >> 2) + 4 * hh + (r & 3);
        so[(w * HD + d) * 32 + q32] = o[n][t][r] * f;
      }
    __syncthreads();
    // thread: query q32, runs of four dims
    int row, head, ps;
    const bool live = query(n * 32 + q32, row, head, ps);
    const size_t slot = ((size_t)it.slot + it.chunk) * a.pg.nkv + kvh;
    if (live && it.c.chunks > 1 && threadIdx.x < 32) a.ml[slot * a.tile + n * 32 + q32] = make_float2(M, L);
    for (int d = (threadIdx.x >> 5) * 4; d < HD; d += 32) {
      float v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[e] = so[(0 * HD + d + e) * 32 + q32];
#pragma unroll
        for (int i = 1; i < 4; ++i) v[e] += so[(i * HD + d + e) * 32 + q32];
      }
      if (!live) continue;
      if (it.c.chunks > 1) {
#pragma unroll
        for (int e = 0; e < 4; ++e) a.part[(slot * HD + d + e) * a.tile + n * 32 + q32] = v[e];
      } else {
        const float inv = 1.f / L;
        const size_t at = (size_t)row * a.ldo + (size_t)head * HD + d;
        if constexpr (QB) {
          *(uint2*)((uint16_t*)a.out + at) = uint2{f2bf_pair(v[0] * inv, v[1] * inv), f2bf_pair(v[2] * inv, v[3] * inv)};
        } else {
          *(f32x4*)((float*)a.out + at) = f32x4{v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv};
        }
      }
    }
  }
}

// ------------------------------------------------------------------ the join

// One tile of several chunks: threads of 32 queries and runs of four dims, 32
// queries at a time
__global__ __launch_bounds__(256) void k_page_join(PageAttnArgs a) {
  const int kvh = blockIdx.x % a.pg.nkv, HD = a.pg.hd;
  const int per = units_per_item(a);
  Item it;
  if (!find<true>(a, per, blockIdx.x / a.pg.nkv, it)) return;
  const int G = a.nq / a.pg.nkv, NX = it.c.R * G;
  int first, last, lo, hi;
  tile_span(a, it, G, first, last, lo, hi);
  const int units = (hi - lo + kUnit - 1) / kUnit;
  const int chunks = min(it.c.chunks, (units + per - 1) / per);   // those with keys of the tile
  const int q32 = threadIdx.x & 31;
  const size_t slot0 = (size_t)it.slot * a.pg.nkv + kvh;
  for (int n = 0; n < a.tile; n += 32) {
    const int x = it.tile * a.tile + n + q32;
    if (x >= NX) continue;
    const int i = x / G, row = it.c.r0 + i, head = kvh * G + (x - i * G);
    float M = -INFINITY, L = 0.f;
    for (int c = 0; c < chunks; ++c) M = fmaxf(M, a.ml[(slot0 + (size_t)c * a.pg.nkv) * a.tile + n + q32].x);
    const float base = M == -INFINITY ? 0.f : M;
    for (int c = 0; c < chunks; ++c) {
      const float2 v = a.ml[(slot0 + (size_t)c * a.pg.nkv) * a.tile + n + q32];
      L += v.y * __builtin_amdgcn_exp2f(v.x - base);
    }
    const float inv = 1.f / L;
    for (int d = (threadIdx.x >> 5) * 4; d < HD; d += 32) {
      float v[4] = {0.f, 0.f, 0.f, 0.f};
      for (int c = 0; c < chunks; ++c) {
        const size_t slot = slot0 + (size_t)c * a.pg.nkv;
        const float f = __builtin_amdgcn_exp2f(a.ml[slot * a.tile + n + q32].x - base);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = fmaf(a.part[(slot * HD + d + e) * a.tile + n + q32], f, v[e]);
      }
      const size_t at = (size_t)row * a.ldo + (size_t)head * HD + d;
      if (a.bf16) *(uint2*)((uint16_t*)a.out + at) = uint2{f2bf_pair(v[0] * inv, v[1] * inv), f2bf_pair(v[2] * inv, v[3] * inv)};
      else *(f32x4*)((float*)a.out + at) = f32x4{v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv};
    }
  }
}

// tiles that windows of a step's rows have together, at most
long long most_tiles(const PageArgs& pg, int rows, int nq, int tile) {
  const long long n = std::min(pg.n_windows, rows), queries = (long long)rows * (nq / pg.nkv);
  return n + (queries - n) / tile;   // 1 + (x - 1) / tile of x queries
}
constexpr int kFewTarget = 1024;
int tile_of(const PageArgs& pg, int rows, int nq) {
  return (long long)rows * (nq / pg.nkv) <= 32ll * pg.n_windows ? 32 : 64;
}
// Items of tiles cut into several chunks: work / per + tiles of them, and their
// tiles are fewer than work / per; in all KV heads twice the target
long long most_slots(const PageArgs& pg) { return 2ll * kFewTarget + pg.nkv; }

template <bool KVB, int HD>
hipError_t launch_few(const PageAttnArgs& a, dim3 grid, hipStream_t s) {
  if (a.bf16) {
    if (a.tile == 32) hipLaunchKernelGGL((k_page_few<KVB, HD, true, 1>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((k_page_few<KVB, HD, true, 2>), grid, dim3(256), 0, s, a);
  } else {
    if (a.tile == 32) hipLaunchKernelGGL((k_page_few<KVB, HD, false, 1>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((k_page_few<KVB, HD, false, 2>), grid, dim3(256), 0, s, a);
  }
  return hipGetLastError();
}
template <bool KVB>
hipError_t launch_few(const PageAttnArgs& a, dim3 grid, hipStream_t s) {
  switch (a.pg.hd) {
    case 32: return launch_few<KVB, 32>(a, grid, s);
    case 64: return launch_few<KVB, 64>(a, grid, s);
    case 96: return launch_few<KVB, 96>(a, grid, s);
    case 128: return launch_few<KVB, 128>(a, grid, s);
  }
  return hipErrorInvalidValue;
}

}  // namespace

size_t page_attend_workspace_bytes(const PageArgs& pg, int rows, int nq) {
  const int tile = tile_of(pg, rows, nq);
  return (size_t)most_slots(pg) * tile * (pg.hd * sizeof(float) + sizeof(float2));
}

hipError_t launch_page_attend(PageAttnArgs a, void* ws, hipStream_t s) {
  a.qlo = 1;
  a.qhi = INT_MAX;
  a.tile = tile_of(a.pg, a.rows, a.nq);
  a.target = kFewTarget;
  a.least = 1;
  a.ml = (float2*)ws;
  a.part = (float*)(a.ml + (size_t)most_slots(a.pg) * a.tile);
  const long long tiles = most_tiles(a.pg, a.rows, a.nq, a.tile), items = a.target / a.pg.nkv + 1 + tiles;
  if (items * a.pg.nkv > INT_MAX) return hipErrorInvalidValue;
  const dim3 grid((unsigned)(items * a.pg.nkv));
  hipError_t e = a.pg.kvb ? launch_few<true>(a, grid, s) : launch_few<false>(a, grid, s);
  if (e != hipSuccess) return e;
  const long long joins = std::min(tiles, (long long)a.target / a.pg.nkv + 1);
  hipLaunchKernelGGL(k_page_join, dim3((unsigned)(joins * a.pg.nkv)), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace dsi
