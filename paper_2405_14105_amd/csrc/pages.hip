// Attention of a step's rows over their windows' pages.
//
//   o = sum_j p_j v_j / sum_j p_j,  p_j = e^{scale q k_j - m},  m the maximum
//
// Rows and the heads that share a KV head are numbered together (query x = row
// * G + head of the group), so that tiles of queries are full whatever the
// group; a tile's keys are cut into chunks, an item is one chunk of one tile and
// KV head.  Lengths are the device's: every workgroup works out the cut itself
// from the windows' lengths and rows (about 2 us), so that items are about equally
// long and as many as the card takes whatever the windows are.
// S^T = K Q^T and O^T = V^T P^T in 32 x 32 x 16 MFMAs: the rows of the K operand
// are taken in an order in which a lane's scores are already its fragments of
// P^T, and a block's layout is such that every operand is 16 contiguous bytes.
// Parts of a tile are joined by a second launch.
// Windows of up to 64 queries of a KV head (few rows) are bound by reading the pages,
// others by the matrix cores: two kernels, or one launch of both.
#include <algorithm>
#include <climits>
#include <type_traits>

#include "pages.h"

namespace dsi {

namespace {

typedef __attribute__((__vector_size__(16 * sizeof(float)))) float f32x16;

constexpr int kUnit = 128;        // keys of a unit, in which chunks are counted

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

// A window of the class: tiles of 32 qw queries
struct Win {
  int r0, R, len, bad;  // bad: its rows do not fit
  int tiles, qw, units; // units of kUnit keys that a tile's rows see, at most
};
__device__ __forceinline__ Win window_at(const PageAttnArgs& a, const PageClass& cl, int b) {
  Win w{0, 0, 0, 0, 0, 1, 0};
  if (b >= a.pg.n_windows) return w;
  int r1;
  window_rows(a.pg, a.rows, b, w.r0, r1);
  w.R = r1 - w.r0;
  const int queries = w.R * a.G;
  if (queries < cl.qlo || queries > cl.qhi) return w;
  w.len = a.pg.len[b];
  w.bad = w.len < 0 || (long long)w.len + w.R > window_positions(a.pg);
  if (w.bad) w.len = 0;
  w.qw = cl.qw ? cl.qw : queries > 32 ? 2 : 1;
  const int T = 32 * w.qw;
  w.tiles = (unsigned)(queries + T - 1) / (unsigned)T;
  int span = w.bad ? 1 : w.len + w.R;
  if (a.reach) span = min(span, a.reach + (int)((unsigned)(T + a.G - 2) / (unsigned)a.G) + 31);   // a tile's rows, from a block's first position on
  w.units = (span + kUnit - 1) / kUnit;
  return w;
}
// How a class is cut: units of an item at most, and all items, or with JOIN the groups
// of 32 queries of tiles that are cut.  Up to 64 windows every lane of every wave works
// it out, a window a lane: the window's items, and the slots of their parts, with those
// of the lanes before.  For more windows a launch of its own has written it down.
struct Plan {
  Win w;
  int per, total;
  int n, incl, split, sincl;
};
// chunks of a tile: the last one may be a quarter longer than the others
__device__ __forceinline__ int chunks_of(int units, int per) {
  return max(1, (int)((unsigned)(units + per - 1 - (per >> 2)) / (unsigned)per));
}
template <bool JOIN>
__device__ __forceinline__ void count(Plan& p) {
  const int chunks = chunks_of(p.w.units, p.per), items = p.w.tiles * chunks;
  p.split = chunks > 1 ? items * p.w.qw : 0;
  p.n = JOIN ? (chunks > 1 ? p.w.tiles * p.w.qw : 0) : items;
  p.incl = wave_scan_incl(p.n);
  p.sincl = wave_scan_incl(p.split);
}
// one item for each workgroup that the card holds where that leaves items short,
// more of them, at most `most`, where they would be long
__device__ __forceinline__ int units_per_item(const PageClass& cl, double work, bool& once_enough) {
  const double once = ceil(work * cl.inv_once), fine = ceil(work * cl.inv_most);
  once_enough = once <= cl.enough;
  return (int)fmin(fmax(fmax(fine, fmin(once, (double)cl.enough)), 1.0), 1e9);
}
template <bool JOIN>
__device__ __forceinline__ Plan plan_of(const PageAttnArgs& a, const PageClass& cl) {
  Plan p;
  if (cl.plan) {
    p.per = cl.plan[0];
    p.total = cl.plan[JOIN ? 2 : 1];
    return p;
  }
  p.w = window_at(a, cl, threadIdx.x & 63);
  bool once_enough;
  p.per = units_per_item(cl, wave_sum((double)(p.w.tiles * p.w.qw) * p.w.units) * a.pg.nkv, once_enough);
  // chunks are whole: a few units more where they are a few items too many for one turn
  if (once_enough && (long long)wave_total(p.w.tiles * p.w.qw) * a.pg.nkv <= cl.once) {
    for (int i = 0; i < 6; ++i) {
      const int items = wave_total(p.w.tiles * p.w.qw * chunks_of(p.w.units, p.per));
      if ((long long)items * a.pg.nkv <= cl.once) break;
      p.per += (p.per + 7) >> 3;
    }
  }
  count<JOIN>(p);
  p.total = __builtin_amdgcn_readlane(p.incl, 63);
  return p;
}
// The cut of more than 64 windows, a workgroup a class: units of an item, items, groups
// of 32 queries to join; then items, groups and slots of the windows up to and with each
constexpr int kPlanHead = 4, kPlanWindows = 4;   // windows a thread
// Sums of items stop at the largest int (items of windows in order are far fewer: 2^28
// queries are 2^21 tiles, and cuts add what the workspace holds).  Rows that thousands of
// windows claim may have more; sums that wrapped would put items outside their windows.
__device__ __forceinline__ int capped_sum(int a, int b) { return (int)min((unsigned)a + (unsigned)b, (unsigned)INT_MAX); }
__global__ __launch_bounds__(1024) void k_page_plan(PageAttnArgs a, PageClass few, PageClass many, int first) {
  __shared__ double works[16];
  __shared__ int sums[3][16];
  const PageClass& cl = (int)blockIdx.x + first ? many : few;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  Win win[kPlanWindows];
  double work = 0.0;
#pragma unroll
  for (int i = 0; i < kPlanWindows; ++i) {
    win[i] = window_at(a, cl, threadIdx.x * kPlanWindows + i);
    work += (double)(win[i].tiles * win[i].qw) * win[i].units;
  }
  work = wave_sum(work);
  if (lane == 0) works[w] = work;
  __syncthreads();
  work = 0.0;
  for (int i = 0; i < 16; ++i) work += works[i];
  bool once_enough;
  const int per = units_per_item(cl, work * a.pg.nkv, once_enough);
  int v[3][kPlanWindows], before[3] = {0, 0, 0};
#pragma unroll
  for (int i = 0; i < kPlanWindows; ++i) {
    const int chunks = chunks_of(win[i].units, per), items = win[i].tiles * chunks;
    v[0][i] = before[0] = capped_sum(before[0], items);
    v[1][i] = before[1] += chunks > 1 ? win[i].tiles * win[i].qw : 0;
    v[2][i] = before[2] += chunks > 1 ? items * win[i].qw : 0;
  }
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    int incl = before[k];
    dpp_steps([&](auto s) { incl = capped_sum(incl, dpp_from<decltype(s)::ctrl, decltype(s)::rows>(0, incl)); });
    if (lane == 63) sums[k][w] = incl;
    before[k] = __shfl_up(incl, 1);
    if (lane == 0) before[k] = 0;
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    int total = 0;
    for (int i = 0; i < 16; ++i) {
      if (i < w) before[k] = capped_sum(before[k], sums[k][i]);
      total = capped_sum(total, sums[k][i]);
    }
#pragma unroll
    for (int i = 0; i < kPlanWindows; ++i) {
      const int b = threadIdx.x * kPlanWindows + i;
      if (b < a.pg.n_windows) cl.plan[kPlanHead + k * a.pg.n_windows + b] = capped_sum(before[k], v[k][i]);
    }
    if (threadIdx.x == 0 && k < 2) cl.plan[1 + k] = total;
  }
  if (threadIdx.x == 0) cl.plan[0] = per;
}
// One item: chunk `chunk` of `chunks` of a tile; JOIN: the 32 queries `sub` of a
// tile of several chunks
struct Item {
  Win w;
  int b, per;           // units of a chunk of this window: as even as they come
  int tile, chunk, chunks, sub;
  int slot;             // of the tile's first 32 queries and chunk 0 (qw slots a chunk)
};
template <bool JOIN>
__device__ __forceinline__ bool find(const PageAttnArgs& a, const PageClass& cl, const Plan& p, int t, Item& it) {
  if (t >= p.total) return false;
  const int lane = threadIdx.x & 63;
  auto at = [&](int v, int l) { return __builtin_amdgcn_readlane(v, l); };
  int in, slot;         // the item's number in its window, slots of the windows before
  if (cl.plan) {
    const int n = a.pg.n_windows;
    const int* upto = cl.plan + kPlanHead + (JOIN ? n : 0);
    const int v = upto[min(lane * 64 + 63, n - 1)];
    const int g = __ffsll((long long)__ballot(v > t)) - 1;
    const int u = upto[min(g * 64 + lane, n - 1)];
    const int l = __ffsll((long long)__ballot(u > t)) - 1;
    it.b = g * 64 + l;
    in = t - (l ? at(u, l - 1) : g ? at(v, g - 1) : 0);
    slot = it.b ? cl.plan[kPlanHead + 2 * n + it.b - 1] : 0;
    it.w = window_at(a, cl, it.b);
  } else {
    const int l = __ffsll((long long)__ballot(p.incl > t)) - 1;
    it.b = l;
    in = t - at(p.incl - p.n, l);
    slot = at(p.sincl - p.split, l);
    it.w = Win{at(p.w.r0, l), at(p.w.R, l), at(p.w.len, l), at(p.w.bad, l), at(p.w.tiles, l), at(p.w.qw, l), at(p.w.units, l)};
  }
  it.chunks = chunks_of(it.w.units, p.per);
  it.per = (unsigned)(it.w.units + it.chunks - 1) / (unsigned)it.chunks;
  if (JOIN) {
    it.tile = (unsigned)in / (unsigned)it.w.qw;
    it.sub = in - it.tile * it.w.qw;
    it.chunk = 0;
  } else {
    const int tile = (unsigned)in / (unsigned)it.chunks;
    it.chunk = in - tile * it.chunks;
    it.tile = it.w.tiles - 1 - tile;   // the longest first
    it.sub = 0;
  }
  it.slot = slot + it.tile * it.chunks * it.w.qw;
  // rows of windows that overlap may need more than there are: no output (NaN)
  if (it.chunks > 1 && it.slot + it.chunks * it.w.qw > cl.slots) it.w.bad = 1;
  return true;
}
// positions of the first and the last row of queries [x0, x0 + n) of a window,
// and the positions [lo, hi) that they see, lo the first of its block
struct Span {
  int first, last, lo, hi;
};
__device__ __forceinline__ Span span_of(const PageAttnArgs& a, const Win& w, int x0, int n) {
  Span s;
  s.first = w.len + (int)((unsigned)x0 / (unsigned)a.G);
  s.last = w.len + min(w.R - 1, (int)((unsigned)(x0 + n - 1) / (unsigned)a.G));
  s.lo = a.reach ? max(0, s.first - a.reach + 1) & ~31 : 0;
  s.hi = s.last + 1;
  return s;
}
// query x of a window (the last one past the end): row, head of the KV head's group, position
__device__ __forceinline__ bool query_at(const PageAttnArgs& a, const Win& w, int x, int& row, int& g, int& pos) {
  const int NX = w.R * a.G, y = min(x, NX - 1), i = (unsigned)y / (unsigned)a.G;
  row = w.r0 + i;
  g = y - i * a.G;
  pos = w.len + i;
  return x < NX;
}
template <bool QB>
__device__ __forceinline__ void store_out(const PageAttnArgs& a, size_t at, const float (&v)[4]) {
  if constexpr (QB) *(uint2*)((uint16_t*)a.out + at) = uint2{f2bf_pair(v[0], v[1]), f2bf_pair(v[2], v[3])};
  else *(f32x4*)((float*)a.out + at) = f32x4{v[0], v[1], v[2], v[3]};
}

// ------------------------------------------------------------------ operands

// the parts of eight fp32 numbers in bf16
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
// Where a lane's entries of a block's fragments lie in it: keys [hd/32][32][32],
// the key of operand row q32 in the order that leaves P^T in place; values [hd][32]
__device__ __forceinline__ int key_offset(int lane, int ds) {
  const int r = lane & 31, key = 16 * (r >> 4) + 8 * ((r >> 2) & 1) + 4 * ((r >> 3) & 1) + (r & 3);
  return (ds >> 1) * 1024 + key * 32 + (ds & 1) * 16 + (lane >> 5) * 8;
}
__device__ __forceinline__ int value_offset(int lane, int t, int h) { return (t * 32 + (lane & 31)) * 32 + h * 16 + (lane >> 5) * 8; }

// what a wave needs of its 32 queries: fragment ds, part i
template <bool KVB, bool QB>
__device__ __forceinline__ void load_query(const PageAttnArgs& a, size_t at, u32x4 (&p)[KVB ? (QB ? 1 : 3) : 2]) {
  if constexpr (QB && KVB) {
    p[0] = *(const u32x4*)((const uint16_t*)a.q + at);
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
      split_parts<3>(v, p);
    } else {
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) p[i][e] = __float_as_uint(v[4 * i + e]);
    }
  }
}
// s += K Q^T of one fragment; p: the query's parts (fp32 caches: its eight entries)
template <bool KVB, int N>
__device__ __forceinline__ void scores(f32x16& s, const Frag<KVB>& k, const u32x4 (&p)[N]) {
  if constexpr (KVB) {
#pragma unroll
    for (int i = 0; i < N; ++i) s = mfma32(k.p[0], p[i], s);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      s = __builtin_amdgcn_mfma_f32_32x32x2f32(f32_of(k, e), __uint_as_float(p[e >> 2][e & 3]), s, 0, 0, 0);
  }
}

// A wave's running softmax of 32 queries: lane (query lane & 31), its half of the keys
struct Running {
  float m, l;           // maximum (base 2, scaled) of all lanes of the query; sum of this lane's keys
};
// Scores of keys that a query does not see become -inf, and vis gets a bit for each
// of the others: lane's entry r is key 16 (r / 8) + 8 (lane / 32) + r % 8 from p0 on.
// A block without a page has NaN for every key that is seen.
__device__ __forceinline__ void mask_scores(f32x16& s, uint32_t& vis, bool page, int p0, int pos, int from) {
  const int hh = (threadIdx.x & 63) >> 5;
  vis = 0;
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const int kp = p0 + 16 * (r >> 3) + 8 * hh + (r & 7);
    const bool in = kp <= pos && kp >= from;
    vis |= in ? 1u << r : 0u;
    s[r] = in ? (page ? s[r] : NAN) : -INFINITY;
  }
}
// Scores of NB blocks to probabilities.  True if the maximum of a lane moved: what
// is summed so far is to be multiplied by alpha.
template <int NB>
__device__ __forceinline__ bool probabilities(f32x16 (&s)[NB], Running& run, float& alpha, float scale2) {
  float mx = s[0][0];
#pragma unroll
  for (int n = 0; n < NB; ++n)
#pragma unroll
    for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[n][r]);
  const float mnew = fmaxf(run.m, max_over_32(mx) * scale2);
  const float base = mnew == -INFINITY ? 0.f : mnew;
  alpha = __builtin_amdgcn_exp2f(run.m - base);
  const bool moved = mnew != run.m;
  float sum = 0.f;
#pragma unroll
  for (int n = 0; n < NB; ++n)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      s[n][r] = __builtin_amdgcn_exp2f(fmaf(s[n][r], scale2, -base));
      sum += s[n][r];
    }
  run.l = run.l * alpha + sum;
  run.m = mnew;
  return moved;
}

// whether a value fragment holds anything that is not finite (this lane's part)
__device__ __forceinline__ bool not_finite(const Frag<true>& f) {
  bool x = false;
#pragma unroll
  for (int e = 0; e < 4; ++e) x |= (f.p[0][e] & 0x7F80u) == 0x7F80u || (f.p[0][e] & 0x7F800000u) == 0x7F800000u;
  return x;
}
__device__ __forceinline__ bool not_finite(const Frag<false>& f) {
  bool x = false;
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) x |= (f.p[i][e] & 0x7F800000u) == 0x7F800000u;
  return x;
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
// Values that only some rows see, or none (dead positions of a page): what is not
// finite among them is taken out and counted apart with the rows that see it, so
// that it reaches no other row's sum (0 * NaN)
template <bool KVB>
__device__ __forceinline__ void guard_values(f32x16& o, Frag<KVB>& v, uint32_t vis8) {
  Frag<KVB> ind;
  if (!part_finite(v, ind)) return;
  f32x16 c = zero16();
  if constexpr (KVB) {
    u32x4 one;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t two = vis8 >> (2 * e);
      one[e] = (two & 1 ? 0x3F80u : 0u) | (two & 2 ? 0x3F800000u : 0u);
    }
    c = mfma32(ind.p[0], one, c);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(f32_of(ind, e), vis8 >> e & 1 ? 1.f : 0.f, c, 0, 0, 0);
  }
#pragma unroll
  for (int r = 0; r < 16; ++r) o[r] = c[r] > 0.f ? NAN : o[r];
}
// o += V^T P^T of one fragment; pf: the probabilities' parts (fp32 caches: none), s
// the probabilities, h the half of the block
template <bool KVB, int N>
__device__ __forceinline__ void outputs(f32x16& o, const Frag<KVB>& v, const u32x4 (&pf)[N], const f32x16& s, int h) {
  if constexpr (KVB) {
#pragma unroll
    for (int i = 0; i < N; ++i) o = mfma32(v.p[0], pf[i], o);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) o = __builtin_amdgcn_mfma_f32_32x32x2f32(f32_of(v, e), s[8 * h + e], o, 0, 0, 0);
  }
}
template <int N>
__device__ __forceinline__ void half_parts(const f32x16& s, int h, u32x4 (&p)[N]) {
  float v[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = s[8 * h + e];
  split_parts<N>(v, p);
}

// the outputs of a window whose rows do not fit, or of one tile's queries: NaN
template <bool QB, int HD>
__device__ __forceinline__ void store_nan(const PageAttnArgs& a, const Item& it, int kvh) {
  const int T = 32 * it.w.qw;
  for (int i = threadIdx.x; i < T * (HD / 4); i += blockDim.x) {
    int row, g, pos;
    if (!query_at(a, it.w, it.tile * T + i / (HD / 4), row, g, pos)) continue;
    const float v[4] = {NAN, NAN, NAN, NAN};
    store_out<QB>(a, (size_t)row * a.ldo + (size_t)(kvh * a.G + g) * HD + i % (HD / 4) * 4, v);
  }
}

// ------------------------------------------------------------------ few rows

// One item of a tile of 32 or 64 queries: waves take 32 of them each, and the
// chunk's blocks of 32 keys in turn (four waves a block apart, or two pairs), each
// with a maximum, a sum and outputs of its own; they meet in LDS at the end.  A
// block's keys and values go from memory to registers, the next block's while
// this one's are worked on; queries lie in LDS in fragment order.
// Bound by reading the pages: 8B, 32 single rows over 100 to 31131 positions (2.05 GB)
// 352 us, 5.8 TB/s.  Few and short windows are bound by a chain of loads (rows and
// lengths, table, keys) and the meeting of the waves: 4 rows of 1B over up to 512
// positions 8.3 us, 7 x 6 fp32 rows of 8B over 2048 (61 MB) 18.5.  64 queries in one
// wave took 65 us there, with the spills of its 128 outputs a lane.
// A query over a bf16 cache is one bf16 part, or three for fp32 queries (exact); a
// probability two, 2^-16 of it left, or three; fp32 caches take fp32 MFMAs.
template <bool KVB, int HD, bool QB>
struct FewShared {
  static constexpr int QT = KVB ? (QB ? 1 : 3) : 2, DS = HD / 16, OS = HD + 4;
  static constexpr int kQ = 2 * QT * DS * 64, kO = 4 * 32 * OS / 4;
  u32x4 sm[kQ > kO ? kQ : kO];
  float wm[4][32], wl[4][32];
};
template <bool KVB, int HD, bool QB>
__device__ __forceinline__ void few_item(const PageAttnArgs& a, const PageClass& cl, const Item& it, int kvh, FewShared<KVB, HD, QB>& sh) {
  constexpr int QT = KVB ? (QB ? 1 : 3) : 2, PT = KVB ? (QB ? 2 : 3) : 1;
  constexpr int DS = HD / 16, DT = HD / 32;
  constexpr int OS = HD + 4;                               // floats from a query's outputs to the next's in LDS
  u32x4* const sm = sh.sm;
  auto& wm = sh.wm;
  auto& wl = sh.wl;
  const int lane = threadIdx.x & 63, q32 = lane & 31, hh = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (it.w.bad) {
    store_nan<QB, HD>(a, it, kvh);
    return;
  }
  const int qw = it.w.qw, T = 32 * qw, kw = 4 / qw;        // waves along the keys
  const int wq = w & (qw - 1), wk = qw == 1 ? w : w >> 1;
  const Span sp = span_of(a, it.w, it.tile * T, T);
  const Span my = span_of(a, it.w, it.tile * T + wq * 32, 32);
  // blocks of this wave: kb0 + wk + kw i; lane l knows the pool's block of i = 64 g + l
  const int kb0 = (int)min((long long)(sp.lo >> 5) + (long long)it.chunk * it.per * (kUnit / 32), 1ll << 30);
  const int kb1 = (int)min((long long)kb0 + (long long)it.per * (kUnit / 32), (long long)((sp.hi + 31) >> 5));
  const int nb = kb1 > kb0 + wk ? (kb1 - kb0 - wk + kw - 1) / kw : 0;
  int mine = -1;
  auto look = [&](int i0) {
    const int kb = kb0 + wk + kw * (i0 + lane);
    mine = kb < kb1 ? (int)block_of(a.pg, it.b, kvh, kb) : -1;
  };
  if (nb) look(0);
  int row, g, pos;
  query_at(a, it.w, it.tile * T + wq * 32 + q32, row, g, pos);
  const int from = a.reach ? pos - a.reach + 1 : 0;
  // queries into LDS, each group of 32 by the waves that work on it
  for (int ds = wk; ds < DS; ds += kw) {
    u32x4 p[QT];
    load_query<KVB, QB>(a, (size_t)row * a.ldq + (size_t)(kvh * a.G + g) * HD + ds * 16 + hh * 8, p);
#pragma unroll
    for (int i = 0; i < QT; ++i) sm[((wq * DS + ds) * QT + i) * 64 + lane] = p[i];
  }
  Frag<KVB> kf[DS], vf[DT][2];
  // of a block without a page, block 0 of the pool is read, and masked
  auto load_k = [&](int blk) {
#pragma unroll
    for (int ds = 0; ds < DS; ++ds) kf[ds] = load_frag<KVB>(a.pg.k, (size_t)max(blk, 0) * (32 * HD) + key_offset(lane, ds));
  };
  auto load_v = [&](int blk) {
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
      for (int h = 0; h < 2; ++h) vf[t][h] = load_frag<KVB>(a.pg.v, (size_t)max(blk, 0) * (32 * HD) + value_offset(lane, t, h));
  };
  Running run{-INFINITY, 0.f};
  f32x16 o[DT];
#pragma unroll
  for (int t = 0; t < DT; ++t) o[t] = zero16();
  int blk = -1;
  if (nb) {
    blk = __builtin_amdgcn_readlane(mine, 0);
    load_k(blk);
    load_v(blk);
  }
  __syncthreads();
  for (int i = 0; i < nb; ++i) {
    const int p0 = (kb0 + wk + kw * i) * 32;
    const bool more = i + 1 < nb;
    int next = -1;
    if (more) {
      if (((i + 1) & 63) == 0) look(i + 1);
      next = __builtin_amdgcn_readlane(mine, (i + 1) & 63);
    }
    asm volatile("" ::: "memory");   // the queries are read again in each turn, not kept in registers
    f32x16 s[1] = {zero16()};
#pragma unroll
    for (int ds = 0; ds < DS; ++ds) {
      u32x4 p[QT];
#pragma unroll
      for (int e = 0; e < QT; ++e) p[e] = sm[((wq * DS + ds) * QT + e) * 64 + lane];
      scores<KVB>(s[0], kf[ds], p);
    }
    if (more) load_k(next);
    // not every query sees every key
    if (blk < 0 || p0 + 31 > my.first || (a.reach && p0 <= my.last - a.reach)) {
      uint32_t vis;
      mask_scores(s[0], vis, blk >= 0, p0, pos, from);
#pragma unroll
      for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int h = 0; h < 2; ++h) guard_values<KVB>(o[t], vf[t][h], vis >> (8 * h));
    }
    float alpha;
    if (__ballot(probabilities(s, run, alpha, a.scale2))) {
#pragma unroll
      for (int t = 0; t < DT; ++t) o[t] *= alpha;
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      u32x4 pf[PT];
      if constexpr (KVB) half_parts<PT>(s[0], h, pf);
#pragma unroll
      for (int t = 0; t < DT; ++t) outputs<KVB>(o[t], vf[t][h], pf, s[0], h);
    }
    if (more) load_v(next);
    blk = next;
  }

  // the waves meet
  run.l = sum_over_32(run.l);
  if (hh == 0) {
    wm[w][q32] = run.m;
    wl[w][q32] = run.l;
  }
  __syncthreads();   // and the queries are no longer read
  float* const so = (float*)sm;
  {
    float M = -INFINITY;
    for (int i = 0; i < kw; ++i) M = fmaxf(M, wm[wq + i * qw][q32]);
    const float f = __builtin_amdgcn_exp2f(run.m - (M == -INFINITY ? 0.f : M));
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        *(f32x4*)(so + (w * 32 + q32) * OS + t * 32 + 8 * j + 4 * hh) = f32x4{o[t][4 * j] * f, o[t][4 * j + 1] * f, o[t][4 * j + 2] * f, o[t][4 * j + 3] * f};
  }
  __syncthreads();
  // HD / 4 threads a query
  for (int i = threadIdx.x; i < T * (HD / 4); i += 256) {
    const int q = i / (HD / 4), d = i % (HD / 4) * 4, n = q >> 5, qq = q & 31;
    if (!query_at(a, it.w, it.tile * T + q, row, g, pos)) continue;
    float M = -INFINITY, L = 0.f;
    for (int k = 0; k < kw; ++k) M = fmaxf(M, wm[n + k * qw][qq]);
    const float base = M == -INFINITY ? 0.f : M;
    f32x4 v = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int k = 0; k < kw; ++k) {
      const int ww = n + k * qw;
      L += wl[ww][qq] * __builtin_amdgcn_exp2f(wm[ww][qq] - base);
      v += *(const f32x4*)(so + (ww * 32 + qq) * OS + d);
    }
    if (it.chunks > 1) {
      const size_t slot = ((size_t)it.slot + it.chunk * qw + n) * a.pg.nkv + kvh;
      *(f32x4*)(cl.part + (slot * 32 + qq) * HD + d) = v;
      if (d == 0) cl.ml[slot * 32 + qq] = make_float2(M, L);
    } else {
      const float inv = 1.f / L, y[4] = {v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv};
      store_out<QB>(a, (size_t)row * a.ldo + (size_t)(kvh * a.G + g) * HD + d, y);
    }
  }
}

// ------------------------------------------------------------------ many rows

// One item of a tile of 128 queries: each of four waves takes 32 of them, and all of
// them the same stages of KS blocks of 32 keys, which go through LDS in fragment
// order, the next one's on their way while one is worked on.  Queries stay in
// registers.  Bound by the matrix cores, the fragment reads from LDS and the
// exponentials: 8B, 2048 rows after 30000 positions 1.44 ms, 0.72 PFLOP/s of the
// formula's products and 1.08 of those done (the second one twice), where a large
// library product reaches 1.14.  (All with one part, 1.10: fragments from memory to
// registers, each wave its own: 1.88 ms.  Eight waves and stages through registers:
// 1.28.  Four waves that way: 2.87, out of registers.)  A wave's loads of its queries have to be waited for
// before the loop: the compiler's wait for them in it would be one for the stage just
// asked for.
// A probability of bf16 queries is two bf16 parts, 2^-16 of it left, as where rows are
// few: the call's rows, not what a caller asks for, say which kernel a row meets.  One
// part is a third less matrix work (2048 rows at 30000: 1.07 ms instead of 1.44; 13B,
// 512 + 7 rows: 138 us instead of 149), but its rounding, 2^-8, adds as much to the
// outputs as their own (off by 2.0e-3 of their norm in all, two parts 1.7e-3).
template <bool KVB, int HD>
struct ManyShared {
  static constexpr int KS = KVB ? 2 : 1, FP = KVB ? 1 : 2, DS = HD / 16, DT = HD / 32;
  static constexpr int FB = DS + 2 * DT, FR = KS * FB;     // fragments of a block, of a stage
  u32x4 kv[2][FR][FP][64];
};
// 16 bytes a lane from memory (`off` bytes behind `from`, by the lane) into LDS, lane
// by lane from `to` on, past the registers; in order with the wave's loads, and
// complete once vmcnt says so
__device__ __forceinline__ void load_lds(const void* from, uint32_t off, uint32_t to) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(from), "s"(to) : "memory");
}
template <bool KVB, int HD, bool QB>
__device__ __forceinline__ void many_item(const PageAttnArgs& a, const PageClass& cl, int block, ManyShared<KVB, HD>& sh) {
  constexpr int NW = 4, QT = KVB ? (QB ? 1 : 3) : 2, PT = KVB ? (QB ? 2 : 3) : 1;
  typedef ManyShared<KVB, HD> S;
  constexpr int KS = S::KS, FP = S::FP, DS = S::DS, DT = S::DT, FB = S::FB, FR = S::FR;
  static_assert(sizeof(S) <= 1 << 16, "offsets of 16 bits");
  constexpr int MINE = (FR + NW - 1) / NW;                  // fragments loaded by one wave
  const int lane = threadIdx.x & 63, q32 = lane & 31, hh = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kvh = block % a.pg.nkv;
  Item it;
  if (!find<false>(a, cl, plan_of<false>(a, cl), block / a.pg.nkv, it)) return;
  if (it.w.bad) {
    store_nan<QB, HD>(a, it, kvh);
    return;
  }
  const int T = 32 * NW, x0 = it.tile * T + w * 32;
  const bool live = x0 < it.w.R * a.G;
  const Span sp = span_of(a, it.w, it.tile * T, T);
  const Span my = span_of(a, it.w, x0, 32);
  const int kb0 = (int)min((long long)(sp.lo >> 5) + (long long)it.chunk * it.per * (kUnit / 32), 1ll << 30);
  const int kb1 = (int)min((long long)kb0 + (long long)it.per * (kUnit / 32), (long long)((sp.hi + 31) >> 5));
  const int ns = kb1 > kb0 ? (kb1 - kb0 + KS - 1) / KS : 0;     // stages
  // lane l knows the pool's block of kb0 + 64 g + l
  int mine = -1;
  auto look = [&](int i0) {
    const int kb = kb0 + i0 + lane;
    mine = kb < kb1 ? (int)block_of(a.pg, it.b, kvh, kb) : -1;
  };
  int row, g, pos;
  query_at(a, it.w, x0 + q32, row, g, pos);
  const int from = a.reach ? pos - a.reach + 1 : 0;
  u32x4 q[DS][QT];
#pragma unroll
  for (int ds = 0; ds < DS; ++ds) load_query<KVB, QB>(a, (size_t)row * a.ldq + (size_t)(kvh * a.G + g) * HD + ds * 16 + hh * 8, q[ds]);

  // all that the wave loaded into registers is there: what it waits for in the loop
  // must not be the next stage
  look(0);
#pragma unroll
  for (int ds = 0; ds < DS; ++ds)
#pragma unroll
    for (int i = 0; i < QT; ++i) asm volatile("" : "+v"(q[ds][i]));
  asm volatile("" : "+v"(mine));

  const uint32_t lds = (uint32_t)(size_t)(__attribute__((address_space(3))) void*)&sh.kv[0][0][0][0];
  // of a block without a page, or past the last, block 0 of the pool is read, and masked
  auto load_stage = [&](const int (&b)[KS], int buf) {
#pragma unroll
    for (int j = 0; j < MINE; ++j) {
      const int f = w + NW * j, n = KS == 1 ? 0 : f / FB, r = f - n * FB;
      if (FR % NW && f >= FR) continue;
      const size_t at = (size_t)max(b[n], 0) * (32 * HD) + (r < DS ? key_offset(0, r) : value_offset(0, (r - DS) >> 1, (r - DS) & 1));
      const char* src = (const char*)(r < DS ? a.pg.k : a.pg.v) + at * (KVB ? 2 : 4);
      const uint32_t off = (uint32_t)(r < DS ? key_offset(lane, 0) : value_offset(lane, 0, 0)) * (KVB ? 2 : 4);
#pragma unroll
      for (int i = 0; i < FP; ++i) load_lds(src + 16 * i, off, lds + (uint32_t)(((buf * FR + f) * FP + i) * 1024));
    }
  };
  auto frag = [&](int buf, int f) {
    Frag<KVB> x;
#pragma unroll
    for (int i = 0; i < FP; ++i) x.p[i] = sh.kv[buf][f][i][lane];
    return x;
  };
  Running run{-INFINITY, 0.f};
  f32x16 o[DT];
#pragma unroll
  for (int t = 0; t < DT; ++t) o[t] = zero16();
  auto values = [&](auto guarded, const f32x16 (&s)[KS], const uint32_t (&vis)[KS], int buf) {
#pragma unroll
    for (int n = 0; n < KS; ++n)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        u32x4 pf[PT];
        if constexpr (KVB) half_parts<PT>(s[n], h, pf);
#pragma unroll
        for (int t = 0; t < DT; ++t) {
          Frag<KVB> v = frag(buf, n * FB + DS + 2 * t + h);
          if constexpr (decltype(guarded)::value) guard_values<KVB>(o[t], v, vis[n] >> (8 * h));
          outputs<KVB>(o[t], v, pf, s[n], h);
        }
      }
  };
  int b[KS] = {};       // the stage's blocks
  if (ns) {
#pragma unroll
    for (int n = 0; n < KS; ++n) b[n] = __builtin_amdgcn_readlane(mine, n);
    load_stage(b, 0);
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  for (int st = 0; st < ns; ++st) {
    const int buf = st & 1, p0 = (kb0 + KS * st) * 32;
    int next[KS] = {};
    if (st + 1 < ns) {
      if (((KS * (st + 1)) & 63) == 0) look(KS * (st + 1));
#pragma unroll
      for (int n = 0; n < KS; ++n) next[n] = __builtin_amdgcn_readlane(mine, (KS * (st + 1) + n) & 63);
      load_stage(next, buf ^ 1);
    }
    if (live && p0 <= my.last && p0 + 32 * KS - 1 >= my.lo) {
      f32x16 s[KS];
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int n = 0; n < KS; ++n) s[n] = zero16();
#pragma unroll
      for (int ds = 0; ds < DS; ++ds)
#pragma unroll
        for (int n = 0; n < KS; ++n) scores<KVB>(s[n], frag(buf, n * FB + ds), q[ds]);
      __builtin_amdgcn_s_setprio(0);
      // not every query sees every key
      bool some = p0 + 32 * KS - 1 > my.first || (a.reach && p0 <= my.last - a.reach);
#pragma unroll
      for (int n = 0; n < KS; ++n) some |= b[n] < 0;
      uint32_t vis[KS];
      if (some) {
#pragma unroll
        for (int n = 0; n < KS; ++n) mask_scores(s[n], vis[n], b[n] >= 0, p0 + 32 * n, pos, from);
        bool odd = false;   // values that need a guard
#pragma unroll
        for (int f = 0; f < KS * 2 * DT; ++f) odd |= not_finite(frag(buf, f / (2 * DT) * FB + DS + f % (2 * DT)));
        some = __ballot(odd) != 0;
      }
      float alpha;
      if (__ballot(probabilities(s, run, alpha, a.scale2))) {
#pragma unroll
        for (int t = 0; t < DT; ++t) o[t] *= alpha;
      }
      __builtin_amdgcn_s_setprio(1);
      if (__builtin_expect(some, 0)) values(std::true_type{}, s, vis, buf);
      else values(std::false_type{}, s, vis, buf);
      __builtin_amdgcn_s_setprio(0);
    }
#pragma unroll
    for (int n = 0; n < KS; ++n) b[n] = next[n];
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // the next stage is in LDS, this wave's part
    __syncthreads();
  }
  run.l = sum_over_32(run.l);
  if (x0 + q32 >= it.w.R * a.G) return;
  if (it.chunks > 1) {
    const size_t slot = ((size_t)it.slot + it.chunk * NW + w) * a.pg.nkv + kvh;
    float* po = cl.part + (slot * 32 + q32) * HD + 4 * hh;
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
      for (int j = 0; j < 4; ++j) *(f32x4*)(po + t * 32 + 8 * j) = f32x4{o[t][4 * j], o[t][4 * j + 1], o[t][4 * j + 2], o[t][4 * j + 3]};
    if (hh == 0) cl.ml[slot * 32 + q32] = make_float2(run.m, run.l);
    return;
  }
  const float inv = 1.f / run.l;
  const size_t at = (size_t)row * a.ldo + (size_t)(kvh * a.G + g) * HD + 4 * hh;
#pragma unroll
  for (int t = 0; t < DT; ++t)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float y[4] = {o[t][4 * j] * inv, o[t][4 * j + 1] * inv, o[t][4 * j + 2] * inv, o[t][4 * j + 3] * inv};
      store_out<QB>(a, at + t * 32 + 8 * j, y);
    }
}

// Items of windows of few rows: `blocks` workgroups take them in turn, so that a call
// of few items has few workgroups that look for one
template <bool KVB, int HD, bool QB>
__device__ __forceinline__ void few_items(const PageAttnArgs& a, const PageClass& cl, int block, int blocks, FewShared<KVB, HD, QB>& sh) {
  const Plan p = plan_of<false>(a, cl);
  Item it;
  for (int t = block; find<false>(a, cl, p, t / a.pg.nkv, it); t += blocks) {
    if (t != block) __syncthreads();   // the item before has been read
    few_item(a, cl, it, t % a.pg.nkv, sh);
  }
}

template <bool KVB, int HD, bool QB>
__global__ __launch_bounds__(256, KVB || HD < 128 ? 2 : 1) void k_page_few(PageAttnArgs a, PageClass cl) {
  __shared__ FewShared<KVB, HD, QB> sh;
  few_items<KVB, HD, QB>(a, cl, blockIdx.x, gridDim.x, sh);
}
// Two workgroups fit a CU but where fp32 queries or keys of wide heads take more than
// 256 registers.  (bf16 ones of head dim 128 take all of them and 20 bytes of scratch a lane.)
constexpr bool many_two(bool kvb, int hd, bool qb) { return hd <= 64 || (kvb && qb); }
template <bool KVB, int HD, bool QB>
__global__ __launch_bounds__(256, many_two(KVB, HD, QB) ? 2 : 1) void k_page_many(PageAttnArgs a, PageClass cl) {
  __shared__ ManyShared<KVB, HD> sh;
  many_item<KVB, HD, QB>(a, cl, blockIdx.x, sh);
}

// Both in one launch where two workgroups of either fit a CU: those for few rows come
// first, one for each CU, and items of many rows beside them.  (1B, 500 rows beside
// 15 single ones: 41 us one after the other, 36 together; 8B, 300 beside 8 x 6: 41 and
// 28; 13B, 512 beside 7: 153 and 141, where both read much.)
template <bool KVB, int HD, bool QB>
__global__ __launch_bounds__(256, 2) void k_page_both(PageAttnArgs a, PageClass few, PageClass many, int nfew) {
  __shared__ union Both {
    ManyShared<KVB, HD> m;
    FewShared<KVB, HD, QB> f;
    __device__ Both() {}
  } sh;
  if ((int)blockIdx.x < nfew) few_items<KVB, HD, QB>(a, few, blockIdx.x, nfew, sh.f);
  else many_item<KVB, HD, QB>(a, many, (int)blockIdx.x - nfew, sh.m);
}

// ------------------------------------------------------------------ the join

// Eight queries of a tile of several chunks: HD / 4 threads hold a query's outputs,
// and as many groups of them as there are threads for share its chunks, kJoinBatch
// of them in flight each.  jfew and jall count groups of 32 queries, at most.
constexpr int kJoinBatch = 4, kJoinQ = 8;
template <bool QB, int HD>
__global__ __launch_bounds__(256) void k_page_join(PageAttnArgs a, PageClass few, PageClass many, int jfew, int jall) {
  constexpr int PER = HD / 4, GR = 256 / PER;               // groups, eight or more
  __shared__ f32x4 so[GR][PER];
  __shared__ float2 sml[GR];
  const int gr = threadIdx.x / PER, d = threadIdx.x % PER;
  auto join = [&](const PageClass& cl, const Item& it, int kvh, int part) {
    const int qw = it.w.qw, T = 32 * qw, x0 = it.tile * T + it.sub * 32 + part * kJoinQ;
    const int live = it.w.bad ? 0 : min(kJoinQ, it.w.R * a.G - x0);
    if (live < 1) return;
    const Span sp = span_of(a, it.w, it.tile * T, T);
    const int units = (sp.hi - sp.lo + kUnit - 1) / kUnit;
    const int chunks = min(it.chunks, (int)((unsigned)(units + it.per - 1) / (unsigned)it.per));   // those with keys of the tile
    const size_t step = (size_t)qw * a.pg.nkv;               // slots from a chunk to the next
    const size_t slot0 = ((size_t)it.slot + it.sub) * a.pg.nkv + kvh;
    const int share = (unsigned)GR / (unsigned)live;         // groups of a query
    const int qq = (unsigned)gr / (unsigned)share, k = gr - qq * share;
    const bool on = qq < live;
    float M = -INFINITY, L = 0.f;
    f32x4 v = f32x4{0.f, 0.f, 0.f, 0.f};
    if (on) {
      const float2* ml = cl.ml + slot0 * 32 + part * kJoinQ + qq;
      const float* po = cl.part + (slot0 * 32 + part * kJoinQ + qq) * HD + d * 4;
      for (int c0 = k; c0 < chunks; c0 += share * kJoinBatch) {
        float2 x[kJoinBatch];
        f32x4 y[kJoinBatch];
#pragma unroll
        for (int i = 0; i < kJoinBatch; ++i) {
          const int c = c0 + i * share;
          x[i] = make_float2(-INFINITY, 0.f);
          y[i] = f32x4{0.f, 0.f, 0.f, 0.f};
          if (c < chunks) {
            x[i] = ml[c * step * 32];
            y[i] = *(const f32x4*)(po + c * step * 32 * HD);
          }
        }
        float mn = M;
#pragma unroll
        for (int i = 0; i < kJoinBatch; ++i) mn = fmaxf(mn, x[i].x);
        const float base = mn == -INFINITY ? 0.f : mn, f = __builtin_amdgcn_exp2f(M - base);
        L *= f;
        v *= f;
#pragma unroll
        for (int i = 0; i < kJoinBatch; ++i) {
          const float w = __builtin_amdgcn_exp2f(x[i].x - base);
          L += x[i].y * w;
          v += y[i] * w;
        }
        M = mn;
      }
    }
    if (share > 1) {
      __syncthreads();   // the item before has been read
      if (gr < GR) {
        so[gr][d] = v;
        if (d == 0) sml[gr] = make_float2(M, L);
      }
      __syncthreads();
      if (on && k == 0) {
        float mx = M;
        for (int i = 1; i < share; ++i) mx = fmaxf(mx, sml[gr + i].x);
        const float base = mx == -INFINITY ? 0.f : mx;
        L = 0.f;
        v = f32x4{0.f, 0.f, 0.f, 0.f};
        for (int i = 0; i < share; ++i) {
          const float w = __builtin_amdgcn_exp2f(sml[gr + i].x - base);
          L += sml[gr + i].y * w;
          v += so[gr + i][d] * w;
        }
      }
    }
    if (!on || k) return;
    int row, g, pos;
    query_at(a, it.w, x0 + qq, row, g, pos);
    const float inv = 1.f / L, y[4] = {v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv};
    store_out<QB>(a, (size_t)row * a.ldo + (size_t)(kvh * a.G + g) * HD + d * 4, y);
  };
  constexpr int PARTS = 32 / kJoinQ;
  const int per_sub = a.pg.nkv * PARTS;
  auto all = [&](const PageClass& cl, int i0, int i1, int first) {
    const Plan p = plan_of<true>(a, cl);
    Item it;
    for (int id = first; id < i1 * per_sub && find<true>(a, cl, p, id / per_sub - i0, it); id += gridDim.x)
      join(cl, it, id % per_sub % a.pg.nkv, id % per_sub / a.pg.nkv);
  };
  int id = blockIdx.x;
  if (jfew) all(few, 0, jfew, id);
  if (jall > jfew) {
    while (id < jfew * per_sub) id += gridDim.x;
    all(many, jfew, jall, id);
  }
}

// ------------------------------------------------------------------ launches

// tiles of 32 qw queries that a step's windows have together, at most: 1 + (x - 1) / (32 qw)
// of x queries
long long most_tiles(const PageArgs& pg, int rows, int nq, int qw) {
  const long long n = std::min(pg.n_windows, rows), queries = (long long)rows * (nq / pg.nkv);
  return n + (queries - n) / (32 * qw);
}
// Slots (32 queries of an item of a tile that is cut): tiles * qw * chunks of them are
// less than twice tiles * qw * units / per, which is at most `most`; and no tile has
// more chunks than the windows' pages have units
long long slots(const PageClass& c, const PageArgs& pg, int rows, int nq) {
  const int qw = c.qw ? c.qw : 1, windows = std::min(pg.n_windows, rows);
  const long long units = ((long long)pg.max_pages * pg.bpp * 32 + kUnit - 1) / kUnit;
  const long long tiles = most_tiles(pg, rows, nq, qw) * qw + windows;   // of 32 queries, the last of a window's tile empty
  return std::min(2ll * c.most, tiles * pg.nkv * units);
}

constexpr int kSlots = 512;   // workgroups that the card holds at once, two a CU
constexpr int kJoinGrid = 1024;   // of the join, which takes parts in turn (512: 32 decoding windows 8.8 us, 1024 8.0)

struct Classes {
  PageClass few, many;
  bool use_few, use_many;
};
// Windows of up to kFewQueries queries of a KV head are few rows.  A call that has no
// more than kAllFew in all takes every window for one of few, and a single window is
// of the kind that its call's rows say: a launch of a kind that has nothing to do costs
// 4 us (7 x 6 rows of 8B: 24 us without, 29 with).  64 rows of 8B over 16000 positions, 256
// queries: 55 us as few rows, 46 as many.
constexpr int kFewQueries = 64, kAllFew = 256;
Classes classes_of(const PageArgs& pg, int rows, int nq, bool bf16) {
  const long long queries = (long long)rows * (nq / pg.nkv);
  Classes c{};
  c.use_many = queries > (pg.n_windows > 1 ? kAllFew : kFewQueries);
  c.use_few = !c.use_many || pg.n_windows > 1;
  c.few.qlo = 1;
  c.few.qhi = c.use_many ? kFewQueries : INT_MAX;
  c.few.once = kSlots;
  // items of 1024 keys are long enough to hide how they begin and end, and what is cut
  // finer than one for each workgroup evens out: 8B, 32 windows of up to 31131 positions,
  // 512 items 404 us, 2048 353, 4096 361; 12 windows of 1 or 8 rows over up to 30000:
  // items of 8 units 68 us, of 4 73, of 16 78
  c.few.most = 4 * kSlots;
  c.few.enough = 8;
  c.many.qlo = c.use_few ? kFewQueries + 1 : 1;
  c.many.qhi = INT_MAX;
  c.many.qw = 4;
  c.many.once = c.many.most = 4 * (many_two(pg.kvb, pg.hd, bf16) ? kSlots : kSlots / 2);
  c.many.enough = INT_MAX;
  for (PageClass* cl : {&c.few, &c.many}) {
    cl->inv_once = 1.0 / cl->once;   // powers of two: exact
    cl->inv_most = 1.0 / cl->most;
  }
  return c;
}

// of a class's written cut
size_t plan_bytes(const PageArgs& pg) {
  return pg.n_windows > 64 ? (((size_t)kPlanHead + 3 * pg.n_windows) * sizeof(int) + 15) & ~(size_t)15 : 0;
}

template <bool KVB, int HD, bool QB>
hipError_t launch_all(PageAttnArgs a, void* ws, hipStream_t s) {
  Classes c = classes_of(a.pg, a.rows, a.nq, QB);
  const bool both = many_two(KVB, HD, QB) && c.use_few && c.use_many;   // in one launch
  if (both) {
    c.few.once = kSlots / 2;
    c.few.inv_once = 1.0 / c.few.once;
  }
  const int nkv = a.pg.nkv, windows = std::min(a.pg.n_windows, a.rows);
  long long nfew = 0, nmany = 0, jfew = 0, jmany = 0;
  if (c.use_few) {
    const long long tiles = most_tiles(a.pg, a.rows, a.nq, 1), cuts = c.few.most / nkv + 1;
    nfew = std::min((cuts + tiles) * nkv, (long long)kSlots);
    // the last tile of a window may have 32 queries that are empty
    jfew = std::min(tiles + windows, cuts);
  }
  if (c.use_many) {
    const long long tiles = most_tiles(a.pg, a.rows, a.nq, 4);
    nmany = (c.many.most / 4 / nkv + 1 + tiles) * nkv;
    jmany = std::min(tiles * 4, (long long)c.many.most / nkv + 1);
  }
  if (both) nfew = std::min(nfew, (long long)kSlots / 2);
  if (nmany + (both ? nfew : 0) > kMaxStepBlocks) return hipErrorInvalidConfiguration;
  char* at = (char*)ws;
  const size_t planned = plan_bytes(a.pg);
  if (planned) {
    c.few.plan = (int*)at;
    c.many.plan = (int*)(at + planned);
    at += 2 * planned;
    const int first = c.use_few ? 0 : 1, classes = c.use_few + c.use_many;
    hipLaunchKernelGGL(k_page_plan, dim3(classes), dim3(1024), 0, s, a, c.few, c.many, first);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  for (PageClass* cl : {&c.few, &c.many}) {
    if (cl == &c.few ? !c.use_few : !c.use_many) continue;
    const long long n = slots(*cl, a.pg, a.rows, a.nq);
    cl->slots = (int)(n / a.pg.nkv);
    cl->ml = (float2*)at;
    cl->part = (float*)(cl->ml + n * 32);
    at = (char*)(cl->part + n * 32 * HD);
  }
  if constexpr (many_two(KVB, HD, QB)) {
    if (both)
      hipLaunchKernelGGL((k_page_both<KVB, HD, QB>), dim3((unsigned)(nfew + nmany)), dim3(256), 0, s, a, c.few, c.many, (int)nfew);
  }
  if (nmany && !both) hipLaunchKernelGGL((k_page_many<KVB, HD, QB>), dim3((unsigned)nmany), dim3(256), 0, s, a, c.many);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (nfew && !both) hipLaunchKernelGGL((k_page_few<KVB, HD, QB>), dim3((unsigned)nfew), dim3(256), 0, s, a, c.few);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  const long long joins = (jfew + jmany) * nkv * (32 / kJoinQ);
  hipLaunchKernelGGL((k_page_join<QB, HD>), dim3((unsigned)std::min(joins, (long long)kJoinGrid)), dim3(256), 0, s, a, c.few, c.many, (int)jfew, (int)(jfew + jmany));
  return hipGetLastError();
}

template <bool KVB, bool QB>
hipError_t launch_hd(const PageAttnArgs& a, void* ws, hipStream_t s) {
  switch (a.pg.hd) {
    case 32: return launch_all<KVB, 32, QB>(a, ws, s);
    case 64: return launch_all<KVB, 64, QB>(a, ws, s);
    case 96: return launch_all<KVB, 96, QB>(a, ws, s);
    case 128: return launch_all<KVB, 128, QB>(a, ws, s);
  }
  return hipErrorInvalidValue;
}

}  // namespace

size_t page_attend_workspace_bytes(const PageArgs& pg, int rows, int nq) {
  size_t most = 0;
  for (bool bf16 : {false, true}) {   // whatever the call's type
    const Classes c = classes_of(pg, rows, nq, bf16);
    most = std::max(most, (size_t)((c.use_few ? slots(c.few, pg, rows, nq) : 0) + (c.use_many ? slots(c.many, pg, rows, nq) : 0)));
  }
  return 2 * plan_bytes(pg) + most * 32 * (pg.hd * sizeof(float) + sizeof(float2));
}

hipError_t launch_page_attend(const PageAttnArgs& a, void* ws, hipStream_t s) {
  if (a.pg.kvb) return a.bf16 ? launch_hd<true, true>(a, ws, s) : launch_hd<true, false>(a, ws, s);
  return a.bf16 ? launch_hd<false, true>(a, ws, s) : launch_hd<false, false>(a, ws, s);
}

}  // namespace dsi
