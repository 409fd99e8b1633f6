// Log probabilities of given tokens, entropy and most probable alternatives of
// rows of logits, in one pass over them.
//
// With x_v = (z_v - M) / T, M the row's maximum and S = sum_v e^{x_v}:
//   log p_t = x_t - log S;  entropy = log S - (1 / S) sum_v x_v e^{x_v};
//   the alternatives are the n largest logits, ties to the lowest id.
// A row is cut into U runs of 1024-entry steps, one wave a run: 16 entries a
// lane and step, the next step's loads in flight while one is worked on.  A
// lane keeps a running maximum, and sums relative to it that are rescaled when
// it moves: the 16 terms of a step are added in fp32, the steps in fp64.  The
// entries equal to the maximum are counted, not summed: log S = log c + log1p(s / c)
// of c such entries and the others' sum s keeps its digits where a row is sure of
// one token.
// Alternatives: a wave keeps its largest entries sorted across its lanes, key =
// (logit in unsigned order, id complemented).  A step whose lanes hold nothing
// above the n-th key costs one ballot.  Otherwise a few alternatives are taken
// one by one, largest first; for more, the entries not below the n-th largest
// lane maximum (n entries are at least that) are gathered in LDS, 64 at a time
// sorted across the lanes and merged with the list.  No wave waits for another.
// A second launch, one wave a row, joins the runs: statistics in fp64, and the
// runs' lists, best ranks first, 64 keys at a time.
// Bound by reading the logits where there are many rows (2048 x 128256 fp32, one
// alternative: 1.05 GB, 175 us, 6.0 TB/s).  A few rows are bound by the two
// launches and what a wave does once: 42 x 128256 take 12.0 us without
// alternatives, 17.0 with one, 22 with 5, 29 with 20 (taken one by one, 20 cost 106 us
// on 300 x 32003 where the gathered ones cost 27); 1 x 32000 with 5 takes 11 us.
#include <math.h>

#include "scan.h"

namespace dsi {

namespace {

constexpr int LPW = 4;                 // waves (runs) per workgroup of the first launch
constexpr int LPE = 16;                // entries per lane and step
constexpr int LPS = 64 * LPE;          // entries per step
constexpr int LPG = 4;                 // runs per lane of the join
constexpr int kLpRuns = 64 * LPG;      // runs per row at most
constexpr int kLpWaves = 3 * 1024;     // waves of a call: three a SIMD
// up to so many alternatives are taken one by one (42 x 128256: 2 of them 18.7 us,
// 4 21.9; 5 gathered 22.1)
constexpr int kLpFew = 4;

typedef unsigned long long u64;

__device__ __forceinline__ u64 lane_key(u64 v, int l) {
  return ((u64)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), l) << 32) |
         (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, l);
}
// order of floats as unsigned words; NaN below everything, -0 as 0
__device__ __forceinline__ uint32_t order_of(float z) {
  const uint32_t b = __float_as_uint(z + 0.f);
  const uint32_t o = b & 0x80000000u ? ~b : b | 0x80000000u;
  return z != z ? 0u : o;
}
__device__ __forceinline__ float from_order(uint32_t o) {
  return __uint_as_float(o & 0x80000000u ? o & 0x7FFFFFFFu : ~o);
}
__device__ __forceinline__ uint32_t wave_umax(uint32_t v) {
  dpp_steps([&](auto s) {
    const uint32_t o = (uint32_t)dpp_from<decltype(s)::ctrl, decltype(s)::rows>((int)v, (int)v);
    v = v > o ? v : o;
  });
  return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}
// the value of lane l ^ J, by lane swaps and DPP patterns (a shuffle goes
// through LDS: a merge of 64 keys took 2 us by itself that way)
template <int J>
__device__ __forceinline__ uint32_t lane_xor(uint32_t v, int lane) {
  const int x = (int)v;
  if constexpr (J == 1) return (uint32_t)__builtin_amdgcn_update_dpp(x, x, 0xB1, 0xF, 0xF, false);
  if constexpr (J == 2) return (uint32_t)__builtin_amdgcn_update_dpp(x, x, 0x4E, 0xF, 0xF, false);
  if constexpr (J == 4) {   // 7 - l of eight lanes, then 3 - l of four
    const int y = __builtin_amdgcn_update_dpp(x, x, 0x141, 0xF, 0xF, false);
    return (uint32_t)__builtin_amdgcn_update_dpp(y, y, 0x1B, 0xF, 0xF, false);
  }
  if constexpr (J == 8) return (uint32_t)__builtin_amdgcn_update_dpp(x, x, 0x128, 0xF, 0xF, false);
  if constexpr (J == 16) {
    const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    return lane & 16 ? a[0] : a[1];
  }
  const auto a = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return lane & 32 ? a[0] : a[1];
}
template <int J>
__device__ __forceinline__ u64 lane_xor(u64 v, int lane) {
  return ((u64)lane_xor<J>((uint32_t)(v >> 32), lane) << 32) | lane_xor<J>((uint32_t)v, lane);
}
// Bitonic sort of 64 values across the lanes: in a sequence of size K, lane l
// keeps the larger of the pair (l, l ^ J) when its bits K and J are equal (DOWN:
// largest value first), or when they differ.
constexpr u64 keep_larger(int k, int j, bool down) {   // a bit per lane
  u64 m = 0;
  for (int l = 0; l < 64; ++l)
    if ((((l & k) == 0) == ((l & j) == 0)) == down) m |= 1ull << l;
  return m;
}
template <int K, int J, bool DOWN, typename V>
__device__ __forceinline__ void sort_steps(V& v, int lane) {
  const V o = lane_xor<J>(v, lane);
  constexpr u64 kLarger = keep_larger(K, J, DOWN);
  const bool larger = __builtin_amdgcn_inverse_ballot_w64(kLarger);
  v = (o > v) == larger ? o : v;
  if constexpr (J > 1) sort_steps<K, J / 2, DOWN>(v, lane);
}
template <bool DOWN, int K = 2, typename V>
__device__ __forceinline__ void wave_sort(V& v, int lane) {
  sort_steps<K, K / 2, DOWN>(v, lane);
  if constexpr (K < 64) wave_sort<DOWN, 2 * K>(v, lane);
}
// the 64 largest of a sorted list (largest first) and 64 keys in any order, sorted
__device__ __forceinline__ void merge_keys(u64& list, u64 keys, int lane) {
  wave_sort<false>(keys, lane);
  list = list > keys ? list : keys;   // the larger ones, as a bitonic sequence
  sort_steps<64, 32, true>(list, lane);
}
// what the wave's lanes wrote to LDS is there for all of them: the LDS takes a
// wave's accesses in their order, the compiler is told to keep it
__device__ __forceinline__ void lanes_see() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}
// the lane above takes this lane's value (wave_shr:1); lane 0 keeps its own
__device__ __forceinline__ u64 from_lane_below(u64 v) {
  const int hi = __builtin_amdgcn_update_dpp((int)(v >> 32), (int)(v >> 32), 0x138, 0xF, 0xF, false);
  const int lo = __builtin_amdgcn_update_dpp((int)(uint32_t)v, (int)(uint32_t)v, 0x138, 0xF, 0xF, false);
  return ((u64)(uint32_t)hi << 32) | (uint32_t)lo;
}

// One step's 16 entries of a lane: granules of 16 bytes, 64 granules (one per
// lane) after each other.  `a` is the row's offset from 16-byte alignment in
// entries: entry v sits at position v + a of the aligned granules.
template <typename T>
struct Step {
  static constexpr int PG = 16 / sizeof(T), NG = LPE / PG;   // entries per granule, granules per lane
  u32x4 g[NG];
};
__device__ __forceinline__ float entry_of(const Step<float>& s, int i) { return __uint_as_float(s.g[i >> 2][i & 3]); }
__device__ __forceinline__ float entry_of(const Step<uint16_t>& s, int i) {
  const uint32_t w = s.g[i >> 3][(i & 7) >> 1];
  return __uint_as_float(i & 1 ? w & 0xFFFF0000u : w << 16);
}
// the aligned position of entry i of lane l in step st
template <typename T>
__device__ __forceinline__ int position(int st, int l, int i) {
  constexpr int PG = Step<T>::PG;
  return st * LPS + ((i / PG) * 64 + l) * PG + i % PG;
}
template <typename T>
__device__ __forceinline__ void load_step(Step<T>& s, const T* row, int a, int V, int st, int lane) {
  constexpr int PG = Step<T>::PG, NG = Step<T>::NG;
  const T* base = row - a;
  if (st * LPS >= a && (st + 1) * LPS <= V + a) {   // the same for the whole wave
#pragma unroll
    for (int i = 0; i < NG; ++i)
      s.g[i] = __builtin_nontemporal_load((const u32x4*)(base + position<T>(st, lane, i * PG)));
    return;
  }
  // a step at an end of the row: only its own entries are read, the others are NaN
#pragma unroll
  for (int i = 0; i < NG; ++i) {
    u32x4 x;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int v = position<T>(st, lane, i * PG + e) - a;
        x[e] = v >= 0 && v < V ? __float_as_uint(row[v]) : 0x7FC00000u;
      }
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int v = position<T>(st, lane, i * PG + 2 * e) - a;
        const uint32_t lo = v >= 0 && v < V ? row[v] : 0x7FC0u, hi = v + 1 >= 0 && v + 1 < V ? row[v + 1] : 0x7FC0u;
        x[e] = lo | hi << 16;
      }
    }
    s.g[i] = x;
  }
}

template <typename T>
__global__ __launch_bounds__(LPW * 64) void k_lp_rows(LogprobArgs a) {
  __shared__ u64 gather[LPW][128];
  const int lane = threadIdx.x & 63;
  u64* const held = gather[threadIdx.x >> 6];
  const int run = __builtin_amdgcn_readfirstlane(blockIdx.x * LPW + (threadIdx.x >> 6));
  if (run >= a.rows * a.U) return;
  const int r = run / a.U, u = run - r * a.U;
  const T* row = (const T*)a.z + (size_t)r * a.ld;
  const int off = (int)(((uintptr_t)row & 15) / sizeof(T));
  const int steps = (a.V + off + LPS - 1) / LPS;
  const int st0 = (int)((long long)steps * u / a.U), st1 = (int)((long long)steps * (u + 1) / a.U);
  float m = -INFINITY, cnt = 0.f;
  double rest = 0.0, t = 0.0;
  u64 list = 0;              // lane i: the i-th largest key so far (0: none)
  uint32_t tau = 0;          // order of the n-th
  Step<T> cur;
  load_step(cur, row, off, a.V, st0, lane);   // U is at most the number of steps: a run has one
  for (int st = st0; st < st1; ++st) {
    Step<T> next = cur;
    if (st + 1 < st1) load_step(next, row, off, a.V, st + 1, lane);
    const bool whole = st * LPS >= off && (st + 1) * LPS <= a.V + off;
    float z[LPE];
#pragma unroll
    for (int i = 0; i < LPE; ++i) z[i] = entry_of(cur, i);
    float best = z[0];
#pragma unroll
    for (int i = 1; i < LPE; ++i) best = fmaxf(best, z[i]);
    const float mnew = fmaxf(m, best);
    const float b = mnew == -INFINITY ? 0.f : mnew;
    if (mnew > m) {   // what equalled the old maximum joins the sums
      const float d = m == -INFINITY ? 0.f : fmaxf((m - b) * a.k2, -1024.f);
      const double f = __builtin_amdgcn_exp2f(d), all = rest + (double)cnt;
      t = (t + d * all) * f;
      rest = all * f;
      cnt = 0.f;
      m = mnew;
    }
    float s = 0.f, ts = 0.f, c = 0.f;
#pragma unroll
    for (int i = 0; i < LPE; ++i) {
      const bool top = z[i] == mnew;
      float y = (z[i] - b) * a.k2;
      y = y < -1024.f ? -1024.f : y;   // e^x is 0, and 0 times -inf is not
      float e = __builtin_amdgcn_exp2f(y);
      e = top ? 0.f : e;
      if (!whole) {   // entries that are not the row's
        const int v = position<T>(st, lane, i) - off;
        e = v >= 0 && v < a.V ? e : 0.f;
        y = v >= 0 && v < a.V ? y : 0.f;
      }
      c += top ? 1.f : 0.f;
      s += e;
      ts = fmaf(e, y, ts);
    }
    if (mnew != -INFINITY) cnt += c;
    rest += (double)s;
    t += (double)ts;
    if (a.n) {
      uint32_t bo = order_of(best);
      if (!__ballot(bo > tau)) {
      } else if (a.n <= kLpFew) {
        uint32_t o[LPE];
#pragma unroll
        for (int i = 0; i < LPE; ++i) o[i] = order_of(z[i]);
        do {
          const uint32_t mx = wave_umax(bo);
          int idx = LPE;
#pragma unroll
          for (int i = LPE - 1; i >= 0; --i) idx = o[i] == mx ? i : idx;
          const uint32_t v = idx < LPE ? (uint32_t)(position<T>(st, lane, idx) - off) : ~0u;
          // the lowest id among equals: the largest complement
          const uint32_t nv = wave_umax(idx < LPE ? ~v : 0u);
          const u64 key = ((u64)mx << 32) | nv;
          const int pos = __popcll(__ballot(list > key));
          const u64 below = from_lane_below(list);
          list = lane > pos ? below : lane == pos ? key : list;
          tau = (uint32_t)(lane_key(list, a.n - 1) >> 32);
          // taken: out of the step
          const bool mine = idx < LPE && ~v == nv;
          bo = 0;
#pragma unroll
          for (int i = 0; i < LPE; ++i) {
            o[i] = mine && i == idx ? 0u : o[i];
            bo = bo > o[i] ? bo : o[i];
          }
        } while (__ballot(bo > tau));
      } else {
        // what equals the n-th key of the steps before has a larger id; within
        // the step ids come in any order, and equals are kept
        uint32_t o[LPE], s = bo;
#pragma unroll
        for (int i = 0; i < LPE; ++i) o[i] = order_of(z[i]);
        wave_sort<true>(s, lane);
        uint32_t bar = (uint32_t)__builtin_amdgcn_readlane((int)s, a.n - 1);
        bar = bar > tau ? bar : tau + 1;
        int have = 0;
#pragma unroll
        for (int i = 0; i < LPE; ++i) {
          const bool in = o[i] >= bar;
          const u64 mask = __ballot(in);
          if (!mask) continue;
          if (in) {
            const int at = have + __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
            held[at] = ((u64)o[i] << 32) | ~(uint32_t)(position<T>(st, lane, i) - off);
          }
          have += __popcll(mask);
          if (have >= 64) {
            lanes_see();
            merge_keys(list, held[lane], lane);
            have -= 64;
            if (lane < have) held[lane] = held[64 + lane];
            lanes_see();
            tau = (uint32_t)(lane_key(list, a.n - 1) >> 32);
            bar = bar > tau ? bar : tau;
          }
        }
        if (have) {
          lanes_see();
          merge_keys(list, lane < have ? held[lane] : 0, lane);
          lanes_see();
          tau = (uint32_t)(lane_key(list, a.n - 1) >> 32);
        }
      }
    }
    cur = next;
  }
  // the lanes' statistics, relative to the wave's maximum
  const float M = wave_max(m);
  const float b = M == -INFINITY ? 0.f : M;
  const float d = m == -INFINITY ? 0.f : fmaxf((m - b) * a.k2, -1024.f);
  const double f = m == M || m == -INFINITY ? 1.0 : (double)__builtin_amdgcn_exp2f(d);
  double ws = m == M ? rest : (rest + (double)cnt) * f;
  double wt = m == M || m == -INFINITY ? t : (t + d * (rest + (double)cnt)) * f;
  const double wc = m == M ? (double)cnt : 0.0;
  ws = wave_sum(ws);
  wt = wave_sum(wt);
  const double all = wave_sum(wc);
  if (lane == 0) a.stat[run] = LpStat{ws, wt, M, (float)all};
  if (lane < a.n) a.keys[((size_t)r * a.n + lane) * a.U + u] = list;   // rank by rank
}

__global__ __launch_bounds__(64) void k_lp_join(LogprobArgs a) {
  const int r = blockIdx.x, lane = threadIdx.x;
  const LpStat* st = a.stat + (size_t)r * a.U;
  // the row's maximum, sums and count
  LpStat x[LPG];
  float M = -INFINITY;
#pragma unroll
  for (int j = 0; j < LPG; ++j) {
    const int u = lane + 64 * j;
    x[j] = u < a.U ? st[u] : LpStat{0.0, 0.0, -INFINITY, 0.f};
    M = fmaxf(M, x[j].m);
  }
  M = wave_max(M);
  // c entries equal the row's maximum, the others' sum is s: S = c + s
  double c = 0.0, s = 0.0, t = 0.0;
  const double ln2 = 0.69314718055994530942;
#pragma unroll
  for (int j = 0; j < LPG; ++j) {
    const double all = x[j].rest + (double)x[j].cnt;
    if (x[j].m == M || x[j].m == -INFINITY) {
      c += (double)x[j].cnt;
      s += x[j].rest;
      t += x[j].t * ln2;
    } else {
      const double d = ((double)x[j].m - (double)M) * a.inv_temperature, f = exp(d);
      s += all * f;
      t += f > 0.0 ? (x[j].t * ln2 + d * all) * f : 0.0;
    }
  }
  c = wave_sum(c);
  s = wave_sum(s);
  t = wave_sum(t);
  // a row of -inf, and one with +inf, has no distribution
  const bool none = !isfinite(M);
  const double lse = none ? (double)NAN : log(c) + log1p(s / c);
  if (lane == 0) {
    if (a.entropy) a.entropy[r] = (float)(lse - t / (c + s));
    if (a.logprob) {
      const int tok = a.tokens[r];
      float lp = NAN;
      if (tok >= 0 && tok < a.V) {
        const float z = a.bf16 ? bf_bits2f(((const uint16_t*)a.z)[(size_t)r * a.ld + tok])
                               : ((const float*)a.z)[(size_t)r * a.ld + tok];
        lp = (float)(((double)z - (double)M) * a.inv_temperature - lse);
      }
      a.logprob[r] = lp;
    }
  }
  if (!a.n) return;
  // the runs' keys, best ranks first: 64 at a time, the next ones in flight
  const u64* keys = a.keys + (size_t)r * a.n * a.U;
  const int total = a.n * a.U;
  u64 list = 0, next = lane < total ? keys[lane] : 0;
  u64 last = 0;   // the n-th key
  for (int i0 = 0; i0 < total; i0 += 64) {
    const u64 k = next;
    next = i0 + 64 + lane < total ? keys[i0 + 64 + lane] : 0;
    if (!__ballot(k > last)) continue;
    merge_keys(list, k, lane);
    last = lane_key(list, a.n - 1);
  }
  if (lane < a.n) {
    const size_t o = (size_t)r * a.n + lane;
    a.top_ids[o] = list ? (int)~(uint32_t)list : -1;
    a.top_logprob[o] = list ? (float)(((double)from_order((uint32_t)(list >> 32)) - (double)M) * a.inv_temperature - lse) : NAN;
  }
}

// Runs per row: three waves a SIMD over the whole call, whole steps.  Both launches
// of 42 x 128256 (5 alternatives), 300 x 32003 (bf16, 20) and 2048 x 128256 (one), us,
// with two waves: 22.9, 34.0, 193; three 23.6, 30.0, 182; four 25.1, 30.9, 183; eight
// 23.4, 34.1, 180.
int lp_runs(long long rows, int V) {
  const long long steps = ((long long)V + LPS - 1) / LPS;
  long long u = (kLpWaves + rows - 1) / rows;
  u = u < steps ? u : steps;
  return (int)(u < 1 ? 1 : u < kLpRuns ? u : kLpRuns);
}

}  // namespace

size_t logprobs_workspace_bytes(int rows, int V, int n) {
  return (size_t)rows * lp_runs(rows, V) * (sizeof(LpStat) + (size_t)n * sizeof(u64));
}

hipError_t launch_logprobs(LogprobArgs a, void* ws, hipStream_t s) {
  if (a.rows < 1 || a.V < 1 || a.n < 0 || a.n > 64) return hipErrorInvalidValue;
  a.U = lp_runs(a.rows, a.V);
  a.stat = (LpStat*)ws;
  a.keys = (u64*)(a.stat + (size_t)a.rows * a.U);
  const dim3 grid((unsigned)(((long long)a.rows * a.U + LPW - 1) / LPW));
  if (a.bf16) hipLaunchKernelGGL((k_lp_rows<uint16_t>), grid, dim3(LPW * 64), 0, s, a);
  else hipLaunchKernelGGL((k_lp_rows<float>), grid, dim3(LPW * 64), 0, s, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(k_lp_join, dim3(a.rows), dim3(64), 0, s, a);
  return hipGetLastError();
}

}  // namespace dsi
