// Windows that continue one prompt: forking a window's cache into others, and
// attention that reads the prefix they share once for all of them.
//
// Attention of row i of window b (position L_b + i) over keys [0, L_b + i] is
// split at s, the largest multiple of 32 up to which every window of a group
// holds what the window they were forked from holds.  Softmax sums over
// disjoint keys join exactly: with (m, l, O) = (max, sum of e^(z - m), sum of
// e^(z - m) v) of each part,
//   M = max m_c,  out = sum_c e^(m_c - M) O_c / sum_c e^(m_c - M) l_c.
// The keys [0, s) are every row's, so the B R rows of a group are one product
// without a mask, over one copy of the prefix; the rest is each window's own.
// The first launch runs the prefix in chunks, and what a window has of its own
// beyond its last kShareLast cached keys and the rows of the call (mostly nothing).
// The second attends to those last keys and joins the parts: rows and masks are
// its business alone, and no third launch reads what it computed.
#include <limits.h>
#include <math.h>

#include "scan.h"

namespace dsi {

namespace {

constexpr int SW = 8;                  // waves per workgroup of the first launch
constexpr int LW = 4;                  // and of the second
constexpr int kOwnChunk = SW * 32;     // keys of a window's own per workgroup of the first launch: a multiple of this

__device__ __forceinline__ int wave_min(int v) {
  dpp_steps([&](auto s) { v = min(v, dpp_from<decltype(s)::ctrl, decltype(s)::rows>(v, v)); });
  return __builtin_amdgcn_readlane(v, 63);
}

// positions of the prefix that the group's windows share, whole blocks of 32
// (each wave finds it for itself); never so many that the rows would not fit
// behind them, whatever a length says
__device__ __forceinline__ int group_prefix(const ShareArgs& a, const ShareGroup& g) {
  int s = a.maxlen - a.R;
  for (int i = threadIdx.x & 63; i < g.count; i += 64) {
    const int w = a.window0 + g.first + i;
    int x = a.f.lens[w];
    if (w != g.root) x = a.f.root[w] == g.root ? min(x, a.f.shared[w]) : 0;
    s = min(s, x);
  }
  s = wave_min(s) & ~31;
  return s < kMinShared ? 0 : s;
}
__device__ __forceinline__ int window_prefix(const ShareArgs& a, int win) {
  for (int g = 0; g < a.n_groups; ++g)
    if (win >= a.group[g].first && win < a.group[g].first + a.group[g].count) return group_prefix(a, a.group[g]);
  return 0;
}
// keys per chunk of a prefix: p_chunks chunks at most, of 128 keys at least, or
// 192 where a part has up to 256 queries and the prefix over 2048 keys: a chunk
// leaves HD * 4 bytes per query, which are read again, and up to 2048 keys there
// are too few chunks for the CUs (a step, us, with 128 and 192: 8B, 8 x 8 rows over
// 1024 keys 22.8 and 24.1, 2000 29.1 and 31.1, 2100 31.0 and 30.7, 3000 32.3 and
// 31.8, 4096 38.6 and 35.0; 64 x 1 over 2048 37.2 and 38.7, 3500 48.6 and 44.4)
__device__ __forceinline__ int prefix_chunk(const ShareArgs& a, int s) {
  return max(a.p_tile > 128 && s > 2048 ? 192 : 128, ((s + a.p_chunks - 1) / a.p_chunks + 63) & ~63);
}
__device__ __forceinline__ int own_chunk(int keys, int most) {
  return ((keys + most - 1) / most + kOwnChunk - 1) / kOwnChunk * kOwnChunk;
}
// keys [s, own_end) of a window of len cached positions are attended by the
// first launch: whole blocks, all of them cached
__device__ __forceinline__ int own_end(int s, int len) { return len - s <= kShareLast ? s : s + (len - s - 1) / kShareLast * kShareLast; }

// Queries of one part: `rows` consecutive rows from row0 on, times the G query
// heads of KV head kvh; query q is row q % rows of head q / rows.
struct QuerySet {
  int row0, rows, kvh;
};
// Keys [k0, k1) of cache window `win`, k0 a multiple of 32, and k1 too unless
// the range holds the rows of the call (LAST): those are keys own .. k1 - 1, and
// key own + j is seen by rows i >= j of the window (tree: by those that have bit
// j).
struct KeyRange {
  int win, k0, k1, own;
};

// One part on the direct path: 16 queries, NW waves that take every NW-th 32-key
// step, keys and values straight from the cache into fragments (as in the window
// attention: 16x16 MFMAs, S^T = K Q^T and O^T += V^T P^T, queries and
// probabilities of a bf16 cache as hi + lo).  The waves' sums are left in LDS
// (WaveSums) to be joined.
// LAST: the second launch's part, with the rows of the call.  Values are summed
// for VD of the head's dims, from d0 on.
template <int NW, int VD>
struct WaveSums {
  float m[NW][16], l[NW][16];
  f32x4 o[NW][VD / 16][64];
};

// range(): the keys, which depend on lengths in memory; asked for once the loads
// of the queries are on their way
template <int KVB, int HD, int VD, int LAST, int NW, typename F>
__device__ __forceinline__ void direct_sums(const ShareArgs& a, const QuerySet& qs, F&& range, int y, int d0,
                                            WaveSums<NW, VD>& sums) {
  constexpr int DS = HD / 32, DT = VD / 16;
  const int lane = threadIdx.x & 63;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int G = a.n_heads / a.n_kv, r16 = lane & 15, kgrp = (lane >> 4) * 8;
  const int qn = G * qs.rows;
  const int qi = y * 16 + r16;
  const bool qvalid = qi < qn;
  const int gh = qvalid ? qi / qs.rows : 0, ri = qvalid ? qi % qs.rows : 0;
  const int m = qs.row0 + ri, head = qs.kvh * G + gh;
  const unsigned long long anc = LAST && a.anc && qvalid ? a.anc[m] : ~0ull;
  const float* qrow = a.q + (size_t)m * (a.n_heads * HD) + head * HD;
  F8 qf[DS];
#pragma unroll
  for (int ds = 0; ds < DS; ++ds) {   // an invalid lane reads its first row, and drops it
    qf[ds].a = *(const float4*)(qrow + ds * 32 + kgrp);
    qf[ds].b = *(const float4*)(qrow + ds * 32 + kgrp + 4);
  }
  const KeyRange ks = range();
  const int qpos = qvalid ? ks.own + ri : -1;
  const size_t base = ((size_t)ks.win * a.n_kv + qs.kvh) * (size_t)a.maxlen * HD;
  const float scale2 = a.scale * 1.44269504088896340736f;   // log2 e
  struct KV16 {
    u32x4 k[2][DS], v[DT];
  };
  struct KV32 {
    F8 k[2][DS], v[DT];
  };
  KV16 b16;
  KV32 b32;
  auto load_k = [&](int p0) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int key = p0 + (r16 >> 2) * 8 + t * 4 + (r16 & 3);
#pragma unroll
      for (int ds = 0; ds < DS; ++ds) {
        const size_t i = base + kc_off(key, ds * 32 + kgrp, HD);
        if (KVB) {
          b16.k[t][ds] = *(const u32x4*)((const uint16_t*)a.kc + i);
        } else {
          b32.k[t][ds].a = *(const float4*)((const float*)a.kc + i);
          b32.k[t][ds].b = *(const float4*)((const float*)a.kc + i + 4);
        }
      }
    }
  };
  auto load_v = [&](int p0) {
#pragma unroll
    for (int t = 0; t < DT; ++t) {
      const size_t i = base + vc_off(p0 + kgrp, d0 + t * 16 + r16, HD);
      if (KVB) {
        b16.v[t] = *(const u32x4*)((const uint16_t*)a.vc + i);
      } else {
        b32.v[t].a = *(const float4*)((const float*)a.vc + i);
        b32.v[t].b = *(const float4*)((const float*)a.vc + i + 4);
      }
    }
  };
  // the first loads of a wave without keys (its step lies past k1) are of the
  // part's first keys and not used: registers that are loaded on one path only
  // are not left to the compiler
  int p0 = ks.k0 + 32 * w;
  load_k(p0 < ks.k1 ? p0 : ks.k0);
  load_v(p0 < ks.k1 ? p0 : ks.k0);
#pragma unroll
  for (int ds = 0; ds < DS; ++ds) {
    const float4 x = qf[ds].a, z = qf[ds].b;
    qf[ds].a = float4{qvalid ? x.x : 0.f, qvalid ? x.y : 0.f, qvalid ? x.z : 0.f, qvalid ? x.w : 0.f};
    qf[ds].b = float4{qvalid ? z.x : 0.f, qvalid ? z.y : 0.f, qvalid ? z.z : 0.f, qvalid ? z.w : 0.f};
  }
  bf16x8 qh[DS], ql[DS];
  if (KVB) {
#pragma unroll
    for (int ds = 0; ds < DS; ++ds) {
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = f8_get(qf[ds], e);
      u32x4 h, l;
      split8(v, h, l);
      qh[ds] = as_bf16x8(h);
      ql[ds] = as_bf16x8(l);
    }
  }
  float mrun = -INFINITY, lrun = 0.f;
  f32x4 o[DT];
#pragma unroll
  for (int t = 0; t < DT; ++t) o[t] = f32x4{0.f, 0.f, 0.f, 0.f};

  for (; p0 < ks.k1; p0 += 32 * NW) {
    const int pn = p0 + 32 * NW;
    f32x4 st[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      st[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ds = 0; ds < DS; ++ds) {
        if (KVB) {
          const bf16x8 kb = as_bf16x8(b16.k[t][ds]);
          st[t] = mfma_bf16(kb, qh[ds], st[t]);
          st[t] = mfma_bf16(kb, ql[ds], st[t]);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) st[t] = mfma_f32(f8_get(b32.k[t][ds], e), f8_get(qf[ds], e), st[t]);
        }
      }
    }
    if (pn < ks.k1) load_k(pn);
    // lane: keys p0 + kgrp + e of query r16, base-2 units
    const bool full = !LAST || p0 + 32 <= ks.own;
    float pv[8];
    unsigned seen = 0xFF;
    float mloc = -INFINITY;
    if (!full) {
      seen = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int key = p0 + kgrp + e;
        bool vis = key <= qpos && key < ks.k1;
        vis = vis && (key < ks.own || ((anc >> ((key - ks.own) & 63)) & 1ull));
        seen |= vis ? 1u << e : 0u;
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      pv[e] = seen >> e & 1 ? st[e >> 2][e & 3] * scale2 : -INFINITY;
      mloc = fmaxf(mloc, pv[e]);
    }
    mloc = max_over_16_32(mloc);
    const float mnew = fmaxf(mrun, mloc);
    const float b = mnew == -INFINITY ? 0.f : mnew;
    float lsum = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      pv[e] = __builtin_amdgcn_exp2f(pv[e] - b);
      lsum += pv[e];
    }
    if (__ballot(mnew != mrun)) {
      const float alpha = __builtin_amdgcn_exp2f(mrun - b);
      lrun *= alpha;
#pragma unroll
      for (int t = 0; t < DT; ++t) o[t] *= alpha;
    }
    lrun += lsum;
    mrun = mnew;
    // A step that some query does not see whole: values past k1 are dead cache
    // rows and become 0, whatever they hold.  A value of the call's rows that
    // is not finite would reach the rows before it as 0 * inf: it becomes 0 as
    // well, and joins the rows that see it one by one.
    if (!full) {
      const int nv = ks.k1 - (p0 + kgrp);
      bool odd = false;
      if (KVB) {
        uint32_t keep[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) keep[i] = (2 * i < nv ? 0x0000FFFFu : 0u) | (2 * i + 1 < nv ? 0xFFFF0000u : 0u);
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t x = b16.v[t][i] & keep[i];
            b16.v[t][i] = x;
            odd = odd || (x & 0x7F80u) == 0x7F80u || (x & 0x7F800000u) == 0x7F800000u;
          }
      } else {
#pragma unroll
        for (int t = 0; t < DT; ++t) {
          float x[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            x[e] = e < nv ? f8_get(b32.v[t], e) : 0.f;
            odd = odd || !(fabsf(x[e]) < INFINITY);
          }
          b32.v[t].a = float4{x[0], x[1], x[2], x[3]};
          b32.v[t].b = float4{x[4], x[5], x[6], x[7]};
        }
      }
      if (__ballot(odd)) {
#pragma unroll
        for (int t = 0; t < DT; ++t) {
          if (KVB) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint32_t x = b16.v[t][i];
              b16.v[t][i] = x & (((x & 0x7F80u) == 0x7F80u ? 0u : 0x0000FFFFu) | ((x & 0x7F800000u) == 0x7F800000u ? 0u : 0xFFFF0000u));
            }
          } else {
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              x[e] = f8_get(b32.v[t], e);
              x[e] = fabsf(x[e]) < INFINITY ? x[e] : 0.f;
            }
            b32.v[t].a = float4{x[0], x[1], x[2], x[3]};
            b32.v[t].b = float4{x[4], x[5], x[6], x[7]};
          }
        }
        // rolled: the usual step pays no registers for it
#pragma unroll 1
        for (int k = 0; k < 32; ++k) {
          float pe = pv[0];
#pragma unroll
          for (int e = 1; e < 8; ++e) pe = (k & 7) == e ? pv[e] : pe;
          const float p = __shfl(pe, r16 + 16 * (k >> 3));
          const unsigned vis = __shfl(seen, r16 + 16 * (k >> 3));
          if (!(vis >> (k & 7) & 1)) continue;
#pragma unroll
          for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const size_t i = base + vc_off(p0 + k, d0 + t * 16 + (lane >> 4) * 4 + j, HD);
              const float v = KVB ? bf_bits2f(((const uint16_t*)a.vc)[i]) : ((const float*)a.vc)[i];
              if (!(fabsf(v) < INFINITY)) o[t][j] += p * v;
            }
        }
      }
    }
    if (KVB) {
      u32x4 h, l;
      split8(pv, h, l);
      const bf16x8 ph = as_bf16x8(h), pl = as_bf16x8(l);
#pragma unroll
      for (int t = 0; t < DT; ++t) {
        const bf16x8 vv = as_bf16x8(b16.v[t]);
        o[t] = mfma_bf16(vv, ph, o[t]);
        o[t] = mfma_bf16(vv, pl, o[t]);
      }
    } else {
#pragma unroll
      for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int e = 0; e < 8; ++e) o[t] = mfma_f32(f8_get(b32.v[t], e), pv[e], o[t]);
    }
    if (pn < ks.k1) load_v(pn);
  }

  lrun = sum_over_16_32(lrun);
  if (lane < 16) {
    sums.m[w][lane] = mrun;
    sums.l[w][lane] = lrun;
  }
#pragma unroll
  for (int t = 0; t < DT; ++t) sums.o[w][t][lane] = o[t];
  __syncthreads();
}

// sums of query q (of 16) over the waves: dims 16 t + 4 (l / 16) + 0..3 of it, l % 16 = q
template <int NW, int VD>
__device__ __forceinline__ void join_waves(const WaveSums<NW, VD>& sums, int t, int l, float& M, float& L, f32x4& acc) {
  const int q = l & 15;
  M = sums.m[0][q];
#pragma unroll
  for (int x = 1; x < NW; ++x) M = fmaxf(M, sums.m[x][q]);
  const float b = M == -INFINITY ? 0.f : M;
  acc = f32x4{0.f, 0.f, 0.f, 0.f};
  L = 0.f;
#pragma unroll
  for (int x = 0; x < NW; ++x) {
    const float f = __builtin_amdgcn_exp2f(sums.m[x][q] - b);
    acc += sums.o[x][t][l] * f;
    L += sums.l[x][q] * f;
  }
}

// 16 queries over keys without a mask, as chunk `slot` of the partials
template <int KVB, int HD>
__device__ void direct_part(const ShareArgs& a, const QuerySet& qs, int win, int k0, int k1, int y, int slot, char* lds) {
  WaveSums<SW, HD>& sums = *(WaveSums<SW, HD>*)lds;
  direct_sums<KVB, HD, HD, 0>(a, qs, [&] { return KeyRange{win, k0, k1, 0}; }, y, 0, sums);
  const int G = a.n_heads / a.n_kv;
  for (int it = threadIdx.x; it < HD / 16 * 64; it += SW * 64) {
    const int t = it >> 6, l = it & 63, qc = y * 16 + (l & 15);
    if (qc >= G * qs.rows) continue;
    float M, L;
    f32x4 acc;
    join_waves(sums, t, l, M, L, acc);
    const size_t r = ((size_t)slot * a.B * a.R + qs.row0 + qc % qs.rows) * a.n_heads + qs.kvh * G + qc / qs.rows;
    *(f32x4*)(a.part_o + r * HD + t * 16 + (l >> 4) * 4) = acc;
    if (t == 0 && l < 16) a.part_ml[r] = make_float2(M, L);
  }
}

typedef __attribute__((__vector_size__(16 * sizeof(float)))) float f32x16;
__device__ __forceinline__ f32x16 mfma32_bf16(const bf16x8& a, const bf16x8& b, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

// One part of a bf16 prefix for many queries: QT tiles of 32 queries, one a
// wave, and KS = 8 / QT waves per tile that take the stage's 32-key blocks in
// turn.  A stage's keys and values go through LDS once for all queries (two
// stages, the next one's loads in flight in registers), so a CU takes in
// HD * 128 bytes per 32 keys for 32 QT queries: from some 64 queries on computing
// takes longer than that.
// 32x32x16 MFMAs, S^T[key][query] = K Q^T and O^T[dim][query] += V^T P^T: lane l
// holds query l % 32 in all of them.  Row rho of S^T stands for key
// 16 (j >> 1) + 8 h + 4 (j & 1) + i of the block, rho = 8 j + 4 h + i, so that
// the 16 scores a lane gets are keys 16 c + 8 (l / 32) + 0..7, c = 0, 1: its
// B operands of the second product.
// A block of the cache is HD / 16 tiles of 1 KB for K (16 positions x 32 dims)
// and for V (16 dims x 32 positions), rows of four 16-byte pieces.  They are
// loaded as they lie; piece q of row r goes to r * 64 + (q ^ r / 4 % 4) * 16 in
// LDS, so that the 16 rows a fragment read takes the same piece of lie in 16
// different groups of banks.
// Queries (times scale and log2 e) and probabilities are hi + lo bf16, as in
// the window attention, which leaves 2^-18 of each: twice the products for an
// error of 5e-6 of the output where fp32 sums leave 1e-6.  The running maximum
// moves only when a score is 2^8 above it, so most blocks rescale nothing.
// 256 queries over 32768 keys (8 KV heads of 128): 79 us, 0.87 PFLOP/s of these
// products, where a library product of 8192^3 reaches 1.2 on the same card.  The
// matrix instructions are busy 38 % of that and the vector ones 31 %: the products
// of the scores, the softmax and the products of the values of a block follow each
// other, with two waves a SIMD to fill in.  40 KV heads with 42 queries over 8191
// keys: 43 us, 5.5 TB/s once running, 16 us of it launch, first loads, the waves'
// join and the partials' stores.  Four waves with 64 queries each, a SIMD to
// themselves: 93 and 70 us.
// An infinite value meets the zeros of low halves and gives NaN, whatever its weight.
template <int HD, int QT>
constexpr int tile_stage_blocks() { return SW / QT < 2 ? 2 : SW / QT; }
template <int HD, int QT>
constexpr int tile_lds() { return 2 * tile_stage_blocks<HD, QT>() * HD * 128 + SW * 32 * 8; }

template <int HD, int QT>
__device__ void tile_part(const ShareArgs& a, const QuerySet& qs, const ShareGroup& g, int y, int c, char* lds) {
  constexpr int KS = SW / QT, SB = tile_stage_blocks<HD, QT>();
  constexpr int TK = HD / 16, TB = 2 * TK, NPW = SB * TB / SW;
  constexpr int DS = HD / 16, DT = HD / 32;
  const int lane = threadIdx.x & 63, h = lane >> 5, c32 = lane & 31;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int qt = w % QT, ks = w / QT;
  const int G = a.n_heads / a.n_kv, qn = G * qs.rows;
  const int qi = (y * QT + qt) * 32 + c32;
  const bool qvalid = qi < qn;
  const int m = qs.row0 + (qvalid ? qi % qs.rows : 0), head = qs.kvh * G + (qvalid ? qi / qs.rows : 0);
  // the queries' loads do not wait for the lengths
  const float* qrow = a.q + ((size_t)m * a.n_heads + head) * HD + h * 8;
  F8 qf[DS];
#pragma unroll
  for (int ds = 0; ds < DS; ++ds) {
    qf[ds].a = *(const float4*)(qrow + ds * 16);
    qf[ds].b = *(const float4*)(qrow + ds * 16 + 4);
  }
  const int shared = group_prefix(a, g), per = prefix_chunk(a, shared);
  const int k0 = c * per, k1 = min(shared, k0 + per), slot = c;
  if (k0 >= k1) return;
  const size_t base = ((size_t)g.root * a.n_kv + qs.kvh) * (size_t)a.maxlen * HD * 2;
  const char* kc = (const char*)a.kc + base;
  const char* vc = (const char*)a.vc + base;
  const int blk0 = k0 >> 5, nblk = (k1 - k0) >> 5, stages = (nblk + SB - 1) / SB;
  const int dst = (lane >> 2) * 64 + ((lane & 3) ^ (lane >> 4)) * 16;   // of this lane's piece in a tile in LDS

  u32x4 sr[NPW];
  auto load_stage = [&](int st) {
#pragma unroll
    for (int j = 0; j < NPW; ++j) {
      const int i = w * NPW + j, tile = i % TB;
      const size_t blk = (size_t)(blk0 + min(st * SB + i / TB, nblk - 1)) * (HD * 64);
      const char* p = tile < TK ? kc + blk + tile * 1024 : vc + blk + (tile - TK) * 1024;
      sr[j] = *(const u32x4*)(p + lane * 16);
    }
  };
  auto store_stage = [&](int buf) {
#pragma unroll
    for (int j = 0; j < NPW; ++j)
      *(u32x4*)(lds + buf * (SB * TB * 1024) + (w * NPW + j) * 1024 + dst) = sr[j];
  };
  load_stage(0);
  const float scale2 = a.scale * 1.44269504088896340736f;   // log2 e
  bf16x8 qh[DS], ql[DS];
#pragma unroll
  for (int ds = 0; ds < DS; ++ds) {
    const float4 x = qf[ds].a, z = qf[ds].b;
    const float f = qvalid ? scale2 : 0.f;
    const float v[8] = {x.x * f, x.y * f, x.z * f, x.w * f, z.x * f, z.y * f, z.z * f, z.w * f};
    u32x4 hi, lo;
    split8(v, hi, lo);
    qh[ds] = as_bf16x8(hi);
    ql[ds] = as_bf16x8(lo);
  }
  float mrun = -INFINITY, lrun = 0.f;
  f32x16 o[DT];
#pragma unroll
  for (int t = 0; t < DT; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[t][i] = 0.f;
  const int key = 16 * (c32 >> 4) + 8 * (c32 >> 2 & 1) + 4 * (c32 >> 3 & 1) + (c32 & 3);
  const int koff = (key >> 4) * 1024 + (key & 15) * 64 + (h ^ (key >> 2 & 3)) * 16;
  const int voff = TK * 1024 + (c32 >> 4) * 1024 + (c32 & 15) * 64 + (h ^ (c32 >> 2 & 3)) * 16;

  // one block of 32 keys
  auto block = [&](const char* p) {
    f32x16 s, s2;   // two independent chains
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = s2[i] = 0.f;
#pragma unroll
    for (int ds = 0; ds < DS; ++ds) {
      const bf16x8 kf = as_bf16x8(*(const u32x4*)(p + (koff ^ (ds & 1) * 32) + (ds >> 1) * 2048));
      s = mfma32_bf16(kf, qh[ds], s);
      s2 = mfma32_bf16(kf, ql[ds], s2);
    }
    s += s2;
    float mx = s[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) mx = fmaxf(mx, s[i]);
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
    mx = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
    if (__ballot(mx > mrun + 8.f)) {
      const float mnew = fmaxf(mrun, mx);
      const float alpha = mnew == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(mrun - mnew);
      mrun = mnew;
      lrun *= alpha;
#pragma unroll
      for (int t = 0; t < DT; ++t) o[t] *= alpha;
    }
    const float b = mrun == -INFINITY ? 0.f : mrun;
    float pv[2][8], ls[2] = {0.f, 0.f};
    auto weight = [&](int half, int i) {
      pv[half][i] = __builtin_amdgcn_exp2f(s[half * 8 + i] - b);
      ls[i & 1] += pv[half][i];
    };
#pragma unroll
    for (int i = 0; i < 8; ++i) weight(0, i);
    // the second 16 keys' weights between the first's matrix instructions
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      u32x4 hi, lo;
      split8(pv[half], hi, lo);
      const bf16x8 ph = as_bf16x8(hi), pl = as_bf16x8(lo);
      bf16x8 vf[DT];
#pragma unroll
      for (int t = 0; t < DT; ++t) vf[t] = as_bf16x8(*(const u32x4*)(p + (voff ^ half * 32) + t * 2048));
  #pragma unroll
      for (int t = 0; t < DT; ++t) {
        o[t] = mfma32_bf16(vf[t], ph, o[t]);
        if (half == 0) {
#pragma unroll
          for (int i = t * 8 / DT; i < (t + 1) * 8 / DT; ++i) weight(1, i);
        }
      }
#pragma unroll
      for (int t = 0; t < DT; ++t) o[t] = mfma32_bf16(vf[t], pl, o[t]);
      }
    lrun += ls[0] + ls[1];
  };

  const bool live = (y * QT + qt) * 32 < qn;   // a wave without queries loads for the others
  auto compute = [&](int st) {
    const char* p = lds + (st & 1) * (SB * TB * 1024);
#pragma unroll
    for (int i = 0; i < SB; i += KS)
      if (live && st * SB + i + ks < nblk) block(p + (i + ks) * (TB * 1024));
  };
  store_stage(0);
  __syncthreads();
  for (int st = 0; st < stages; ++st) {
    if (st + 1 < stages) load_stage(st + 1);
    compute(st);
    if (st + 1 < stages) store_stage((st + 1) & 1);
    __syncthreads();
  }

  {
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(lrun), __float_as_uint(lrun), false, false);
    lrun = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
  }
  if constexpr (KS > 1) {   // the tile's waves, in order
    float2(*ml)[32] = (float2(*)[32])(lds + 2 * SB * TB * 1024);
    f32x4(*so)[DT * 4][64] = (f32x4(*)[DT * 4][64])lds;
    if (lane < 32) ml[w][lane] = make_float2(mrun, lrun);
    if (ks) {
#pragma unroll
      for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          so[w - QT][t * 4 + j][lane] = f32x4{o[t][4 * j], o[t][4 * j + 1], o[t][4 * j + 2], o[t][4 * j + 3]};
    }
    __syncthreads();
    if (ks) return;
    float M = mrun;
#pragma unroll
    for (int x = 1; x < KS; ++x) M = fmaxf(M, ml[x * QT + qt][c32].x);
    const float b = M == -INFINITY ? 0.f : M;
    const float f0 = __builtin_amdgcn_exp2f(mrun - b);
    float L = lrun * f0;
#pragma unroll
    for (int t = 0; t < DT; ++t) o[t] *= f0;
#pragma unroll
    for (int x = 1; x < KS; ++x) {
      const float2 v = ml[x * QT + qt][c32];
      const float f = __builtin_amdgcn_exp2f(v.x - b);
      L += v.y * f;
#pragma unroll
      for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const f32x4 z = so[x * QT + qt - QT][t * 4 + j][lane];
#pragma unroll
          for (int i = 0; i < 4; ++i) o[t][4 * j + i] += z[i] * f;
        }
    }
    mrun = M;
    lrun = L;
  }
  if (!qvalid) return;
  const size_t r = ((size_t)slot * a.B * a.R + m) * a.n_heads + head;
  float* po = a.part_o + r * HD + 4 * h;
#pragma unroll
  for (int t = 0; t < DT; ++t)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      *(f32x4*)(po + t * 32 + j * 8) = f32x4{o[t][4 * j], o[t][4 * j + 1], o[t][4 * j + 2], o[t][4 * j + 3]};
  if (lane < 32) a.part_ml[r] = make_float2(mrun, lrun);
}

// the rows' keys and values of one window and KV head into the slots behind its
// length, rounded to the cache's type: keys by dims, values by positions, so that
// neighbouring threads write neighbours.  The host has checked that they fit, but
// for calls that the caller replays: there is nothing cached where they do not.
template <int KVB, int HD>
__device__ void append_rows(const ShareArgs& a, int win, int kvh) {
  const int len = a.f.lens[a.window0 + win];
  const int n = a.R;
  if (len > a.max_len - n) {
    if (kvh == 0 && threadIdx.x == 0) atomicOr(a.err, 32);
    return;
  }
  const size_t base = ((size_t)(a.window0 + win) * a.n_kv + kvh) * (size_t)a.maxlen * HD;
  const size_t row = (size_t)a.n_kv * HD, from = (size_t)win * a.R * row + (size_t)kvh * HD;
  for (int i = threadIdx.x; i < n * HD; i += SW * 64) {
    const int kj = i / HD, kd = i % HD, vj = i % n, vd = i / n;
    const float k = a.k_new[from + kj * row + kd], v = a.v_new[from + vj * row + vd];
    const size_t ki = base + kc_off(len + kj, kd, HD), vi = base + vc_off(len + vj, vd, HD);
    if (KVB) {
      ((uint16_t*)a.kc)[ki] = f2bf_bits(k);
      ((uint16_t*)a.vc)[vi] = f2bf_bits(v);
    } else {
      ((float*)a.kc)[ki] = k;
      ((float*)a.vc)[vi] = v;
    }
  }
}

// First launch.  QT: query tiles of 32 per workgroup of the prefix's parts
// (tile_part), or 0: 16 queries on the direct path (fp32 caches, whose keys are
// read again for every 16 queries)
template <int KVB, int HD, int QT>
__global__ __launch_bounds__(SW * 64) void k_share(ShareArgs a) {
  constexpr int kDirectLds = sizeof(WaveSums<SW, HD>);
  constexpr int kTileLds = QT ? tile_lds<HD, QT ? QT : 8>() : 0;
  __shared__ __align__(16) char lds[kDirectLds > kTileLds ? kDirectLds : kTileLds];
  // ids of one KV head are equal mod n_kv: with eight or a multiple of eight
  // KV heads, the parts that read the same keys run on one XCD
  const int n_prefix = a.n_groups * a.n_kv * a.p_tiles * a.p_chunks;
  int id = blockIdx.x;
  if (id < n_prefix) {
    const int kvh = id % a.n_kv;
    id /= a.n_kv;
    const ShareGroup& g = a.group[id % a.n_groups];
    id /= a.n_groups;
    const int y = id % a.p_tiles, c = id / a.p_tiles;
    const QuerySet qs{g.first * a.R, g.count * a.R, kvh};
    if (y * (QT ? 32 * QT : 16) >= qs.rows * (a.n_heads / a.n_kv)) return;
    if constexpr (QT > 0) {
      tile_part<HD, QT>(a, qs, g, y, c, lds);
    } else {
      const int s = group_prefix(a, g), per = prefix_chunk(a, s);
      if (c * per < s) direct_part<KVB, HD>(a, qs, g.root, c * per, min(s, c * per + per), y, c, lds);
    }
    return;
  }
  id -= n_prefix;
  const int kvh = id % a.n_kv;
  id /= a.n_kv;
  // the windows of a row are turned by one each time: where B is a multiple of
  // four, the few that have keys of their own would meet the same quarter of an
  // XCD in every row (8 x 8 rows, two windows with 6000: 68 and 45 us)
  const int row = id / a.B, win = (id + row) % a.B;
  const int y = row % a.t_tiles, c = row / a.t_tiles;
  // no part of this launch reads the slots of the call's rows
  if (a.k_new && y == 0 && c == 0) append_rows<KVB, HD>(a, win, kvh);
  const int s = window_prefix(a, win);
  const int keys = own_end(s, min(a.f.lens[a.window0 + win], a.maxlen - a.R)) - s, per = own_chunk(keys, a.t_chunks);
  if (c * per >= keys) return;
  direct_part<KVB, HD>(a, QuerySet{win * a.R, a.R, kvh}, a.window0 + win, s + c * per, s + min(keys, c * per + per), y,
                       a.p_chunks + c, lds);
}

// Bound by latency (launch, lengths, keys, partials: 6 us for 4 windows of one
// row, 1B) or, where a group has many queries, by the partials, eight of which are
// loaded, waited for and joined at a time: 256 queries and 32 chunks leave 33 MB, 17
// us, 2.3 TB/s.
// Second launch: one workgroup per (window, KV head, 16 queries, VD dims) attends
// to the window's last keys and the rows, and joins that with the partials of its
// queries, in order.  Heads of more than 64 dims are halved: twice the workgroups
// read the partials, for a second reading of the few keys.
// What is known without the lengths is loaded before they are: the queries, and
// the first CB partials (of chunks that may turn out not to exist).
// Two workgroups a CU have to fit the registers: with one, 480 of them (13B, 6 x 7
// rows) took 15.4 us, with two 11.3.
template <int KVB, int HD>
__global__ __launch_bounds__(LW * 64, KVB ? 2 : 1) void k_share_last(ShareArgs a) {
  constexpr int NV = HD > 64 ? 2 : 1, VD = HD / NV, CB = 8;
  static_assert(VD / 16 * 64 <= LW * 64, "a piece of four dims of a query per thread");
  __shared__ __align__(16) WaveSums<LW, VD> sums;
  int id = blockIdx.x;
  const int kvh = id % a.n_kv;
  id /= a.n_kv;
  const int d0 = id % NV * VD;
  id /= NV;
  const int win = id % a.B, y = id / a.B;
  const int G = a.n_heads / a.n_kv;
  // this thread's piece of the result
  const int t = threadIdx.x >> 6, l = threadIdx.x & 63;
  const int qc = min(y * 16 + (l & 15), G * a.R - 1);
  const int m = win * a.R + qc % a.R, head = kvh * G + qc / a.R, d = d0 + t * 16 + (l >> 4) * 4;
  const size_t rows = (size_t)a.B * a.R * a.n_heads, r = (size_t)m * a.n_heads + head;
  const bool piece = t < VD / 16;
  float2 ml[CB];
  f32x4 o[CB];
#pragma unroll
  for (int j = 0; j < CB; ++j) {
    const size_t slot = (size_t)min(j, a.p_chunks + a.t_chunks - 1) * rows + r;
    ml[j] = a.part_ml[slot];
    o[j] = *(const f32x4*)(a.part_o + slot * HD + (piece ? d : 0));
  }
  int s, e, len;
  direct_sums<KVB, HD, VD, 1>(a, QuerySet{win * a.R, a.R, kvh}, [&] {
    s = window_prefix(a, win);
    len = min(a.f.lens[a.window0 + win], a.maxlen - a.R);
    e = own_end(s, len);
    return KeyRange{a.window0 + win, e, len + a.R, len};
  }, y, d0, sums);
  if (!piece || y * 16 + (l & 15) >= G * a.R) return;
  const int np = s ? (s + prefix_chunk(a, s) - 1) / prefix_chunk(a, s) : 0;
  const int nc = np + (e > s ? (e - s + own_chunk(e - s, a.t_chunks) - 1) / own_chunk(e - s, a.t_chunks) : 0);
  float M, L;
  f32x4 acc;
  join_waves(sums, t, l, M, L, acc);
  for (int c0 = 0; c0 < nc; c0 += CB) {
    if (c0 || np < min(nc, CB)) {   // else they are the partials loaded above
#pragma unroll
      for (int j = 0; j < CB; ++j) {
        const int c = min(c0 + j, nc - 1);
        const size_t slot = (size_t)(c < np ? c : a.p_chunks + c - np) * rows + r;
        ml[j] = a.part_ml[slot];
        o[j] = *(const f32x4*)(a.part_o + slot * HD + d);
      }
    }
    float Mn = M;
#pragma unroll
    for (int j = 0; j < CB; ++j)
      if (c0 + j < nc) Mn = fmaxf(Mn, ml[j].x);
    const float b = Mn == -INFINITY ? 0.f : Mn;
    const float f0 = __builtin_amdgcn_exp2f(M - b);
    L *= f0;
    acc *= f0;
    M = Mn;
#pragma unroll
    for (int j = 0; j < CB; ++j)
      if (c0 + j < nc) {
        const float f = __builtin_amdgcn_exp2f(ml[j].x - b);
        L += ml[j].y * f;
        acc += o[j] * f;
      }
  }
  // a replayed call's rows that did not fit were not cached: no result
  const float inv = a.k_new && a.f.lens[a.window0 + win] > a.max_len - a.R ? NAN : 1.0f / L;
  const float y4[4] = {acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv};
  if (a.out_rows) *(float4*)(a.out_rows + r * HD + d) = float4{y4[0], y4[1], y4[2], y4[3]};
  else pack_store4(a.out, a.wtype, m, head * HD + d, y4);
}

template <int KVB, int HD, int QT>
hipError_t launch_shared_qt(const ShareArgs& a, hipStream_t s) {
  const long long wgs = (long long)a.n_groups * a.n_kv * a.p_tiles * a.p_chunks + (long long)a.B * a.n_kv * a.t_tiles * a.t_chunks;
  if (wgs > INT_MAX) return hipErrorInvalidValue;
  if (wgs) hipLaunchKernelGGL((k_share<KVB, HD, QT>), dim3((unsigned)wgs), dim3(SW * 64), 0, s, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((k_share_last<KVB, HD>), dim3((unsigned)a.B * a.n_kv * a.t_tiles * (HD > 64 ? 2 : 1)), dim3(LW * 64),
                     0, s, a);
  return hipGetLastError();
}

template <int HD>
hipError_t launch_shared_hd(int kv_bf16, const ShareArgs& a, hipStream_t s) {
  if (!kv_bf16) return launch_shared_qt<0, HD, 0>(a, s);
  switch (a.p_tile) {
    case 256: return launch_shared_qt<1, HD, 8>(a, s);
    case 128: return launch_shared_qt<1, HD, 4>(a, s);
    case 64: return launch_shared_qt<1, HD, 2>(a, s);
  }
  return hipErrorInvalidValue;
}

__global__ void k_kv_advance(int* lens, int window0, int B, int rows, int max_len) {
  for (int b = threadIdx.x; b < B; b += blockDim.x)
    if (lens[window0 + b] <= max_len - rows) lens[window0 + b] += rows;
}

__global__ void k_fork_cut(ForkState f, int window, int new_len) { fork_cut(f, window, new_len); }

// Copies positions [0, len) of window src into n windows: one workgroup per
// 32-position block of a (layer, KV head), which holds its keys and values in
// registers and stores them n times: the source is read once, 16 bytes a lane
// on both sides.  Bound by memory: 8B, 2048 positions into 6 windows, 1.88 GB
// moved, 364 us, 5.16 TB/s, where a copy of 1 GiB reaches 5.21 (reads and writes
// together); 1B, 509 positions into 3, 67 MB, 16.4 us.  The positions behind len in its last
// block stay as they are in the windows.  The first workgroup sets the lengths
// and the record of what is shared: nothing else of this launch reads those.
template <int ESZ>
__global__ __launch_bounds__(256) void k_kv_fork(ForkArgs a) {
  const int have = a.f.lens[a.src];
  const int len = a.len < 0 ? have : a.len;
  const bool first = blockIdx.x == 0 && blockIdx.y == 0;
  // a replayed commit of the caller's may have carried a length past the cache's end
  const bool bad = len > have || len > a.most;
  constexpr int VE = 16 / ESZ;           // elements per 16 bytes
  constexpr int MOST = 128 * 32 / VE / 256;   // 16-byte pieces per thread of a block's keys (and values)
  const int pieces = a.hd * 32 / VE;
  const int layer = blockIdx.y / a.n_kv, h = blockIdx.y % a.n_kv;
  const size_t head = (size_t)h * a.maxlen * a.hd * ESZ;
  char* kc = (char*)a.kc + layer * a.layer_bytes + head;
  char* vc = (char*)a.vc + layer * a.layer_bytes + head;
  for (int blk = blockIdx.x; blk * 32 < len && !bad; blk += gridDim.x) {
    const size_t at = (size_t)blk * 32 * a.hd * ESZ;
    const int live = min(32, len - blk * 32);
    u32x4 k[MOST], v[MOST];
#pragma unroll
    for (int i = 0; i < MOST; ++i) {
      const int p = i * 256 + threadIdx.x;
      if (p < pieces) {
        k[i] = ((const u32x4*)(kc + a.src * a.win_bytes + at))[p];
        v[i] = ((const u32x4*)(vc + a.src * a.win_bytes + at))[p];
      }
    }
    for (int w = a.window0; w < a.window0 + a.n; ++w) {
      u32x4* dk = (u32x4*)(kc + w * a.win_bytes + at);
      u32x4* dv = (u32x4*)(vc + w * a.win_bytes + at);
#pragma unroll
      for (int i = 0; i < MOST; ++i) {
        const int p = i * 256 + threadIdx.x;
        if (p >= pieces) continue;
        if (live == 32) {
          dk[p] = k[i];
          dv[p] = v[i];
        } else {
          // a piece of keys is VE dims of one position, one of values VE positions of one dim
          if (p * VE / 32 % 32 < live) dk[p] = k[i];
          const int p0 = p * VE % 32;
#pragma unroll
          for (int e = 0; e < VE; ++e)
            if (p0 + e < live) {
              if constexpr (ESZ == 2) ((uint16_t*)(dv + p))[e] = (uint16_t)(v[i][e / 2] >> (e % 2 * 16));
              else ((uint32_t*)(dv + p))[e] = v[i][e];
            }
        }
      }
    }
  }
  if (!first) return;
  if (bad && threadIdx.x == 0) atomicOr(a.err, 16);
  // what other windows shared with the overwritten ones ends
  for (int w = threadIdx.x; w < a.f.n_windows; w += 256) {
    const bool into = w >= a.window0 && w < a.window0 + a.n;
    if (into) {
      a.f.lens[w] = bad ? 0 : len;
      a.f.root[w] = a.src;
      a.f.shared[w] = bad ? 0 : len;
    } else if (a.f.root[w] >= a.window0 && a.f.root[w] < a.window0 + a.n) {
      a.f.shared[w] = 0;
    }
  }
}

}  // namespace

int share_tile(int kv_bf16, int queries) { return !kv_bf16 ? 16 : queries > 128 ? 256 : queries > 64 ? 128 : 64; }

hipError_t launch_attention_shared(int kv_bf16, int hd, const ShareArgs& a, hipStream_t s) {
  if (a.B < 1 || a.R < 1 || a.t_tiles < 1 || a.t_chunks < 0 || (a.k_new && a.t_chunks < 1) || a.n_groups < 0 || a.n_groups > kMaxForkGroups ||
      (a.n_groups && (a.p_tiles < 1 || a.p_chunks < 1)) || a.p_chunks < 0)
    return hipErrorInvalidValue;
  switch (hd) {
    case 32: return launch_shared_hd<32>(kv_bf16, a, s);
    case 64: return launch_shared_hd<64>(kv_bf16, a, s);
    case 96: return launch_shared_hd<96>(kv_bf16, a, s);
    case 128: return launch_shared_hd<128>(kv_bf16, a, s);
  }
  return hipErrorInvalidValue;
}

hipError_t launch_kv_advance(int* lens, int window0, int B, int rows, int max_len, hipStream_t s) {
  hipLaunchKernelGGL(k_kv_advance, dim3(1), dim3(64), 0, s, lens, window0, B, rows, max_len);
  return hipGetLastError();
}

hipError_t launch_fork_cut(const ForkState& f, int window, int new_len, hipStream_t s) {
  hipLaunchKernelGGL(k_fork_cut, dim3(1), dim3(64), 0, s, f, window, new_len);
  return hipGetLastError();
}

// max_len: a bound on the positions taken, for the grid only
hipError_t launch_kv_fork(const ForkArgs& a, int max_len, hipStream_t s) {
  if (a.n < 1 || a.hd % 32 || a.hd > 128) return hipErrorInvalidValue;
  const dim3 grid(max_len > 32 ? (max_len + 31) / 32 : 1, a.n_layers * a.n_kv);
  if (a.esz == 2) hipLaunchKernelGGL((k_kv_fork<2>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((k_kv_fork<4>), grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace dsi
