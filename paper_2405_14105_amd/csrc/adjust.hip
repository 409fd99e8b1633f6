// Penalties for tokens that were seen, biases and a grammar's mask on rows of
// logits, in one pass over them.
//
//   c > 0: z = z > 0 ? z / r : z r;  z = z - f c - (c > 0 ? p : 0) + bias;
//   -inf where the mask forbids the token
// A workgroup takes a chunk of kAdjChunk entries of the vocabulary and a few
// rows of one window.  One word of LDS an entry holds how often the text so far
// has its token (low 21 bits) and which bias it has (high bits: the largest
// index of an entry of its id, so that the last one counts whatever the order of
// the atomics).  The window's tokens are counted once for the workgroup's rows;
// then each row's own token is added before the row is worked on.  The first
// row's logits are on their way meanwhile.
// In place, only 16-byte runs with something to change are read and written.
// Bound by reading and writing the rows where there are many (7 x 6 x 128256 fp32, 44
// MB: 13 us; 64 x 128256: 16 us, 4.1 TB/s), by the chain from the tokens to the stores
// where there are few (1 x 32000: 5.4 us).
#include <algorithm>

#include "device_util.h"

namespace dsi {

namespace {

constexpr int kAdjThreads = 256;
constexpr int kAdjChunk = 4096;
// workgroups up to which a window's rows are spread (7 x 6 x 128256, 2048 tokens seen:
// 16.0 us with 256, 13.5 with 512 or 1024; 16 x 4 in bf16: 15.8, 16.0, 12.6, with 2048 14.0)
constexpr int kAdjFull = 1024;
static_assert(kMaxBias < 1 << 11 && kMaxCount == 1 << 21, "a word holds both");

// 16 bytes of a row, whose alignment is the type's (T holds bit patterns:
// uint32_t for fp32, uint16_t for bf16)
template <typename T>
struct Run;
template <>
struct Run<uint32_t> {
  static constexpr int N = 4;
  typedef uint32_t vec __attribute__((ext_vector_type(4), aligned(4)));
};
template <>
struct Run<uint16_t> {
  static constexpr int N = 8;
  typedef uint32_t vec __attribute__((ext_vector_type(4), aligned(2)));
};
template <typename T>
__device__ __forceinline__ u32x4 load_run(const T* row, int v, int V) {
  typedef typename Run<T>::vec vec;
  if (v + Run<T>::N <= V) return *(const vec*)(row + v);
  u32x4 x = u32x4{0, 0, 0, 0};
#pragma unroll
  for (int e = 0; e < Run<T>::N; ++e)
    if (v + e < V) x[e * sizeof(T) / 4] |= (uint32_t)row[v + e] << (sizeof(T) == 2 ? 16 * (e & 1) : 0);
  return x;
}
template <typename T>
__device__ __forceinline__ void store_run(T* row, int v, int V, const u32x4& x) {
  typedef typename Run<T>::vec vec;
  if (v + Run<T>::N <= V) {
    *(vec*)(row + v) = x;
    return;
  }
#pragma unroll
  for (int e = 0; e < Run<T>::N; ++e)
    if (v + e < V) row[v + e] = (T)(sizeof(T) == 4 ? x[e] : x[e >> 1] >> (16 * (e & 1)));
}
template <typename T>
__device__ __forceinline__ float entry(const u32x4& x, int e) {
  if constexpr (sizeof(T) == 4) return __uint_as_float(x[e]);
  return __uint_as_float(e & 1 ? x[e >> 1] & 0xFFFF0000u : x[e >> 1] << 16);
}

template <typename T, bool PLACE>
__global__ __launch_bounds__(kAdjThreads) void k_adjust(AdjustArgs a) {
  constexpr int N = Run<T>::N, PER = kAdjChunk / N / kAdjThreads;   // runs of a thread
  __shared__ uint32_t word[kAdjChunk];
  const int tid = threadIdx.x;
  const int c = blockIdx.x % a.chunks, bg = blockIdx.x / a.chunks;
  const int g = bg % a.groups, b = bg / a.groups;
  const int v0 = c * kAdjChunk;
  const int i0 = g * a.rpg, i1 = min(i0 + a.rpg, a.R);
  auto row_of = [&](int i) { return (const T*)a.z + ((size_t)b * a.R + i) * a.ld; };
  u32x4 z[PER];
  uint32_t ok[PER];   // the mask's bits, of a run's entries the lowest
  auto load_row = [&](int i) {
    const uint32_t* mask = a.allowed ? a.allowed + ((size_t)b * a.R + i) * a.lda : nullptr;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int v = v0 + (j * kAdjThreads + tid) * N;
      if (v >= a.V) continue;
      if constexpr (!PLACE) z[j] = load_run(row_of(i), v, a.V);
      ok[j] = mask ? mask[v >> 5] >> (v & 31) : ~0u;
    }
  };
  load_row(i0);
  for (int j = tid; j < kAdjChunk / 4; j += kAdjThreads) ((u32x4*)word)[j] = u32x4{0, 0, 0, 0};
  __syncthreads();
  for (int j = tid; j < a.n_bias; j += kAdjThreads) {
    const uint32_t at = (uint32_t)a.bias_ids[(size_t)b * a.n_bias + j] - (uint32_t)v0;
    if (at < (uint32_t)kAdjChunk) atomicMax(&word[at], (uint32_t)(j + 1) << 21);
  }
  if (a.n_bias) __syncthreads();
  auto count = [&](int tok) {
    const uint32_t at = (uint32_t)tok - (uint32_t)v0;
    if (at < (uint32_t)kAdjChunk) atomicAdd(&word[at], 1u);
  };
  if (a.seen) {
    const int* s = a.seen + (size_t)b * a.ldseen;
    const int n = min(max(a.n_seen[b], 0), (int)a.ldseen);
    // eight loads of a thread in flight (one after the other they were half the time
    // of 7 windows x 6 rows x 128256 with 2048 tokens seen)
    for (int j0 = tid; j0 < n; j0 += 8 * kAdjThreads) {
      int tok[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) tok[k] = j0 + k * kAdjThreads < n ? s[j0 + k * kAdjThreads] : -1;
#pragma unroll
      for (int k = 0; k < 8; ++k) count(tok[k]);
    }
  }
  const int* own = a.tokens ? a.tokens + (size_t)b * a.R : nullptr;
  if (own)
    for (int j = tid; j < i0; j += kAdjThreads) count(own[j]);
  const float r = a.repetition ? a.repetition[b] : 1.f;
  const float f = a.frequency ? a.frequency[b] : 0.f;
  const float p = a.presence ? a.presence[b] : 0.f;
  const float* bias = a.bias + (size_t)b * a.n_bias;
  for (int i = i0; i < i1; ++i) {
    if (own && tid == 0) count(own[i]);
    __syncthreads();
    T* out = (T*)a.out + ((size_t)b * a.R + i) * a.ldo;
    u32x4 y[PER];
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int at = (j * kAdjThreads + tid) * N, v = v0 + at;
      if (v >= a.V) continue;
      uint32_t w[N], any = 0;
#pragma unroll
      for (int e = 0; e < N; ++e) any |= w[e] = word[at + e];
      const bool all = (~ok[j] & ((1u << N) - 1)) == 0;
      if (PLACE && !any && all) continue;
      const u32x4 x = PLACE ? load_run(row_of(i), v, a.V) : z[j];
      uint32_t o[N];
#pragma unroll
      for (int e = 0; e < N; ++e) {
        float t = entry<T>(x, e);
        const uint32_t n = w[e] & (kMaxCount - 1);
        if (n) {
          t = t > 0.f ? t / r : t * r;
          t = t - f * (float)n - p;
        }
        if (w[e] >> 21) t += bias[(w[e] >> 21) - 1];
        if (!(ok[j] >> e & 1)) t = -INFINITY;
        o[e] = __float_as_uint(t);
      }
      if constexpr (sizeof(T) == 4) {
        y[j] = u32x4{o[0], o[1], o[2], o[3]};
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) y[j][e] = f2bf_pair(__uint_as_float(o[2 * e % N]), __uint_as_float(o[(2 * e + 1) % N]));
      }
      if constexpr (PLACE) store_run(out, v, a.V, y[j]);
    }
    if (i + 1 < i1) {
      load_row(i + 1);
      __syncthreads();   // the words are read before the next row's token enters them
    }
    if constexpr (!PLACE) {
#pragma unroll
      for (int j = 0; j < PER; ++j) {
        const int v = v0 + (j * kAdjThreads + tid) * N;
        if (v < a.V) store_run(out, v, a.V, y[j]);
      }
    }
  }
}

}  // namespace

hipError_t launch_adjust(AdjustArgs a, hipStream_t s) {
  a.chunks = (a.V - 1) / kAdjChunk + 1;
  // rows of a window share what it has seen, where there is work for the card without them
  const long long each = (long long)a.chunks * a.B;
  a.groups = (int)std::min((long long)a.R, (kAdjFull + each - 1) / each);
  a.rpg = (a.R + a.groups - 1) / a.groups;
  a.groups = (a.R + a.rpg - 1) / a.rpg;
  if (each * a.groups > kMaxStepBlocks) return hipErrorInvalidConfiguration;
  const dim3 grid((unsigned)(each * a.groups)), block(kAdjThreads);
  const bool place = a.z == a.out && a.ld == a.ldo;
  if (a.bf16) {
    if (place) hipLaunchKernelGGL((k_adjust<uint16_t, true>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((k_adjust<uint16_t, false>), grid, block, 0, s, a);
  } else {
    if (place) hipLaunchKernelGGL((k_adjust<uint32_t, true>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((k_adjust<uint32_t, false>), grid, block, 0, s, a);
  }
  return hipGetLastError();
}

}  // namespace dsi
