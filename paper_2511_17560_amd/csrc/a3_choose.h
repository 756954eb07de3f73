// Reading rows of logits and choosing the best of them: shared by the log probabilities (a3_logits.hip) and by what follows several
// candidates (a3_candidates.hip).
#pragma once

#include <type_traits>

#include "a3_internal.h"

namespace {

constexpr int kLpThreads = 256, kLpValues = 32, kLpTop = 64, kLpCands = 576;
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.693147180559945309417f;

// Order of the alternatives as one number: larger logit, then lower index; -0 equals 0, NaN below everything (0: no value).
__device__ __forceinline__ uint32_t top_order(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);
  return x != x ? 0u : (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ unsigned long long top_key(float x, int v) { return ((unsigned long long)top_order(x) << 32) | (uint32_t)~v; }
__device__ __forceinline__ float top_value(unsigned long long key) {
  const uint32_t o = (uint32_t)(key >> 32);
  return o == 0u ? __uint_as_float(0x7fc00000u) : __uint_as_float((o & 0x80000000u) ? o & 0x7fffffffu : ~o);
}

constexpr int kLpChunks = 20;        // chunks whose maxima are noted before their alternatives are chosen: rows up to 163840 in one go
constexpr int kLpQueue = 512;

struct lp_shared {
  float red[4][4];
  uint32_t bound[4];
  int count, queued, total;
  unsigned short queue[kLpQueue];    // noted chunks to look at: chunk * 256 + thread
  unsigned long long best[4], list[kLpTop], cand[kLpCands];
};

// Sum and maximum over a wave, in every lane, by data-parallel moves (a shuffle through LDS takes 130 cycles).
#define A3_WAVE_REDUCE(OP, X, NONE)                                                                                                    \
  X = OP(X, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, NONE), __builtin_bit_cast(int, X), 0x111, 0xf, 0xf, false))); \
  X = OP(X, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, NONE), __builtin_bit_cast(int, X), 0x112, 0xf, 0xf, false))); \
  X = OP(X, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, NONE), __builtin_bit_cast(int, X), 0x114, 0xf, 0xf, false))); \
  X = OP(X, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, NONE), __builtin_bit_cast(int, X), 0x118, 0xf, 0xf, false))); \
  X = OP(X, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, NONE), __builtin_bit_cast(int, X), 0x142, 0xa, 0xf, false))); \
  X = OP(X, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, NONE), __builtin_bit_cast(int, X), 0x143, 0xc, 0xf, false))); \
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, X), 63));
__device__ __forceinline__ float lp_add(float a, float b) { return a + b; }
__device__ __forceinline__ float wave_sum(float x) { A3_WAVE_REDUCE(lp_add, x, 0.f) }
__device__ __forceinline__ float wave_max(float x) { A3_WAVE_REDUCE(fmaxf, x, -INFINITY) }
#undef A3_WAVE_REDUCE

// (from - to) in units of log 2: what moves a sum from reference `from` to the larger `to`.  Bounded, so that a sum whose weight
// is 0 (masks of the type's lowest value: the difference overflows) leaves no NaN.
__device__ __forceinline__ float lp_shift(float from, float to) { return from == -INFINITY ? 0.f : fmaxf((from - to) * kLog2e, -1e30f); }

// (m, z, t) of a workgroup's threads as one, in every thread
__device__ __forceinline__ void lp_join_workgroup(lp_shared &s, float &m, float &z, float &t) {
  const int wave = threadIdx.x >> 6;
  const float mw = wave_max(m), dw = lp_shift(m, mw), fw = __builtin_amdgcn_exp2f(dw);
  const float tw = wave_sum(fw * fmaf(dw, z, t)), zw = wave_sum(fw * z);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) { s.red[wave][0] = mw; s.red[wave][1] = zw; s.red[wave][2] = tw; }
  __syncthreads();
  m = fmaxf(fmaxf(s.red[0][0], s.red[1][0]), fmaxf(s.red[2][0], s.red[3][0]));
  z = t = 0.f;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const float d = lp_shift(s.red[w][0], m), f = __builtin_amdgcn_exp2f(d);
    t += f * fmaf(d, s.red[w][1], s.red[w][2]);
    z += f * s.red[w][1];
  }
}

// The n-th largest of a wave's numbers, J of so many bits a lane (0: fewer than n are not 0).
template <int BITS, int J>
__device__ __forceinline__ uint32_t wave_nth(const uint32_t (&x)[J], int n) {
  uint32_t b = 0;
#pragma unroll 4
  for (int i = BITS - 1; i >= 0; --i) {
    const uint32_t t = b | 1u << i;
    int count = 0;
#pragma unroll
    for (int j = 0; j < J; ++j) count += __popcll(__ballot(x[j] >= t));
    if (count >= n) b = t;
  }
  return b;
}

__device__ __forceinline__ void lp_push(lp_shared &s, unsigned long long k, unsigned long long last) {
  if (k <= last) return;
  const int at = atomicAdd(&s.count, 1);
  if (at < kLpCands) s.cand[at] = k;
}

// list becomes the n best candidates: every candidate's place is the number of larger ones (all differ; 0: none).
__device__ __forceinline__ void lp_rank(lp_shared &s, int n) {
  const int count = s.count;
  for (int c = threadIdx.x; c < count; c += kLpThreads) {
    const unsigned long long k = s.cand[c];
    int rank = 0;
#pragma unroll 8
    for (int o = 0; o < count; ++o) rank += s.cand[o] > k;
    if (rank < n && k) s.list[rank] = k;
  }
  __syncthreads();
}

// The other way where there is no room for the candidates (NaN nearly everywhere, or one thread's values far above all others'):
// one after the other, the largest below the last one taken.  below(prev): the thread's largest key below prev.
template <class Below>
__device__ __forceinline__ void lp_one_by_one(lp_shared &s, int n, Below below) {
  const int tid = threadIdx.x;
  __syncthreads();
  if (tid < n) s.cand[tid] = s.list[tid];                      // the list before
  __syncthreads();
  unsigned long long prev = ~0ull;
  int old = 0;
  for (int j = 0; j < n; ++j) {
    unsigned long long k = below(prev);
    for (int o = 32; o; o >>= 1) { const unsigned long long x = __shfl_xor(k, o); k = x > k ? x : k; }
    if ((tid & 63) == 0) s.best[tid >> 6] = k;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 4; ++w) k = s.best[w] > k ? s.best[w] : k;
    const unsigned long long from_list = s.cand[old];
    if (from_list > k) { k = from_list; ++old; } else prev = k;
    __syncthreads();
    if (tid == 0) s.list[j] = k;
  }
  __syncthreads();
}

// A row as aligned vectors: vector v holds elements v V - skew .. (skew: how far the row starts behind a 16-byte border); a slice is
// vectors v0 .. v1 - 1, a chunk 256 U of them, element i of a thread's 32 in vector c + 256 (i / V) + thread.
// ANYWHERE: vectors as the row stands (skew 0), loaded from any place an element can have, so that what is summed in which order does not
// depend on where the row starts.
template <typename E, bool ANYWHERE = false>
struct lp_row {
  typedef E T;
  static constexpr int V = a3_elem<T>::kVec, U = kLpValues / V, kChunk = U * kLpThreads;
  typedef T vec_t __attribute__((ext_vector_type(V)));
  typedef T vec_any __attribute__((ext_vector_type(V), aligned(sizeof(T))));
  typedef typename std::conditional<ANYWHERE, vec_any, vec_t>::type load_t;
  const T *x;
  int vocab, skew, v0, v1;
  __device__ __forceinline__ vec_t vec(int v) const {          // -inf where the slice has none
    const int e = v * V - skew;
    if (v < v1 && e >= 0 && e + V <= vocab) return *reinterpret_cast<const load_t *>(x + e);
    vec_t r;
#pragma unroll
    for (int i = 0; i < V; ++i) r[i] = (T)-INFINITY;
    if (v < v1)                                                // the first or the last of a row
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (e + i >= 0 && e + i < vocab) r[i] = x[e + i];
    return r;
  }
  __device__ __forceinline__ unsigned long long key(int v, int i, float y) const {
    const int e = v * V - skew + i;
    return v < v1 && (unsigned)e < (unsigned)vocab ? top_key(y, e) : 0ull;
  }
};

// The n best of the list so far and of chunks g0 .. (vectors) up to g1, whose maxima are noted.  most, second: the order of the largest
// values of two halves of chunks of the thread's, 0 if there may be none but NaN.
template <class R>
__device__ void lp_choose(lp_shared &s, const R &r, const float (*noted)[kLpThreads], int n, int g0, int g1, uint32_t most, uint32_t second) {
  typedef typename R::T T;
  constexpr int V = R::V, kChunk = R::kChunk;
  const int tid = threadIdx.x, chunks = (g1 - g0 + kChunk - 1) / kChunk;
  constexpr int kBits = 8 * sizeof(T);                         // of a value's order: bf16 values differ in the upper 16
  const uint32_t mine = wave_nth<kBits, 2>({most >> (32 - kBits), second >> (32 - kBits)}, n);
  if ((tid & 63) == 0) s.bound[tid >> 6] = mine;
  for (int pass = 0;; ++pass) {                                // 0: what reaches the bound; 1: what exceeds it, and the first equal ones
    if (tid == 0) { s.count = n; s.queued = 0; s.total = 0; }
    __syncthreads();
    const uint32_t bound = max(max(s.bound[0], s.bound[1]), max(s.bound[2], s.bound[3])) + pass;
    const unsigned long long last = s.list[n - 1];
    if (tid < n) s.cand[tid] = s.list[tid];
    for (int c = 0; c < chunks; ++c) {
      const float y = noted[c][tid];
      // (a chunk of NaN notes -inf: without a bound everything is looked at)
      if (bound == 0 || top_order(y) >> (32 - kBits) >= bound) {
        const int at = atomicAdd(&s.queued, 1);
        if (at < kLpQueue) s.queue[at] = (unsigned short)(c * kLpThreads + tid);
      }
    }
    __syncthreads();
    const int queued = s.queued;
    if (queued <= kLpQueue) {
      constexpr int Q = 4, kHalves = kLpThreads / 32;          // half a wave a chunk, the loads of four on their way together
      for (int q0 = tid >> 5; q0 < queued; q0 += Q * kHalves) {
        T y[Q];
        int e[Q];
#pragma unroll
        for (int k = 0; k < Q; ++k) {
          const int id = s.queue[min(q0 + k * kHalves, queued - 1)], i = tid & 31;
          const int v = g0 + id / kLpThreads * kChunk + i / V * kLpThreads + id % kLpThreads, at = v * V - r.skew + i % V;
          e[k] = q0 + k * kHalves < queued && v < r.v1 && (unsigned)at < (unsigned)r.vocab ? at : -1;
          y[k] = r.x[max(e[k], 0)];
        }
#pragma unroll
        for (int k = 0; k < Q; ++k) {
          const unsigned long long key = top_key((float)y[k], e[k]);
          if (e[k] >= 0 && (uint32_t)(key >> (64 - kBits)) >= bound) lp_push(s, key, last);
        }
      }
    }
    __syncthreads();
    if (pass == 1 && queued <= kLpQueue) {
      for (int v = g0;; v += kLpThreads) {                     // the equal ones in the row's order
        const typename R::vec_t raw = r.vec(v + tid);
        int found = 0;
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const unsigned long long k = r.key(v + tid, i, (float)raw[i]);
          found += k != 0 && (uint32_t)(k >> (64 - kBits)) == bound - 1;
        }
        const int incl = a3_wave_prefix(found);
        if ((tid & 63) == 63) s.bound[tid >> 6] = incl;        // (the bounds are not needed any more)
        const int before = s.total;
        __syncthreads();
        int at = before + incl - found;
        for (int w = 0; w < (tid >> 6); ++w) at += s.bound[w];
        const int all = before + s.bound[0] + s.bound[1] + s.bound[2] + s.bound[3];
        if (found && at < n)
#pragma unroll
          for (int i = 0; i < V; ++i) {
            const unsigned long long k = r.key(v + tid, i, (float)raw[i]);
            if (k != 0 && (uint32_t)(k >> (64 - kBits)) == bound - 1 && at++ < n) lp_push(s, k, last);
          }
        __syncthreads();
        if (tid == 0) s.total = all;
        __syncthreads();
        if (all >= n || v + kLpThreads >= g1) break;
      }
    }
    if (queued <= kLpQueue && s.count <= kLpCands) break;
    if (pass == 0) { __syncthreads(); continue; }
    lp_one_by_one(s, n, [&](unsigned long long prev) {
      unsigned long long b = 0;
      for (int v = g0 + tid; v < g1; v += kLpThreads) {
        const typename R::vec_t raw = r.vec(v);
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const unsigned long long k = r.key(v, i, (float)raw[i]);
          if (k < prev && k > b) b = k;
        }
      }
      return b;
    });
    return;
  }
  lp_rank(s, n);
}

}  // namespace
