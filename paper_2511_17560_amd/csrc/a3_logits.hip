// From hidden rows to the next token: the product with the vocabulary's weights, and log probabilities of its rows.
#include "a3_internal.h"
#include "a3_gemm_pp.h"

namespace {

// ---------------------------------------------------------------------------------------
// logits, bf16: the row-tiled MFMA GEMM of a3_gemm_pp.h, float out
// ---------------------------------------------------------------------------------------
struct logits_args {
  const void *x;           // [*, K]
  const int *row_idx;
  int n_rows;
  const void *w;           // [N, K]
  float *out;
  long long ld;
  int K, N;
  int n_wtiles, n_tok_tiles, group;
};

template <class P>
__global__ void __launch_bounds__(512)
logits_bf16_kernel(logits_args a) {
  constexpr int IB = P::kIB, JB = P::kJB, L = P::L;
  extern __shared__ __align__(16) unsigned char lds[];
  int wt, xt;
  if (!gemm_tile_of(a.n_wtiles, a.n_tok_tiles, a.group, blockIdx.x, wt, xt)) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, lg = lane >> 4, grp = wave >> 2, wn = wave & 3;
  f32x4 acc[IB][JB];
  P::mainloop(
      acc, lds, a.K / 64,
      [&](int) -> const char * { return reinterpret_cast<const char *>((const bf16_t *)a.w + (size_t)wt * P::BM * a.K); },
      [&](int r) -> uint32_t {
        int q, f;
        P::row_of(r % (16 * IB), q, f);
        f += (r / (16 * IB)) * (P::BM / 2) + 8 * IB * q;
        return (uint32_t)min(f, a.N - 1 - wt * P::BM) * (uint32_t)a.K * 2u;      // clamp: computed but never stored
      },
      [&](int) -> const char * { return reinterpret_cast<const char *>(a.x); },
      [&](int r) -> uint32_t {
        const int m = min(xt * P::BN + r, a.n_rows - 1);
        return (uint32_t)(a.row_idx ? a.row_idx[m] : m) * (uint32_t)a.K * 2u;
      });
  // a lane holds L consecutive features of half 0 and of half 1 of one row
  const int feat = wt * P::BM + grp * (P::BM / 2) + L * lg;
#pragma unroll
  for (int j = 0; j < JB; ++j) {
    const int tok = xt * P::BN + 16 * (JB * wn + j) + l16;
    float lo[L], hi[L];
    gemm_lane_values<IB, JB>(acc, j, lo, hi);
    if (tok >= a.n_rows) continue;
    float *p = a.out + (size_t)tok * a.ld;
#pragma unroll
    for (int e = 0; e < L; ++e) {
      if (feat + e < a.N) p[feat + e] = lo[e];
      if (feat + 8 * IB + e < a.N) p[feat + 8 * IB + e] = hi[e];
    }
  }
}

// ---------------------------------------------------------------------------------------
// logits, fp32: 64 weight rows x 16 rows a workgroup
// ---------------------------------------------------------------------------------------
__global__ void __launch_bounds__(256)
logits_f32_kernel(logits_args a) {
  constexpr int R = 16, F = 64, BK = 32;
  __shared__ float xs[R][BK + 1], ws[F][BK + 1];
  const int f0 = blockIdx.x * F, m0 = blockIdx.y * R, tid = threadIdx.x, ty = tid >> 4, tx = tid & 15;
  float acc[4] = {0.f, 0.f, 0.f, 0.f};
  for (int k0 = 0; k0 < a.K; k0 += BK) {
    for (int i = tid; i < R * BK; i += 256) {
      const int m = min(m0 + i / BK, a.n_rows - 1);
      xs[i / BK][i % BK] = ((const float *)a.x)[(size_t)(a.row_idx ? a.row_idx[m] : m) * a.K + k0 + i % BK];
    }
    for (int i = tid; i < F * BK; i += 256)
      ws[i / BK][i % BK] = ((const float *)a.w)[(size_t)min(f0 + i / BK, a.N - 1) * a.K + k0 + i % BK];
    __syncthreads();
    for (int c = 0; c < BK; ++c)
#pragma unroll
      for (int f = 0; f < 4; ++f) acc[f] = fmaf(xs[ty][c], ws[tx + 16 * f][c], acc[f]);
    __syncthreads();
  }
  if (m0 + ty >= a.n_rows) return;
#pragma unroll
  for (int f = 0; f < 4; ++f)
    if (f0 + tx + 16 * f < a.N) a.out[(size_t)(m0 + ty) * a.ld + f0 + tx + 16 * f] = acc[f];
}

// ---------------------------------------------------------------------------------------
// log probabilities: every row read once
// ---------------------------------------------------------------------------------------
// A workgroup reads a row, or with few rows a slice of one, in chunks of 32 values a thread.  Sums: every thread keeps the maximum m of
// its own values, z = sum e^(x - m) and t = sum e^(x - m) (x - m) in units of log 2 and rescales them when a chunk brings a larger value
// (t' = f (t + (m - m') z), f = 2^(m - m')).  Alternatives: while it reads, a thread only notes the maximum of each of its chunks.
// Then the n-th largest of a wave's 64 lane maxima is found bit by bit with ballots: at least n values of the row are no smaller, so
// what lies below the largest of the four waves' bounds is out, and only the chunks that reach it are looked at again (some n of
// them, from cache) and their values ranked.  The order has no ties (a value's index is part of it), so rows of equal or masked
// values leave no more than a few hundred candidates either.  Slices of a row are put together by a second kernel in the same way.
struct logprob_args {
  const void *x;
  long long ld;
  int vocab, n_given, n_top;
  const int *tokens;
  float *logprob, *entropy, *top_logprob;
  int *top_idx;
  int slices;                        // of a row; 1: no second kernel
  float4 *part;                      // [n_rows, slices] (m, z, t) of a slice
  unsigned long long *part_top;      // [n_rows, slices, n_top]
};

constexpr int kLpThreads = 256, kLpValues = 32, kLpTop = 64, kLpCands = 1024;
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

struct lp_shared {
  float red[4][4];
  unsigned long long bound[4];
  int count;
  unsigned long long best[4], list[kLpTop], cand[kLpCands];
};

// The n-th largest of a wave's 64 keys, or something below it that no more values reach; 0 if fewer than n lanes have a key.
__device__ __forceinline__ unsigned long long wave_bound(unsigned long long key, int n) {
  const uint32_t hi = (uint32_t)(key >> 32), lo = (uint32_t)key;
  uint32_t b = 0;
#pragma unroll 4
  for (int i = 31; i >= 0; --i) {
    const uint32_t t = b | 1u << i;
    if (__popcll(__ballot(hi >= t)) >= n) b = t;
  }
  const unsigned long long equal = __ballot(hi == b && key != 0);
  const int want = n - __popcll(__ballot(hi > b));             // of the lanes whose value is the n-th largest, those of lowest index
  uint32_t l = 0;
  if (__popcll(equal) > want)
#pragma unroll 4
    for (int i = 31; i >= 0; --i) {
      const uint32_t t = l | 1u << i;
      if (__popcll(__ballot(lo >= t) & equal) >= want) l = t;
    }
  return (unsigned long long)b << 32 | l;
}

// list (the n best so far, sorted, 0: none) becomes the n best of itself and of the values behind all threads' `top` keys (the largest of
// a thread's values).  gather(bound, push) hands push() every key of the thread from `bound` on; below(key): the thread's largest
// key below it.  All keys differ, except for 0, which is none.
template <class Gather, class Below>
__device__ __forceinline__ void top_update(lp_shared &s, int n, unsigned long long top, Gather gather, Below below) {
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const unsigned long long b = wave_bound(top, n);
  if (tid == 0) s.count = n;
  if ((tid & 63) == 0) s.bound[wave] = b;
  if (tid < n) s.cand[tid] = s.list[tid];
  __syncthreads();
  unsigned long long bound = s.list[n - 1] + 1;
#pragma unroll
  for (int w = 0; w < 4; ++w) bound = s.bound[w] > bound ? s.bound[w] : bound;
  if (top >= bound)
    gather(bound, [&](unsigned long long k) {
      const int at = atomicAdd(&s.count, 1);
      if (at < kLpCands) s.cand[at] = k;
    });
  __syncthreads();
  const int count = s.count;
  if (count <= kLpCands) {                                     // every candidate's place is the number of larger ones
    for (int c = tid; c < count; c += kLpThreads) {
      const unsigned long long k = s.cand[c];
      int rank = 0;
#pragma unroll 8
      for (int o = 0; o < count; ++o) rank += s.cand[o] > k;
      if (rank < n && k) s.list[rank] = k;
    }
    __syncthreads();
    return;
  }
  // more than there is room for (NaN everywhere, or one thread's values far above all others'): one after the other, the largest
  // below the last one taken (s.cand[0 .. n - 1]: the list before)
  unsigned long long prev = ~0ull;
  int old = 0;
  for (int j = 0; j < n; ++j) {
    unsigned long long k = below(prev);
    for (int o = 32; o; o >>= 1) { const unsigned long long x = __shfl_xor(k, o); k = x > k ? x : k; }
    if ((tid & 63) == 0) s.best[wave] = k;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 4; ++w) k = s.best[w] > k ? s.best[w] : k;
    const unsigned long long from_list = s.cand[old];
    if (from_list > k) { k = from_list; ++old; } else prev = k;
    if (tid == 0) s.list[j] = k;
    __syncthreads();
  }
}

// What a row's m, z, t and best values give.
template <typename T>
__device__ __forceinline__ void logprobs_write(const logprob_args &a, const lp_shared &s, int row, const T *x, float m, float z, float t) {
  const float log_z = logf(z);
  const bool none = m == -INFINITY;
  if (threadIdx.x == 0 && a.entropy) a.entropy[row] = none ? __uint_as_float(0x7fc00000u) : log_z - kLn2 * t / z;
  for (int j = threadIdx.x; j < a.n_given; j += kLpThreads) {
    const int tok = a.tokens[(size_t)row * a.n_given + j];
    a.logprob[(size_t)row * a.n_given + j] = tok < 0 || tok >= a.vocab ? -INFINITY : ((float)x[tok] - m) - log_z;
  }
  for (int j = threadIdx.x; j < a.n_top; j += kLpThreads) {
    const unsigned long long k = s.list[j];
    a.top_idx[(size_t)row * a.n_top + j] = (int)~(uint32_t)k;
    a.top_logprob[(size_t)row * a.n_top + j] = (top_value(k) - m) - log_z;
  }
}

// (from - to) in units of log 2: what moves a sum from reference `from` to the larger `to`.  Bounded, so that a sum whose weight
// is 0 (masks of the type's lowest value: the difference overflows) leaves no NaN.
__device__ __forceinline__ float lp_shift(float from, float to) { return from == -INFINITY ? 0.f : fmaxf((from - to) * kLog2e, -1e30f); }

// (m, z, t) of a workgroup's threads, or of pieces, as one
__device__ __forceinline__ void lp_join(float &m, float &z, float &t, float m1, float z1, float t1) {
  const float top = fmaxf(m, m1);
  const float d = lp_shift(m, top), d1 = lp_shift(m1, top);
  const float f = __builtin_amdgcn_exp2f(d), f1 = __builtin_amdgcn_exp2f(d1);
  t = f * fmaf(d, z, t) + f1 * fmaf(d1, z1, t1);
  z = f * z + f1 * z1;
  m = top;
}
__device__ __forceinline__ void lp_join_workgroup(lp_shared &s, float &m, float &z, float &t) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    // both sides of a pair form the same numbers: the lower lane's first
    const float m1 = __shfl_xor(m, o), z1 = __shfl_xor(z, o), t1 = __shfl_xor(t, o);
    if (threadIdx.x & o) { float a = m1, b = z1, c = t1; lp_join(a, b, c, m, z, t); m = a; z = b; t = c; }
    else lp_join(m, z, t, m1, z1, t1);
  }
  const int wave = threadIdx.x >> 6;
  __syncthreads();
  if ((threadIdx.x & 63) == 0) { s.red[wave][0] = m; s.red[wave][1] = z; s.red[wave][2] = t; }
  __syncthreads();
  m = s.red[0][0]; z = s.red[0][1]; t = s.red[0][2];
  for (int w = 1; w < 4; ++w) lp_join(m, z, t, s.red[w][0], s.red[w][1], s.red[w][2]);
}

// ONE: no slice has more than one chunk, whose values then stay in registers.
template <typename T, bool ONE>
__global__ void __launch_bounds__(kLpThreads)
logprobs_kernel(logprob_args a) {
  constexpr int V = a3_elem<T>::kVec, U = kLpValues / V, kChunk = U * kLpThreads;
  typedef T vec_t __attribute__((ext_vector_type(V)));
  __shared__ lp_shared s;
  __shared__ float noted[ONE ? 1 : kLpChunks][kLpThreads];
  const int row = blockIdx.x / a.slices, slice = blockIdx.x - row * a.slices, tid = threadIdx.x;
  const T *x = (const T *)a.x + (size_t)row * a.ld;
  // the row as aligned vectors: vector v holds elements v V - skew .. (skew: how far the row starts behind a 16-byte border)
  const int skew = (int)(((uintptr_t)x & 15) / sizeof(T)), n_vec = (int)(((long long)a.vocab + skew + V - 1) / V);
  const int v0 = (int)((long long)n_vec * slice / a.slices), v1 = (int)((long long)n_vec * (slice + 1) / a.slices);
  for (int j = tid; j < a.n_top; j += kLpThreads) s.list[j] = 0;
  // the thread's 32 values of the chunk at vector c, -inf where the row has none; their elements
  auto load = [&](int c, vec_t (&raw)[U]) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int v = c + u * kLpThreads + tid, e = v * V - skew;
      if (v < v1 && e >= 0 && e + V <= a.vocab) raw[u] = *reinterpret_cast<const vec_t *>(x + e);
      else
#pragma unroll
        for (int i = 0; i < V; ++i) raw[u][i] = v < v1 && e + i >= 0 && e + i < a.vocab ? x[e + i] : (T)-INFINITY;
    }
  };
  auto index = [&](int c, int i) { return (c + i / V * kLpThreads + tid) * V - skew + i % V; };
  auto key = [&](int c, int i, float y) {
    const bool inside = c + i / V * kLpThreads + tid < v1 && (unsigned)index(c, i) < (unsigned)a.vocab;
    return inside ? top_key(y, index(c, i)) : 0ull;
  };
  auto largest = [&](const vec_t (&raw)[U]) {
    float top = (float)raw[0][0];
#pragma unroll
    for (int i = 1; i < kLpValues; ++i) top = fmaxf(top, (float)raw[i / V][i % V]);
    return top;
  };
  // largest key below prev, of the 32 values
  auto largest_below = [&](int c, const vec_t (&raw)[U], unsigned long long prev) {
    unsigned long long b = 0;
#pragma unroll
    for (int i = 0; i < kLpValues; ++i) {
      const unsigned long long k = key(c, i, (float)raw[i / V][i % V]);
      if (k < prev && k > b) b = k;
    }
    return b;
  };
  float m = -INFINITY, z = 0.f, t = 0.f;
  vec_t raw[U];
  load(v0, raw);
  for (int g0 = v0; g0 < v1; g0 += kLpChunks * kChunk) {       // chunks between two choices of alternatives
    const int g1 = min(v1, g0 + kLpChunks * kChunk);
    float best = -INFINITY;
    int best_at = g0;
    for (int c = g0; c < g1; c += kChunk) {
      float y[kLpValues];
#pragma unroll
      for (int i = 0; i < kLpValues; ++i) y[i] = (float)raw[i / V][i % V];
      if (!ONE && c + kChunk < v1) load(c + kChunk, raw);      // on its way while this chunk is worked on
      float top = y[0];
#pragma unroll
      for (int i = 1; i < kLpValues; ++i) top = fmaxf(top, y[i]);
      if (!ONE) noted[(c - g0) / kChunk][tid] = top;
      if (top > best) { best = top; best_at = c; }
      if (top > m) {
        const float d = lp_shift(m, top), f = __builtin_amdgcn_exp2f(d);
        t = f * fmaf(d, z, t);
        z *= f;
        m = top;
      }
      const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
      for (int i = 0; i < kLpValues; ++i) {
        const float d = (y[i] - ref) * kLog2e, e = __builtin_amdgcn_exp2f(d);
        z += e;
        t = fmaf(e, fmaxf(d, -1e30f), t);                      // -inf: e = 0 (NaN stays in z)
      }
    }
    if (a.n_top == 0) continue;
    __syncthreads();                                           // (list of the last choice, or cleared)
    if constexpr (ONE) {
      top_update(s, a.n_top, largest_below(v0, raw, ~0ull),
                 [&](unsigned long long bound, auto push) {
#pragma unroll
                   for (int i = 0; i < kLpValues; ++i) {
                     const unsigned long long k = key(v0, i, (float)raw[i / V][i % V]);
                     if (k >= bound) push(k);
                   }
                 },
                 [&](unsigned long long prev) { return largest_below(v0, raw, prev); });
    } else {
      vec_t again[U];
      load(best_at, again);
      top_update(s, a.n_top, largest_below(best_at, again, ~0ull),
                 [&](unsigned long long bound, auto push) {
                   const float value = top_value(bound);       // NaN: every chunk has to be looked at
                   for (int c = g0; c < g1; c += kChunk) {
                     if (noted[(c - g0) / kChunk][tid] < value) continue;
                     load(c, again);
#pragma unroll
                     for (int i = 0; i < kLpValues; ++i) {
                       const float y = (float)again[i / V][i % V];
                       if (y < value) continue;
                       const unsigned long long k = key(c, i, y);
                       if (k >= bound) push(k);
                     }
                   }
                 },
                 [&](unsigned long long prev) {
                   unsigned long long b = 0;
                   for (int c = g0; c < g1; c += kChunk) {
                     load(c, again);
                     const unsigned long long k = largest_below(c, again, prev);
                     b = k > b ? k : b;
                   }
                   return b;
                 });
    }
  }
  lp_join_workgroup(s, m, z, t);
  if (a.slices == 1) {
    logprobs_write(a, s, row, x, m, z, t);
    return;
  }
  if (tid == 0) a.part[blockIdx.x] = make_float4(m, z, t, 0.f);
  for (int j = tid; j < a.n_top; j += kLpThreads) a.part_top[(size_t)blockIdx.x * a.n_top + j] = s.list[j];
}

template <typename T>
__global__ void __launch_bounds__(kLpThreads)
logprobs_join_kernel(logprob_args a) {
  __shared__ lp_shared s;
  const int row = blockIdx.x, tid = threadIdx.x;
  float m = -INFINITY, z = 0.f, t = 0.f;
  if (tid < a.slices) {
    const float4 p = a.part[(size_t)row * a.slices + tid];
    m = p.x; z = p.y; t = p.z;
  }
  const unsigned long long *keys = a.part_top + (size_t)row * a.slices * a.n_top;
  constexpr int N = 16;                                        // kLpSlices * kLpTop / kLpThreads
  unsigned long long k[N], top = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) k[i] = i * kLpThreads + tid < a.slices * a.n_top ? keys[i * kLpThreads + tid] : 0ull;
  for (int j = tid; j < a.n_top; j += kLpThreads) s.list[j] = 0;
  lp_join_workgroup(s, m, z, t);
#pragma unroll
  for (int i = 0; i < N; ++i) top = k[i] > top ? k[i] : top;
  if (a.n_top)
    top_update(s, a.n_top, top,
               [&](unsigned long long bound, auto push) {
#pragma unroll
                 for (int i = 0; i < N; ++i)
                   if (k[i] >= bound) push(k[i]);
               },
               [&](unsigned long long prev) {
                 unsigned long long b = 0;
#pragma unroll
                 for (int i = 0; i < N; ++i)
                   if (k[i] < prev && k[i] > b) b = k[i];
                 return b;
               });
  logprobs_write(a, s, row, (const T *)a.x + (size_t)row * a.ld, m, z, t);
}

// Slices of a row: few rows are cut so that some thousand workgroups share the reading, into pieces of no less than two vectors a thread.
constexpr int kLpSlices = 64;
static_assert(kLpSlices * kLpTop == 16 * kLpThreads, "logprobs_join_kernel's keys");
int logprob_slices(int n_rows, int vocab, int elem) {
  const int by_rows = (1024 + n_rows - 1) / n_rows, by_size = (int)((long long)vocab * elem / (16 * 2 * kLpThreads));
  const int n = by_rows < by_size ? by_rows : by_size;
  return n < 1 ? 1 : n > kLpSlices ? kLpSlices : n;
}
size_t logprob_ws(int n_rows, int slices, int n_top, void *base, logprob_args *a) {
  if (slices == 1) return 256;
  a3_ws_cursor cur(base, 0);
  float4 *part = (float4 *)cur.take((size_t)n_rows * slices * sizeof(float4));
  unsigned long long *top = (unsigned long long *)cur.take((size_t)n_rows * slices * n_top * sizeof(unsigned long long));
  if (a) { a->part = part; a->part_top = top; }
  return cur.off;
}

}  // namespace

extern "C" a3_status a3_lm_head(const a3_layout *L, const void *hidden, const int *row_idx, int n_rows, const void *w, int vocab,
                                float *logits, long long ld, void *stream) {
  a3_status s = a3_check_layout(L, "a3_lm_head", false);
  if (s != A3_OK) return s;
  A3_REQUIRE(n_rows >= 0 && (row_idx || n_rows <= L->total_tokens), A3_ERR_INVALID_ARG, "a3_lm_head: n_rows %d outside [0, %d]", n_rows,
             L->total_tokens);
  A3_REQUIRE(vocab > 0 && ld >= vocab, A3_ERR_INVALID_ARG, "a3_lm_head: vocab %d, ld %lld", vocab, ld);
  if (n_rows == 0) return A3_OK;
  A3_REQUIRE(hidden && w && logits, A3_ERR_INVALID_ARG, "a3_lm_head: NULL tensor");
  A3_REQUIRE(a3_aligned16(hidden) && a3_aligned16(w) && ((uintptr_t)logits & 3) == 0, A3_ERR_INVALID_ARG,
             "a3_lm_head: tensors must be 16-byte aligned (logits 4)");
  logits_args a{hidden, row_idx, n_rows, w, logits, ld, L->hidden, vocab, 0, 0, 0};
  hipStream_t st = (hipStream_t)stream;
  if (L->dtype == A3_BF16) {
    A3_REQUIRE(L->hidden % 64 == 0, A3_ERR_UNSUPPORTED, "a3_lm_head: bf16 needs hidden %% 64 == 0, got %d", L->hidden);
    A3_REQUIRE((long long)L->total_tokens * L->hidden * 2 < (1LL << 32), A3_ERR_UNSUPPORTED, "a3_lm_head: hidden tensor larger than 4 GiB");
    return gemm_with_tile(gemm_choose_tile(vocab, n_rows, L->hidden / 64, 1).tile, [&](auto t) -> a3_status {
      using P = decltype(t);
      auto kern = logits_bf16_kernel<P>;
      static a3_once_per_device lds_once;
      if (a3_once(lds_once, [&]() { return hipFuncSetAttribute((const void *)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)P::kLdsBytes); }) != hipSuccess)
        return a3_fail(A3_ERR_HIP, "a3_lm_head: cannot raise the dynamic LDS limit");
      logits_args b = a;
      b.n_wtiles = (vocab + P::BM - 1) / P::BM;
      b.n_tok_tiles = (n_rows + P::BN - 1) / P::BN;
      b.group = gemm_tile_group(b.n_wtiles, b.n_tok_tiles);
      hipLaunchKernelGGL(kern, dim3(gemm_tile_grid(b.n_wtiles, b.n_tok_tiles)), dim3(512), P::kLdsBytes, st, b);
      A3_CHECK_LAUNCH("a3_lm_head");
      return A3_OK;
    });
  }
  A3_REQUIRE((n_rows + 15) / 16 <= 65535, A3_ERR_UNSUPPORTED, "a3_lm_head: too many rows");
  hipLaunchKernelGGL(logits_f32_kernel, dim3((vocab + 63) / 64, (n_rows + 15) / 16), dim3(256), 0, st, a);
  A3_CHECK_LAUNCH("a3_lm_head");
  return A3_OK;
}

extern "C" size_t a3_token_logprobs_ws_bytes(int n_rows, int vocab, int n_top) {
  if (n_rows < 0 || vocab <= 0 || n_top < 0) return 0;
  return n_rows == 0 ? 256 : logprob_ws(n_rows, logprob_slices(n_rows, vocab, 4), n_top, nullptr, nullptr);   // (bf16: no more slices)
}

extern "C" a3_status a3_token_logprobs(int dtype, const void *logits, int n_rows, int vocab, long long ld, const int *tokens, int n_given,
                                       int n_top, float *logprob, float *entropy, int *top_idx, float *top_logprob, void *ws,
                                       size_t ws_bytes, void *stream) {
  A3_REQUIRE(dtype == A3_F32 || dtype == A3_BF16, A3_ERR_INVALID_ARG, "a3_token_logprobs: unknown dtype %d", dtype);
  A3_REQUIRE(n_rows >= 0 && vocab > 0 && ld >= vocab, A3_ERR_INVALID_ARG, "a3_token_logprobs: n_rows %d, vocab %d, ld %lld", n_rows, vocab, ld);
  A3_REQUIRE(vocab < (1 << 30), A3_ERR_UNSUPPORTED, "a3_token_logprobs: vocab %d (2^30 and more)", vocab);
  A3_REQUIRE(n_given >= 0 && n_top >= 0 && n_top <= vocab, A3_ERR_INVALID_ARG, "a3_token_logprobs: n_given %d, n_top %d of %d", n_given,
             n_top, vocab);
  A3_REQUIRE(n_top <= 64, A3_ERR_UNSUPPORTED, "a3_token_logprobs: n_top %d (64 at most)", n_top);
  if (n_rows == 0) return A3_OK;
  A3_REQUIRE(logits && (n_given == 0 || (tokens && logprob)) && (n_top == 0 || (top_idx && top_logprob)), A3_ERR_INVALID_ARG,
             "a3_token_logprobs: NULL tensor");
  A3_REQUIRE(a3_aligned16(logits), A3_ERR_INVALID_ARG, "a3_token_logprobs: logits must be 16-byte aligned");
  const size_t need = a3_token_logprobs_ws_bytes(n_rows, vocab, n_top);
  A3_REQUIRE(ws && a3_aligned16(ws) && ws_bytes >= need, A3_ERR_WORKSPACE, "a3_token_logprobs: workspace %zu bytes (16-byte aligned), need %zu",
             ws ? ws_bytes : 0, need);
  logprob_args a{logits, ld, vocab, n_given, n_top, tokens, logprob, entropy, top_logprob, top_idx,
                 logprob_slices(n_rows, vocab, dtype == A3_BF16 ? 2 : 4), nullptr, nullptr};
  A3_REQUIRE((long long)n_rows * a.slices < (1LL << 31), A3_ERR_UNSUPPORTED, "a3_token_logprobs: too many rows");
  logprob_ws(n_rows, a.slices, n_top, ws, &a);
  const int elem = dtype == A3_BF16 ? 2 : 4;
  const bool one = (long long)(vocab + 2LL * a.slices * (16 / elem)) * elem <= (long long)a.slices * kLpThreads * kLpValues * elem;
  auto launch = [&](auto e) {
    typedef decltype(e) T;
    auto kern = one ? logprobs_kernel<T, true> : logprobs_kernel<T, false>;
    hipLaunchKernelGGL(kern, dim3((unsigned)(n_rows * a.slices)), dim3(kLpThreads), 0, (hipStream_t)stream, a);
    if (a.slices > 1) hipLaunchKernelGGL(logprobs_join_kernel<T>, dim3((unsigned)n_rows), dim3(kLpThreads), 0, (hipStream_t)stream, a);
  };
  if (dtype == A3_BF16) launch(bf16_t{});
  else launch(0.f);
  A3_CHECK_LAUNCH("a3_token_logprobs");
  return A3_OK;
}
