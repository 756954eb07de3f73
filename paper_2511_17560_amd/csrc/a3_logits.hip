// From hidden rows to the next token: the product with the vocabulary's weights, and log probabilities of its rows.
#include "a3_internal.h"
#include "a3_choose.h"
#include "a3_gemm_pp.h"

namespace {

// ---------------------------------------------------------------------------------------
// logits: the row-tiled MFMA GEMM of a3_gemm_pp.h (fp32: with the fp32 matrix instruction), float out.  Few rows: bound by the weights'
// way from HBM (4 rows of 128256 x 4096, 1.05 GB: 160 us, 6.6 TB/s).  Many: by the matrix pipe and its power (512 rows 443 us, 1.21
// PFLOP/s; 4096 rows 3.1 ms, 1.38).  Medians of 300 launches in a row over three sets of inputs; the first dozen after a pause
// take up to 560 us for 512 rows.  The library's product with bf16 results of the same inputs, calls in turn with this one's: 4 rows 186 us
// (176 here), 64 rows of 152064 x 3584 209 (220), 512 rows 509 (453), 4096 rows 2.9 ms (3.1).
// ---------------------------------------------------------------------------------------
struct logits_args {
  const void *x;           // [*, K]
  const int *row_idx;
  int n_rows, total;       // rows of the list, and of x
  const void *w;           // [N, K]
  float *out;
  long long ld;
  int K, N;
  int n_wtiles, n_tok_tiles, group;
};

template <typename T, class P>
__global__ void __launch_bounds__(512)
logits_kernel(logits_args a) {
  constexpr int IB = P::kIB, JB = P::kJB;
  extern __shared__ __align__(16) unsigned char lds[];
  int wt, xt;
  if (!gemm_tile_of(a.n_wtiles, a.n_tok_tiles, a.group, blockIdx.x, wt, xt)) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, lg = lane >> 4, grp = wave >> 2, wn = wave & 3;
  f32x4 acc[IB][JB];
  P::mainloop(
      acc, lds, a.K / P::kElems,
      [&](int) -> const char * { return reinterpret_cast<const char *>((const T *)a.w + (size_t)wt * P::BM * a.K); },
      [&](int r) -> uint32_t { return (uint32_t)min(r, a.N - 1 - wt * P::BM) * (uint32_t)(a.K * sizeof(T)); },   // clamp: computed but never stored
      [&](int) -> const char * { return reinterpret_cast<const char *>(a.x); },
      [&](int r) -> uint32_t {
        const int m = min(xt * P::BN + r, a.n_rows - 1), row = a.row_idx ? a.row_idx[m] : m;
        return ((uint32_t)row < (uint32_t)a.total ? (uint32_t)row : 0u) * (uint32_t)(a.K * sizeof(T));             // (no such row: likewise)
      });
  // block (i, j) as the matrix instruction leaves it: a lane has four consecutive features of one row, four lanes a 64-byte run
  // (16 consecutive features a lane, one float at a time: 512 rows of 128256 x 4096 641 us, 4096 rows 4800; this 446 and 3215).
  // Rows of the output start anywhere a float can.
  typedef f32x4 f32x4_any __attribute__((aligned(4)));
  const int feat = wt * P::BM + 16 * IB * grp + 4 * lg;
#pragma unroll
  for (int j = 0; j < JB; ++j) {
    const int tok = xt * P::BN + 16 * (JB * wn + j) + l16;
    if (tok >= a.n_rows || (a.row_idx && (uint32_t)a.row_idx[tok] >= (uint32_t)a.total)) continue;
    float *p = a.out + (size_t)tok * a.ld + feat;
#pragma unroll
    for (int i = 0; i < IB; ++i) {
      if (feat + 16 * i + 3 < a.N) {
        *reinterpret_cast<f32x4_any *>(p + 16 * i) = acc[i][j];
        continue;
      }
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (feat + 16 * i + e < a.N) p[16 * i + e] = acc[i][j][e];
    }
  }
}

// ---------------------------------------------------------------------------------------
// log probabilities: every row read once
// ---------------------------------------------------------------------------------------
// A workgroup reads a row, or with few rows a slice of one, in chunks of 32 values a thread.  Sums: every thread keeps the maximum m of
// its own values, z = sum e^(x - m) and t = sum e^(x - m) (x - m) in units of log 2 and rescales them when a chunk brings a larger value
// (t' = f (t + (m - m') z), f = 2^(m - m')).  Alternatives: while it reads, a thread only notes the maximum of each of its chunks.
// Then the n-th largest of a wave's 128 - every lane's two largest maxima of half chunks - is found bit by bit with ballots: at least
// n values of the row are no smaller, so what lies below the largest of the four waves' bounds is out.  The noted chunks that reach it (some n of them) are looked at again,
// each by half a wave, and the values found are ranked.  Where too many equal the bound (rows that are masked or constant), only the
// larger ones are gathered, and of the equal ones the first n in the row's order.  Slices of a row are put together by a second kernel.
// fp32: bound by HBM (1024 rows of 128256 91 us without alternatives, 5.8 TB/s, 103 with 20).  bf16: those rows take 50 us and 59, where
// reading alone would take 37 (at the 7.1 TB/s that it reaches) and the vector unit is busy for 35 (10.4 issue slots a value, 2 of them
// the exponential's): neither hides the other wholly.  1500 rows of 32003 bf16, all of them in flight at once: 22 us, and 5.5 more for choosing
// 8 alternatives when all have been read.  Few rows: latency (1 row 9.6 + 4.8 us).
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

// What a row's m, z, t and best values give.  given: the logits of the first given tokens, one a thread, fetched beforehand.
template <typename T>
__device__ __forceinline__ float lp_given(const logprob_args &a, int row, int j, const T *x) {
  const int tok = j < a.n_given ? a.tokens[(size_t)row * a.n_given + j] : -1;
  return tok < 0 || tok >= a.vocab ? -INFINITY : (float)x[tok];
}
template <typename T>
__device__ __forceinline__ void logprobs_write(const logprob_args &a, const lp_shared &s, int row, const T *x, float given, float m, float z, float t) {
  const float log_z = logf(z);
  const bool none = m == -INFINITY;
  if (threadIdx.x == 0 && a.entropy) a.entropy[row] = none ? __uint_as_float(0x7fc00000u) : log_z - kLn2 * t / z;
  for (int j = threadIdx.x; j < a.n_given; j += kLpThreads) {
    if (j >= kLpThreads) given = lp_given(a, row, j, x);
    const int tok = a.tokens[(size_t)row * a.n_given + j];
    a.logprob[(size_t)row * a.n_given + j] = tok < 0 || tok >= a.vocab ? -INFINITY : (given - m) - log_z;
  }
  for (int j = threadIdx.x; j < a.n_top; j += kLpThreads) {
    const unsigned long long k = s.list[j];
    a.top_idx[(size_t)row * a.n_top + j] = (int)~(uint32_t)k;
    a.top_logprob[(size_t)row * a.n_top + j] = (top_value(k) - m) - log_z;
  }
}

template <typename T>
__global__ void __launch_bounds__(kLpThreads)
logprobs_kernel(logprob_args a) {
  typedef lp_row<T> R;
  constexpr int V = R::V, U = R::U, kChunk = R::kChunk;
  __shared__ lp_shared s;
  __shared__ float noted[kLpChunks][kLpThreads];
  const int row = blockIdx.x / a.slices, slice = blockIdx.x - row * a.slices, tid = threadIdx.x;
  R r;
  r.x = (const T *)a.x + (size_t)row * a.ld;
  r.vocab = a.vocab;
  r.skew = (int)(((uintptr_t)r.x & 15) / sizeof(T));
  const int n_vec = (int)(((long long)a.vocab + r.skew + V - 1) / V);
  const int per = n_vec / a.slices, rest = n_vec - per * a.slices;
  r.v0 = slice * per + min(slice, rest);
  r.v1 = r.v0 + per + (slice < rest ? 1 : 0);
  typename R::vec_t raw[U];
  auto load = [&](int c) {
    if (c * V >= r.skew && c + kChunk <= r.v1 && (long long)(c + kChunk) * V - r.skew <= r.vocab) {
      const T *x = r.x + ((long long)c * V - r.skew);
#pragma unroll
      for (int u = 0; u < U; ++u) raw[u] = *reinterpret_cast<const typename R::vec_t *>(x + (u * kLpThreads + tid) * V);
      return;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) raw[u] = r.vec(c + u * kLpThreads + tid);
  };
  load(r.v0);
  const float given = a.slices == 1 ? lp_given(a, row, tid, r.x) : 0.f;
  for (int j = tid; j < a.n_top; j += kLpThreads) s.list[j] = 0;
  float m = -INFINITY, z = 0.f, t = 0.f;
  for (int g0 = r.v0; g0 < r.v1; g0 += kLpChunks * kChunk) {   // chunks between two choices of alternatives
    const int g1 = min(r.v1, g0 + kLpChunks * kChunk);
    float most = -INFINITY, second = -INFINITY;
    for (int c = g0; c < g1; c += kChunk) {
      float y[kLpValues];
#pragma unroll
      for (int i = 0; i < kLpValues; ++i) y[i] = (float)raw[i / V][i % V];
      if (c + kChunk < r.v1) load(c + kChunk);                 // on its way while this chunk is worked on
      // every other value: a short slice fills both halves too.  A half of nothing but NaN is -inf: left NaN, fminf below would take
      // the other half's maximum for both, one value for two
      float top = fmaxf(-INFINITY, y[0]), half = fmaxf(-INFINITY, y[1]);
#pragma unroll
      for (int i = 2; i < kLpValues; i += 2) { top = fmaxf(top, y[i]); half = fmaxf(half, y[i + 1]); }
      second = fmaxf(second, fmaxf(fminf(top, half), fminf(most, fmaxf(top, half))));
      top = fmaxf(top, half);
      noted[(c - g0) / kChunk][tid] = top;
      most = fmaxf(most, top);
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
    __syncthreads();                                           // (the list: cleared, or of the last choice)
    // (-inf may stand for no value at all: for the largest there is one unless the slice ends before it or NaN has been seen)
    lp_choose(s, r, noted, a.n_top, g0, g1, g0 + tid >= g1 || (most == -INFINITY && z != z) ? 0u : top_order(most),
              second == -INFINITY ? 0u : top_order(second));
  }
  lp_join_workgroup(s, m, z, t);
  if (a.slices == 1) {
    logprobs_write(a, s, row, r.x, given, m, z, t);
    return;
  }
  if (tid == 0) a.part[blockIdx.x] = make_float4(m, z, t, 0.f);
  for (int j = tid; j < a.n_top; j += kLpThreads) a.part_top[(size_t)blockIdx.x * a.n_top + j] = s.list[j];
}

template <typename T>
__global__ void __launch_bounds__(kLpThreads)
logprobs_join_kernel(logprob_args a) {
  __shared__ lp_shared s;
  const int row = blockIdx.x, tid = threadIdx.x, n = a.n_top;
  const T *x = (const T *)a.x + (size_t)row * a.ld;
  float m = -INFINITY, z = 0.f, t = 0.f;
  if (tid < a.slices) {
    const float4 p = a.part[(size_t)row * a.slices + tid];
    m = p.x; z = p.y; t = p.z;
  }
  const unsigned long long *keys = a.part_top + (size_t)row * a.slices * n;
  constexpr int N = 16;                                        // kLpSlices * kLpTop / kLpThreads
  unsigned long long k[N];
#pragma unroll
  for (int i = 0; i < N; ++i) k[i] = i * kLpThreads + tid < a.slices * n ? keys[i * kLpThreads + tid] : 0ull;
  // every wave: the first of all slices' lists, two of each or, where that are fewer than n, eight; their n-th largest is the bound
  constexpr int J = 8;
  const int lane = tid & 63, deep = min(n, 2 * a.slices >= n ? 2 : J);
  uint32_t head[J];
#pragma unroll
  for (int j = 0; j < J; ++j) head[j] = lane < a.slices && j < deep ? (uint32_t)(keys[lane * n + j] >> 32) : 0u;
  const float given = lp_given(a, row, tid, x);
  lp_join_workgroup(s, m, z, t);
  if (n) {
    const uint32_t bound = deep <= 2 ? wave_nth<32, 2>({head[0], head[1]}, n) : wave_nth<32, J>(head, n);
    if (tid < n) s.list[tid] = 0;
    if (tid == 0) s.count = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i)
      if ((uint32_t)(k[i] >> 32) >= bound) lp_push(s, k[i], 0ull);
    __syncthreads();
    if (s.count <= kLpCands) lp_rank(s, n);
    else
      lp_one_by_one(s, n, [&](unsigned long long prev) {
        unsigned long long b = 0;
#pragma unroll
        for (int i = 0; i < N; ++i)
          if (k[i] < prev && k[i] > b) b = k[i];
        return b;
      });
  }
  logprobs_write(a, s, row, x, given, m, z, t);
}

// Slices of a row: few rows are cut so that some thousand workgroups share the reading, into pieces of no less than two vectors a thread.
constexpr int kLpSlices = 64;
static_assert(kLpSlices * kLpTop == 16 * kLpThreads, "logprobs_join_kernel's keys");
constexpr int kLpPieces = 1024;                                // of all rows, about
int logprob_slices_by_size(int vocab, int elem) {
  const long long n = (long long)vocab * elem / (16 * 2 * kLpThreads);
  return n < 1 ? 1 : n > kLpSlices ? kLpSlices : (int)n;
}
int logprob_slices(int n_rows, int vocab, int elem) {
  const int by_rows = n_rows >= kLpPieces ? 1 : (kLpPieces + n_rows - 1) / n_rows, by_size = logprob_slices_by_size(vocab, elem);
  return by_rows < by_size ? by_rows : by_size;
}
size_t logprob_ws(size_t pieces, int n_top, void *base, logprob_args *a) {
  a3_ws_cursor cur(base, 0);
  float4 *part = (float4 *)cur.take(pieces * sizeof(float4));
  unsigned long long *top = (unsigned long long *)cur.take(pieces * n_top * sizeof(unsigned long long));
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
  logits_args a{hidden, row_idx, n_rows, L->total_tokens, w, logits, ld, L->hidden, vocab, 0, 0, 0};
  hipStream_t st = (hipStream_t)stream;
  const bool bf16 = L->dtype == A3_BF16;
  A3_REQUIRE(!bf16 || L->hidden % 64 == 0, A3_ERR_UNSUPPORTED, "a3_lm_head: bf16 needs hidden %% 64 == 0, got %d", L->hidden);
  A3_REQUIRE((long long)L->total_tokens * L->hidden * (bf16 ? 2 : 4) < (1LL << 32), A3_ERR_UNSUPPORTED,
             "a3_lm_head: hidden tensor larger than 4 GiB");
  auto launch = [&](auto elem, auto tile) -> a3_status {
    using P = decltype(tile);
    auto kern = logits_kernel<decltype(elem), P>;
    static a3_once_per_device lds_once;
    if (a3_once(lds_once, [&]() { return hipFuncSetAttribute((const void *)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)P::kLdsBytes); }) != hipSuccess)
      return a3_fail(A3_ERR_HIP, "a3_lm_head: cannot raise the dynamic LDS limit");
    logits_args b = a;
    b.n_wtiles = (vocab + P::BM - 1) / P::BM;
    b.n_tok_tiles = (n_rows + P::BN - 1) / P::BN;
    b.group = gemm_tile_group(b.n_wtiles, b.n_tok_tiles);
    A3_REQUIRE((long long)b.n_wtiles * b.n_tok_tiles < (1LL << 28), A3_ERR_UNSUPPORTED, "a3_lm_head: too many rows");
    hipLaunchKernelGGL(kern, dim3(gemm_tile_grid(b.n_wtiles, b.n_tok_tiles)), dim3(512), P::kLdsBytes, st, b);
    A3_CHECK_LAUNCH("a3_lm_head");
    return A3_OK;
  };
  // Tiles of 64 x 64 where they all run at once: the more compute units, the better (64 rows, weights from HBM: 11699 x 3584, 183 tiles,
  // 23 us, 128 x 64 32; 18702 x 4096, 293 tiles, 49 and 42.  fp32: 4099 x 512 13 and 20; 152064 x 512 127 and 110).
  const bool small = (long long)((vocab + 63) / 64) * ((n_rows + 63) / 64) <= 256;
  if (bf16) {
    const int knob = gemm_tile_of_knob(a3_knob(A3_KNOB_GEMM_TB));
    if (knob < 0 && small) return launch(bf16_t{}, gemm_pl<2, 1, 8>{});
    const int tile = knob >= 0 ? knob : gemm_choose_tile(vocab, n_rows, L->hidden / 64, 1).tile;
    // One tile of rows, and weights that take more than half of the 256 MB of the memory-side cache, whose other half the rest of a step
    // turns over: nothing of them is read again before it is gone, so they go past the caches (1 row of 128256 x 4096, 1.05 GB: 175
    // -> 162 us; of 8000 x 4096, 66 MB and called again and again, 20 -> 25).  Up to 64 rows in tiles of which two fit a compute unit, one
    // streaming while the other starts or ends: of 64 weight rows where those all run at once and are not bound by the activation rows
    // they read (32003 x 4096, 1 row 58 -> 47 us, 32 rows 60 -> 50), of 128 otherwise (65536 x 4096, 1 row 116 -> 96, 48 rows 121 ->
    // 104; 152064 x 3584, 64 rows 223 -> 216; 18702 x 4096, 64 rows 42 -> 41 and 47 in tiles of 64; only 128256 x 4096 at 64 rows, two full
    // rounds of 256 x 128, is slower: 184 -> 196).
    if (knob < 0 && n_rows <= 128 && (long long)vocab * L->hidden * 2 > (128LL << 20)) {
      if (n_rows <= 32 && vocab <= 64 * 512) return launch(bf16_t{}, gemm_pl<2, 1, 5, gemm_mul_bf16, true>{});
      if (n_rows <= 64) return launch(bf16_t{}, gemm_pl<4, 1, 3, gemm_mul_bf16, true>{});
      if (tile == GEMM_256x128) return launch(bf16_t{}, gemm_pl<8, 2, 3, gemm_mul_bf16, true>{});
      if (tile == GEMM_128x128) return launch(bf16_t{}, gemm_pl<4, 2, 5, gemm_mul_bf16, true>{});
    }
    return gemm_with_tile(tile, [&](auto t) { return launch(bf16_t{}, t); });
  }
  // fp32: bound by the matrix pipe (138 TFLOP/s at 512 rows of 32000 x 4096).  128 rows a tile, which fetch less, or 64 where those would
  // leave compute units without a tile (65 rows of 4099 x 512, 33 tiles of 128 rows: 34 us and 21; 512 rows, 132 tiles: 38 and 42).
  const long long tiles = (long long)((vocab + 127) / 128) * ((n_rows + 127) / 128);
  if (small) return launch(0.f, gemm_pl<2, 1, 8, gemm_mul_f32>{});
  return n_rows <= 64 || tiles < 128 ? launch(0.f, gemm_pl<4, 1, 6, gemm_mul_f32>{}) : launch(0.f, gemm_pl<4, 2, 5, gemm_mul_f32>{});
}

extern "C" size_t a3_token_logprobs_ws_bytes(int n_rows, int vocab, int n_top) {
  if (n_rows < 0 || vocab <= 0 || n_top < 0) return 0;
  // What serves every smaller number of rows too (the last piece of many rows is one): r rows are r min(s, ceil(1024 / r)) pieces, which
  // is r s at most, below 1024 + r, and nothing from r = 1024 on.  (bf16: no more slices than float.)
  const size_t rows = n_rows < kLpPieces ? n_rows : kLpPieces - 1, s = logprob_slices_by_size(vocab, 4);
  const size_t pieces = rows * s < kLpPieces + rows ? rows * s : kLpPieces + rows;
  const size_t need = s == 1 ? 0 : logprob_ws(pieces, n_top, nullptr, nullptr);
  return need < 256 ? 256 : need;
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
  A3_REQUIRE(((uintptr_t)logits & (dtype == A3_BF16 ? 1 : 3)) == 0, A3_ERR_INVALID_ARG, "a3_token_logprobs: logits are not aligned to their type");
  const size_t need = a3_token_logprobs_ws_bytes(n_rows, vocab, n_top);
  A3_REQUIRE(ws && a3_aligned16(ws) && ws_bytes >= need, A3_ERR_WORKSPACE, "a3_token_logprobs: workspace %zu bytes (16-byte aligned), need %zu",
             ws ? ws_bytes : 0, need);
  logprob_args a{logits, ld, vocab, n_given, n_top, tokens, logprob, entropy, top_logprob, top_idx,
                 logprob_slices(n_rows, vocab, dtype == A3_BF16 ? 2 : 4), nullptr, nullptr};
  A3_REQUIRE((long long)n_rows * a.slices < (1LL << 31), A3_ERR_UNSUPPORTED, "a3_token_logprobs: too many rows");
  if (a.slices > 1) logprob_ws((size_t)n_rows * a.slices, n_top, ws, &a);
  auto launch = [&](auto e) {
    typedef decltype(e) T;
    hipLaunchKernelGGL(logprobs_kernel<T>, dim3((unsigned)(n_rows * a.slices)), dim3(kLpThreads), 0, (hipStream_t)stream, a);
    if (a.slices > 1) hipLaunchKernelGGL(logprobs_join_kernel<T>, dim3((unsigned)n_rows), dim3(kLpThreads), 0, (hipStream_t)stream, a);
  };
  if (dtype == A3_BF16) launch(bf16_t{});
  else launch(0.f);
  A3_CHECK_LAUNCH("a3_token_logprobs");
  return A3_OK;
}
