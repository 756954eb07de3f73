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
// log probabilities: one workgroup per row, the row read once for each of its maximum, its sums and its alternatives
// ---------------------------------------------------------------------------------------
struct logprob_args {
  const void *x;
  long long ld;
  int vocab, n_given, n_top;
  const int *tokens;
  float *logprob, *entropy, *top_logprob;
  int *top_idx;
};

// Order of the alternatives as one number: larger logit, then lower index; -0 equals 0, NaN below everything.
__device__ __forceinline__ unsigned long long top_key(float x, int v) {
  const unsigned b = __float_as_uint(x + 0.f);
  const unsigned o = x != x ? 0u : (b & 0x80000000u) ? ~b : b | 0x80000000u;
  return ((unsigned long long)o << 32) | (unsigned)~v;
}
__device__ __forceinline__ float top_value(unsigned long long key) {
  const unsigned o = (unsigned)(key >> 32);
  return o == 0u ? __uint_as_float(0x7fc00000u) : __uint_as_float((o & 0x80000000u) ? o & 0x7fffffffu : ~o);
}

template <typename T>
__global__ void __launch_bounds__(256)
logprobs_kernel(logprob_args a) {
  __shared__ float red[4][2];
  __shared__ unsigned long long best[4];
  const int row = blockIdx.x, tid = threadIdx.x, wave = tid >> 6;
  const T *x = (const T *)a.x + (size_t)row * a.ld;
  float m = -INFINITY;
  bool nan = false;
  for (int v = tid; v < a.vocab; v += 256) { const float f = (float)x[v]; m = fmaxf(m, f); nan |= f != f; }
  for (int o = 32; o; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
  if ((tid & 63) == 0) red[wave][0] = m;
  nan = __syncthreads_or(nan);
  m = fmaxf(fmaxf(red[0][0], red[1][0]), fmaxf(red[2][0], red[3][0]));
  __syncthreads();
  float z = 0.f, t = 0.f;
  for (int v = tid; v < a.vocab; v += 256) {
    const float d = (float)x[v] - m, e = expf(d);
    z += e;
    if (e > 0.f) t += e * d;
  }
  for (int o = 32; o; o >>= 1) { z += __shfl_xor(z, o); t += __shfl_xor(t, o); }
  if ((tid & 63) == 0) { red[wave][0] = z; red[wave][1] = t; }
  __syncthreads();
  z = (red[0][0] + red[1][0]) + (red[2][0] + red[3][0]);
  t = (red[0][1] + red[1][1]) + (red[2][1] + red[3][1]);
  if (nan || m == INFINITY || m == -INFINITY) z = __uint_as_float(0x7fc00000u);
  const float log_z = logf(z);
  if (tid == 0 && a.entropy) a.entropy[row] = log_z - t / z;
  for (int j = tid; j < a.n_given; j += 256) {
    const int tok = a.tokens[(size_t)row * a.n_given + j];
    a.logprob[(size_t)row * a.n_given + j] = tok < 0 || tok >= a.vocab ? -INFINITY : ((float)x[tok] - m) - log_z;
  }
  unsigned long long last = ~0ull;
  for (int j = 0; j < a.n_top; ++j) {
    unsigned long long b = 0;
    for (int v = tid; v < a.vocab; v += 256) {
      const unsigned long long k = top_key((float)x[v], v);
      if (k < last && k > b) b = k;
    }
    for (int o = 32; o; o >>= 1) { const unsigned long long k = __shfl_xor(b, o); b = k > b ? k : b; }
    __syncthreads();
    if ((tid & 63) == 0) best[wave] = b;
    __syncthreads();
    for (int w = 0; w < 4; ++w) b = best[w] > b ? best[w] : b;
    if (tid == 0) {
      a.top_idx[(size_t)row * a.n_top + j] = (int)~(unsigned)b;
      a.top_logprob[(size_t)row * a.n_top + j] = (top_value(b) - m) - log_z;
    }
    last = b;
  }
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
  return 256;
}

extern "C" a3_status a3_token_logprobs(int dtype, const void *logits, int n_rows, int vocab, long long ld, const int *tokens, int n_given,
                                       int n_top, float *logprob, float *entropy, int *top_idx, float *top_logprob, void *ws,
                                       size_t ws_bytes, void *stream) {
  A3_REQUIRE(dtype == A3_F32 || dtype == A3_BF16, A3_ERR_INVALID_ARG, "a3_token_logprobs: unknown dtype %d", dtype);
  A3_REQUIRE(n_rows >= 0 && vocab > 0 && ld >= vocab, A3_ERR_INVALID_ARG, "a3_token_logprobs: n_rows %d, vocab %d, ld %lld", n_rows, vocab, ld);
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
  logprob_args a{logits, ld, vocab, n_given, n_top, tokens, logprob, entropy, top_logprob, top_idx};
  if (dtype == A3_BF16) hipLaunchKernelGGL(logprobs_kernel<bf16_t>, dim3(n_rows), dim3(256), 0, (hipStream_t)stream, a);
  else hipLaunchKernelGGL(logprobs_kernel<float>, dim3(n_rows), dim3(256), 0, (hipStream_t)stream, a);
  A3_CHECK_LAUNCH("a3_token_logprobs");
  return A3_OK;
}
