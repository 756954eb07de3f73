// What follows several candidates of a request: the accepted path of a drafted tree, cache rows moved to other slots, and the best
// continuations of beams.
#include "a3_pages.h"

namespace {

constexpr int kMaxRows = 1024, kMaxPath = 64, kMaxSet = 64, kMaxBeams = 64, kMaxBest = 64;

// Order of logits as one number: larger, then lower index; -0 equals 0, NaN below everything.
__device__ __forceinline__ unsigned long long logit_key(float x, int v) {
  const uint32_t b = __float_as_uint(x + 0.f), o = x != x ? 0u : (b & 0x80000000u) ? ~b : b | 0x80000000u;
  return ((unsigned long long)o << 32) | (uint32_t)~v;
}
__device__ __forceinline__ unsigned long long wave_max_key(unsigned long long k) {
  for (int o = 32; o; o >>= 1) { const unsigned long long x = __shfl_xor(k, o); k = x > k ? x : k; }
  return k;
}

// ---------------------------------------------------------------------------------------
// the accepted path
// ---------------------------------------------------------------------------------------
struct accept_args {
  const void *x;
  long long ld;
  int vocab;
  int *picked;
  const int *tokens, *parent, *start, *len;
  int n_groups, n_rows, max_rows, max_path;
  int *count, *path, *next, *src, *dst;
};

template <typename T>
__global__ void __launch_bounds__(256)
pick_kernel(accept_args a) {
  __shared__ unsigned long long best[4];
  const int tid = threadIdx.x;
  const T *x = (const T *)a.x + (size_t)blockIdx.x * a.ld;
  unsigned long long k = 0;
  for (int v = tid; v < a.vocab; v += 256) { const unsigned long long y = logit_key((float)x[v], v); k = y > k ? y : k; }
  k = wave_max_key(k);
  if ((tid & 63) == 0) best[tid >> 6] = k;
  __syncthreads();
  if (tid == 0) {
    for (int w = 1; w < 4; ++w) k = best[w] > k ? best[w] : k;
    a.picked[blockIdx.x] = (int)~(uint32_t)k;
  }
}

// One wave a group: every step looks for the first child of the last row among 64 rows at a time.
__global__ void __launch_bounds__(64)
follow_kernel(accept_args a) {
  const int g = blockIdx.x, lane = threadIdx.x;
  const int first = a.start[g], end = a.start[g + 1];
  const int n = first < 0 || end > a.n_rows || end < first ? 0 : min(end - first, a.max_rows);
  int mine = -1, count = 0, last = 0;                          // lane m keeps path[m]
  while (n > 0) {
    if (lane == count) mine = last;
    if (++count == a.max_path) break;
    const int tok = a.picked[first + last];
    int child = -1;
    for (int c0 = last + 1; c0 < n && child < 0; c0 += 64) {
      const int c = c0 + lane;
      const unsigned long long hit = __ballot(c < n && a.parent[first + min(c, n - 1)] == last && a.tokens[first + min(c, n - 1)] == tok);
      if (hit) child = c0 + __builtin_ctzll(hit);
    }
    if (child < 0) break;
    last = child;
  }
  if (lane == 0) {
    a.count[g] = count;
    a.next[g] = n > 0 ? a.picked[first + last] : -1;
  }
  if (lane < a.max_path) {
    const size_t i = (size_t)g * a.max_path + lane;
    a.path[i] = lane < count ? mine : -1;
    if (a.src) {
      const int L = a.len[g];
      a.src[i] = lane < count ? L + mine : -1;
      a.dst[i] = lane < count ? L + lane : -1;
    }
  }
}

// ---------------------------------------------------------------------------------------
// cache rows moved
// ---------------------------------------------------------------------------------------
constexpr int kLayersAtOnce = 64;
struct move_args {
  pages_args p;                        // (pools: of the layers below)
  char *pools[2 * kLayersAtOnce];      // K and V of every layer
  const int *src_req, *src_slot, *dst_req, *dst_slot, *n_slots;
  int max_slots, set_size, row_bytes, q8;
  size_t head_bytes;
};

__device__ __forceinline__ long long slot_of(const pages_args &p, int req, long long slot) {
  if (req < 0 || req >= p.n_req || slot < 0 || slot >= p.slots) return -1;
  const int page = p.table[(size_t)req * p.max_pages + (slot >> p.page_shift)];
  return page < 0 || page >= p.n_pages ? -1 : ((long long)page << p.page_shift) + (slot & ((1 << p.page_shift) - 1));
}

// A thread has four bytes of one KV head at one o, of all moves of its set: it reads them all, then writes them all.
template <int N>
__global__ void __launch_bounds__(256)
move_kernel(move_args a) {
  const int set = blockIdx.y, words = a.row_bytes / 4 + a.q8, per_o = a.p.Hkv * words;
  char *pool = a.pools[blockIdx.z];
  for (long long u = (long long)blockIdx.x * 256 + threadIdx.x; u < (long long)a.max_slots * per_o; u += (long long)gridDim.x * 256) {
    const int o = (int)(u / per_o), rest = (int)(u - (long long)o * per_o), h = rest / words, c = rest - h * words;
    auto where = [&](long long at) {
      const long long page = at >> a.p.page_shift, in = at & ((1 << a.p.page_shift) - 1);
      return ((size_t)page * a.p.Hkv + h) * a.head_bytes + (4 * c < a.row_bytes ? in * a.row_bytes + 4 * c : ((size_t)a.row_bytes << a.p.page_shift) + 4 * in);
    };
    uint32_t x[N];
    long long to[N];
#pragma unroll
    for (int m = 0; m < N; ++m) {
      to[m] = -1;
      if (m >= a.set_size) continue;
      const int i = set * a.set_size + m;
      if (o >= (a.n_slots ? a.n_slots[i] : 1) || a.src_slot[i] < 0 || a.dst_slot[i] < 0) continue;
      const long long from = slot_of(a.p, a.src_req ? a.src_req[i] : set, (long long)a.src_slot[i] + o);
      to[m] = slot_of(a.p, a.dst_req ? a.dst_req[i] : set, (long long)a.dst_slot[i] + o);
      if (from < 0 || from == to[m]) to[m] = -1;
      if (to[m] >= 0) x[m] = *reinterpret_cast<const uint32_t *>(pool + where(from));
    }
#pragma unroll
    for (int m = 0; m < N; ++m)
      if (to[m] >= 0) *reinterpret_cast<uint32_t *>(pool + where(to[m])) = x[m];
  }
}

// ---------------------------------------------------------------------------------------
// beams
// ---------------------------------------------------------------------------------------
struct beam_args {
  const void *x;
  long long ld;
  int vocab, n_beams, n_best, end;
  const float *score;
  const int *done;
  float *best_score;
  int *best_row, *best_token;
  double *base;            // [rows] score - m - log Z: what a logit is added to; -inf: the beam goes on with nothing
};

template <typename T>
__global__ void __launch_bounds__(256)
beam_row_kernel(beam_args a) {
  __shared__ float top[4];
  __shared__ double sums[4];
  const int row = blockIdx.x, tid = threadIdx.x, wave = tid >> 6;
  const T *x = (const T *)a.x + (size_t)row * a.ld;
  float m = -INFINITY;
  bool nan = false;
  for (int v = tid; v < a.vocab; v += 256) { const float y = (float)x[v]; m = fmaxf(m, y); nan |= y != y; }
  for (int o = 32; o; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
  if ((tid & 63) == 0) top[wave] = m;
  nan = __syncthreads_or(nan);
  m = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
  double z = 0.0;
  for (int v = tid; v < a.vocab; v += 256) z += (double)expf((float)x[v] - m);
  for (int o = 32; o; o >>= 1) z += __shfl_xor(z, o);
  if ((tid & 63) == 0) sums[wave] = z;
  __syncthreads();
  if (tid != 0) return;
  const float s = a.score[row];
  const bool on = !nan && m > -INFINITY && m < INFINITY && s > -INFINITY && s < INFINITY;
  a.base[row] = on ? (double)s - (double)m - log(sums[0] + sums[1] + sums[2] + sums[3]) : -INFINITY;
}

template <typename T>
__global__ void __launch_bounds__(1024)
beam_choose_kernel(beam_args a) {
  __shared__ double value[16];
  __shared__ unsigned long long where[16];
  const int g = blockIdx.x, tid = threadIdx.x, wave = tid >> 6;
  double last = INFINITY;
  unsigned long long at = 0;
  for (int j = 0; j < a.n_best; ++j) {
    double v = -INFINITY;
    unsigned long long w = ~0ull;
    auto offer = [&](double y, unsigned long long i) {
      if (y > -INFINITY && (y < last || (y == last && i > at)) && (y > v || (y == v && i < w))) { v = y; w = i; }
    };
    for (int b = 0; b < a.n_beams; ++b) {
      const int row = g * a.n_beams + b;
      if (a.done && a.done[row]) {
        const float s = a.score[row];
        if (tid == 0 && s < INFINITY) offer((double)s, ((unsigned long long)b << 32) | (uint32_t)a.end);
        continue;
      }
      const double base = a.base[row];
      const T *x = (const T *)a.x + (size_t)row * a.ld;
      if (base > -INFINITY)
        for (int t = tid; t < a.vocab; t += 1024) offer(base + (double)(float)x[t], ((unsigned long long)b << 32) | (uint32_t)t);
    }
    auto join = [&](double y, unsigned long long i) { if (y > v || (y == v && i < w)) { v = y; w = i; } };
    for (int o = 32; o; o >>= 1) join(__shfl_xor(v, o), __shfl_xor(w, o));
    __syncthreads();
    if ((tid & 63) == 0) { value[wave] = v; where[wave] = w; }
    __syncthreads();
    for (int i = 0; i < 16; ++i) join(value[i], where[i]);
    const bool none = !(v > -INFINITY);
    if (tid == 0) {
      a.best_score[(size_t)g * a.n_best + j] = none ? -INFINITY : (float)v;
      a.best_row[(size_t)g * a.n_best + j] = none ? -1 : g * a.n_beams + (int)(w >> 32);
      a.best_token[(size_t)g * a.n_best + j] = none ? -1 : (int)(uint32_t)w;
    }
    if (none) { v = -INFINITY; w = ~0ull; }
    last = v;
    at = w;
  }
}

template <class F>
void with_dtype(int dtype, F f) {
  if (dtype == A3_BF16) f(bf16_t{});
  else f(0.f);
}

}  // namespace

extern "C" size_t a3_tree_accept_ws_bytes(int n_rows, int vocab) {
  if (n_rows < 0 || vocab <= 0) return 0;
  return 256;
}

extern "C" a3_status a3_tree_accept(int dtype, const void *logits, int vocab, long long ld, int *picked, const int *tokens, const int *parent,
                                    int n_groups, const int *group_start, const int *group_len, int n_rows, int max_rows, int max_path,
                                    int *count, int *path, int *next_token, int *src_slot, int *dst_slot, void *ws, size_t ws_bytes,
                                    void *stream) {
  A3_REQUIRE(logits == nullptr || dtype == A3_F32 || dtype == A3_BF16, A3_ERR_INVALID_ARG, "a3_tree_accept: unknown dtype %d", dtype);
  A3_REQUIRE(logits == nullptr || (vocab > 0 && ld >= vocab), A3_ERR_INVALID_ARG, "a3_tree_accept: vocab %d, ld %lld", vocab, ld);
  A3_REQUIRE(logits == nullptr || vocab < (1 << 30), A3_ERR_UNSUPPORTED, "a3_tree_accept: vocab %d (2^30 and more)", vocab);
  A3_REQUIRE(n_groups >= 0 && n_rows >= 0, A3_ERR_INVALID_ARG, "a3_tree_accept: n_groups %d, n_rows %d", n_groups, n_rows);
  A3_REQUIRE(max_rows >= 1 && max_path >= 1, A3_ERR_INVALID_ARG, "a3_tree_accept: max_rows %d, max_path %d", max_rows, max_path);
  A3_REQUIRE(max_rows <= kMaxRows && max_path <= kMaxPath, A3_ERR_UNSUPPORTED, "a3_tree_accept: max_rows %d (%d at most), max_path %d (%d at most)",
             max_rows, kMaxRows, max_path, kMaxPath);
  if (n_groups == 0 && n_rows == 0) return A3_OK;
  A3_REQUIRE(n_rows == 0 || (picked && tokens && parent), A3_ERR_INVALID_ARG, "a3_tree_accept: NULL tensor");
  A3_REQUIRE(n_groups == 0 || (group_start && count && path && next_token), A3_ERR_INVALID_ARG, "a3_tree_accept: NULL tensor");
  A3_REQUIRE((src_slot == nullptr) == (dst_slot == nullptr) && (src_slot == nullptr || group_len), A3_ERR_INVALID_ARG,
             "a3_tree_accept: src_slot, dst_slot and group_len go together");
  A3_REQUIRE(((uintptr_t)logits & (dtype == A3_BF16 ? 1 : 3)) == 0, A3_ERR_INVALID_ARG, "a3_tree_accept: logits are not aligned to their type");
  const size_t need = a3_tree_accept_ws_bytes(n_rows, vocab);
  A3_REQUIRE(logits == nullptr || (ws && a3_aligned16(ws) && ws_bytes >= need), A3_ERR_WORKSPACE,
             "a3_tree_accept: workspace %zu bytes (16-byte aligned), need %zu", ws ? ws_bytes : 0, need);
  accept_args a{logits, ld, vocab, picked, tokens, parent, group_start, group_len, n_groups, n_rows, max_rows, max_path,
                count, path, next_token, src_slot, dst_slot};
  if (logits && n_rows)
    with_dtype(dtype, [&](auto e) { hipLaunchKernelGGL(pick_kernel<decltype(e)>, dim3((unsigned)n_rows), dim3(256), 0, (hipStream_t)stream, a); });
  if (n_groups) hipLaunchKernelGGL(follow_kernel, dim3((unsigned)n_groups), dim3(64), 0, (hipStream_t)stream, a);
  A3_CHECK_LAUNCH("a3_tree_accept");
  return A3_OK;
}

extern "C" a3_status a3_paged_move(const a3_pages *layers, int n_layers, const int *src_req, const int *src_slot, const int *dst_req,
                                   const int *dst_slot, const int *n_slots, int max_slots, int n_sets, int set_size, void *stream) {
  A3_REQUIRE(n_layers >= 0 && n_sets >= 0 && max_slots >= 0, A3_ERR_INVALID_ARG, "a3_paged_move: n_layers %d, n_sets %d, max_slots %d", n_layers,
             n_sets, max_slots);
  A3_REQUIRE(set_size >= 1, A3_ERR_INVALID_ARG, "a3_paged_move: set_size %d", set_size);
  A3_REQUIRE(set_size <= kMaxSet, A3_ERR_UNSUPPORTED, "a3_paged_move: set_size %d (%d at most)", set_size, kMaxSet);
  A3_REQUIRE(n_layers == 0 || layers, A3_ERR_INVALID_ARG, "a3_paged_move: layers is NULL");
  for (int l = 0; l < n_layers; ++l) {
    const a3_pages *P = layers + l;
    const a3_status s = check_pages(P, "a3_paged_move", true);
    if (s != A3_OK) return s;
    A3_REQUIRE(P->format == layers->format && P->dtype == layers->dtype && P->n_q_heads == layers->n_q_heads && P->n_kv_heads == layers->n_kv_heads &&
                   P->head_dim == layers->head_dim && P->page_size == layers->page_size && P->n_pages == layers->n_pages &&
                   P->n_req == layers->n_req && P->max_pages == layers->max_pages && P->page_table == layers->page_table,
               A3_ERR_INVALID_ARG, "a3_paged_move: the pages of layer %d are not laid out as those of layer 0", l);
  }
  if (n_layers == 0 || n_sets == 0 || max_slots == 0) return A3_OK;
  A3_REQUIRE(src_slot && dst_slot, A3_ERR_INVALID_ARG, "a3_paged_move: NULL tensor");
  A3_REQUIRE((src_req && dst_req) || n_sets <= layers->n_req, A3_ERR_INVALID_ARG, "a3_paged_move: %d sets without requests for %d requests", n_sets,
             layers->n_req);
  A3_REQUIRE(n_sets <= 65535, A3_ERR_UNSUPPORTED, "a3_paged_move: %d sets (65535 at most)", n_sets);
  const bool q8 = layers->format == A3_PAGES_Q8;
  move_args a{};
  a.p = args_of(layers);
  a.src_req = src_req; a.src_slot = src_slot; a.dst_req = dst_req; a.dst_slot = dst_slot; a.n_slots = n_slots;
  a.max_slots = n_slots ? max_slots : 1;
  a.set_size = set_size;
  a.row_bytes = layers->head_dim * (q8 ? 1 : elem_bytes(layers));
  a.q8 = q8;
  a.head_bytes = page_head_bytes(layers->format, elem_bytes(layers), layers->page_size, layers->head_dim);
  const long long units = (long long)a.max_slots * layers->n_kv_heads * (a.row_bytes / 4 + a.q8), blocks = (units + 255) / 256;
  for (int l0 = 0; l0 < n_layers; l0 += kLayersAtOnce) {
    const int n = n_layers - l0 < kLayersAtOnce ? n_layers - l0 : kLayersAtOnce;
    for (int l = 0; l < n; ++l) {
      a.pools[2 * l] = (char *)layers[l0 + l].k_pool;
      a.pools[2 * l + 1] = (char *)layers[l0 + l].v_pool;
    }
    const dim3 grid((unsigned)(blocks < 1024 ? blocks : 1024), (unsigned)n_sets, (unsigned)(2 * n));
    if (set_size <= 4) hipLaunchKernelGGL(move_kernel<4>, grid, dim3(256), 0, (hipStream_t)stream, a);
    else if (set_size <= 8) hipLaunchKernelGGL(move_kernel<8>, grid, dim3(256), 0, (hipStream_t)stream, a);
    else if (set_size <= 16) hipLaunchKernelGGL(move_kernel<16>, grid, dim3(256), 0, (hipStream_t)stream, a);
    else hipLaunchKernelGGL(move_kernel<64>, grid, dim3(256), 0, (hipStream_t)stream, a);
    A3_CHECK_LAUNCH("a3_paged_move");
  }
  return A3_OK;
}

extern "C" size_t a3_beam_select_ws_bytes(int n_groups, int n_beams, int vocab, int n_best) {
  if (n_groups < 0 || n_beams < 1 || n_beams > kMaxBeams || vocab <= 0 || n_best < 1 || n_best > kMaxBest) return 0;
  return a3_align_up((size_t)n_groups * n_beams * sizeof(double), 256) + 256;
}

extern "C" a3_status a3_beam_select(int dtype, const void *logits, int n_groups, int n_beams, int vocab, long long ld, const float *score,
                                    const int *done, int end_token, int n_best, float *best_score, int *best_row, int *best_token, void *ws,
                                    size_t ws_bytes, void *stream) {
  A3_REQUIRE(dtype == A3_F32 || dtype == A3_BF16, A3_ERR_INVALID_ARG, "a3_beam_select: unknown dtype %d", dtype);
  A3_REQUIRE(n_groups >= 0 && n_beams >= 1 && n_best >= 1, A3_ERR_INVALID_ARG, "a3_beam_select: n_groups %d, n_beams %d, n_best %d", n_groups, n_beams,
             n_best);
  A3_REQUIRE(n_beams <= kMaxBeams && n_best <= kMaxBest, A3_ERR_UNSUPPORTED, "a3_beam_select: n_beams %d, n_best %d (%d at most)", n_beams, n_best,
             kMaxBest);
  A3_REQUIRE(vocab > 0 && ld >= vocab, A3_ERR_INVALID_ARG, "a3_beam_select: vocab %d, ld %lld", vocab, ld);
  A3_REQUIRE(vocab < (1 << 30) && (long long)n_groups * n_beams < (1LL << 30), A3_ERR_UNSUPPORTED, "a3_beam_select: vocab %d, %d groups", vocab, n_groups);
  A3_REQUIRE(done == nullptr || end_token >= 0, A3_ERR_INVALID_ARG, "a3_beam_select: end_token %d", end_token);
  if (n_groups == 0) return A3_OK;
  A3_REQUIRE(logits && score && best_score && best_row && best_token, A3_ERR_INVALID_ARG, "a3_beam_select: NULL tensor");
  A3_REQUIRE(((uintptr_t)logits & (dtype == A3_BF16 ? 1 : 3)) == 0, A3_ERR_INVALID_ARG, "a3_beam_select: logits are not aligned to their type");
  const size_t need = a3_beam_select_ws_bytes(n_groups, n_beams, vocab, n_best);
  A3_REQUIRE(ws && a3_aligned16(ws) && ws_bytes >= need, A3_ERR_WORKSPACE, "a3_beam_select: workspace %zu bytes (16-byte aligned), need %zu",
             ws ? ws_bytes : 0, need);
  beam_args a{logits, ld, vocab, n_beams, n_best, end_token, score, done, best_score, best_row, best_token, (double *)ws};
  with_dtype(dtype, [&](auto e) {
    hipLaunchKernelGGL(beam_row_kernel<decltype(e)>, dim3((unsigned)(n_groups * n_beams)), dim3(256), 0, (hipStream_t)stream, a);
    hipLaunchKernelGGL(beam_choose_kernel<decltype(e)>, dim3((unsigned)n_groups), dim3(1024), 0, (hipStream_t)stream, a);
  });
  A3_CHECK_LAUNCH("a3_beam_select");
  return A3_OK;
}
