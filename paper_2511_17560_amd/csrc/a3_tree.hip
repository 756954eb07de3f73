// Attention of drafted tokens: the rows of a group see their request's whole cache and, among the group's own slots, what a mask says.
#include "a3_pages.h"

namespace {

struct tree_args {
  pages_args p;
  const void *q;
  void *out;
  const int *start, *req, *len, *mask;
  int n_groups, n_rows, max_rows, mask_words;
  float scale;             // of the logits, in units of log 2
};

// Rows of a group, first of all rows: none where its bounds are not in order.
__device__ __forceinline__ int group_rows(const tree_args &a, int g, int &first) {
  first = a.start[g];
  const int end = a.start[g + 1];
  return first < 0 || end > a.n_rows || end < first ? 0 : min(end - first, a.max_rows);
}

// One workgroup a row and query head, a wave every fourth slot.
template <typename T, int D, bool Q8>
__global__ void __launch_bounds__(256)
tree_attention_kernel(tree_args a) {
  constexpr int E = D / 64;
  __shared__ float2 ml[4];
  __shared__ int any[4];
  __shared__ float os[4][D];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int g = blockIdx.x / a.max_rows, j = blockIdx.x - g * a.max_rows, h = blockIdx.y, kv = h / (a.p.Hq / a.p.Hkv);
  int first;
  const int n = group_rows(a, g, first), req = a.req ? a.req[g] : g;
  if (j >= n || req < 0 || req >= a.p.n_req) return;
  const int L = max(0, min(a.len[g], a.p.slots)), end = (int)min((long long)L + n, (long long)a.p.slots);
  const size_t row = (size_t)first + j, at = (row * a.p.Hq + h) * D + lane * E;
  float q[E], o[E], m = -INFINITY, l = 0.f;
  bool seen = false;
#pragma unroll
  for (int e = 0; e < E; ++e) { q[e] = (float)((const T *)a.q)[at + e]; o[e] = 0.f; }
  const size_t head_bytes = page_head_bytes(Q8 ? A3_PAGES_Q8 : A3_PAGES_PLAIN, sizeof(T), 1 << a.p.page_shift, D);
  for (int u = wave; u < end; u += 4) {
    const int t = u - L;
    if (t >= 0 && !(a.mask ? (a.mask[row * a.mask_words + (t >> 5)] >> (t & 31)) & 1 : t <= j)) continue;
    const int page = a.p.table[(size_t)req * a.p.max_pages + (u >> a.p.page_shift)], in = u & ((1 << a.p.page_shift) - 1);
    if (page < 0 || page >= a.p.n_pages) continue;
    const char *kp = a.p.k_pool + ((size_t)page * a.p.Hkv + kv) * head_bytes, *vp = a.p.v_pool + ((size_t)page * a.p.Hkv + kv) * head_bytes;
    float k[E], v[E], s = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const size_t c = (size_t)in * D + lane * E + e;
      if constexpr (Q8) {
        const size_t sc = ((size_t)D << a.p.page_shift) + 4 * in;
        k[e] = (float)((const signed char *)kp)[c] * *(const float *)(kp + sc);
        v[e] = (float)((const signed char *)vp)[c] * *(const float *)(vp + sc);
      } else {
        k[e] = (float)((const T *)kp)[c];
        v[e] = (float)((const T *)vp)[c];
      }
      s = fmaf(q[e], k[e], s);
    }
    for (int x = 32; x; x >>= 1) s += __shfl_xor(s, x);
    s *= a.scale;
    seen = true;
    const float next = fmaxf(m, s), f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - next);
    const float w = s == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(s - (next == -INFINITY ? 0.f : next));
    l = l * f + w;
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = o[e] * f + w * v[e];
    m = next;
  }
  if (lane == 0) { ml[wave] = make_float2(m, l); any[wave] = seen; }
#pragma unroll
  for (int e = 0; e < E; ++e) os[wave][lane * E + e] = o[e];
  __syncthreads();
  if (wave != 0) return;
  float M = -INFINITY, sum = 0.f, y[E] = {};
  for (int w = 0; w < 4; ++w) M = fmaxf(M, ml[w].x);
  for (int w = 0; w < 4; ++w) {
    const float f = ml[w].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml[w].x - M);
    sum += ml[w].x == -INFINITY ? ml[w].y : ml[w].y * f;
#pragma unroll
    for (int e = 0; e < E; ++e) y[e] += ml[w].x == -INFINITY ? os[w][lane * E + e] : os[w][lane * E + e] * f;
  }
  const bool some = any[0] | any[1] | any[2] | any[3];
#pragma unroll
  for (int e = 0; e < E; ++e) ((T *)a.out)[at + e] = (T)(some ? y[e] / sum : 0.f);
}

constexpr int kMaxRows = 1024;

}  // namespace

extern "C" size_t a3_tree_attention_ws_bytes(const a3_pages *P, int n_groups, int max_rows) {
  if (check_pages(P, "a3_tree_attention_ws_bytes", false) != A3_OK || n_groups < 0 || max_rows < 1 || max_rows > kMaxRows) return 0;
  return 256;
}

extern "C" a3_status a3_tree_attention(const a3_pages *P, const void *q, int n_groups, const int *group_start, const int *group_req,
                                       const int *group_len, const int *mask, int mask_words, int n_rows, int max_rows, void *out,
                                       void *ws, size_t ws_bytes, void *stream) {
  a3_status s = check_pages(P, "a3_tree_attention", true);
  if (s != A3_OK) return s;
  A3_REQUIRE(n_groups >= 0 && n_rows >= 0, A3_ERR_INVALID_ARG, "a3_tree_attention: n_groups %d, n_rows %d", n_groups, n_rows);
  A3_REQUIRE(max_rows >= 1, A3_ERR_INVALID_ARG, "a3_tree_attention: max_rows %d", max_rows);
  A3_REQUIRE(max_rows <= kMaxRows, A3_ERR_UNSUPPORTED, "a3_tree_attention: max_rows %d (%d at most)", max_rows, kMaxRows);
  if (n_groups == 0 || n_rows == 0) return A3_OK;
  A3_REQUIRE(q && out && group_start && group_len, A3_ERR_INVALID_ARG, "a3_tree_attention: NULL tensor");
  A3_REQUIRE(group_req || n_groups <= P->n_req, A3_ERR_INVALID_ARG, "a3_tree_attention: %d groups without group_req for %d requests", n_groups,
             P->n_req);
  A3_REQUIRE(mask == nullptr || (mask_words >= 1 && mask_words <= kMaxRows / 32 && mask_words * 32 >= max_rows), A3_ERR_INVALID_ARG,
             "a3_tree_attention: masks of %d words for groups of up to %d rows", mask_words, max_rows);
  A3_REQUIRE(a3_aligned16(q) && a3_aligned16(out), A3_ERR_INVALID_ARG, "a3_tree_attention: tensors must be 16-byte aligned");
  const size_t need = a3_tree_attention_ws_bytes(P, n_groups, max_rows);
  A3_REQUIRE(ws && a3_aligned16(ws) && ws_bytes >= need, A3_ERR_WORKSPACE, "a3_tree_attention: workspace %zu bytes (16-byte aligned), need %zu",
             ws ? ws_bytes : 0, need);
  tree_args a{args_of(P), q, out, group_start, group_req, group_len, mask, n_groups, n_rows, max_rows, mask_words,
              (float)((P->sm_scale != 0.f ? (double)P->sm_scale : 1.0 / sqrt((double)P->head_dim)) * 1.4426950408889634074)};
  A3_REQUIRE((long long)n_groups * max_rows < (1LL << 31), A3_ERR_UNSUPPORTED, "a3_tree_attention: too many groups");
  with_format(P, [&](auto elem, auto d, auto q8) {
    hipLaunchKernelGGL((tree_attention_kernel<decltype(elem), d.value, q8.value>), dim3((unsigned)(n_groups * max_rows), (unsigned)P->n_q_heads),
                       dim3(256), 0, (hipStream_t)stream, a);
  });
  A3_CHECK_LAUNCH("a3_tree_attention");
  return A3_OK;
}
