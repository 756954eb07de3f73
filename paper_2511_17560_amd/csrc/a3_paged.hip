// Generating on the fused cache: K and V of new tokens into pages, and the attention of single tokens over them.
#include "a3_internal.h"
#include "a3_q8.h"

namespace {

// ---------------------------------------------------------------------------------------
// pages
// ---------------------------------------------------------------------------------------
// What the kernels need of an a3_pages.  Page p of a pool, KV head h: [page_size, d] elements, 8-bit pages: codes, then
// page_size float scales.
struct pages_args {
  char *k_pool, *v_pool;
  const int *table;
  const float2 *rope_cs;
  int n_req, max_pages, n_pages, n_pos, page_shift, Hkv, Hq;
  int slots;               // of a request: max_pages << page_shift, at most 2^31 - 1
  int rope_layout;
};

__host__ __device__ inline size_t page_head_bytes(int format, int elem, int page_size, int d) {
  return format == A3_PAGES_Q8 ? (size_t)page_size * (d + 4) : (size_t)page_size * d * elem;
}

__global__ void __launch_bounds__(256)
pages_rope_kernel(float2 *cs, long long total, int half, double base) {
  const long long gid = (long long)blockIdx.x * 256 + threadIdx.x;
  if (gid >= total) return;
  const long long p = gid / half;
  const int i = (int)(gid - p * half);
  double s, c;
  sincos((double)p * pow(base, -(double)i / (double)half), &s, &c);
  cs[gid] = make_float2((float)c, (float)s);
}

// ---------------------------------------------------------------------------------------
// append
// ---------------------------------------------------------------------------------------
// A lane holds 16 coordinates of one head of one row, as two runs of 8 so that both RoPE pairings are inside it (half pairing:
// 8c .. and d / 2 + 8c ..); d / 16 lanes a head, a wave 64 * 16 / d heads of one row, the row's heads in the order K, V, Q.
// Everything a wave looks up (request, slot, position, page) is the same for all its lanes.
struct append_args {
  pages_args p;
  const void *k, *v, *q;
  void *q_out;
  const int *row_req, *row_slot, *row_pos;
  int n_rows, units;       // units: waves per row
};

template <typename T, int D, bool Q8>
__global__ void __launch_bounds__(256)
paged_append_kernel(append_args a) {
  constexpr int kLanes = D / 16, kHeads = 64 / kLanes;
  typedef T vec8 __attribute__((ext_vector_type(8)));
  const int lane = threadIdx.x & 63;
  const unsigned wid = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const unsigned row = wid / (unsigned)a.units;
  if (row >= (unsigned)a.n_rows) return;
  const int head = (int)(wid - row * a.units) * kHeads + lane / kLanes, c = lane % kLanes;
  const int Hkv = a.p.Hkv, heads = 2 * Hkv + (a.q ? a.p.Hq : 0);
  const bool on = head < heads, is_k = head < Hkv, is_v = !is_k && head < 2 * Hkv;
  const int h = is_k ? head : is_v ? head - Hkv : head - 2 * Hkv;

  const int req = a.row_req ? a.row_req[row] : (int)row, slot = a.row_slot[row];
  const int pos = a.row_pos ? a.row_pos[row] : 0;
  if (req < 0 || req >= a.p.n_req || slot < 0 || slot >= a.p.slots || (a.row_pos && (pos < 0 || pos >= a.p.n_pos))) return;
  const int page = a.p.table[(size_t)req * a.p.max_pages + (slot >> a.p.page_shift)];
  if (page < 0 || page >= a.p.n_pages) return;
  const int at = slot & ((1 << a.p.page_shift) - 1);

  const bool rotate = a.row_pos && !is_v, inter = a.p.rope_layout == A3_ROPE_INTERLEAVED;
  const bool split = a.row_pos && !inter;                      // the two runs lie d / 2 apart
  const int e0 = split ? 8 * c : 16 * c, e1 = split ? D / 2 + 8 * c : 16 * c + 8;
  vec8 ra = {}, rb = {};
  if (on) {
    const T *src = (is_k ? (const T *)a.k + ((size_t)row * Hkv + h) * D : is_v ? (const T *)a.v + ((size_t)row * Hkv + h) * D
                                                                               : (const T *)a.q + ((size_t)row * a.p.Hq + h) * D);
    ra = *reinterpret_cast<const vec8 *>(src + e0);
    rb = *reinterpret_cast<const vec8 *>(src + e1);
  }
  float cs[16], sn[16];                                        // of the pair that coordinate e belongs to (e and e + 8: half pairing)
  if (rotate) {
    const float2 *t = a.p.rope_cs + (size_t)pos * (D / 2);
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const float2 v = t[inter ? 8 * c + (e >> 1) : 8 * c + (e & 7)];
      cs[e] = v.x;
      sn[e] = v.y;
    }
  }
  if (Q8 && (is_k || is_v)) {
    // 8-bit pages: the turned key in double (products of floats are exact there), so that a code is that of the exact value
    signed char *base = (signed char *)(is_k ? a.p.k_pool : a.p.v_pool) +
                        ((size_t)page * Hkv + h) * page_head_bytes(A3_PAGES_Q8, 0, 1 << a.p.page_shift, D);
    float x[16], scale;
    double y[16];
#pragma unroll
    for (int e = 0; e < 8; ++e) { x[e] = (float)ra[e]; x[8 + e] = (float)rb[e]; }
    double amax = 0.0;
    if (rotate) {
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int m = inter ? e ^ 1 : e ^ 8;                   // the pair's other coordinate
        const bool first = inter ? !(e & 1) : e < 8;
        y[e] = first ? (double)x[e] * cs[e] - (double)x[m] * sn[e] : (double)x[m] * sn[e] + (double)x[e] * cs[e];
        amax = fmax(amax, fabs(y[e]));
      }
    } else {
      float m = 0.f;
#pragma unroll
      for (int e = 0; e < 16; ++e) m = fmaxf(m, fabsf(x[e]));
      amax = m;
    }
#pragma unroll
    for (int m = 1; m < kLanes; m <<= 1) amax = fmax(amax, __shfl_xor(amax, m));
    scale = q8_scale(amax);
    if (!on) return;
    i8x16 code;
    if (rotate) {
#pragma unroll
      for (int e = 0; e < 16; ++e) code[e] = (signed char)(int)q8_code(y[e], scale);
    } else {
      code = q8_codes(x, scale);
    }
    signed char *dst = base + (size_t)at * D;
    *reinterpret_cast<i8x8 *>(dst + e0) = __builtin_shufflevector(code, code, 0, 1, 2, 3, 4, 5, 6, 7);
    *reinterpret_cast<i8x8 *>(dst + e1) = __builtin_shufflevector(code, code, 8, 9, 10, 11, 12, 13, 14, 15);
    if (c == 0) reinterpret_cast<float *>(base + ((size_t)D << a.p.page_shift))[at] = scale;
    return;
  }
  if (!on) return;
  T *dst = is_k || is_v ? (T *)(is_k ? a.p.k_pool : a.p.v_pool) + ((((size_t)page * Hkv + h) << a.p.page_shift) + at) * D
                        : (T *)a.q_out + ((size_t)row * a.p.Hq + h) * D;
  if (rotate) {
    float x[16], y[16];
#pragma unroll
    for (int e = 0; e < 8; ++e) { x[e] = (float)ra[e]; x[8 + e] = (float)rb[e]; }
    if (inter) {
#pragma unroll
      for (int e = 0; e < 16; e += 2) a3_rotate_pair(x[e], x[e + 1], make_float2(cs[e], sn[e]), y[e], y[e + 1]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) a3_rotate_pair(x[e], x[e + 8], make_float2(cs[e], sn[e]), y[e], y[e + 8]);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) { ra[e] = (T)y[e]; rb[e] = (T)y[8 + e]; }
  }
  *reinterpret_cast<vec8 *>(dst + e0) = ra;
  *reinterpret_cast<vec8 *>(dst + e1) = rb;
}

// ---------------------------------------------------------------------------------------
// attention of single tokens
// ---------------------------------------------------------------------------------------
// One workgroup per (row, query head), 256 slots a step: every thread scores one slot, then sums one coordinate over the 256.
struct attend_args {
  pages_args p;
  const void *q;
  void *out;
  const int *row_req, *row_len;
  int n_rows;
  float scale;
};

template <typename T, int D, bool Q8>
__global__ void __launch_bounds__(256)
paged_attention_kernel(attend_args a) {
  __shared__ float qs[D], w[256], red[4], part[256];
  const int row = blockIdx.x / a.p.Hq, hq = blockIdx.x % a.p.Hq, G = a.p.Hq / a.p.Hkv, h = hq / G, tid = threadIdx.x;
  const int req = a.row_req ? a.row_req[row] : row;
  if (req < 0 || req >= a.p.n_req) return;
  const int len = min(a.row_len[row], a.p.slots), page_size = 1 << a.p.page_shift;
  const size_t head_bytes = page_head_bytes(Q8 ? A3_PAGES_Q8 : A3_PAGES_PLAIN, sizeof(T), page_size, D);
  const size_t qo = ((size_t)row * a.p.Hq + hq) * D;
  if (tid < D) qs[tid] = (float)((const T *)a.q)[qo + tid];
  __syncthreads();
  auto block_of = [&](char *pool, int slot) -> char * {
    const int page = a.p.table[(size_t)req * a.p.max_pages + (slot >> a.p.page_shift)];
    return page < 0 || page >= a.p.n_pages ? nullptr : pool + ((size_t)page * a.p.Hkv + h) * head_bytes;
  };
  float m = -INFINITY, l = 0.f, o = 0.f;
  bool any = false;
  for (int u0 = 0; u0 < len; u0 += 256) {
    const int slot = u0 + tid;
    float s = -INFINITY;
    bool here = false;
    if (slot < len) {
      const char *b = block_of(a.p.k_pool, slot);
      const int at = slot & (page_size - 1);
      if (b) {
        here = true;
        s = 0.f;
        for (int e = 0; e < D; ++e)
          s += qs[e] * (Q8 ? (float)((const signed char *)b)[at * D + e] : (float)((const T *)b)[at * D + e]);
        if (Q8) s *= ((const float *)(b + (size_t)page_size * D))[at];
        s *= a.scale;
      }
    }
    any = __syncthreads_or(here) || any;
    float mx = s;
    for (int x = 32; x; x >>= 1) mx = fmaxf(mx, __shfl_xor(mx, x));
    if ((tid & 63) == 0) red[tid >> 6] = mx;
    __syncthreads();
    mx = fmaxf(m, fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3])));
    const float ref = mx == -INFINITY ? 0.f : mx, keep = expf(m - ref);
    w[tid] = here ? expf(s - ref) : 0.f;
    __syncthreads();
    o *= keep;
    l *= keep;
    m = mx;
    const int e = tid % D, lo = tid / D * D, n = min(256, len - u0);           // each group of D threads sums D of the 256 slots
    for (int j = lo; j < min(n, lo + D); ++j) {
      const char *b = block_of(a.p.v_pool, u0 + j);
      const int at = (u0 + j) & (page_size - 1);
      if (!b) continue;
      const float v = Q8 ? (float)((const signed char *)b)[at * D + e] * ((const float *)(b + (size_t)page_size * D))[at]
                         : (float)((const T *)b)[at * D + e];
      o += w[j] * v;
      l += w[j];
    }
    __syncthreads();
  }
  part[tid] = o;
  w[tid] = l;
  __syncthreads();
  if (tid >= D) return;
  o = l = 0.f;
  for (int j = tid; j < 256; j += D) { o += part[j]; l += w[j]; }
  ((T *)a.out)[qo + tid] = (T)(any ? o / l : 0.f);
}

// ---------------------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------------------
int elem_bytes(const a3_pages *P) { return P->dtype == A3_BF16 ? 2 : 4; }

a3_status check_pages(const a3_pages *P, const char *who, bool pools) {
  A3_REQUIRE(P != nullptr, A3_ERR_INVALID_ARG, "%s: pages is NULL", who);
  A3_REQUIRE(P->dtype == A3_F32 || P->dtype == A3_BF16, A3_ERR_INVALID_ARG, "%s: unknown dtype %d", who, P->dtype);
  A3_REQUIRE(P->format == A3_PAGES_PLAIN || P->format == A3_PAGES_Q8, A3_ERR_INVALID_ARG, "%s: unknown format %d", who, P->format);
  A3_REQUIRE(P->rope_layout == A3_ROPE_INTERLEAVED || P->rope_layout == A3_ROPE_HALF, A3_ERR_INVALID_ARG,
             "%s: unknown rope_layout %d", who, P->rope_layout);
  A3_REQUIRE(P->n_q_heads > 0 && P->n_kv_heads > 0 && P->n_q_heads % P->n_kv_heads == 0, A3_ERR_INVALID_ARG,
             "%s: n_q_heads %d is not a positive multiple of n_kv_heads %d", who, P->n_q_heads, P->n_kv_heads);
  A3_REQUIRE(P->n_q_heads / P->n_kv_heads <= 16, A3_ERR_UNSUPPORTED, "%s: more than 16 query heads per KV head", who);
  A3_REQUIRE(P->head_dim == 64 || P->head_dim == 128, A3_ERR_UNSUPPORTED, "%s: head_dim %d (64 or 128 only)", who, P->head_dim);
  A3_REQUIRE(P->rope_base > 1.0, A3_ERR_INVALID_ARG, "%s: rope_base must be > 1", who);
  A3_REQUIRE(P->sm_scale >= 0.f, A3_ERR_INVALID_ARG, "%s: sm_scale must be >= 0", who);
  A3_REQUIRE(P->page_size >= 32 && P->page_size <= 1024 && (P->page_size & (P->page_size - 1)) == 0, A3_ERR_UNSUPPORTED,
             "%s: page_size %d (a power of two from 32 to 1024)", who, P->page_size);
  A3_REQUIRE(P->n_pages > 0 && P->n_req > 0 && P->max_pages > 0 && P->n_pos >= 0, A3_ERR_INVALID_ARG,
             "%s: n_pages, n_req and max_pages must be positive", who);
  if (pools) {
    A3_REQUIRE(P->k_pool && P->v_pool && P->page_table, A3_ERR_INVALID_ARG, "%s: NULL pool or page table", who);
    A3_REQUIRE(a3_aligned16(P->k_pool) && a3_aligned16(P->v_pool), A3_ERR_INVALID_ARG, "%s: pools must be 16-byte aligned", who);
  }
  return A3_OK;
}

pages_args args_of(const a3_pages *P) {
  pages_args p;
  p.k_pool = (char *)P->k_pool;
  p.v_pool = (char *)P->v_pool;
  p.table = P->page_table;
  p.rope_cs = (const float2 *)P->rope_cs;
  p.n_req = P->n_req;
  p.max_pages = P->max_pages;
  p.n_pages = P->n_pages;
  p.n_pos = P->n_pos;
  p.page_shift = __builtin_ctz((unsigned)P->page_size);
  p.Hkv = P->n_kv_heads;
  p.Hq = P->n_q_heads;
  const long long slots = (long long)P->max_pages * P->page_size;
  p.slots = slots > 0x7fffffffLL ? 0x7fffffff : (int)slots;
  p.rope_layout = P->rope_layout;
  return p;
}

// f(type of a row's element, head_dim, whether the pages are 8-bit)
template <class F>
void with_format(const a3_pages *P, F f) {
  auto by_dim = [&](auto elem, auto q8) {
    if (P->head_dim == 64) f(elem, std::integral_constant<int, 64>{}, q8);
    else f(elem, std::integral_constant<int, 128>{}, q8);
  };
  auto by_format = [&](auto elem) {
    if (P->format == A3_PAGES_Q8) by_dim(elem, std::true_type{});
    else by_dim(elem, std::false_type{});
  };
  if (P->dtype == A3_BF16) by_format(bf16_t{});
  else by_format(0.f);
}

}  // namespace

extern "C" size_t a3_page_bytes(const a3_pages *P) {
  if (check_pages(P, "a3_page_bytes", false) != A3_OK) return 0;
  return (size_t)P->n_kv_heads * page_head_bytes(P->format, elem_bytes(P), P->page_size, P->head_dim);
}

extern "C" a3_status a3_pages_prepare(const a3_pages *P, void *stream) {
  a3_status s = check_pages(P, "a3_pages_prepare", false);
  if (s != A3_OK) return s;
  if (P->n_pos == 0) return A3_OK;
  A3_REQUIRE(P->rope_cs, A3_ERR_INVALID_ARG, "a3_pages_prepare: rope_cs is NULL");
  const long long total = (long long)P->n_pos * (P->head_dim / 2);
  hipLaunchKernelGGL(pages_rope_kernel, dim3((unsigned)((total + 255) / 256)), dim3(256), 0, (hipStream_t)stream,
                     (float2 *)P->rope_cs, total, P->head_dim / 2, P->rope_base);
  A3_CHECK_LAUNCH("a3_pages_prepare");
  return A3_OK;
}

extern "C" a3_status a3_paged_append(const a3_pages *P, const void *k, const void *v, const int *row_req, const int *row_slot,
                                     const int *row_pos, int n_rows, const void *q, void *q_out, void *stream) {
  a3_status s = check_pages(P, "a3_paged_append", true);
  if (s != A3_OK) return s;
  A3_REQUIRE(n_rows >= 0, A3_ERR_INVALID_ARG, "a3_paged_append: n_rows %d is negative", n_rows);
  if (n_rows == 0) return A3_OK;
  A3_REQUIRE(k && v && row_slot, A3_ERR_INVALID_ARG, "a3_paged_append: NULL tensor");
  A3_REQUIRE(row_req || n_rows <= P->n_req, A3_ERR_INVALID_ARG, "a3_paged_append: %d rows without row_req for %d requests", n_rows, P->n_req);
  A3_REQUIRE((q == nullptr) == (q_out == nullptr) && (q == nullptr || row_pos), A3_ERR_INVALID_ARG,
             "a3_paged_append: q needs q_out and row_pos");
  A3_REQUIRE(row_pos == nullptr || P->rope_cs, A3_ERR_INVALID_ARG, "a3_paged_append: row_pos without rope_cs");
  for (const void *p : {k, v, q, (const void *)q_out})
    A3_REQUIRE(a3_aligned16(p), A3_ERR_INVALID_ARG, "a3_paged_append: tensors must be 16-byte aligned");
  append_args a{args_of(P), k, v, q, q_out, row_req, row_slot, row_pos, n_rows, 0};
  const int heads = 2 * P->n_kv_heads + (q ? P->n_q_heads : 0), per_wave = 64 / (P->head_dim / 16);
  a.units = (heads + per_wave - 1) / per_wave;
  const long long waves = (long long)n_rows * a.units;
  A3_REQUIRE(waves < (1LL << 31), A3_ERR_UNSUPPORTED, "a3_paged_append: too many rows");
  with_format(P, [&](auto elem, auto d, auto q8) {
    hipLaunchKernelGGL((paged_append_kernel<decltype(elem), d.value, q8.value>), dim3((unsigned)((waves + 3) / 4)), dim3(256), 0,
                       (hipStream_t)stream, a);
  });
  A3_CHECK_LAUNCH("a3_paged_append");
  return A3_OK;
}

extern "C" size_t a3_paged_attention_ws_bytes(const a3_pages *P, int n_rows) {
  if (check_pages(P, "a3_paged_attention_ws_bytes", false) != A3_OK || n_rows < 0) return 0;
  return 256;
}

extern "C" a3_status a3_paged_attention(const a3_pages *P, const void *q, const int *row_req, const int *row_len, int n_rows,
                                        void *out, void *ws, size_t ws_bytes, void *stream) {
  a3_status s = check_pages(P, "a3_paged_attention", true);
  if (s != A3_OK) return s;
  A3_REQUIRE(n_rows >= 0, A3_ERR_INVALID_ARG, "a3_paged_attention: n_rows %d is negative", n_rows);
  if (n_rows == 0) return A3_OK;
  A3_REQUIRE(q && row_len && out, A3_ERR_INVALID_ARG, "a3_paged_attention: NULL tensor");
  A3_REQUIRE(row_req || n_rows <= P->n_req, A3_ERR_INVALID_ARG, "a3_paged_attention: %d rows without row_req for %d requests", n_rows,
             P->n_req);
  A3_REQUIRE(a3_aligned16(q) && a3_aligned16(out), A3_ERR_INVALID_ARG, "a3_paged_attention: tensors must be 16-byte aligned");
  A3_REQUIRE((long long)n_rows * P->n_q_heads < (1LL << 31), A3_ERR_UNSUPPORTED, "a3_paged_attention: too many rows");
  const size_t need = a3_paged_attention_ws_bytes(P, n_rows);
  A3_REQUIRE(ws && a3_aligned16(ws) && ws_bytes >= need, A3_ERR_WORKSPACE, "a3_paged_attention: workspace %zu bytes (16-byte aligned), need %zu",
             ws ? ws_bytes : 0, need);
  attend_args a{args_of(P), q, out, row_req, row_len, n_rows, P->sm_scale != 0.f ? P->sm_scale : 1.0f / sqrtf((float)P->head_dim)};
  with_format(P, [&](auto elem, auto d, auto q8) {
    hipLaunchKernelGGL((paged_attention_kernel<decltype(elem), d.value, q8.value>), dim3((unsigned)(n_rows * P->n_q_heads)), dim3(256), 0,
                       (hipStream_t)stream, a);
  });
  A3_CHECK_LAUNCH("a3_paged_attention");
  return A3_OK;
}
