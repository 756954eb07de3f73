// The paged cache as the kernels of a3_paged.hip, a3_tree.hip and a3_candidates.hip see it.
#pragma once

#include <type_traits>

#include "a3_internal.h"

namespace {

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

// Eight codes as bf16 (whole numbers up to 127: exact, the high half of the float).
__device__ __forceinline__ uint32_t pack_codes(float lo, float hi) {
  return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
}
__device__ __forceinline__ bf16x8 codes8(const uint32_t (&w)[2]) {
  uint32_t x[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    x[i] = pack_codes((float)(signed char)(w[i >> 1] >> 16 * (i & 1)), (float)(signed char)(w[i >> 1] >> (16 * (i & 1) + 8)));
  return __builtin_bit_cast(bf16x8, make_uint4(x[0], x[1], x[2], x[3]));
}

// One number at a wave-uniform place of an array that no kernel in flight writes, by a scalar load: a vector load would be waited for
// together with all the slabs requested before it (they come back in order).
__device__ __forceinline__ int scalar_at(const int *p, size_t i) {
  return reinterpret_cast<const __attribute__((address_space(4))) int *>(reinterpret_cast<uintptr_t>(p))[i];
}

inline int elem_bytes(const a3_pages *P) { return P->dtype == A3_BF16 ? 2 : 4; }

inline a3_status check_pages(const a3_pages *P, const char *who, bool pools) {
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

inline pages_args args_of(const a3_pages *P) {
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
