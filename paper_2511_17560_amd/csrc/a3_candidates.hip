// What follows several candidates of a request: the accepted path of a drafted tree, cache rows moved to other slots, and the best
// continuations of beams.
#include "a3_choose.h"
#include "a3_pages.h"

namespace {

constexpr int kMaxRows = 1024, kMaxPath = 64, kMaxSet = 64, kMaxBeams = 64, kMaxBest = 64;

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
  int slices;                          // of a row
  unsigned long long *part;            // [n_rows, slices] largest keys
};

// The largest key of 2^k neighbouring lanes, in all of them.
__device__ __forceinline__ unsigned long long max_of_lanes(unsigned long long k, int lanes) {
  for (int o = lanes >> 1; o; o >>= 1) { const unsigned long long x = __shfl_xor(k, o); k = x > k ? x : k; }
  return k;
}

// The largest logit of a slice of a row.  A thread keeps the maximum of its values and the chunk of 32 that it came from: one instruction a
// value, so that reading is all that counts.  The key of the largest is found in that chunk afterwards, by the threads that have it alone.  (A
// maximum of -inf says nothing: all may be NaN.)  Bound by one trip to memory where there are few rows: 16 rows of 128256 floats (8.2 MB) 5.7 us,
// 403 of 32003 bf16 (26 MB) 11.3 us, 2.3 TB/s (of 32000, whose rows are aligned, no less); 403 of 128256 floats (207 MB) 44 us the whole call.
template <typename T>
__global__ void __launch_bounds__(kLpThreads)
pick_kernel(accept_args a) {
  typedef lp_row<T, true> R;
  constexpr int V = R::V, U = R::U, kChunk = R::kChunk;
  __shared__ unsigned long long best;
  __shared__ float tops[4];
  const int row = blockIdx.x / a.slices, slice = blockIdx.x - row * a.slices, tid = threadIdx.x;
  R r;
  r.x = (const T *)a.x + (size_t)row * a.ld;
  r.vocab = a.vocab;
  r.skew = 0;
  const int n_vec = (a.vocab + V - 1) / V, per = n_vec / a.slices, rest = n_vec - per * a.slices;
  r.v0 = slice * per + min(slice, rest);
  r.v1 = r.v0 + per + (slice < rest ? 1 : 0);
  // Where the slice or the row ends some of it is read again: the maximum minds no value twice, and the loads need no branches.
  typename R::vec_t raw[U];
  auto element = [&](int c, int u) {
    const int e = min(c + u * kLpThreads + tid, r.v1 - 1) * V;
    return r.vocab >= V ? min(e, r.vocab - V) : e;
  };
  auto load = [&](int c) {
#pragma unroll
    for (int u = 0; u < U; ++u)
      raw[u] = r.vocab >= V ? *reinterpret_cast<const typename R::vec_any *>(r.x + element(c, u)) : r.vec(0);
  };
  float m = -INFINITY;
  int from = r.v0, c = r.v0;
  for (;; c += kChunk) {
    load(c);
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < kLpValues; ++i) top = fmaxf(top, (float)raw[i / V][i % V]);
    if (top > m) { m = top; from = c; }
    if (c + kChunk >= r.v1) break;
  }
  const float mw = wave_max(m);
  if ((tid & 63) == 0) tops[tid >> 6] = mw;
  if (tid == 0) best = 0;
  __syncthreads();
  const float M = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
  const bool all = M == -INFINITY;                             // nothing but -inf and NaN: every value is looked at
  if (all || m == M) {
    unsigned long long k = 0;
    for (int at = all ? r.v0 : from; at < r.v1; at = all ? at + kChunk : r.v1) {
      if (at != c) load(at);
      c = at;
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const int e = element(at, u) + i;
          const unsigned long long x = e < r.vocab ? top_key((float)raw[u][i], e) : 0ull;
          k = x > k ? x : k;
        }
    }
    atomicMax(&best, k);                                       // (the order does not matter)
  }
  __syncthreads();
  if (tid == 0) a.part[blockIdx.x] = best;
}

// Workgroup g < n_groups follows the tree of group g; the others write the picks of 64 rows each (rows may be in no group).
// A chain of latencies: the slices' keys and the tree in one round trip, then a look at LDS for every row of the path (3 - 4 us).
__global__ void __launch_bounds__(256)
follow_kernel(accept_args a) {
  __shared__ int picked[kMaxRows], parent[kMaxRows], token[kMaxRows];
  const int tid = threadIdx.x, g = blockIdx.x;
  // picks of rows first .. first + n - 1 into `to`: as many lanes a row as there are threads for
  auto join = [&](int first, int n, int *to) {
    int lanes = 64;
    while (lanes > 1 && lanes * n > 256) lanes >>= 1;
    for (int r0 = 0; r0 < n; r0 += 256 / lanes) {
      const int r = r0 + tid / lanes;
      unsigned long long k = 0;
      if (r < n) {
        const unsigned long long *p = a.part + (size_t)(first + r) * a.slices;
#pragma unroll 4
        for (int s = tid % lanes; s < a.slices; s += lanes) k = p[s] > k ? p[s] : k;
      }
      k = max_of_lanes(k, lanes);
      if (r < n && tid % lanes == 0) to[r] = (int)~(uint32_t)k;
    }
  };
  if (g >= a.n_groups) {
    const int first = (g - a.n_groups) * 64;
    join(first, min(64, a.n_rows - first), a.picked + first);
    return;
  }
  const int first = a.start[g], end = a.start[g + 1], L = a.len ? max(a.len[g], 0) : 0;
  const int n = first < 0 || end > a.n_rows || end < first ? 0 : min(end - first, a.max_rows);
  for (int i = tid; i < n; i += 256) {
    parent[i] = a.parent[first + i];
    token[i] = a.tokens[first + i];
    if (!a.x) picked[i] = a.picked[first + i];
  }
  if (a.x) join(first, n, picked);
  __syncthreads();
  if (tid >= 64) return;
  int mine = -1, count = 0, last = 0;                          // lane m keeps path[m]
  while (n > 0) {
    if (tid == count) mine = last;
    if (++count == a.max_path) break;
    const int tok = picked[last];
    int child = -1;
    for (int c0 = last + 1; c0 < n && child < 0; c0 += 64) {
      const int c = min(c0 + tid, n - 1);
      const unsigned long long hit = __ballot(c0 + tid < n && parent[c] == last && token[c] == tok);
      if (hit) child = c0 + __builtin_ctzll(hit);
    }
    if (child < 0) break;
    last = child;
  }
  if (tid == 0) {
    a.count[g] = count;
    a.next[g] = n > 0 ? picked[last] : -1;
  }
  if (tid < a.max_path) {
    const size_t i = (size_t)g * a.max_path + tid;
    a.path[i] = tid < count ? mine : -1;
    if (a.src) {
      a.src[i] = tid < count ? L + mine : -1;
      a.dst[i] = tid < count ? L + tid : -1;
    }
  }
}

// Slices of a row: few rows are cut so that some thousand workgroups share the reading, into pieces of a chunk at least.
constexpr int kPickPieces = 2048;
int pick_slices(int n_rows, int vocab) {
  const int by_rows = n_rows >= kPickPieces ? 1 : (kPickPieces + n_rows - 1) / n_rows;
  const int by_size = (int)(((long long)vocab + kLpValues * kLpThreads - 1) / (kLpValues * kLpThreads));
  return by_size < by_rows ? by_size : by_rows < 128 ? by_rows : 128;
}

// ---------------------------------------------------------------------------------------
// cache rows moved
// ---------------------------------------------------------------------------------------
constexpr int kLayersAtOnce = 64, kMoveGroups = 8192, kMoveSlots = 256;      // (slots of all moves of a set that a workgroup has at once)
struct move_args {
  pages_args p;                        // (pools: of the layers below)
  char *pools[2 * kLayersAtOnce];      // K and V of every layer
  const int *src_req, *src_slot, *dst_req, *dst_slot, *n_slots;
  int max_slots, set_size, row_bytes, q8;
  // a workgroup: 2^row_shift vectors of a row, 2^slot_shift slots, `heads` KV heads (256 >> both shifts); groups of those, units: of all pools
  int row_shift, slot_shift, heads, groups, units;
  size_t head_bytes;
};

// The physical slot of a request's, -1 where there is none.
__device__ __forceinline__ long long place_of(const pages_args &p, int req, int first, uint32_t o) {
  const long long slot = (long long)first + o;
  if (req < 0 || req >= p.n_req || first < 0 || slot >= p.slots) return -1;
  const int page = p.table[(size_t)req * p.max_pages + (size_t)(slot >> p.page_shift)];
  return page >= 0 && page < p.n_pages ? ((long long)page << p.page_shift) + (slot & ((1 << p.page_shift) - 1)) : -1;
}

// A thread has 16 bytes of one KV head at one slot o of the runs, of all N moves of its set: it reads them all, then writes them all, and no
// other thread touches what it does, so that a set needs neither a barrier nor a copy in between.  8-bit pages: then the scales, four bytes
// a slot.  Where the slots are is the same in every pool and head: looked up once, for every gridDim.z-th of them.  Bound by memory (reading and
// writing the rows that change their place): 24 rows' worth of 32 layers' caches among 32 beams, 1.56 GB, 277 us = 5.6 TB/s, where torch's copy of
// 2 GiB reaches 4.9 (looked up for each pool and head, by every thread, 426); the same rows in 8-bit pages, 0.80 GB, 155 us.
template <int N>
__global__ void __launch_bounds__(256)
move_kernel(move_args a) {
  const int set = blockIdx.y, tid = threadIdx.x, slots = 1 << a.slot_shift, slot_mask = (1 << a.p.page_shift) - 1;
  struct place { long long from, to; int from_slot, to_slot; };        // of a page in the pool (to < 0: nothing to move); a slot of it
  __shared__ place places[N * (kMoveSlots / N)];
  __shared__ int last[N];
  const size_t first = (size_t)set * a.set_size;
  const int m_of = tid & (N - 1), m_at = min(m_of, a.set_size - 1);
  const int from = a.src_slot[first + m_at], to = a.dst_slot[first + m_at], n = m_of < a.set_size ? min(a.n_slots ? a.n_slots[first + m_at] : 1, a.max_slots) : 0,
            from_req = a.src_req ? a.src_req[first + m_at] : set, to_req = a.dst_req ? a.dst_req[first + m_at] : set;
  if (tid < N) last[tid] = n;
  __syncthreads();
  int most = 0;
#pragma unroll 8
  for (int m = 0; m < N; ++m) most = max(most, last[m]);       // (up to 2^31 - 1: what comes behind it is counted unsigned)
  // Moves words W of slot `so` of these, of KV heads h, h + heads a pool, ..: the lane's `at` bytes into the slot's `width` bytes.
  auto move = [&](auto word, int so, int h, size_t at, int width) {
    typedef decltype(word) W;
    const place *p = places + so * N;
    for (int unit = blockIdx.z; unit < a.units; unit += gridDim.z) {
      const int pool_no = unit / a.groups, head = (unit - pool_no * a.groups) * a.heads + h;
      char *pool = a.pools[pool_no] + (size_t)head * a.head_bytes + at;
      if (head >= a.p.Hkv) continue;
      W x[N];
#pragma unroll
      for (int m = 0; m < N; ++m)
        if (p[m].to >= 0) x[m] = *reinterpret_cast<const W *>(pool + p[m].from + (uint32_t)(p[m].from_slot * width));
#pragma unroll
      for (int m = 0; m < N; ++m)
        if (p[m].to >= 0) *reinterpret_cast<W *>(pool + p[m].to + (uint32_t)(p[m].to_slot * width)) = x[m];
    }
  };
  for (uint32_t o0 = blockIdx.x * slots; o0 < (uint32_t)most; o0 += gridDim.x * slots) {
    for (int i = tid; i < N * slots; i += 256) {               // (256 is a multiple of N: a thread has one move of the set)
      const uint32_t o = o0 + i / N;
      const bool on = (long long)o < n;
      const long long x = on ? place_of(a.p, from_req, from, o) : -1, y = on ? place_of(a.p, to_req, to, o) : -1;
      const size_t page_bytes = a.p.Hkv * a.head_bytes;
      places[i] = x >= 0 && y >= 0 && x != y ? place{(long long)((x >> a.p.page_shift) * page_bytes), (long long)((y >> a.p.page_shift) * page_bytes),
                                                     (int)(x & slot_mask), (int)(y & slot_mask)}
                                             : place{0, -1, 0, 0};
    }
    __syncthreads();
    move(a3_u32x4{}, (tid >> a.row_shift) & (slots - 1), tid >> (a.row_shift + a.slot_shift), 16 * (tid & ((1 << a.row_shift) - 1)), a.row_bytes);
    if (a.q8 && tid < slots * a.heads) move(uint32_t{}, tid & (slots - 1), tid >> a.slot_shift, (size_t)a.row_bytes << a.p.page_shift, 4);
    __syncthreads();
  }
}

// ---------------------------------------------------------------------------------------
// beams
// ---------------------------------------------------------------------------------------
// A workgroup reads a row, or a slice of one, as the log probabilities do (a3_logits.hip): maximum and sum of a thread's own values, the
// maxima of its chunks of 32 noted, and the best n_best values chosen when all have been read.  Its vectors lie as the row stands, wherever
// that starts, so that beams that are the same have the same sums.  A chunk's 32 exponentials are summed in float, chunks in double.
// A second kernel, one workgroup a group, makes worths of its lists (one of every slice of every beam, best first) in double and puts
// them together: the n_best-th of the lists' heads (or of their first few, where there are fewer lists) bounds what can be among the best,
// what reaches it is gathered, n_best^2 values at most, and ranked by counting.  It is a chain of latencies: three trips to
// memory, and nothing that goes through all lists one by one.  1 x 4 beams of 128256 floats: 7.6 + 6.8 us; 64 x 8 of 152064 floats: 56 us (311 MB,
// 5.6 TB/s) + 6.8 us; of 152064 bf16 (156 MB) 45 us the whole call.
struct beam_args {
  const void *x;
  long long ld;
  int vocab, n_beams, n_best, end, slices;
  const float *score;
  const int *done;
  float *best_score;
  int *best_row, *best_token;
  double2 *part;                       // [rows, slices] maximum and sum of a slice
  unsigned long long *part_top;        // [rows, slices, n_best] its best values, best first (0: none)
};

template <typename T>
__global__ void __launch_bounds__(kLpThreads)
beam_row_kernel(beam_args a) {
  typedef lp_row<T, true> R;
  constexpr int V = R::V, U = R::U, kChunk = R::kChunk;
  __shared__ lp_shared s;
  __shared__ float noted[kLpChunks][kLpThreads];
  __shared__ double sums[4];
  const int row = blockIdx.x / a.slices, slice = blockIdx.x - row * a.slices, tid = threadIdx.x;
  if (a.done && a.done[row]) return;                           // (its logits are not looked at, nor what would be left of them)
  R r;
  r.x = (const T *)a.x + (size_t)row * a.ld;
  r.vocab = a.vocab;
  r.skew = 0;
  const int n_vec = (a.vocab + V - 1) / V, per = n_vec / a.slices, rest = n_vec - per * a.slices;
  r.v0 = slice * per + min(slice, rest);
  r.v1 = r.v0 + per + (slice < rest ? 1 : 0);
  typename R::vec_t raw[U];
  auto load = [&](int c) {
    if (c + kChunk <= r.v1 && (long long)(c + kChunk) * V <= r.vocab) {
      const T *x = r.x + (long long)c * V;
#pragma unroll
      for (int u = 0; u < U; ++u) raw[u] = *reinterpret_cast<const typename R::vec_any *>(x + (u * kLpThreads + tid) * V);
      return;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) raw[u] = r.vec(c + u * kLpThreads + tid);
  };
  load(r.v0);
  for (int j = tid; j < a.n_best; j += kLpThreads) s.list[j] = 0;
  float m = -INFINITY;
  double z = 0.0;
  for (int g0 = r.v0; g0 < r.v1; g0 += kLpChunks * kChunk) {   // chunks between two choices of the best
    const int g1 = min(r.v1, g0 + kLpChunks * kChunk);
    float most = -INFINITY, second = -INFINITY;
    for (int c = g0; c < g1; c += kChunk) {
      float y[kLpValues];
#pragma unroll
      for (int i = 0; i < kLpValues; ++i) y[i] = (float)raw[i / V][i % V];
      if (c + kChunk < r.v1) load(c + kChunk);                 // on its way while this chunk is worked on
      float top = fmaxf(-INFINITY, y[0]), half = fmaxf(-INFINITY, y[1]);   // (halves of nothing but NaN: -inf)
#pragma unroll
      for (int i = 2; i < kLpValues; i += 2) { top = fmaxf(top, y[i]); half = fmaxf(half, y[i + 1]); }
      second = fmaxf(second, fmaxf(fminf(top, half), fminf(most, fmaxf(top, half))));
      top = fmaxf(top, half);
      noted[(c - g0) / kChunk][tid] = top;
      most = fmaxf(most, top);
      if (top > m) {
        z *= (double)__builtin_amdgcn_exp2f(lp_shift(m, top));
        m = top;
      }
      const float ref = m == -INFINITY ? 0.f : m;
      float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < kLpValues; ++i) sum[i & 3] += __builtin_amdgcn_exp2f((y[i] - ref) * kLog2e);
      z += (double)((sum[0] + sum[1]) + (sum[2] + sum[3]));
    }
    __syncthreads();                                           // (the list: cleared, or of the last choice)
    lp_choose(s, r, noted, a.n_best, g0, g1, g0 + tid >= g1 || (most == -INFINITY && z != z) ? 0u : top_order(most),
              second == -INFINITY ? 0u : top_order(second));
  }
  const float mw = wave_max(m);
  z *= (double)__builtin_amdgcn_exp2f(lp_shift(m, mw));
  for (int o = 32; o; o >>= 1) z += __shfl_xor(z, o);
  __syncthreads();
  if ((tid & 63) == 0) { s.red[tid >> 6][0] = mw; sums[tid >> 6] = z; }
  __syncthreads();
  if (tid == 0) {
    const float top = fmaxf(fmaxf(s.red[0][0], s.red[1][0]), fmaxf(s.red[2][0], s.red[3][0]));
    double all = 0.0;
#pragma unroll
    for (int w = 0; w < 4; ++w) all += sums[w] * (double)__builtin_amdgcn_exp2f(lp_shift(s.red[w][0], top));
    a.part[blockIdx.x] = make_double2((double)top, all);
  }
  for (int j = tid; j < a.n_best; j += kLpThreads) a.part_top[(size_t)blockIdx.x * a.n_best + j] = s.list[j];
}

// Larger worth, then lower beam, then larger logit, then lower token; worth -inf: no candidate.  Worths of one beam differ as its logits do: where
// a large score leaves a double no room for the difference, the logits decide, which the lists are ordered by.
struct candidate { double worth; int beam; unsigned long long key; };       // key: the logit's, as in the lists
__device__ __forceinline__ bool before(const candidate &a, const candidate &b) {
  return a.worth > b.worth || (a.worth == b.worth && (a.beam < b.beam || (a.beam == b.beam && a.key > b.key)));
}
// How many of n candidates are before one of them: worths first, the rest only where some are equal.
__device__ __forceinline__ int rank_of(const candidate &c, const candidate *of, int n) {
  int rank = 0, equal = 0;
#pragma unroll 4
  for (int o = 0; o < n; ++o) {
    rank += of[o].worth > c.worth;
    equal += of[o].worth == c.worth;
  }
  if (equal > 1)
    for (int o = 0; o < n; ++o) rank += of[o].worth == c.worth && before(of[o], c);
  return rank;
}

constexpr int kBeamLists = 512, kBeamHeads = kBeamLists + kMaxBest, kHeadsAThread = (kBeamHeads + 255) / 256;
__global__ void __launch_bounds__(256)
beam_join_kernel(beam_args a) {
  extern __shared__ candidate gathered[];                      // [n_best * n_best]
  __shared__ candidate head[kBeamHeads], bound;
  __shared__ double base[kMaxBeams];
  __shared__ unsigned char kind[kMaxBeams];                    // 0: no candidates, 1: logits, 2: has ended
  __shared__ unsigned short place[kBeamHeads], chosen[kMaxBest];       // of the heads kept; lists that may have more of the best
  __shared__ uint32_t bounds[4];
  __shared__ int count, kept, n_lists;
  const int g = blockIdx.x, tid = threadIdx.x, lists = a.n_beams * a.slices, first = g * a.n_beams;
  // the lists' first `deep`: n_best of them at least, more where there are threads for them
  const int deep = min(a.n_best, max((a.n_best + lists - 1) / lists, 256 / lists)), heads = lists * deep;
  const unsigned long long *tops = a.part_top + (size_t)first * a.slices * a.n_best;
  unsigned long long keys[kHeadsAThread];                      // (on their way while the beams' sums are joined)
#pragma unroll
  for (int q = 0; q < kHeadsAThread; ++q) {
    const int i = min(tid + 256 * q, heads - 1);
    keys[q] = tops[(size_t)(i / deep) * a.n_best + i % deep];
  }
  if (tid == 0) { bound = candidate{-INFINITY, 0, 0}; count = kept = n_lists = 0; }
  // worth of a logit: base + x; as many lanes a beam as it has slices
  int lanes = 1;
  while (lanes < 64 && lanes < a.slices) lanes <<= 1;
  for (int b0 = 0; b0 < a.n_beams; b0 += 256 / lanes) {
    const int b = b0 + tid / lanes, bb = min(b, a.n_beams - 1);
    const float s = a.score[first + bb];
    const bool ended = a.done && a.done[first + bb];
    int k = !(fabsf(s) < INFINITY) ? 0 : ended ? 2 : 1;
    double M = -INFINITY, Z = 0.0;
    if (k == 1) {                                              // (the same in all lanes of a beam)
      const double2 *p = a.part + (size_t)(first + bb) * a.slices;
      for (int i = tid % lanes; i < a.slices; i += lanes) {
        const double2 x = p[i];
        if (x.x == -INFINITY && x.y == 0.0) continue;
        const double up = fmax(M, x.x);
        Z = (M == up ? Z : Z * exp(M - up)) + (x.x == up ? x.y : x.y * exp(x.x - up));
        M = up;
      }
      double up = M;
      for (int o = lanes >> 1; o; o >>= 1) up = fmax(up, __shfl_xor(up, o));
      Z = M == up || Z == 0.0 ? Z : Z * exp(M - up);
      for (int o = lanes >> 1; o; o >>= 1) Z += __shfl_xor(Z, o);
      M = up;
      if (!(Z > 0.0 && Z < INFINITY && fabs(M) < INFINITY)) k = 0;
    }
    if (b < a.n_beams && tid % lanes == 0) {
      kind[b] = (unsigned char)k;
      base[b] = k == 2 ? (double)s : (double)s - M - log(Z);
    }
  }
  __syncthreads();
  auto made = [&](int list, int j, unsigned long long key) {   // the jth of a list
    const int b = list / a.slices;
    const candidate none{-INFINITY, 0, 0};
    if (kind[b] == 0) return none;
    if (kind[b] == 2) return list == b * a.slices && j == 0 ? candidate{base[b], b, top_key(0.f, a.end)} : none;
    return key ? candidate{base[b] + (double)top_value(key), b, key} : none;
  };
  // A first bound: the largest of the waves' n_best-th heads, in float; the heads that reach it are ranked.
  candidate mine[kHeadsAThread];
  uint32_t order[kHeadsAThread];
#pragma unroll
  for (int q = 0; q < kHeadsAThread; ++q) {
    const int i = tid + 256 * q;
    mine[q] = i < heads ? made(i / deep, i % deep, keys[q]) : candidate{-INFINITY, 0, 0};
    order[q] = mine[q].worth > -INFINITY ? max(top_order((float)mine[q].worth), 1u) : 0u;
  }
  const uint32_t nth = wave_nth<32, kHeadsAThread>(order, a.n_best);
  if ((tid & 63) == 0) bounds[tid >> 6] = nth;
  __syncthreads();
  const uint32_t reach = max(max(bounds[0], bounds[1]), max(max(bounds[2], bounds[3]), 1u));
#pragma unroll
  for (int q = 0; q < kHeadsAThread; ++q)
    if (order[q] >= reach) {
      const int to = atomicAdd(&kept, 1);
      head[to] = mine[q];
      place[to] = (unsigned short)(tid + 256 * q);
    }
  __syncthreads();
  const int n_heads = kept;
  for (int i = tid; i < n_heads; i += 256) {
    const candidate c = head[i];
    const int rank = rank_of(c, head, n_heads);
    if (rank >= a.n_best) continue;
    if (rank == a.n_best - 1) bound = c;
    gathered[atomicAdd(&count, 1)] = c;
    if (deep < a.n_best && place[i] % deep == deep - 1) chosen[atomicAdd(&n_lists, 1)] = (unsigned short)(place[i] / deep);
  }
  __syncthreads();
  const candidate last = bound;                                // (none: all there are)
  const int more = a.n_best - deep;
  for (int i = tid; i < n_lists * more; i += 256) {
    const int list = chosen[i / more], j = deep + i % more;
    const candidate c = made(list, j, tops[(size_t)list * a.n_best + j]);
    if (c.worth > -INFINITY && !(last.worth > -INFINITY && before(last, c))) gathered[atomicAdd(&count, 1)] = c;
  }
  __syncthreads();
  const int n = count;
  for (int i = tid; i < n; i += 256) {
    const candidate c = gathered[i];
    const int rank = rank_of(c, gathered, n);
    if (rank < a.n_best) {
      const size_t to = (size_t)g * a.n_best + rank;
      a.best_score[to] = (float)c.worth;
      a.best_row[to] = first + c.beam;
      a.best_token[to] = (int)~(uint32_t)c.key;
    }
  }
  for (int j = n + tid; j < a.n_best; j += 256) {
    const size_t to = (size_t)g * a.n_best + j;
    a.best_score[to] = -INFINITY;
    a.best_row[to] = a.best_token[to] = -1;
  }
}

// Slices of a row: few rows are cut so that some thousand workgroups share the reading, into pieces of no less than two vectors a thread, and
// so that a group has no more lists than kBeamLists.
constexpr int kBeamPieces = 1024;
int beam_slices(long long rows, int n_beams, int vocab, int elem) {
  const long long by_size = (long long)vocab * elem / (16 * 2 * kLpThreads), by_rows = rows >= kBeamPieces ? 1 : (kBeamPieces + rows - 1) / rows;
  long long n = by_rows < kBeamLists / n_beams ? by_rows : kBeamLists / n_beams;
  if (by_size < n) n = by_size;
  return n < 1 ? 1 : (int)n;
}
size_t beam_ws(size_t pieces, int n_best, void *base, beam_args *a) {
  a3_ws_cursor cur(base, 0);
  double2 *part = (double2 *)cur.take(pieces * sizeof(double2));
  unsigned long long *top = (unsigned long long *)cur.take(pieces * n_best * sizeof(unsigned long long));
  if (a) { a->part = part; a->part_top = top; }
  return cur.off;
}

template <class F>
void with_dtype(int dtype, F f) {
  if (dtype == A3_BF16) f(bf16_t{});
  else f(0.f);
}

}  // namespace

extern "C" size_t a3_tree_accept_ws_bytes(int n_rows, int vocab) {
  if (n_rows < 0 || vocab <= 0) return 0;
  // (r rows are r min(128, ceil(2048 / r)) pieces at most: below 2048 + r, and r from r = 2048 on)
  const size_t r = n_rows < kPickPieces ? n_rows : kPickPieces - 1, some = r * 128 < kPickPieces + r ? r * 128 : kPickPieces + r;
  return ((size_t)n_rows > some ? (size_t)n_rows : some) * sizeof(unsigned long long) + 256;
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
                count, path, next_token, src_slot, dst_slot, n_rows ? pick_slices(n_rows, vocab) : 1,
                (unsigned long long *)ws};
  const int more = logits ? (int)(((long long)n_rows + 63) / 64) : 0;
  if (n_groups + (long long)more == 0) return A3_OK;           // (no trees, and the picks are given)
  A3_REQUIRE((long long)n_rows * a.slices < (1LL << 31) && (long long)n_groups + more < (1LL << 31), A3_ERR_UNSUPPORTED, "a3_tree_accept: too many rows");
  if (logits && n_rows)
    with_dtype(dtype, [&](auto e) {
      hipLaunchKernelGGL(pick_kernel<decltype(e)>, dim3((unsigned)(n_rows * a.slices)), dim3(kLpThreads), 0, (hipStream_t)stream, a);
    });
  hipLaunchKernelGGL(follow_kernel, dim3((unsigned)(n_groups + more)), dim3(256), 0, (hipStream_t)stream, a);
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
  a.max_slots = !n_slots ? 1 : max_slots < a.p.slots ? max_slots : a.p.slots;      // (none behind the table's end)
  a.set_size = set_size;
  a.row_bytes = layers->head_dim * (q8 ? 1 : elem_bytes(layers));
  a.q8 = q8;
  a.head_bytes = page_head_bytes(layers->format, elem_bytes(layers), layers->page_size, layers->head_dim);
  a.row_shift = __builtin_ctz((unsigned)(a.row_bytes / 16));
  a.slot_shift = 0;
  int size = 2;
  while (size < set_size) size *= 2;
  while (a.slot_shift < 8 - a.row_shift && (1 << a.slot_shift) < a.max_slots && (size << a.slot_shift) < kMoveSlots) ++a.slot_shift;
  a.heads = 256 >> (a.row_shift + a.slot_shift);
  a.groups = (layers->n_kv_heads + a.heads - 1) / a.heads;
  // (the runs may be shorter than max_slots says: some workgroups that go on along them, not one for each piece that there might be)
  const long long tiles = ((long long)a.max_slots + (1 << a.slot_shift) - 1) >> a.slot_shift;
  for (int l0 = 0; l0 < n_layers; l0 += kLayersAtOnce) {
    const int n = n_layers - l0 < kLayersAtOnce ? n_layers - l0 : kLayersAtOnce;
    for (int l = 0; l < n; ++l) {
      a.pools[2 * l] = (char *)layers[l0 + l].k_pool;
      a.pools[2 * l + 1] = (char *)layers[l0 + l].v_pool;
    }
    a.units = 2 * n * a.groups;
    const long long gx = tiles < kMoveGroups ? tiles : kMoveGroups, others = gx * n_sets, want = (kMoveGroups + others - 1) / others;
    const dim3 grid((unsigned)gx, (unsigned)n_sets, (unsigned)(a.units < want ? a.units : want));
    auto launch = [&](auto size) { hipLaunchKernelGGL(move_kernel<size.value>, grid, dim3(256), 0, (hipStream_t)stream, a); };
    if (size == 2) launch(std::integral_constant<int, 2>{});
    else if (size == 4) launch(std::integral_constant<int, 4>{});
    else if (size == 8) launch(std::integral_constant<int, 8>{});
    else if (size == 16) launch(std::integral_constant<int, 16>{});
    else if (size == 32) launch(std::integral_constant<int, 32>{});
    else launch(std::integral_constant<int, 64>{});
    A3_CHECK_LAUNCH("a3_paged_move");
  }
  return A3_OK;
}

extern "C" size_t a3_beam_select_ws_bytes(int n_groups, int n_beams, int vocab, int n_best) {
  if (n_groups < 0 || n_beams < 1 || n_beams > kMaxBeams || vocab <= 0 || n_best < 1 || n_best > kMaxBest) return 0;
  // (r rows are r min(s, ceil(1024 / r)) pieces at most: below 1024 + r, and r from r = 1024 on)
  const size_t rows = (size_t)n_groups * n_beams, s = beam_slices(1, n_beams, vocab, 4), r = rows < kBeamPieces ? rows : kBeamPieces - 1;
  const size_t some = r * s < kBeamPieces + r ? r * s : kBeamPieces + r;
  return beam_ws(rows > some ? rows : some, n_best, nullptr, nullptr) + 256;
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
  const int rows = n_groups * n_beams;
  beam_args a{logits, ld, vocab, n_beams, n_best, end_token, beam_slices(rows, n_beams, vocab, dtype == A3_BF16 ? 2 : 4), score, done, best_score,
              best_row, best_token, nullptr, nullptr};
  beam_ws((size_t)rows * a.slices, n_best, ws, &a);
  with_dtype(dtype, [&](auto e) {
    hipLaunchKernelGGL(beam_row_kernel<decltype(e)>, dim3((unsigned)(rows * a.slices)), dim3(kLpThreads), 0, (hipStream_t)stream, a);
  });
  static a3_once_per_device lds_once;
  if (a3_once(lds_once, [&]() {
        return hipFuncSetAttribute((const void *)beam_join_kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)(kMaxBest * kMaxBest * sizeof(candidate)));
      }) != hipSuccess)
    return a3_fail(A3_ERR_HIP, "a3_beam_select: cannot raise the dynamic LDS limit");
  hipLaunchKernelGGL(beam_join_kernel, dim3((unsigned)n_groups), dim3(256), (size_t)n_best * n_best * sizeof(candidate), (hipStream_t)stream, a);
  A3_CHECK_LAUNCH("a3_beam_select");
  return A3_OK;
}
