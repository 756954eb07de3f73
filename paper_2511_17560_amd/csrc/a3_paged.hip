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
// Bound by memory for a prompt (16448 rows of 8 KV heads x 128, 135 MB in and out: 29 us, 4.6 TB/s; a copy reaches 5.35; into 8-bit pages,
// 102 MB, 33 us, 3.1 TB/s), by the chain slot - page - store for a step's rows (1 row of 8 KV and 32 query heads 2.7 us; 32 rows into
// 8-bit pages 4.8).
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
    if (rotate) code = q8_codes(y, scale);
    else code = q8_codes(x, scale);
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

// A step of a workgroup is 4 SK slots of one (row, KV head), SK a wave: 32, or 16 with fp32 pages.  The steps of the call, rows first, then
// KV heads, then slots, are cut into as many runs, equal to one step, as there are workgroups, whatever the lengths are: every workgroup
// forms the running sum of the rows' steps itself (lengths live on the device).  An item (row, KV head) that ends up whole in
// one workgroup is finished there; of one that is cut, every workgroup leaves a piece in ws and a second kernel joins them.
//
// Matrix instructions, operands straight from memory to registers, no LDS: S^T = K Q^T puts the query heads of the KV head (16
// columns) beside the slots (rows), and O^T = V^T P^T wants of a lane 8 consecutive slots of one coordinate.
//   - which slot a row of S^T is, is free: row i of block b is slot 8 (i / 4) + 4 b + i % 4, so that the weights a lane (column
//     l16, lane group lg) gets are those of slots 8 lg .. 8 lg + 7, the P^T operand as it stands
//   - which coordinate a row of O^T is, is free too: row l16 of block c is coordinate E l16 + c, so that a lane loads E consecutive
//     coordinates of its 8 slots (a row of the page in 16 lanes) and the V^T operands are a transposition inside the lane
//   - the weights go in as a sum of two bf16 (three where rows are fp32): the matrix pipe is idle most of the time, and the
//     only rounding of bf16 size is then the output's; each part but the last is cut off below the weight, so that none is
//     zero or negative and an infinite value stays one
//   - codes of 8-bit pages are whole numbers that bf16 holds; the scales join the logits and the weights
// The maximum that exponentials refer to moves only when a logit exceeds it by 8 (2^8 is far from any limit of a float): a
// comparison a slab instead of a reduction over lanes.
//
// Bound by HBM; both kernels, 8 KV heads x 128: 64 requests of 32K tokens 1224 us (8.6 GB, 7.0 TB/s), 8 of 64K 317 (6.8 TB/s; 8-bit pages 180,
// 6.2), 128 of 4096 (4 KV heads) 161 (6.7); 8 KV heads x 64: 16 of 16K with fp32 pages 165 (6.5), with fp32 rows over 8-bit pages 69 (4.1).
// About 10 us of a call are not: the start (lengths, page numbers, first slabs: 5 us) and the join (5 us); one request of 16K tokens takes
// 21 us, of 500 12.  Two workgroups of four waves a compute unit, 16 KB a wave on its way (one
// workgroup, or four half as long: up to 40 % and 15 % slower).
struct attend_args {
  pages_args p;
  const void *q;
  void *out;
  const int *row_req, *row_len;
  int n_rows, shares;
  float scale;             // of the logits, in units of log 2
  float *part_o;           // [2 * shares, G, D] pieces: 2 w the one that began before workgroup w, 2 w + 1 the one that goes on after it
  float2 *part_ml;         // [2 * shares, G] (maximum, sum)
  int *part_seen;          // [2 * shares] whether the piece has a slot at all
  int2 *cut;               // [shares] the item that goes on after workgroup w (-1: none), and its pieces; or, with few items,
  int by_item;             // [items] the workgroup that item begins in, and its pieces
};

template <typename T, int D, bool Q8>
struct attend_form {
  static constexpr bool kF32 = sizeof(T) == 4 && !Q8;          // fp32 matrix instructions
  static constexpr int SK = kF32 ? 16 : 32;                    // slots of a wave's slab
  static constexpr int KB = SK / 16;                           // row blocks of S^T
  static constexpr int kRow = Q8 ? D : D * (int)sizeof(T);     // bytes of a slot
  static constexpr int NK = kRow / 64;                         // 16-byte loads of a lane and row block: bytes 64 s + 16 lg ..
  static constexpr int NS = SK / 4;                            // slots whose weights a lane has
  static constexpr int E = kF32 ? 4 : D / 16, NP = D / (16 * E);   // a lane's coordinates: 16 E j + E l16 .. + E - 1, j < NP
  static constexpr int kVWords = E * kRow / D / 4;             // 32-bit words of one of them
  static constexpr int kQParts = Q8 && sizeof(T) == 4 ? 3 : 1, kPParts = sizeof(T) == 4 ? 3 : 2;
  static constexpr int kStep = 4 * SK;
  static constexpr int kAhead = 1;                             // slabs on their way (8-bit pages with two: no faster)
};
// slots of a step by a3_pages (host and device agree through this)
constexpr int step_shift(int dtype, int format) { return dtype == A3_F32 && format == A3_PAGES_PLAIN ? 6 : 7; }

__device__ __forceinline__ int steps_of(const attend_args &a, int req, int len, int shift) {
  if (req < 0 || req >= a.p.n_req) return 0;
  len = min(len, a.p.slots);
  return len <= 0 ? 1 : ((len - 1) >> shift) + 1;                // (a row that sees nothing has its zeros written)
}
__device__ __forceinline__ int steps_of(const attend_args &a, int row, int shift) {
  return steps_of(a, a.row_req ? a.row_req[row] : row, a.row_len[row], shift);
}

// One number at a wave-uniform place of an array that no kernel in flight writes, by a scalar load: a vector load would be waited for
// together with all the slabs requested before it (they come back in order).
__device__ __forceinline__ int scalar_at(const int *p, size_t i) {
  return reinterpret_cast<const __attribute__((address_space(4))) int *>(reinterpret_cast<uintptr_t>(p))[i];
}

template <typename T, int D, bool Q8>
__global__ void __launch_bounds__(256, 2)
paged_attention_kernel(attend_args a) {
  using F = attend_form<T, D, Q8>;
  constexpr int SK = F::SK, kShift = SK == 16 ? 6 : 7, kOS = D + 4;
  static_assert(F::kStep == 1 << kShift, "step");
  __shared__ int scan[8], found[5];
  __shared__ float2 ml[4][16];
  __shared__ __align__(16) float os[4][16][kOS];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, lg = lane >> 4, G = a.p.Hq / a.p.Hkv, Hkv = a.p.Hkv;

  // ---- this workgroup's run of steps -----------------------------------------------------------------------
  // Up to 256 rows: one thread a row.  More: the rows' sum first, then blocks of 256 rows up to the one the run begins in.
  int st = tid < a.n_rows ? steps_of(a, tid, kShift) : 0, incl = a3_wave_prefix(st), sum = incl;
  if (a.n_rows > 256) {
    int mine = st;
    for (int r = tid + 256; r < a.n_rows; r += 256) mine += steps_of(a, r, kShift);
    sum = a3_wave_prefix(mine);
  }
  if (lane == 63) { scan[wave] = sum; scan[4 + wave] = incl; }
  __syncthreads();
  const int total = (scan[0] + scan[1] + scan[2] + scan[3]) * Hkv, w = blockIdx.x;
  const int each = total / a.shares, rest = total - each * a.shares;      // the first `rest` workgroups take one more
  const int first = w * each + min(w, rest), n_steps = each + (w < rest ? 1 : 0);
  if (n_steps == 0) {
    if (tid == 0 && !a.by_item) a.cut[w] = make_int2(-1, 0);
    return;
  }
  for (int r0 = 0, before = 0;;) {                             // before: steps of the rows in front of this block
    int base = before;
    for (int i = 0; i < wave; ++i) base += scan[4 + i];
    const int lo = (base + incl - st) * Hkv, hi = (base + incl) * Hkv;
    if (first >= lo && first < hi) {
      const int r = r0 + tid;
      found[0] = r;
      found[1] = first - lo;
      found[2] = st;
      found[3] = max(0, min(a.row_len[r], a.p.slots));
      found[4] = a.row_req ? a.row_req[r] : r;
    }
    before += scan[4] + scan[5] + scan[6] + scan[7];
    if (before * Hkv > first) break;
    r0 += 256;
    st = r0 + tid < a.n_rows ? steps_of(a, r0 + tid, kShift) : 0;
    incl = a3_wave_prefix(st);
    __syncthreads();
    if (lane == 63) scan[4 + wave] = incl;
    __syncthreads();
  }
  __syncthreads();

  // ---- where the workgroup stands: a step of a row's KV head (all scalar) ------------------------------------------
  struct place { int row, head, step, steps, len, req; };
  place now;
  now.row = __builtin_amdgcn_readfirstlane(found[0]);
  now.steps = __builtin_amdgcn_readfirstlane(found[2]);
  now.len = __builtin_amdgcn_readfirstlane(found[3]);
  now.req = __builtin_amdgcn_readfirstlane(found[4]);
  const int inside = __builtin_amdgcn_readfirstlane(found[1]);
  now.head = inside / now.steps;
  now.step = inside - now.head * now.steps;
  auto enter = [&](place &p) {                                 // another row's own numbers
    const int len = scalar_at(a.row_len, p.row);
    p.req = a.row_req ? scalar_at(a.row_req, p.row) : p.row;
    p.len = max(0, min(len, a.p.slots));
    p.steps = steps_of(a, p.req, len, kShift);
  };
  auto advance = [&](place &p) {
    if (++p.step < p.steps) return;
    p.step = 0;
    if (++p.head < Hkv) return;
    p.head = 0;
    do {
      if (++p.row >= a.n_rows) return;                         // (only behind the last step of all)
      enter(p);
    } while (p.steps == 0);
  };

  // ---- one slab of one wave in registers ------------------------------------------------------------------
  struct slab {
    uint4 k[F::KB][F::NK];
    uint32_t v[F::NS][F::NP][F::kVWords];
    f32x4 ks[Q8 ? 2 : 1], vs[Q8 ? 2 : 1];
    int n;                                                     // slots of it that are seen (0: nothing was loaded)
  };
  const size_t head_bytes = page_head_bytes(Q8 ? A3_PAGES_Q8 : A3_PAGES_PLAIN, sizeof(T), 1 << a.p.page_shift, D);
  uint32_t koff[F::KB], voff;
#pragma unroll
  for (int b = 0; b < F::KB; ++b) koff[b] = (SK == 16 ? l16 : 8 * (l16 >> 2) + 4 * b + (l16 & 3)) * F::kRow + 16 * lg;
  voff = (uint32_t)(F::NS * lg * F::kRow + F::kVWords * 4 * l16);
  auto load = [&](slab &s, const place &p) {
    const int slot = (p.step << kShift) + SK * wave;
    s.n = p.len - slot;
    if (s.n <= 0) { s.n = 0; return; }
    const int page = scalar_at(a.p.table, (size_t)p.req * a.p.max_pages + (slot >> a.p.page_shift));
    if (page < 0 || page >= a.p.n_pages) { s.n = 0; return; }
    const size_t block = ((size_t)page * Hkv + p.head) * head_bytes;
    const int at = slot & ((1 << a.p.page_shift) - 1);
    // a row reads every byte once: nontemporal (8 requests of 64K tokens 362 -> 326 us, 48 of 4000 79 -> 71; rows that name the
    // same request read its bytes again)
    const char *kb = a.p.k_pool + block + at * F::kRow, *vb = a.p.v_pool + block + at * F::kRow;
#pragma unroll
    for (int b = 0; b < F::KB; ++b)
#pragma unroll
      for (int i = 0; i < F::NK; ++i) s.k[b][i] = a3_nt_load(kb + koff[b] + 64 * i);
    if constexpr (Q8) {
      const char *sc = a.p.k_pool + block + ((size_t)D << a.p.page_shift) + 4 * at + 32 * lg;
      s.ks[0] = *reinterpret_cast<const f32x4 *>(sc);
      s.ks[1] = *reinterpret_cast<const f32x4 *>(sc + 16);
      sc += a.p.v_pool - a.p.k_pool;
      s.vs[0] = *reinterpret_cast<const f32x4 *>(sc);
      s.vs[1] = *reinterpret_cast<const f32x4 *>(sc + 16);
    }
#pragma unroll
    for (int i = 0; i < F::NS; ++i)
#pragma unroll
      for (int j = 0; j < F::NP; ++j) {
        typedef uint32_t words __attribute__((ext_vector_type(F::kVWords == 1 ? 1 : F::kVWords)));
        const words w = __builtin_nontemporal_load(reinterpret_cast<const words *>(vb + voff + i * F::kRow + j * 64 * F::kVWords));
#pragma unroll
        for (int u = 0; u < F::kVWords; ++u) s.v[i][j][u] = w[u];
      }
  };

  // ---- queries of the item: operand of S^T, 16 columns ----------------------------------------------------------------
  constexpr int NQ = F::kF32 ? F::NK : D / 32;
  f32x4 qf[F::kF32 ? NQ : 1];
  bf16x8 qb[F::kF32 ? 1 : F::kQParts][F::kF32 ? 1 : NQ];
  auto load_queries = [&](const place &p) {
    // (columns past G repeat the last head: nothing of them is stored)
    const T *q = (const T *)a.q + ((size_t)p.row * a.p.Hq + p.head * G + min(l16, G - 1)) * D;
    if constexpr (F::kF32) {
#pragma unroll
      for (int i = 0; i < NQ; ++i) qf[i] = *reinterpret_cast<const f32x4 *>(q + 16 * i + 4 * lg);
    } else {
#pragma unroll
      for (int i = 0; i < NQ; ++i) {
        const T *at = q + (Q8 ? 64 * (i >> 1) + 16 * lg + 8 * (i & 1) : 32 * i + 8 * lg);
        if constexpr (sizeof(T) == 2) {
          qb[0][i] = *reinterpret_cast<const bf16x8 *>(at);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) {                        // x as the sum of three bf16
            float x = at[e];
#pragma unroll
            for (int k = 0; k < F::kQParts; ++k) {
              const bf16_t h = a3_f2bf(x);
              qb[k][i][e] = h;
              x -= a3_bf2f(h);
              if (!(fabsf(x) < INFINITY)) x = 0.f;             // an infinity has no remainder
            }
          }
        }
      }
    }
  };

  // ---- running state of the item --------------------------------------------------------------------------
  f32x4 o[D / 16];
  float m, l;
  bool seen;
  auto clear = [&]() {
#pragma unroll
    for (int c = 0; c < D / 16; ++c) o[c] = f32x4{0.f, 0.f, 0.f, 0.f};
    m = -INFINITY;
    l = 0.f;
    seen = false;
  };

  auto compute = [&](slab &s) {
    if (s.n == 0) return;
    seen = true;
    f32x4 acc[F::KB];
#pragma unroll
    for (int b = 0; b < F::KB; ++b) acc[b] = f32x4{0.f, 0.f, 0.f, 0.f};
    if constexpr (F::kF32) {
#pragma unroll
      for (int i = 0; i < F::NK; ++i) {
        const f32x4 kf = __builtin_bit_cast(f32x4, s.k[0][i]);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[0] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[e], qf[i][e], acc[0], 0, 0, 0);
      }
    } else if constexpr (Q8) {
#pragma unroll
      for (int i = 0; i < F::NK; ++i)
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int b = 0; b < F::KB; ++b) {
            const uint32_t w[2] = {u ? s.k[b][i].z : s.k[b][i].x, u ? s.k[b][i].w : s.k[b][i].y};
            const bf16x8 kf = codes8(w);
#pragma unroll
            for (int k = 0; k < F::kQParts; ++k) acc[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qb[k][2 * i + u], acc[b], 0, 0, 0);
          }
    } else {
#pragma unroll
      for (int i = 0; i < F::NK; ++i)
#pragma unroll
        for (int b = 0; b < F::KB; ++b)
          acc[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, s.k[b][i]), qb[0][i], acc[b], 0, 0, 0);
    }
    float w[F::NS];
#pragma unroll
    for (int i = 0; i < F::NS; ++i) {
      w[i] = acc[i >> 2][i & 3] * a.scale;
      if constexpr (Q8) w[i] *= s.ks[i >> 2][i & 3];
    }
    if (s.n < SK) {                                            // the row ends in this slab: whatever lies behind counts nothing
#pragma unroll
      for (int i = 0; i < F::NS; ++i)
        if (F::NS * lg + i >= s.n) {
          w[i] = -INFINITY;
          if constexpr (Q8) s.vs[i >> 2][i & 3] = 0.f;
          else
#pragma unroll
            for (int j = 0; j < F::NP; ++j)
#pragma unroll
              for (int u = 0; u < F::kVWords; ++u) s.v[i][j][u] = 0u;
        }
    }
    float top = w[0];
#pragma unroll
    for (int i = 1; i < F::NS; ++i) top = fmaxf(top, w[i]);
    if (__any(top > m + 8.f)) {
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const float next = fmaxf(m, top), f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - next);
      m = next;
      l *= f;
#pragma unroll
      for (int c = 0; c < D / 16; ++c) o[c] *= f;
    }
    const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int i = 0; i < F::NS; ++i) {
      w[i] = __builtin_amdgcn_exp2f(w[i] - ref);
      l += w[i];
      if constexpr (Q8) w[i] *= s.vs[i >> 2][i & 3];
    }
    if constexpr (F::kF32) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int c = 0; c < D / 16; ++c)
          o[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(__builtin_bit_cast(float, s.v[i][c >> 2][c & 3]), w[i], o[c], 0, 0, 0);
    } else {
      bf16x8 pf[F::kPParts];
#pragma unroll
      for (int k = 0; k < F::kPParts; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (k == F::kPParts - 1) { pf[k][i] = a3_f2bf(w[i]); continue; }
          const uint32_t h = __builtin_elementwise_sub_sat(__float_as_uint(w[i]), 1u) & 0xffff0000u;
          pf[k][i] = __builtin_bit_cast(bf16_t, (unsigned short)(h >> 16));
          w[i] -= __uint_as_float(h);
        }
#pragma unroll
      for (int c = 0; c < D / 16; ++c) {
        uint32_t x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if constexpr (Q8)
            x[i] = pack_codes((float)(signed char)(s.v[2 * i][0][c >> 2] >> 8 * (c & 3)), (float)(signed char)(s.v[2 * i + 1][0][c >> 2] >> 8 * (c & 3)));
          else
            x[i] = __builtin_amdgcn_perm(s.v[2 * i + 1][0][c >> 1], s.v[2 * i][0][c >> 1], c & 1 ? 0x07060302u : 0x05040100u);
        }
        const bf16x8 vf = __builtin_bit_cast(bf16x8, make_uint4(x[0], x[1], x[2], x[3]));
#pragma unroll
        for (int k = 0; k < F::kPParts; ++k) o[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[k], o[c], 0, 0, 0);
      }
    }
  };

  // ---- an item, or this workgroup's part of one, is done: join the four waves -----------------------------------------------
  auto finish = [&](const place &p, bool begins, bool ends) {
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (lg == 0) ml[wave][l16] = make_float2(m, l);
    if (lane == 0) scan[wave] = seen;
    A3_LDS_BARRIER();
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < 4; ++w) top = fmaxf(top, ml[w][l16].x);
    const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top);
    if (l16 < G) {
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int j = 0; j < F::NP; ++j)
#pragma unroll
          for (int c = 0; c < F::E; c += 4) {
            const int b = j * F::E + c;
            *reinterpret_cast<f32x4 *>(&os[wave][l16][16 * F::E * j + F::E * (4 * lg + r) + c]) =
                f32x4{o[b][r], o[b + 1][r], o[b + 2][r], o[b + 3][r]} * f;
          }
    }
    const bool any = scan[0] | scan[1] | scan[2] | scan[3];
    A3_LDS_BARRIER();
    const bool whole = begins && ends;
    const int slot = 2 * blockIdx.x + (begins ? 1 : 0);
    for (int e = tid; e < G * (D / 4); e += 256) {
      const int g = e / (D / 4), d = 4 * (e % (D / 4));
      f32x4 sum = {0.f, 0.f, 0.f, 0.f};
      float M = -INFINITY, L = 0.f;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        sum += *reinterpret_cast<const f32x4 *>(&os[w][g][d]);
        M = fmaxf(M, ml[w][g].x);
      }
#pragma unroll
      for (int w = 0; w < 4; ++w) L += ml[w][g].x == -INFINITY ? 0.f : ml[w][g].y * __builtin_amdgcn_exp2f(ml[w][g].x - M);
      if (whole) {
        typedef T vec4 __attribute__((ext_vector_type(4)));
        vec4 y;
#pragma unroll
        for (int u = 0; u < 4; ++u) y[u] = (T)(any ? sum[u] / L : 0.f);
        *reinterpret_cast<vec4 *>((T *)a.out + ((size_t)p.row * a.p.Hq + p.head * G + g) * D + d) = y;
      } else {
        *reinterpret_cast<f32x4 *>(a.part_o + ((size_t)slot * G + g) * D + d) = sum;
        if (d == 0) a.part_ml[(size_t)slot * G + g] = make_float2(M, L);
      }
    }
    if (!whole && tid == 0) a.part_seen[slot] = any;
    A3_LDS_BARRIER();
  };

  // ---- the run of steps: the next slabs are on their way while one is worked on ---------------------------------------
  slab ring[F::kAhead + 1];
  place ahead = now;
  bool begins = now.step == 0;
#pragma unroll
  for (int k = 0; k < F::kAhead; ++k)
    if (k < n_steps) {
      if (k > 0) advance(ahead);
      load(ring[k], ahead);
    }
  load_queries(now);
  clear();
  int cut_item = -1, cut_pieces = 0;
  auto step = [&](int i, slab &cur, slab &new_one) {
    if (i + F::kAhead < n_steps) {
      advance(ahead);
      load(new_one, ahead);
    }
    __builtin_amdgcn_sched_barrier(0);
    compute(cur);
    const bool ends = now.step == now.steps - 1, more = i + 1 < n_steps;
    if (!ends && more) {
      ++now.step;
      return;
    }
    place next = now;
    if (more) {
      advance(next);
      load_queries(next);                                      // on their way while the item is put together
    }
    finish(now, begins, ends);
    if (begins) {
      const int item = now.row * Hkv + now.head;
      int pieces = 1;
      if (!ends) {                                             // goes on in the workgroups behind: how many of them
        // (its last step is `last` of all: in a workgroup of the first `rest`, or behind them)
        const int last = first + i + now.steps - 1 - now.step, fat = rest * (each + 1);
        pieces += (last < fat ? last / (each + 1) : rest + (last - fat) / max(each, 1)) - w;
        cut_item = item;
        cut_pieces = pieces;
      }
      if (a.by_item && tid == 0) a.cut[item] = make_int2(w, pieces);
    }
    begins = true;
    clear();
    now = next;
  };
  constexpr int R = F::kAhead + 1;
  for (int i = 0; i < n_steps; i += R) {
#pragma unroll
    for (int k = 0; k < R; ++k)
      if (i + k < n_steps) step(i + k, ring[k], ring[(k + F::kAhead) % R]);
  }
  if (tid == 0 && !a.by_item) a.cut[w] = make_int2(cut_item, cut_pieces);
}

// Joins the pieces of an item: of item blockIdx.x, query head blockIdx.y (few items), or of the one that goes on after workgroup
// blockIdx.x, as many of its heads' coordinates as there are threads.  A thread sums four coordinates over every kth piece, all
// loads of eight pieces on their way together; then the k partial sums are joined.  Nothing but latency, and as few waves to
// start as possible (1024 threads for each of 512 workgroups: 10 us, where this takes 5).
constexpr int kJoinThreads = 256;
__host__ __device__ inline int join_units(int by_item, int G, int D) {         // four coordinates each, of a workgroup
  return by_item || G * (D / 4) < kJoinThreads ? (by_item ? D / 4 : G * (D / 4)) : kJoinThreads;
}
template <typename T, int D>
__global__ void __launch_bounds__(kJoinThreads)
paged_attention_join_kernel(attend_args a) {
  __shared__ f32x4 os[kJoinThreads];
  __shared__ float2 mls[kJoinThreads];
  const int tid = threadIdx.x, G = a.p.Hq / a.p.Hkv, units = join_units(a.by_item, G, D), groups = kJoinThreads / units;
  const int2 cut = a.cut[blockIdx.x];
  int w = blockIdx.x, item = cut.x;
  const int n = cut.y;
  if (a.by_item) {
    item = blockIdx.x;
    w = cut.x;
    if (steps_of(a, item / a.p.Hkv, 30) == 0) return;          // a row that does not exist: `cut` says nothing
  }
  if (item < 0 || n < 2) return;
  const int gr = tid / units, v = tid - gr * units, u = blockIdx.y * units + v, g = u / (D / 4);
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;
  int seen = 0;
  constexpr int K = 8;
  if (gr < groups && g < G)
    for (int i = gr; i < n; i += K * groups) {
      f32x4 x[K];
      float2 ml[K];
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const int p = min(i + k * groups, n - 1), slot = p == 0 ? 2 * w + 1 : 2 * (w + p);
        x[k] = *reinterpret_cast<const f32x4 *>(a.part_o + (size_t)slot * G * D + 4 * u);
        ml[k] = a.part_ml[(size_t)slot * G + g];
        seen |= a.part_seen[slot];
      }
      float top = m;
#pragma unroll
      for (int k = 0; k < K; ++k) {
        if (i + k * groups >= n) ml[k].x = -INFINITY;
        top = fmaxf(top, ml[k].x);
      }
      const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top);
      o *= f;
      l *= f;
      m = top;
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const float f1 = ml[k].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml[k].x - top);
        // (by number, not by weight: a piece whose logits are all NaN has no maximum, and its NaN stays one times 0)
        if (i + k * groups < n) { o += x[k] * f1; l += ml[k].y * f1; }
      }
    }
  os[tid] = o;
  mls[tid] = make_float2(m, l);
  seen = __syncthreads_or(seen);
  if (gr != 0 || g >= G) return;
#pragma unroll 8
  for (int k = 1; k < groups; ++k) m = fmaxf(m, mls[k * units + v].x);
  o = f32x4{0.f, 0.f, 0.f, 0.f};
  l = 0.f;
#pragma unroll 8
  for (int k = 0; k < groups; ++k) {
    const float2 ml = mls[k * units + v];
    const float f = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml.x - m);
    o += os[k * units + v] * f;
    l += ml.y * f;
  }
  typedef T vec4 __attribute__((ext_vector_type(4)));
  vec4 y;
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] = (T)(seen ? o[e] / l : 0.f);
  *reinterpret_cast<vec4 *>((T *)a.out + ((size_t)(item / a.p.Hkv) * a.p.Hq + (item % a.p.Hkv) * G) * D + 4 * u) = y;
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

// Two workgroups on each of the 256 compute units, fewer where the page table has fewer steps than that.
constexpr int kMaxShares = 512;
static long long attend_steps(const a3_pages *P, int n_rows) {
  const int shift = step_shift(P->dtype, P->format);
  return (((long long)P->max_pages * P->page_size + (1 << shift) - 1) >> shift) * P->n_kv_heads * n_rows;
}
static int attend_shares(const a3_pages *P, int n_rows) {
  const long long steps = attend_steps(P, n_rows);
  return steps < kMaxShares ? (int)steps : kMaxShares;
}
// workspace of `shares` workgroups; base NULL: only its size
static size_t attend_ws(const a3_pages *P, int shares, void *base, attend_args *a) {
  const size_t G = P->n_q_heads / P->n_kv_heads, D = P->head_dim, n = (size_t)shares;
  a3_ws_cursor cur(base, 0);
  float *o = (float *)cur.take(2 * n * G * D * sizeof(float));
  float2 *ml = (float2 *)cur.take(2 * n * G * sizeof(float2));
  int *seen = (int *)cur.take(2 * n * sizeof(int));
  int2 *cut = (int2 *)cur.take(n * sizeof(int2));
  if (a) { a->part_o = o; a->part_ml = ml; a->part_seen = seen; a->cut = cut; }
  return cur.off;
}

extern "C" size_t a3_paged_attention_ws_bytes(const a3_pages *P, int n_rows) {
  if (check_pages(P, "a3_paged_attention_ws_bytes", false) != A3_OK || n_rows < 0) return 0;
  return attend_ws(P, attend_shares(P, n_rows > 0 ? n_rows : 1), nullptr, nullptr);
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
  A3_REQUIRE(attend_steps(P, n_rows) < (1LL << 31) - 1024 && (long long)n_rows * P->n_q_heads < (1LL << 31), A3_ERR_UNSUPPORTED,
             "a3_paged_attention: too many rows for a page table of this width");
  const int shares = attend_shares(P, n_rows), items = n_rows * P->n_kv_heads, G = P->n_q_heads / P->n_kv_heads;
  attend_args a{args_of(P), q, out, row_req, row_len, n_rows, shares,
                (float)((P->sm_scale != 0.f ? (double)P->sm_scale : 1.0 / sqrt((double)P->head_dim)) * 1.4426950408889634074)};
  const size_t need = attend_ws(P, shares, ws, &a);
  A3_REQUIRE(ws && a3_aligned16(ws) && ws_bytes >= need, A3_ERR_WORKSPACE, "a3_paged_attention: workspace %zu bytes (16-byte aligned), need %zu",
             ws ? ws_bytes : 0, need);
  a.by_item = items <= shares && items * G <= kMaxShares;
  const int units = join_units(a.by_item, G, P->head_dim);
  const dim3 join((unsigned)(a.by_item ? items : shares), (unsigned)((G * (P->head_dim / 4) + units - 1) / units));
  with_format(P, [&](auto elem, auto d, auto q8) {
    hipLaunchKernelGGL((paged_attention_kernel<decltype(elem), d.value, q8.value>), dim3((unsigned)shares), dim3(256), 0, (hipStream_t)stream, a);
    hipLaunchKernelGGL((paged_attention_join_kernel<decltype(elem), d.value>), join, dim3(kJoinThreads), 0, (hipStream_t)stream, a);
  });
  A3_CHECK_LAUNCH("a3_paged_attention");
  return A3_OK;
}
