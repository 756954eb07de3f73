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
  int shares, tiles;       // workgroups; most items of a (group, KV head)
  float *part_o;           // [2 * shares] pieces: 2 w the one that began before run w, 2 w + 1 the one that goes on after it; each the
                           // accumulators of an item's columns as the waves hold them
  float2 *part_ml;         // [2 * shares, columns] (maximum, sum; sum < 0: nothing seen)
  int4 *cut;               // of run w: the item that goes on after it (group or -1, KV head and item of it, w, its pieces); with few items, of
  int by_item;             // each: the same, w the run that it begins in
};

// The rows of a group are packed with the query heads of a KV head: column m = row * G + head of it.  An item is 16 NB WC columns of one
// (group, KV head): NB blocks of 16 a wave, WC waves beside each other; the other waves take further slots.  A step of a workgroup
// is WS SK slots, SK a wave: 32, or 16 with fp32 pages.  The steps of the call, groups first, then KV heads, then items, then slots, are cut
// into as many runs, equal to one step, as there are workgroups, whatever the lengths are: every workgroup forms the running sum of the
// groups' steps itself (they live on the device).  An item that ends up whole in one workgroup is finished there; of one that is cut, every
// workgroup leaves a piece in ws and a second kernel joins them in the order of the slots.
//
// Matrix instructions: S^T = K Q^T puts 16 columns beside the slots (rows), and O^T = V^T P^T wants of a lane 8 consecutive slots of one
// coordinate.
//   - which slot a row of S^T is, is free: row i of block b is slot 8 (i / 4) + 4 b + i % 4, so that the weights a lane (column l16, lane group
//     lg) gets are those of slots 8 lg .. 8 lg + 7, the P^T operand as it stands
//   - which coordinate a row of O^T is, is free too: row l16 of block c is coordinate E l16 + c, so that a lane loads E consecutive
//     coordinates of its 8 slots and the V^T operands are a transposition inside the lane, formed once for all NB blocks of columns
//   - the weights go in as a sum of two bf16 (three where rows are fp32), so that the only rounding of bf16 size is the output's; each
//     part but the last is cut off, not rounded, so that a remainder is never negative
//   - codes of 8-bit pages are whole numbers that bf16 holds; the scales join the logits and the weights
// The maximum that exponentials refer to moves only when a logit exceeds it by 8 (2^8 is far from any limit of a float), and to a whole
// number: what moves sums, and weights that wait, is then a power of two.
//
// What bounds it: memory, as long as the cache is read once for all columns; with more columns the half steps below (a slab of 32 slots
// costs a wave of 32 columns 48 matrix instructions and 180 others), in which the matrix unit is busy 38 % of the time and the vector unit 49 %: the
// rest are waits between two barriers that two waves a SIMD do not fill.
// Registers: every form keeps 62 to 136 scalars in lanes of vector registers; bf16 of 128 with two blocks a wave (17 .. 32 columns) has seven vector
// registers too few, 32 bytes a lane in scratch.
//
// Up to 32 columns, up to 64 over 8-bit pages, and fp32 rows: K and V straight from memory to registers.  One slab of registers is enough to have the next one on its
// way: K of the next is asked for as soon as the products with this one's have read it, V as soon as its operands are formed, so that each
// is under way for most of a step.  Nothing of that is conditional (a slab that does not exist is read from the pool's start and counts
// nothing): a wait for V would otherwise have to be one for the next K too.
//
// More columns: the 16 slots that a quarter wave reads of K lie in as many lines, which occupies the address units four times as long as
// whole lines do, once for each of WC waves.  There K and V come through LDS, in whole lines, once for all of them, three steps ahead.  The
// two waves of a SIMD are half a step apart, with a barrier at each half: while one is at the matrix unit (V of its step before, K of this
// one), the other forms weights on the vector unit.
//
// Measured (one MI355X, bf16, 8 KV heads of 128, the whole call): 4 requests of 64K, 32 rows of 128 columns 261 us (4.1 TB/s; four waves of 64
// columns, PV of one step and QK of the next between the weights, 283; without the products 206, without the weights 210); 8 of 8K, 64 rows 127 us
// (0.49 PFLOP/s without the weights' second parts); 8 of 64K: 1 row 335 us (the single-token kernel 328), 4 rows 368, 8 rows 424, 16 rows 456.
//
// A lane's eight slots of a column are eight bits of the row's mask.  Only slabs that reach behind the committed slots look at it: a slot that
// is not seen has weight 0.  0 times a value that is not finite would be NaN in the rows that do not see it, so there such values are taken out
// of the product, and where there are any the rows that see them get them when the item is put together (the result there is not finite
// whatever the weights are).
template <typename T, int D, bool Q8, int NB_, int WC_, int W_>
struct tree_form {
  static constexpr int NB = NB_, WC = WC_, W = W_, WS = W_ / WC_;
  static constexpr bool kF32 = sizeof(T) == 4 && !Q8;          // fp32 matrix instructions
  static constexpr int SK = kF32 ? 16 : 32;                    // slots of a wave's slab
  static constexpr int KB = SK / 16;                           // row blocks of S^T
  static constexpr int kRow = Q8 ? D : D * (int)sizeof(T);     // bytes of a slot
  static constexpr int NK = kRow / 64;                         // 16-byte loads of a lane and row block: bytes 64 s + 16 lg ..
  static constexpr int NS = SK / 4;                            // slots whose weights a lane has
  static constexpr int E = kF32 ? 4 : D / 16, NP = D / (16 * E);   // a lane's coordinates: 16 E j + E l16 .. + E - 1, j < NP
  static constexpr int kVWords = E * kRow / D / 4;             // 32-bit words of one of them
  static constexpr int kQParts = Q8 && sizeof(T) == 4 ? 3 : 1, kPParts = sizeof(T) == 4 ? 3 : 2;
  static constexpr int TC = 16 * NB * WC;                      // columns of an item
  static constexpr int kStep = WS * SK;
  static constexpr bool kOnce = WC_ == 1;                      // a cache is read once: nontemporal
  static constexpr int kBlocks = NB * D / 16;                  // accumulator blocks of a wave
  static constexpr bool kLds = sizeof(T) == 2 && WC_ > 2;      // through LDS: rings of K and V, and of scales, four steps each
  static constexpr int kHalf = SK * kRow, kKV = WS * kHalf, kScaleAt = 8 * kKV;
  static constexpr int kLoads = kRow / 32 >= WC ? kRow / 32 / WC : 1;          // direct-to-LDS loads of a wave, of K and of V, a step
  static constexpr int kPer = 2 * kLoads + (Q8 ? 1 : 0);
  static constexpr int kAtOnce = kLds ? 4 : kBlocks;           // blocks that half of the waves exchange at once, when waves are joined
  static constexpr int kRoomAt = kLds ? kScaleAt + (Q8 ? 8 * WS * 256 : 0) : 0;
  static constexpr int kLdsBytes = kRoomAt + (WS > 1 ? W_ / 2 * kAtOnce * 1024 : 16);
  static constexpr int kWaves = sizeof(T) == 4 && D == 128 && NB_ == 2 ? 1 : 2;             // a SIMD
};

// Steps of a group's item, and items of its KV heads (0 steps: nothing of the group is written).
struct group_work { int first, rows, req, len, end, steps, tiles; };
template <int STEP, int TC>
__device__ __forceinline__ group_work work_of(const tree_args &a, int start, int stop, int req, int len) {
  group_work w;
  w.first = start;
  w.rows = start < 0 || stop > a.n_rows || stop < start ? 0 : min(stop - start, a.max_rows);
  w.req = req;
  w.len = max(0, min(len, a.p.slots));
  w.end = (int)min((long long)w.len + w.rows, (long long)a.p.slots);
  w.steps = w.rows == 0 || req < 0 || req >= a.p.n_req ? 0 : (w.end - 1) / STEP + 1;
  w.tiles = (w.rows * (a.p.Hq / a.p.Hkv) + TC - 1) / TC;
  return w;
}

template <int N, class Fn>
__device__ __forceinline__ void each_of(Fn f) {               // f(0) .. f(N - 1), the numbers as constants
  if constexpr (N > 0) {
    each_of<N - 1>(f);
    f(std::integral_constant<int, N - 1>{});
  }
}

template <class F, typename T, int D, bool Q8>
__global__ void __launch_bounds__(64 * F::W, F::W == 4 ? F::kWaves : 1)
tree_attention_kernel(tree_args a) {
  constexpr int SK = F::SK, NB = F::NB, WS = F::WS, WC = F::WC, W = F::W;
  extern __shared__ __align__(16) unsigned char lds[];
  __shared__ int scan[2][W], found[6], odd_waves[W];
  __shared__ float2 ml[NB][W][16];
  __shared__ int sees[NB][W][16];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, lg = lane >> 4, G = a.p.Hq / a.p.Hkv, Hkv = a.p.Hkv, wc = wave % WC, wsl = wave / WC;

  // ---- this workgroup's run of steps -----------------------------------------------------------------------
  // Up to as many groups as threads: one thread a group.  More: the groups' sum first, then blocks of them up to the one the run begins in.
  struct bounds { int start, stop, req, len; };
  auto bounds_of = [&](int g) {
    return g < a.n_groups ? bounds{a.start[g], a.start[g + 1], a.req ? a.req[g] : g, a.len[g]} : bounds{0, 0, 0, 0};
  };
  auto steps_of = [&](const bounds &b) {
    const group_work w = work_of<F::kStep, F::TC>(a, b.start, b.stop, b.req, b.len);
    return w.steps * w.tiles;
  };
  bounds mine = bounds_of(tid);
  int st = steps_of(mine), incl = a3_wave_prefix(st), sum = incl;
  if (a.n_groups > 64 * W) {
    int all = st;
    for (int g = tid + 64 * W; g < a.n_groups; g += 64 * W) all += steps_of(bounds_of(g));
    sum = a3_wave_prefix(all);
  }
  if (lane == 63) { scan[0][wave] = sum; scan[1][wave] = incl; }
  __syncthreads();
  int total = 0;
#pragma unroll
  for (int i = 0; i < W; ++i) total += scan[0][i];
  total *= Hkv;
  // neighbouring runs, which may read the same slots for other columns, on one of the eight dies (workgroups are dealt out in turn)
  const int w = a.shares % 8 == 0 ? (int)(blockIdx.x % 8) * (a.shares / 8) + blockIdx.x / 8 : blockIdx.x;
  const int each = total / a.shares, rest = total - each * a.shares;      // the first `rest` workgroups take one more
  const int first = w * each + min(w, rest), n_steps = each + (w < rest ? 1 : 0);
  if (tid == 0 && !a.by_item) a.cut[w].x = -1;
  if (n_steps == 0) return;
  for (int g0 = 0, before = 0;;) {                             // before: steps of the groups in front of this block
    int base = before;
    for (int i = 0; i < wave; ++i) base += scan[1][i];
    const int lo = (base + incl - st) * Hkv, hi = (base + incl) * Hkv;
    if (first >= lo && first < hi) {
      found[0] = g0 + tid;
      found[1] = first - lo;
      found[2] = mine.start;
      found[3] = mine.stop;
      found[4] = mine.req;
      found[5] = mine.len;
    }
#pragma unroll
    for (int i = 0; i < W; ++i) before += scan[1][i];
    if (before * Hkv > first) break;
    g0 += 64 * W;
    mine = bounds_of(g0 + tid);
    st = steps_of(mine);
    incl = a3_wave_prefix(st);
    __syncthreads();
    if (lane == 63) scan[1][wave] = incl;
    __syncthreads();
  }
  __syncthreads();

  // ---- where the workgroup stands: a step of an item (all scalar) --------------------------------------------------
  struct place { int g, head, tile, step; group_work k; };
  auto at_lds = [&](int i) { return __builtin_amdgcn_readfirstlane(found[i]); };
  place now;
  now.g = at_lds(0);
  now.k = work_of<F::kStep, F::TC>(a, at_lds(2), at_lds(3), at_lds(4), at_lds(5));
  const int inside = at_lds(1);
  now.head = inside / (now.k.steps * now.k.tiles);
  now.tile = (inside - now.head * now.k.steps * now.k.tiles) / now.k.steps;
  now.step = inside % now.k.steps;
  auto advance = [&](place &p) {
    if (++p.step < p.k.steps) return;
    p.step = 0;
    if (++p.tile < p.k.tiles) return;
    p.tile = 0;
    if (++p.head < Hkv) return;
    p.head = 0;
    do {
      if (++p.g >= a.n_groups) return;                         // (only behind the last step of all)
      p.k = work_of<F::kStep, F::TC>(a, scalar_at(a.start, p.g), scalar_at(a.start, p.g + 1), a.req ? scalar_at(a.req, p.g) : p.g,
                                     scalar_at(a.len, p.g));
    } while (p.k.steps == 0);
  };
  auto slot_of = [&](const place &p) { return p.step * F::kStep + SK * wsl; };      // a wave's first slot

  // ---- the slabs that are asked for, ahead of the work -------------------------------------------------------------
  // Page numbers come 64 at a time into the lanes of a register (one at a time, each is a load that the next thing waits for).
  struct where { size_t block; int at, n; };                   // n: its slots up to the tree's end (<= 0: none of them counts)
  const size_t head_bytes = page_head_bytes(Q8 ? A3_PAGES_Q8 : A3_PAGES_PLAIN, sizeof(T), 1 << a.p.page_shift, D);
  constexpr int kNoPages = -(1 << 30);
  // What was asked for by now is there.  (The compiler's own waits would stand where the values are used, in the loops, and be for all
  // later loads too: it does not know of the direct-to-LDS ones.)
  auto wait_loads = [&]() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(0x0f70);                        // vmcnt(0)
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" ::: "memory");
  };
  place ahead = now;
  int ahead_left = n_steps, pages = 0, pages_from = kNoPages;
  auto look = [&]() {                                          // (behind the run: the pool's start)
    where x{0, 0, 0};
    if (ahead_left > 0) {
      const int slot = slot_of(ahead), last = (ahead.k.end - 1) >> a.p.page_shift, no = min(slot >> a.p.page_shift, last);
      if ((uint32_t)(no - pages_from) >= 64u) {
        pages = a.p.table[(size_t)ahead.k.req * a.p.max_pages + min(no + lane, last)];
        wait_loads();                                          // (here, not in every step)
        pages_from = no;
      }
      const int page = __builtin_amdgcn_readlane(pages, no - pages_from);
      if (slot < ahead.k.end && page >= 0 && page < a.p.n_pages) {
        x.block = ((size_t)page * Hkv + ahead.head) * head_bytes;
        x.at = slot & ((1 << a.p.page_shift) - 1);
        x.n = ahead.k.end - slot;
      }
      if (--ahead_left > 0) {
        const int g = ahead.g;
        advance(ahead);
        if (ahead.g != g) pages_from = kNoPages;
      }
    }
    return x;
  };

  // How many of the next ones need no more than a look at the lane that has their page's number.
  auto count_simple = [&]() {
    const int slot = slot_of(ahead), from = (int)((uint32_t)pages_from << a.p.page_shift), room = (int)((uint32_t)from + (64u << a.p.page_shift) - (uint32_t)slot);
    if (pages_from == kNoPages || slot < from || room <= 0) return 0;
    return min(min(ahead.k.steps - 1 - ahead.step, ahead_left - 1), (room - 1) / F::kStep + 1);
  };
  auto look_simply = [&]() {
    where x{0, 0, 0};
    const int slot = slot_of(ahead), page = __builtin_amdgcn_readlane(pages, (slot >> a.p.page_shift) - pages_from);
    const bool there = (uint32_t)page < (uint32_t)a.p.n_pages;
    x.block = there ? ((size_t)(uint32_t)page * (uint32_t)Hkv + ahead.head) * head_bytes : 0;
    x.at = there ? slot & ((1 << a.p.page_shift) - 1) : 0;
    x.n = there ? ahead.k.end - slot : 0;
    ++ahead.step;
    --ahead_left;
    return x;
  };

  // ---- one slab of one wave in registers: buffer loads, the page in four scalars, a lane's place in one register ---------------------
  const uint32_t koff = (SK == 16 ? l16 : 8 * (l16 >> 2) + (l16 & 3)) * F::kRow + 16 * lg;
  const uint32_t voff = (uint32_t)(F::NS * lg * F::kRow + F::kVWords * 4 * l16);
  uint4 sk[F::KB][F::NK];
  uint32_t sv[F::NS][F::NP][F::kVWords];
  f32x4 ks[Q8 ? 2 : 1], vs[Q8 ? 2 : 1];
  constexpr int kAux = F::kOnce ? 2 : 0;                       // nontemporal
  auto page_of = [&](const char *pool, const where &x) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(pool) + x.block, 0, (int)head_bytes, 0x00020000);
  };
  auto load_k = [&](const where &x) {
    const auto page = page_of(a.p.k_pool, x);
    const int at = x.at * F::kRow;
#pragma unroll
    for (int b = 0; b < F::KB; ++b)
#pragma unroll
      for (int i = 0; i < F::NK; ++i)
        sk[b][i] = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(page, koff + 4 * b * F::kRow + 64 * i, at, kAux));
    if constexpr (Q8) {
      const int sc = (D << a.p.page_shift) + 4 * x.at;
      ks[0] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(page, 32 * lg, sc, 0));
      ks[1] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(page, 32 * lg + 16, sc, 0));
    }
  };
  auto load_v = [&](const where &x) {
    const auto page = page_of(a.p.v_pool, x);
    const int at = x.at * F::kRow;
#pragma unroll
    for (int i = 0; i < F::NS; ++i)
#pragma unroll
      for (int j = 0; j < F::NP; ++j) {
        const uint32_t from = voff + i * F::kRow + j * 64 * F::kVWords;
        if constexpr (F::kVWords == 4) {
          const uint4 y = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(page, from, at, kAux));
          sv[i][j][0] = y.x; sv[i][j][1] = y.y; sv[i][j][2] = y.z; sv[i][j][3] = y.w;
        } else if constexpr (F::kVWords == 2) {
          const uint2 y = __builtin_bit_cast(uint2, __builtin_amdgcn_raw_buffer_load_b64(page, from, at, kAux));
          sv[i][j][0] = y.x; sv[i][j][1] = y.y;
        } else {
          sv[i][j][0] = __builtin_amdgcn_raw_buffer_load_b32(page, from, at, kAux);
        }
      }
    if constexpr (Q8) {
      const int sc = (D << a.p.page_shift) + 4 * x.at;
      vs[0] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(page, 32 * lg, sc, 0));
      vs[1] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(page, 32 * lg + 16, sc, 0));
    }
  };

  // ---- through LDS: the waves that share a slab bring equal parts of it, 1 KB a load, lane after lane 16 bytes ------------------------
  // 16-byte piece c of slot s of K lies at place c ^ key(s) of its row, so that the 16 slots a quarter wave reads at one place lie in all 64
  // banks once.  Step i of a run has place i % 4 of the rings.
  const uint32_t lds_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char *)lds;
  constexpr int kPieces = F::kRow / 16, kRows = 1024 / F::kRow, kHalfLoads = F::kRow / 32;     // pieces of a slot; slots of a load; loads of a slab
  auto key_of = [&](int s) { return ((s >> 3 & 3) << 2 | (s & 3)) >> (F::kRow == 256 ? 0 : F::kRow == 128 ? 1 : 2); };
  const int my_slot = 8 * (l16 >> 2) + (l16 & 3), my_key = key_of(my_slot);    // a lane's row of S^T in block 0 (4 more in block 1)
  uint32_t dma_k[F::kLds ? F::kLoads : 1], dma_v[F::kLds ? F::kLoads : 1];
  if constexpr (F::kLds) {
#pragma unroll
    for (int t = 0; t < F::kLoads; ++t) {
      const int s = (wc * F::kLoads + t) % kHalfLoads * kRows + lane / kPieces, c = lane % kPieces;
      dma_k[t] = (uint32_t)(s * F::kRow + 16 * (c ^ key_of(s)));
      dma_v[t] = (uint32_t)(s * F::kRow + 16 * c);
    }
  }
  // Inline assembly on purpose: the compiler then neither treats these as LDS writes (it would wait for all of them before every LDS
  // read) nor moves memory accesses across them; the waits for them are the explicit s_waitcnt below.
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  auto page_at = [&](const char *pool, size_t block) {
    const uint64_t p = (uint64_t)pool + block;
    return u32x4{(uint32_t)p, (uint32_t)(p >> 32) & 0xffffu, (uint32_t)head_bytes, 0x00020000u};
  };
  auto dma = [&](u32x4 page, uint32_t off, uint32_t at, uint32_t to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(to), "v"(off), "s"(page), "s"(at) : "memory");
  };
  uint32_t missing = 0;                                        // bit q: step t + q does not count (no page, behind the tree's end)
  struct request { u32x4 k, v, scales; uint32_t at, scale_at, to, to_scales; };
  auto request_of = [&](int i, const where &x) {               // step i (a wave has as many loads in every step)
    request r;
    r.k = page_at(a.p.k_pool, x.block);
    r.v = page_at(a.p.v_pool, x.block);
    r.at = (uint32_t)x.at * F::kRow;
    r.to = lds_base + wsl * F::kHalf + (i & 3) * F::kKV;
    if constexpr (Q8) {                                        // 64 scales, of which 32 are the slab's (behind the head's page: zeros)
      r.scales = page_at(wc & 1 ? a.p.v_pool : a.p.k_pool, x.block);
      r.scale_at = (uint32_t)(D << a.p.page_shift) + 4 * x.at;
      r.to_scales = lds_base + F::kScaleAt + ((wc & 1) * 4 + (i & 3)) * WS * 256 + wsl * 256;
    }
    missing = missing >> 1 | (x.n <= 0 ? 8u : 0u);
    return r;
  };
  auto ask_part = [&](const request &r, int t) {               // load t of kPer
    if (t < F::kLoads) {
      dma(r.k, dma_k[t], r.at, r.to + (wc * F::kLoads + t) % kHalfLoads * 1024);
    } else if (t < 2 * F::kLoads) {
      dma(r.v, dma_v[t - F::kLoads], r.at, r.to + 4 * F::kKV + (wc * F::kLoads + t - F::kLoads) % kHalfLoads * 1024);
    } else {
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, %3 offen lds" ::"s"(r.to_scales), "v"(4 * lane), "s"(r.scales),
                   "s"(r.scale_at) : "memory");
    }
  };
  auto ask = [&](const request &r) {
#pragma unroll
    for (int t = 0; t < F::kPer; ++t) ask_part(r, t);
  };

  // ---- the item's columns: their rows and the queries, operand of S^T ----------------------------------------------------
  constexpr int NQ = F::kF32 ? F::NK : D / 32;
  f32x4 qf[F::kF32 ? NB : 1][F::kF32 ? NQ : 1];
  bf16x8 qb[F::kF32 ? 1 : NB][F::kF32 ? 1 : F::kQParts][F::kF32 ? 1 : NQ];
  struct columns { int row[NB]; uint32_t mask[NB][2]; };       // rows of the group, the first two words of their masks
  columns col;
  auto load_queries = [&](const place &p, columns &col) {
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      // (columns past the last repeat it: nothing of them is stored)
      const int m = min(p.tile * F::TC + (wc * NB + nb) * 16 + l16, p.k.rows * G - 1);
      const int j = m / G;
      col.row[nb] = j;
      col.mask[nb][0] = col.mask[nb][1] = 0;
      if (a.mask) {
        const int *w = a.mask + (size_t)(p.k.first + j) * a.mask_words;
        col.mask[nb][0] = (uint32_t)w[0];
        if (a.mask_words > 1) col.mask[nb][1] = (uint32_t)w[1];
      }
      const T *q = (const T *)a.q + ((size_t)(p.k.first + j) * a.p.Hq + p.head * G + (m - j * G)) * D;
      if constexpr (F::kF32) {
#pragma unroll
        for (int i = 0; i < NQ; ++i) qf[nb][i] = *reinterpret_cast<const f32x4 *>(q + 16 * i + 4 * lg);
      } else {
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
          const T *at = q + (Q8 ? 64 * (i >> 1) + 16 * lg + 8 * (i & 1) : 32 * i + 8 * lg);
          if constexpr (sizeof(T) == 2) {
            qb[nb][0][i] = *reinterpret_cast<const bf16x8 *>(at);
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {                      // x as the sum of three bf16
              float x = at[e];
#pragma unroll
              for (int k = 0; k < F::kQParts; ++k) {
                const bf16_t h = a3_f2bf(x);
                qb[nb][k][i][e] = h;
                x -= a3_bf2f(h);
                if (!(fabsf(x) < INFINITY)) x = 0.f;           // an infinity has no remainder
              }
            }
          }
        }
      }
    }
  };
  // ---- running state of the item --------------------------------------------------------------------------
  f32x4 o[NB][D / 16];
  float m[NB], l[NB];
  int seen;                                                    // bit nb: the lane's column of block nb has seen a slot of the lane's
  bool odd;                                                    // a value that is not finite was taken out
  auto clear = [&]() {
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
      for (int c = 0; c < D / 16; ++c) o[nb][c] = f32x4{0.f, 0.f, 0.f, 0.f};
      m[nb] = -INFINITY;
      l[nb] = 0.f;
    }
    seen = 0;
    odd = false;
  };

  auto two_bf16 = [](float x, float y) {
    typedef bf16_t bf16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, bf16x2{a3_f2bf(x), a3_f2bf(y)});
  };

  // ---- parts of a step ----------------------------------------------------------------------------------------------
  typedef f32x4 logits[NB][F::KB];
  typedef uint32_t words4 __attribute__((ext_vector_type(4)));
  struct weights {                                             // two bf16 of a part in a word, or (fp32 pages) as they are
    words4 b[F::kF32 ? 1 : NB][F::kF32 ? 1 : F::kPParts];
    float f[F::kF32 ? NB : 1][F::kF32 ? 4 : 1];
  };
  struct slab_info { int slot, n; bool masked; };              // masked: it reaches behind the committed slots, or does not exist
  auto info_of = [&](const place &p, int n) {
    const int slot = slot_of(p);
    return slab_info{slot, n, n < SK || slot + SK > p.k.len};
  };

  // S^T of step i (its logits but for the scale)
  auto take_k = [&](int i) {
    if constexpr (F::kLds) {
      const unsigned char *slab = lds + (i & 3) * F::kKV + wsl * F::kHalf + my_slot * F::kRow;
#pragma unroll
      for (int x = 0; x < F::NK; ++x)
#pragma unroll
        for (int b = 0; b < F::KB; ++b) sk[b][x] = *reinterpret_cast<const uint4 *>(slab + (((4 * x + lg) ^ my_key) << 4) + 4 * b * F::kRow);
    }
    if constexpr (F::kLds && Q8) {
#pragma unroll
      for (int b = 0; b < 2; ++b)
        ks[b] = *reinterpret_cast<const f32x4 *>(lds + F::kScaleAt + (i & 3) * WS * 256 + wsl * 256 + 32 * lg + 16 * b);
    }
  };
  auto multiply_k_part = [&](logits &acc, int x) {             // with bytes 64 x .. of the slots
    if (x == 0)
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int b = 0; b < F::KB; ++b) acc[nb][b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int b = 0; b < F::KB; ++b) {
        const uint4 kk = sk[b][x];
        if constexpr (F::kF32) {
          const f32x4 kf = __builtin_bit_cast(f32x4, kk);
#pragma unroll
          for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) acc[nb][0] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[e], qf[nb][x][e], acc[nb][0], 0, 0, 0);
        } else if constexpr (Q8) {
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const uint32_t two[2] = {u ? kk.z : kk.x, u ? kk.w : kk.y};
            const bf16x8 kf = codes8(two);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
              for (int k = 0; k < F::kQParts; ++k)
                acc[nb][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qb[nb][k][2 * x + u], acc[nb][b], 0, 0, 0);
          }
        } else {
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
            acc[nb][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kk), qb[nb][0][x], acc[nb][b], 0, 0, 0);
        }
      }
  };
  auto scale_k = [&](logits &acc) {
    if constexpr (Q8) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int b = 0; b < 2; ++b) acc[nb][b] *= ks[b];
    }
  };
  auto multiply_k = [&](logits &acc, int i) {
    take_k(i);
#pragma unroll
    for (int x = 0; x < F::NK; ++x) multiply_k_part(acc, x);
    scale_k(acc);
  };

  // Bits of the lane's slots (t0 .. t0 + NS - 1 of the tree; committed ones below 0) that the row of block nb's column sees.
  auto seen_slots = [&](const place &p, int t0, int nb) -> uint32_t {
    constexpr uint32_t kAll = (1u << F::NS) - 1;
    if (t0 + F::NS <= 0) return kAll;
    const int top = p.k.end - p.k.len - t0;                    // slots in front of the tree's end
    uint32_t bits;
    if (a.mask) {
      const int lo = max(t0, 0), word = lo >> 5;
      uint32_t w0, w1;
      if (a.mask_words <= 2) {
        w0 = word == 0 ? col.mask[nb][0] : word == 1 ? col.mask[nb][1] : 0u;
        w1 = word == 0 ? col.mask[nb][1] : 0u;
      } else {
        const int *w = a.mask + (size_t)(p.k.first + col.row[nb]) * a.mask_words;
        w0 = word < a.mask_words ? (uint32_t)w[word] : 0u;
        w1 = word + 1 < a.mask_words ? (uint32_t)w[word + 1] : 0u;
      }
      bits = (uint32_t)(((uint64_t)w1 << 32 | w0) >> (lo & 31));
      if (t0 < 0) bits = (bits << -t0) | ((1u << -t0) - 1);
    } else {
      const int n = col.row[nb] + 1 - t0;
      bits = n >= F::NS ? kAll : n <= 0 ? 0u : (1u << n) - 1;
    }
    return bits & (top >= F::NS ? kAll : top <= 0 ? 0u : (1u << top) - 1);
  };
  uint32_t vis[NB];                                            // of the step at hand, where it is masked
  auto hide = [&](logits &acc, const place &p, const slab_info &in) {
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      vis[nb] = in.n <= 0 ? 0u : seen_slots(p, in.slot + F::NS * lg - p.k.len, nb);
      if (vis[nb]) seen |= 1 << nb;
#pragma unroll
      for (int i = 0; i < F::NS; ++i)
        if (!(vis[nb] >> i & 1)) acc[nb][i >> 2][i & 3] = -INFINITY;
    }
  };
  // The maximum moves where it has to.
  auto move_maximum = [&](const logits &acc) {
    float top[NB];
    bool far = false;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      top[nb] = acc[nb][0][0];
#pragma unroll
      for (int i = 1; i < F::NS; ++i) top[nb] = fmaxf(top[nb], acc[nb][i >> 2][i & 3]);
      far |= fmaf(top[nb], a.scale, -m[nb]) > 8.f;
    }
    if (__builtin_expect(__any(far), 0)) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        float t = ceilf(top[nb] * a.scale);
        t = fmaxf(t, __shfl_xor(t, 16));
        t = fmaxf(t, __shfl_xor(t, 32));
        const float up = fmaxf(m[nb], t), f = m[nb] == -INFINITY ? 0.f : ldexpf(1.f, (int)fmaxf(m[nb] - up, -1000.f));
        m[nb] = up;
        l[nb] *= f;
#pragma unroll
        for (int c = 0; c < D / 16; ++c) o[nb][c] *= f;
      }
    }
  };
  auto take_scales = [&](int i) {
    if constexpr (F::kLds && Q8) {
#pragma unroll
      for (int b = 0; b < 2; ++b)
        vs[b] = *reinterpret_cast<const f32x4 *>(lds + F::kScaleAt + (4 + (i & 3)) * WS * 256 + wsl * 256 + 32 * lg + 16 * b);
    }
  };
  auto weigh_two = [&](const logits &acc, weights &p, int nb, int q, bool masked) {    // the weights of block nb's slots 2 q and 2 q + 1
    const float ref = m[nb] == -INFINITY ? 0.f : -m[nb];
    float w[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int i = 2 * q + e;
      w[e] = __builtin_amdgcn_exp2f(fmaf(acc[nb][i >> 2][i & 3], a.scale, ref));
      l[nb] += w[e];
      if constexpr (Q8) w[e] = !masked || vis[nb] >> i & 1 ? w[e] * vs[i >> 2][i & 3] : 0.f;       // (behind the tree: any scale)
      if constexpr (F::kF32) p.f[nb][i] = w[e];
    }
    if constexpr (!F::kF32) {
      // (weights are finite or NaN, and a NaN here stays one without its lower half)
#pragma unroll
      for (int k = 0; k + 1 < F::kPParts; ++k) {
        uint32_t x = __builtin_amdgcn_perm(__float_as_uint(w[1]), __float_as_uint(w[0]), 0x07060302u);
        if constexpr (F::kLds) asm volatile("" : "+v"(x));     // (here, not where it is used)
        p.b[nb][k][q] = x;
#pragma unroll
        for (int e = 0; e < 2; ++e) w[e] -= __uint_as_float(__float_as_uint(w[e]) & 0xffff0000u);
      }
      uint32_t x = two_bf16(w[0], w[1]);
      if constexpr (F::kLds) asm volatile("" : "+v"(x));
      p.b[nb][F::kPParts - 1][q] = x;
    }
  };
  auto weigh = [&](const logits &acc, weights &p, int i, bool masked) {
    take_scales(i);
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int q = 0; q < F::NS / 2; ++q) weigh_two(acc, p, nb, q, masked);
  };
  // O^T += V^T P^T of step i
  auto take_v = [&](int i) {
    if constexpr (F::kLds) {
      const unsigned char *slab = lds + (4 + (i & 3)) * F::kKV + wsl * F::kHalf + voff;
#pragma unroll
      for (int x = 0; x < F::NS; ++x) {
        typedef uint32_t words __attribute__((ext_vector_type(F::kVWords)));
        const words y = *reinterpret_cast<const words *>(slab + x * F::kRow);
#pragma unroll
        for (int u = 0; u < F::kVWords; ++u) sv[x][0][u] = y[u];
      }
    }
  };
  auto clean_v = [&](const slab_info &in, int len) {           // of a masked slab
    if constexpr (!Q8) {
      uint32_t bad = 0;                                        // the top bit of a half (bf16) or of all: an exponent of ones
#pragma unroll
      for (int i = 0; i < F::NS; ++i) {
        const bool none = F::NS * lg + i >= in.n;              // behind the tree: anything
#pragma unroll
        for (int j = 0; j < F::NP; ++j)
#pragma unroll
          for (int u = 0; u < F::kVWords; ++u) {
            if (none) sv[i][j][u] = 0u;
            bad |= sizeof(T) == 4 ? (sv[i][j][u] & 0x7f800000u) + 0x00800000u : (sv[i][j][u] & 0x7f807f80u) + 0x00800080u;
          }
      }
      if (__builtin_expect(__any(bad & (sizeof(T) == 4 ? 0x80000000u : 0x80008000u)), 0)) {
#pragma unroll
        for (int i = 0; i < F::NS; ++i) {
          if (in.slot + F::NS * lg + i < len) continue;        // (every row sees the committed ones)
#pragma unroll
          for (int j = 0; j < F::NP; ++j)
#pragma unroll
            for (int u = 0; u < F::kVWords; ++u) {
              uint32_t x = sv[i][j][u];
              if constexpr (sizeof(T) == 4) {
                if ((x & 0x7f800000u) == 0x7f800000u) { x = 0u; odd = true; }
              } else {
                if ((x & 0x7f80u) == 0x7f80u) { x &= 0xffff0000u; odd = true; }
                if ((x & 0x7f800000u) == 0x7f800000u) { x &= 0xffffu; odd = true; }
              }
              sv[i][j][u] = x;
            }
        }
      }
    }
  };
  auto v_operand = [&](int c) {                                // coordinates of block c (bf16)
    uint32_t x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (Q8)
        x[i] = pack_codes((float)(signed char)(sv[2 * i][0][c >> 2] >> 8 * (c & 3)), (float)(signed char)(sv[2 * i + 1][0][c >> 2] >> 8 * (c & 3)));
      else
        x[i] = __builtin_amdgcn_perm(sv[2 * i + 1][0][c >> 1], sv[2 * i][0][c >> 1], c & 1 ? 0x07060302u : 0x05040100u);
    }
    return words4{x[0], x[1], x[2], x[3]};
  };
  auto multiply_v_part = [&](const weights &p, const words4 &v, int c) {
#pragma unroll
    for (int k = 0; k < F::kPParts; ++k)
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
        o[nb][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, v), __builtin_bit_cast(bf16x8, p.b[nb][k]), o[nb][c], 0, 0, 0);
  };
  auto multiply_v = [&](const weights &p) {
    if constexpr (F::kF32) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int c = 0; c < D / 16; ++c)
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
            o[nb][c] = __builtin_amdgcn_mfma_f32_16x16x4f32(__builtin_bit_cast(float, sv[i][c >> 2][c & 3]), p.f[nb][i], o[nb][c], 0, 0, 0);
    } else {
#pragma unroll
      for (int c = 0; c < D / 16; ++c) multiply_v_part(p, v_operand(c), c);
    }
  };

  // Rare: the values that are not finite, of the tree's slots that a column's row sees, decide its result there, whatever the sums are (of
  // several pieces each gets them all).  A wave's columns once more, after they have been written.
  auto piece_at = [&](int slot, int nb, int c) { return a.part_o + ((size_t)slot * F::TC * D + ((wc * NB + nb) * (D / 16) + c) * 256 + 4 * lane); };
  auto write_odd = [&](const place &p, bool whole, int slot) {
    for (int e = 0; e < F::kBlocks * 4; ++e) {
      const int nb = e / (D / 4), c = e / 4 % (D / 16), r = e & 3, at = p.tile * F::TC + (wc * NB + nb) * 16 + l16;
      const int d = 16 * F::E * (c / F::E) + F::E * (4 * lg + r) + c % F::E;
      if (at >= p.k.rows * G) continue;
      const int j = at / G;
      float sum = 0.f;
      for (int s = p.k.len; s < p.k.end; ++s) {
        const int page = a.p.table[(size_t)p.k.req * a.p.max_pages + (s >> a.p.page_shift)], t = s - p.k.len;
        if (page < 0 || page >= a.p.n_pages) continue;
        if (a.mask ? !(a.mask[(size_t)(p.k.first + j) * a.mask_words + (t >> 5)] >> (t & 31) & 1) : t > j) continue;
        const T *v = (const T *)(a.p.v_pool + ((size_t)page * Hkv + p.head) * head_bytes) + (size_t)(s & ((1 << a.p.page_shift) - 1)) * D;
        const float x = (float)v[d];
        if (!(fabsf(x) < INFINITY)) sum += x;
      }
      if (fabsf(sum) < INFINITY) continue;
      if (whole) ((T *)a.out)[((size_t)(p.k.first + j) * a.p.Hq + p.head * G + (at - j * G)) * D + d] = (T)sum;
      else piece_at(slot, nb, c)[r] = sum;
    }
  };

  // ---- an item, or this workgroup's part of one, is done: join the waves that share columns ---------------------------------
  // Every wave brings its sums to the columns' common maximum; then half of the waves add those of the other half to their own, block by block as
  // the registers hold them, until one wave of each has all.
  auto finish = [&](const place &p, bool begins, bool ends) {
    const bool whole = begins && ends;
    const int slot = 2 * w + (begins ? 1 : 0), some_odd = __any(odd);
    if (WS > 1 && lane == 0) odd_waves[wave] = some_odd;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      l[nb] += __shfl_xor(l[nb], 16);
      l[nb] += __shfl_xor(l[nb], 32);
      int any = seen >> nb & 1;
      any |= __shfl_xor(any, 16);
      any |= __shfl_xor(any, 32);
      if (lg == 0) { ml[nb][wave][l16] = make_float2(m[nb], l[nb]); sees[nb][wave][l16] = any; }
    }
    A3_LDS_BARRIER();
    float M[NB], L[NB];
    // (waves that all take the same slots have all seen the same values; with WS = 1 no barrier would keep a wave's next flag from these readers)
    int some[NB], odd_any = some_odd;
#pragma unroll
    for (int x = 0; x < W; ++x)
      if (WS > 1) odd_any |= odd_waves[x];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      M[nb] = -INFINITY;
      L[nb] = 0.f;
      some[nb] = 0;
#pragma unroll
      for (int x = 0; x < WS; ++x) M[nb] = fmaxf(M[nb], ml[nb][x * WC + wc][l16].x);
#pragma unroll
      for (int x = 0; x < WS; ++x) {
        const float2 y = ml[nb][x * WC + wc][l16];
        L[nb] += y.x == -INFINITY ? 0.f : y.y * __builtin_amdgcn_exp2f(y.x - M[nb]);
        some[nb] |= sees[nb][x * WC + wc][l16];
      }
      const float f = m[nb] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[nb] - M[nb]);
#pragma unroll
      for (int c = 0; c < D / 16; ++c) o[nb][c] *= f;
    }
    constexpr int kAtOnce = F::kAtOnce;
    auto room = [&](int q) { return lds + F::kRoomAt + q * kAtOnce * 1024 + 16 * lane; };      // of the qth of the waves that hand over
#pragma unroll
    for (int half = WS / 2; half >= 1; half /= 2)
#pragma unroll
      for (int b0 = 0; b0 < F::kBlocks; b0 += kAtOnce) {
        if (wsl >= half && wsl < 2 * half) {
          unsigned char *to = room((wsl - half) * WC + wc);
#pragma unroll
          for (int b = 0; b < kAtOnce; ++b) *reinterpret_cast<f32x4 *>(to + b * 1024) = o[(b0 + b) / (D / 16)][(b0 + b) % (D / 16)];
        }
        A3_LDS_BARRIER();
        if (wsl < half) {
          const unsigned char *from = room(wsl * WC + wc);
#pragma unroll
          for (int b = 0; b < kAtOnce; ++b) o[(b0 + b) / (D / 16)][(b0 + b) % (D / 16)] += *reinterpret_cast<const f32x4 *>(from + b * 1024);
        }
        if (half > 1 || b0 + kAtOnce < F::kBlocks) A3_LDS_BARRIER();
      }
    if constexpr (F::kLds) wait_loads();                       // the next item's queries, before there are stores to be waited for too
    if (wsl == 0) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const int in = (wc * NB + nb) * 16 + l16, at = p.tile * F::TC + in;  // the column's number in the item, and among the group's
        if (!whole) {                                          // as the registers hold them: whole lines
#pragma unroll
          for (int c = 0; c < D / 16; ++c) *reinterpret_cast<f32x4 *>(piece_at(slot, nb, c)) = o[nb][c];
          if (lg == 0) a.part_ml[(size_t)slot * F::TC + in] = make_float2(M[nb], some[nb] ? L[nb] : -1.f);
        } else if (at < p.k.rows * G) {
          const int j = at / G;
          T *out = (T *)a.out + ((size_t)(p.k.first + j) * a.p.Hq + p.head * G + (at - j * G)) * D;
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int c = 0; c < D / 16; c += F::E) {
              typedef T vec __attribute__((ext_vector_type(F::E)));
              vec y;
#pragma unroll
              for (int u = 0; u < F::E; ++u) y[u] = (T)(some[nb] ? o[nb][c + u][r] / L[nb] : 0.f);
              *reinterpret_cast<vec *>(out + 16 * c + F::E * (4 * lg + r)) = y;
            }
        }
      }
      if constexpr (!Q8) {
        if (__builtin_expect(odd_any, 0)) {
          __builtin_amdgcn_s_waitcnt(0);
          write_odd(p, whole, slot);
        }
      }
    }
  };
  // Which item goes on after this run, and in how many pieces.
  auto note_cut = [&](const place &p, bool ends, int t) {
    if (tid != 0) return;
    int pieces = 1;
    if (!ends) {                                               // goes on in the workgroups behind: how many of them
      // (its last step is `last` of all: in a workgroup of the first `rest`, or behind them)
      const int last = first + t + p.k.steps - 1 - p.step, fat = rest * (each + 1);
      pieces += (last < fat ? last / (each + 1) : rest + (last - fat) / max(each, 1)) - w;
    }
    if (a.by_item) a.cut[((size_t)p.g * Hkv + p.head) * a.tiles + p.tile] = make_int4(p.g, p.head, w, pieces);
    else if (!ends) a.cut[w] = make_int4(p.g, p.head | p.tile << 16, w, pieces);
  };

  // ---- the run of steps ------------------------------------------------------------------------------------------------
  bool begins = now.step == 0;
  clear();
  if constexpr (!F::kLds) {
    where next = look();
    load_queries(now, col);
    __builtin_amdgcn_sched_barrier(0);
    load_k(next);
    __builtin_amdgcn_sched_barrier(0);
    load_v(next);
    __builtin_amdgcn_sched_barrier(0);
    int n = next.n;
    for (int t = 0; t < n_steps; ++t) {
      next = look();
      const bool more = t + 1 < n_steps, ends = now.step == now.k.steps - 1, last = ends || !more;
      place p = now;
      if (!last) ++p.step;
      else if (more) advance(p);
      const slab_info in = info_of(now, n);
      logits acc;
      weights wt;
      columns col_next;
      multiply_k(acc, t);
      __builtin_amdgcn_sched_barrier(0);
      // (loads come back in order: the next item's queries in front of its first K, so that a wait for that K is one for them)
      if (last && more) load_queries(p, col_next);
      __builtin_amdgcn_sched_barrier(0);
      load_k(next);
      __builtin_amdgcn_sched_barrier(0);
      if (in.masked) hide(acc, now, in);
      else seen = (1 << NB) - 1;
      move_maximum(acc);
      weigh(acc, wt, t, in.masked);
      if (in.masked) clean_v(in, now.k.len);
      multiply_v(wt);
      __builtin_amdgcn_sched_barrier(0);
      load_v(next);
      __builtin_amdgcn_sched_barrier(0);
      n = next.n;
      if (last) {
        finish(now, begins, ends);
        if (begins) note_cut(now, ends, t);
        begins = true;
        clear();
        if (more) col = col_next;
      }
      now = p;
    }
  } else {
    // Two phases a step, a barrier behind each: products on the matrix unit (V of the step before, K of this one), then weights on the vector unit.
    // The two waves of a SIMD are a phase apart.
    const bool late = wsl == 1;
    int t = 0;
#pragma unroll 1
    for (int i = 0; i < 3; ++i) ask(request_of(i, look()));
    load_queries(now, col);
    wait_loads();
    request r = request_of(3, look());
    int simple = count_simple();
    A3_LDS_BARRIER();
    if (late) A3_LDS_BARRIER();
    logits acc;
    weights wt;
    words4 vt[D / 16];
    columns col_next = col;
    bool pending = false;
    auto end_phase = [&]() {
      __builtin_amdgcn_sched_barrier(0);
      A3_LDS_BARRIER();
      __builtin_amdgcn_sched_barrier(0);
    };
    for (;; ++t) {
      take_k(t);
      if (pending) {
        each_of<D / 16>([&](auto c) {
          multiply_v_part(wt, vt[c], c);
          each_of<F::kPer * (c + 1) / (D / 16) - F::kPer * c / (D / 16)>([&](auto i) { ask_part(r, F::kPer * c / (D / 16) + i); });
        });
      } else {
        ask(r);
      }
      __builtin_amdgcn_sched_barrier(0);
      take_v(t);
      take_scales(t);
#pragma unroll
      for (int x = 0; x < F::NK; ++x) multiply_k_part(acc, x);
      // (the compiler would else move products behind the barrier)
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
        for (int b = 0; b < F::KB; ++b) asm volatile("" : "+v"(acc[nb][b]));
#pragma unroll
        for (int c = 0; c < D / 16; ++c) asm volatile("" : "+v"(o[nb][c]));
      }
      end_phase();
      scale_k(acc);
      const slab_info in = info_of(now, missing & 1 ? 0 : now.k.end - slot_of(now));
      const bool last = now.step == now.k.steps - 1 || t + 1 == n_steps;
      if (in.masked) hide(acc, now, in);
      else seen = (1 << NB) - 1;
      move_maximum(acc);
      weigh(acc, wt, t, in.masked);
      if (in.masked) clean_v(in, now.k.len);
#pragma unroll
      for (int c = 0; c < D / 16; ++c) {
        vt[c] = v_operand(c);
        asm volatile("" : "+v"(vt[c]));
      }
      // K and V of step t + 1 are there (of this wave's loads; behind the barrier, of all)
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * F::kPer) : "memory");
      if (simple > 0) {
        r = request_of(t + 4, look_simply());
        --simple;
      } else {
        r = request_of(t + 4, look());
        simple = count_simple();
      }
      if (!last) {
        pending = true;
        ++now.step;
        end_phase();
        continue;
      }
      const bool more = t + 1 < n_steps, ends = now.step == now.k.steps - 1;
      place p = now;
      if (more) {
        advance(p);
        load_queries(p, col_next);
      }
#pragma unroll
      for (int c = 0; c < D / 16; ++c) multiply_v_part(wt, vt[c], c);
      if (!late) A3_LDS_BARRIER();                             // (the late waves' products)
      finish(now, begins, ends);
      if (begins) note_cut(now, ends, t);
      if (!more) break;
      if (late) A3_LDS_BARRIER();
      begins = true;
      pending = false;
      clear();
      col = col_next;
      now = p;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");           // (the memory that the last loads go to is another workgroup's next)
  }
}

// Joins the pieces of an item that is cut: of item blockIdx.x (by_item: few of them), or of the one that goes on after workgroup blockIdx.x,
// four accumulator blocks of 16 columns (blockIdx.y).  A wave sums every fourth piece, the loads of four pieces on their way together; then
// the four partial sums are joined.
template <class F, typename T, int D>
__global__ void __launch_bounds__(256)
tree_join_kernel(tree_args a) {
  constexpr int TC = F::TC, E = F::E;
  __shared__ f32x4 os[4][4][64];
  __shared__ float2 mls[4][16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, lg = lane >> 4, G = a.p.Hq / a.p.Hkv;
  int g, head, tile;
  if (a.by_item) {
    g = blockIdx.x / (a.p.Hkv * a.tiles);
    head = blockIdx.x / a.tiles % a.p.Hkv;
    tile = blockIdx.x % a.tiles;
  } else {
    const int4 c = a.cut[blockIdx.x];
    if (c.x < 0) return;
    g = c.x;
    head = c.y & 0xffff;
    tile = c.y >> 16;
  }
  const group_work k = work_of<1, TC>(a, a.start[g], a.start[g + 1], a.req ? a.req[g] : g, a.len[g]);
  if (k.steps == 0 || tile >= k.tiles) return;                 // (no such item: `cut` says nothing)
  const int4 c = a.cut[blockIdx.x];
  const int w = c.z, n = c.w, cb = blockIdx.y / (D / 64), c0 = blockIdx.y % (D / 64) * 4, at = tile * TC + cb * 16 + l16;
  if (n < 2 || tile * TC + cb * 16 >= k.rows * G) return;
  f32x4 o[4];
#pragma unroll
  for (int b = 0; b < 4; ++b) o[b] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = -1.f;                               // l < 0: nothing seen
  auto take = [](f32x4 (&o)[4], float &l, const f32x4 (&x)[4], float2 ml, float top) {
    if (ml.y < 0.f) return;
    const float f = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml.x - top);
#pragma unroll
    for (int b = 0; b < 4; ++b) o[b] += x[b] * f;              // (a piece whose logits are all NaN has no maximum, and its NaN stays one times 0)
    l = (l < 0.f ? 0.f : l) + ml.y * f;
  };
  constexpr int K = 4;
  for (int i = wave; i < n; i += 4 * K) {
    f32x4 x[K][4];
    float2 ml[K];
#pragma unroll
    for (int q = 0; q < K; ++q) {
      const int p = min(i + 4 * q, n - 1), slot = p == 0 ? 2 * w + 1 : 2 * (w + p);
      const float *from = a.part_o + ((size_t)slot * TC * D + (cb * (D / 16) + c0) * 256 + 4 * lane);
#pragma unroll
      for (int b = 0; b < 4; ++b) x[q][b] = *reinterpret_cast<const f32x4 *>(from + 256 * b);
      ml[q] = a.part_ml[(size_t)slot * TC + cb * 16 + l16];
    }
    float top = m;
#pragma unroll
    for (int q = 0; q < K; ++q) {
      if (i + 4 * q >= n) ml[q] = make_float2(-INFINITY, -1.f);
      top = fmaxf(top, ml[q].x);
    }
    const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top);
    if (!(l < 0.f)) {
#pragma unroll
      for (int b = 0; b < 4; ++b) o[b] *= f;
      l *= f;
    }
    m = top;
#pragma unroll
    for (int q = 0; q < K; ++q) take(o, l, x[q], ml[q], top);
  }
#pragma unroll
  for (int b = 0; b < 4; ++b) os[wave][b][lane] = o[b];
  if (lg == 0) mls[wave][l16] = make_float2(m, l);
  __syncthreads();
  if (wave != 0 || at >= k.rows * G) return;
#pragma unroll
  for (int q = 1; q < 4; ++q) m = fmaxf(m, mls[q][l16].x);
#pragma unroll
  for (int b = 0; b < 4; ++b) o[b] = f32x4{0.f, 0.f, 0.f, 0.f};
  l = -1.f;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const f32x4 x[4] = {os[q][0][lane], os[q][1][lane], os[q][2][lane], os[q][3][lane]};
    take(o, l, x, mls[q][l16], m);
  }
  const int j = at / G;
  T *out = (T *)a.out + ((size_t)(k.first + j) * a.p.Hq + head * G + (at - j * G)) * D + 16 * E * (c0 / E) + c0 % E;
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    typedef T vec4 __attribute__((ext_vector_type(4)));
    vec4 y;
#pragma unroll
    for (int u = 0; u < 4; ++u) y[u] = (T)(l < 0.f ? 0.f : o[u][r] / l);
    *reinterpret_cast<vec4 *>(out + E * (4 * lg + r)) = y;
  }
}

constexpr int kMaxRows = 1024;

// What a call runs in: blocks of columns a wave, waves beside each other, waves, workgroups at most.  No more columns than rows need, as each
// costs products.  33 .. 64 columns of bf16 rows, through LDS with a block a wave, or from registers with two and two waves beside each other: a
// tree of 16 over 16K 32 and 34 us, 48 ragged chains (up to 42 columns) 125 and 124, 8 requests of 64K 456 and 505; with 8-bit pages, whose codes
// every wave makes bf16 of, 32 requests of about 5K 157 and 111, of 8K 272 and 207.  From 65 columns on: 128 columns of 4 x 64K 260 and 351 us.
// fp32 rows have no LDS form: three (8-bit pages) or fp32 products a value leave the matrix unit the bound.
struct tree_shape { int nb, wc, waves, wgs; };
tree_shape shape_of(const a3_pages *P, int max_rows) {
  const int cols = max_rows * (P->n_q_heads / P->n_kv_heads);
  const bool wide = P->dtype == A3_F32 && P->head_dim == 128;  // (two blocks a wave: registers for one wave a SIMD)
  if (cols <= 16) return {1, 1, 4, 512};
  if (cols <= 32) return {2, 1, 4, wide ? 256 : 512};
  if (wide) return {2, 4, 4, 256};
  if (P->dtype == A3_F32) return {2, cols <= 64 ? 2 : 4, 8, 256};
  if (cols <= 64 && P->format == A3_PAGES_Q8) return {2, 2, 4, 512};
  return {cols <= 64 ? 1 : 2, 4, 8, 256};
}
template <typename T, int D, bool Q8, class F>
void with_shape(tree_shape s, F f) {
  if (s.nb == 1 && s.wc == 1) f(tree_form<T, D, Q8, 1, 1, 4>{});
  else if (s.wc == 1) f(tree_form<T, D, Q8, 2, 1, 4>{});
  else if constexpr (sizeof(T) == 4 && D == 128) f(tree_form<T, D, Q8, 2, 4, 4>{});
  else if constexpr (sizeof(T) == 4) {
    if (s.wc == 2) f(tree_form<T, D, Q8, 2, 2, 8>{});
    else f(tree_form<T, D, Q8, 2, 4, 8>{});
  }
  else if (s.nb == 2 && s.wc == 4) f(tree_form<T, D, Q8, 2, 4, 8>{});
  else if constexpr (Q8) f(tree_form<T, D, Q8, 2, 2, 4>{});
  else f(tree_form<T, D, Q8, 1, 4, 8>{});
}
struct tree_plan { tree_shape s; int tc, tiles, shares; long long items, steps; };
tree_plan plan_of(const a3_pages *P, int n_groups, int max_rows) {
  tree_plan p;
  p.s = shape_of(P, max_rows);
  p.tc = 16 * p.s.nb * p.s.wc;
  p.tiles = (max_rows * (P->n_q_heads / P->n_kv_heads) + p.tc - 1) / p.tc;
  const int step = p.s.waves / p.s.wc * (P->dtype == A3_F32 && P->format == A3_PAGES_PLAIN ? 16 : 32);
  p.items = (long long)n_groups * P->n_kv_heads * p.tiles;
  p.steps = ((long long)P->max_pages * P->page_size + step - 1) / step * p.items;
  p.shares = p.steps < p.s.wgs ? (int)p.steps : p.s.wgs;
  return p;
}
// workspace; base NULL: only its size
size_t tree_ws(const a3_pages *P, const tree_plan &p, void *base, tree_args *a) {
  a3_ws_cursor cur(base, 0);
  const size_t n = (size_t)p.shares;
  float *o = (float *)cur.take(2 * n * p.tc * P->head_dim * sizeof(float));
  float2 *ml = (float2 *)cur.take(2 * n * p.tc * sizeof(float2));
  int4 *cut = (int4 *)cur.take(n * sizeof(int4));
  if (a) { a->part_o = o; a->part_ml = ml; a->cut = cut; }
  return cur.off;
}

}  // namespace

extern "C" size_t a3_tree_attention_ws_bytes(const a3_pages *P, int n_groups, int max_rows) {
  if (check_pages(P, "a3_tree_attention_ws_bytes", false) != A3_OK || n_groups < 0 || max_rows < 1 || max_rows > kMaxRows) return 0;
  size_t most = 0;                                             // (fewer rows may take another shape, fewer groups fewer workgroups)
  const int G = P->n_q_heads / P->n_kv_heads;
  for (int cols : {16, 32, 64, 128, kMaxRows * 16}) {
    const int rows = cols / G < max_rows ? cols / G : max_rows;
    if (rows < 1) continue;
    const size_t n = tree_ws(P, plan_of(P, n_groups > 0 ? n_groups : 1, rows), nullptr, nullptr);
    most = n > most ? n : most;
  }
  return most;
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
  const tree_plan plan = plan_of(P, n_groups, max_rows);
  A3_REQUIRE(plan.steps < (1LL << 31) - 1024 && (long long)n_rows * P->n_q_heads < (1LL << 31), A3_ERR_UNSUPPORTED,
             "a3_tree_attention: too many groups for a page table of this width");
  a.shares = plan.shares;
  a.tiles = plan.tiles;
  a.by_item = plan.items <= plan.shares;
  tree_ws(P, plan, ws, &a);
  const dim3 join((unsigned)(a.by_item ? plan.items : plan.shares), (unsigned)(plan.tc / 16 * (P->head_dim / 64)));
  with_format(P, [&](auto elem, auto d, auto q8) {
    typedef decltype(elem) T;
    with_shape<T, d.value, q8.value>(plan.s, [&](auto form) {
      typedef decltype(form) F;
      auto kern = tree_attention_kernel<F, T, d.value, q8.value>;
      static a3_once_per_device lds_once;
      if (F::kLdsBytes > 65536 && a3_once(lds_once, [&]() {
            return hipFuncSetAttribute((const void *)kern, hipFuncAttributeMaxDynamicSharedMemorySize, F::kLdsBytes);
          }) != hipSuccess) {
        s = a3_fail(A3_ERR_HIP, "a3_tree_attention: cannot raise the dynamic LDS limit");
        return;
      }
      hipLaunchKernelGGL(kern, dim3((unsigned)plan.shares), dim3(64 * F::W), F::kLdsBytes, (hipStream_t)stream, a);
      hipLaunchKernelGGL((tree_join_kernel<F, T, d.value>), join, dim3(256), 0, (hipStream_t)stream, a);
    });
  });
  if (s != A3_OK) return s;
  A3_CHECK_LAUNCH("a3_tree_attention");
  return A3_OK;
}
