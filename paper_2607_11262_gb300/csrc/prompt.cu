// Attention of packed sequences over themselves with its gradient (gts_prompt_attention, gts_prompt_attention_grad), and of chunks of
// new tokens over a paged cache (gts_chunk_attention).
//
// Mathematics.  Query i of a sequence with n queries and m keys sees the keys j <= i + m - n (causal) or all.  With s_ij = scale *
// q_i . k_j, out_i = sum_j exp(s_ij - max) v_j / sum_j exp(s_ij - max), taken with the maximum and the sum so far.  Backward: with
// p_ij = exp(s_ij - lse_i), e_i = dout_i . out_i - dlse_i and ds_ij = p_ij (dout_i . v_j - e_i): dv_j = sum p_ij dout_i,
// dq_i = scale sum ds_ij k_j, dk_j = scale sum ds_ij q_i.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "internal.h"
#include "tensor.cuh"

namespace {

struct Heads { const void *data; int64_t tok, head; };

struct Args {
  Heads q, k, v, out, low, dout, dq, dk, dv;   // low: what rounding took from out
  float *lse, *delta;
  const float *dlse;
  const int32_t *starts, *lens, *table;
  int64_t k_page, v_page;
  int n_seqs, n_tokens, q_heads, kv_heads, group, causal, zero_rest, paged;
  int n_pages, page_size, max_pages;
  Divisor in_group, in_page;
  float scale;
  int32_t *status;
};

// Every wait ends: after two seconds, or when another warp has given up, the block winds down with an error status.
constexpr uint64_t LIMIT_NS = 2000000000ull, DRAIN_NS = 2000000000ull;   // of a wait; of what a block that winds down has in flight
constexpr int TRIES = 1024, BETWEEN = 64;   // before the timer is read first, and from then on (reading it takes longer than most waits)
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}"
               : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  return ok;
}
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, volatile int *dead) {
  if (bar_try(bar, parity)) return true;
#pragma unroll 1
  for (int n = 0; n < TRIES; n++)
    if (bar_try(bar, parity)) return true;
  const uint64_t from = now_ns();
#pragma unroll 1
  while (!*dead) {
#pragma unroll 1
    for (int n = 0; n < BETWEEN; n++)
      if (bar_try(bar, parity)) return true;
    if (now_ns() - from > LIMIT_NS) *dead = 1;
  }
  return false;
}

// ---------------------------------------------------------------- how the work is cut
// An item is a key head with a tile of rows of one sequence, or (the gradients of keys and values) a tile of 128 keys of it; it
// passes along its tiles of the other side.  All items stand in one line, key head by key head, sequence by sequence, each with a
// weight: what its tiles cost (one for each key or query seen) and what it costs beside them (LEAD of its tiles).  Each block takes an equal
// stretch of the line, rounded to whole tiles, so sequences of any lengths share the SMs evenly, a few rows over many keys are
// split along the keys, and the cut needs no plan from the host.  A sequence's weight up to an item is a sum of an arithmetic series, so a
// block finds its stretch by a sum over the sequences and a bisection.  An item within one block's stretch is finished there; one
// that is cut leaves partial results, which k_join adds up in their order.
constexpr int SMS = 152, TILE = 128, LEAD = 2;
constexpr int NOTHING = -1;

struct Cut {
  int blocks;
  int4 *ends;            // [blocks]: the item that begins in a block and goes on: sequence (or NOTHING), key head, item, further blocks
  float4 *o;             // [blocks][2][D / 4][rows of an item]: parts of the item that began before (0) and of the one that goes on (1)
  float2 *ml;            // [blocks][2][rows]: maximum (of log2 scores) and sum
};

struct Seq { int first, n, keys; };  // first row and number of its queries, and keys

__device__ __forceinline__ Seq sequence(const Args &a, int b) {
  const int from = a.starts[b], to = a.starts[b + 1];
  Seq s;
  s.first = max(0, min(from, a.n_tokens));
  s.n = max(s.first, min(to, a.n_tokens)) - s.first;     // (a difference of what lies within the call: starts may be any numbers)
  bool bad = from != s.first || to != s.first + s.n;
  s.keys = s.n;
  if (a.paged) {
    const int len = a.lens[b], most = a.max_pages * a.page_size;
    s.keys = max(0, min(len, most));
    bad |= len > most;
  }
  if (bad && a.status) *a.status = GTS_ERR_INVALID_PARAMS;
  return s;
}

// Items of rows (BY_KEYS false) and of keys: how many a sequence has, the tiles of one, its weight and that of all before it.
template <bool BY_KEYS> struct Items {
  int q, causal;         // queries of an item (of a tile of rows, by keys)
  int beside = LEAD;
  __device__ __forceinline__ int lead() const { return beside * (BY_KEYS ? q : TILE); }
  __device__ __forceinline__ int count(const Seq &s) const { return BY_KEYS ? (s.keys + TILE - 1) / TILE : (s.n + q - 1) / q; }
  // keys that the item's last query sees, or queries that see the item's first key (rounded to whole items)
  __device__ __forceinline__ int seen(const Seq &s, int t) const {
    if (BY_KEYS) return causal ? s.n - t * TILE : s.n;
    return causal ? max(0, s.keys - s.n + min(s.n, (t + 1) * q)) : s.keys;
  }
  __device__ __forceinline__ int first_tile(int t) const { return BY_KEYS && causal ? t * TILE / q : 0; }
  __device__ __forceinline__ int tiles(const Seq &s, int t) const {
    if (BY_KEYS) return (s.n + q - 1) / q - first_tile(t);
    return max(1, (seen(s, t) + TILE - 1) / TILE);
  }
  __device__ __forceinline__ int64_t weight(const Seq &s, int t) const { return (int64_t)lead() + seen(s, t); }
  __device__ __forceinline__ int64_t before(const Seq &s, int t) const {
    const int64_t x = t;
    if (!causal) return x * (lead() + (BY_KEYS ? s.n : s.keys));
    if (BY_KEYS) return x * ((int64_t)lead() + s.n) - x * (x - 1) / 2 * TILE;
    const int64_t off = (int64_t)s.keys - s.n, none = off < 0 ? min(x, -off / q) : 0;   // items that see nothing
    int64_t sum = x * lead() + (x - none) * off + (x * (x + 1) - none * (none + 1)) / 2 * q;
    if (x > none && x * q > s.n) sum -= x * q - s.n;
    return sum;
  }
  // tiles of an item up to a place in its weight
  __device__ __forceinline__ int tiles_before(int64_t y, int64_t weight, int tiles) const {
    if (y >= weight) return tiles;
    const int64_t in = y - lead() + (BY_KEYS ? q : TILE) / 2;
    return in <= 0 ? 0 : (int)min((int64_t)tiles, in / (BY_KEYS ? q : TILE));
  }
};

// The line of a call, and a block's walk along its stretch of it.
struct Stretch { int64_t head, all, per, x0, x1; int b, t; int64_t pos; int kh, rest_from, rest_to; };

// Where a block begins: every thread of it takes part.  rest_from, rest_to: rows of sequences are between them.  (`scratch`: SCRATCH bytes of shared memory)
constexpr int SCRATCH = 512;
template <bool BY_KEYS, int THREADS>
__device__ __forceinline__ Stretch find_stretch(const Args &a, const Items<BY_KEYS> &items, int blocks, void *scratch) {
  constexpr int WARPS = THREADS / 32;
  int64_t *const sums = (int64_t *)scratch, *const places = sums + WARPS;
  int (*const ends)[2] = (int (*)[2])(places + 1);
  int *const found = (int *)(ends + WARPS);
  static_assert(WARPS * 16 + 16 <= SCRATCH, "room for the sums");
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
  const int each = (a.n_seqs + THREADS - 1) / THREADS, from = min(a.n_seqs, tid * each), to = min(a.n_seqs, from + each);
  int64_t mine = 0;
  int first = a.n_tokens, last = 0;
  for (int b = from; b < to; b++) {
    const Seq s = sequence(a, b);
    if (s.n) first = min(first, s.first), last = max(last, s.first + s.n);
    mine += items.before(s, items.count(s));
  }
  int64_t upto = mine;
#pragma unroll
  for (int o = 1; o < 32; o *= 2) {
    const int64_t x = __shfl_up_sync(~0u, upto, o);
    if (lane >= o) upto += x;
  }
  first = __reduce_min_sync(~0u, first), last = __reduce_max_sync(~0u, last);
  if (lane == 31) sums[warp] = upto;
  if (lane == 0) ends[warp][0] = first, ends[warp][1] = last;
  if (tid == 0) found[0] = -1;
  __syncthreads();
  Stretch s = {};
  s.rest_from = a.n_tokens;
  int64_t earlier = 0;
#pragma unroll
  for (int w = 0; w < THREADS / 32; w++) {
    if (w < warp) earlier += sums[w];
    s.head += sums[w];
    s.rest_from = min(s.rest_from, ends[w][0]), s.rest_to = max(s.rest_to, ends[w][1]);
  }
  if (s.rest_to == 0) s.rest_from = 0;
  s.all = s.head * a.kv_heads;
  s.per = max((int64_t)items.lead(), quotient(s.all + blocks - 1, blocks));
  s.x0 = min(s.all, s.per * blockIdx.x), s.x1 = min(s.all, s.x0 + s.per);
  if (s.x0 >= s.x1) return s;
  s.kh = (int)quotient(s.x0, s.head);
  const int64_t in = s.x0 - s.kh * s.head;
  int64_t at = earlier + upto - mine;
  if (in >= at && in < at + mine) {
    for (int b = from; b < to; b++) {
      const Seq q = sequence(a, b);
      const int count = items.count(q);
      const int64_t w = items.before(q, count);
      if (in < at + w) {
        int lo = 0, hi = count - 1;                    // the last item that begins at `in` or before
        while (lo < hi) {
          const int mid = (lo + hi + 1) / 2;
          if (at + items.before(q, mid) <= in) lo = mid; else hi = mid - 1;
        }
        found[0] = b, found[1] = lo, places[0] = s.kh * s.head + at + items.before(q, lo);
        break;
      }
      at += w;
    }
  }
  __syncthreads();
  s.b = found[0], s.t = found[1], s.pos = places[0];
  if (s.b < 0) s.x0 = s.x1 = 0;                        // (sequences that overlap without end, from starts that fall: their sum may pass 64 bits)
  return s;
}

// What a block does with an item: its tiles from tile0 to tile1 of `tiles`.
struct Item { int b, first, n, keys, kh, t, tile0, tile1, tiles; };

// The next item of a stretch that has tiles in it; false at its end.  `ends`: where an item that goes on is recorded, by one thread.
template <bool BY_KEYS>
__device__ __forceinline__ bool next_item(const Args &a, const Items<BY_KEYS> &items, Stretch &s, Seq &q, Item &i, int4 *ends) {
  while (s.pos < s.x1) {
    if (s.t == 0 || i.b != s.b) q = sequence(a, s.b);
    const int64_t w = items.weight(q, s.t), end = s.pos + w;
    const int n = items.tiles(q, s.t);
    i = {s.b, q.first, q.n, q.keys, s.kh, s.t, s.pos < s.x0 ? items.tiles_before(s.x0 - s.pos, w, n) : 0,
         items.tiles_before(s.x1 - s.pos, w, n), n};
    if (ends && i.tile0 == 0 && i.tile1 > 0 && i.tile1 < n) {
      int64_t last = quotient(end - 1, s.per);
      if (items.tiles_before(last * s.per - s.pos, w, n) == n) last--;
      *ends = make_int4(s.b, s.kh, s.t, (int)(last - blockIdx.x));
    }
    s.pos = end;
    if (++s.t == items.count(q)) {
      s.t = 0;
      do {
        if (++s.b == a.n_seqs) s.b = 0, s.kh++;
      } while (s.pos < s.x1 && sequence(a, s.b).n == 0);
    }
    if (i.tile1 > i.tile0) return true;
  }
  return false;
}

template <typename T> __device__ __forceinline__ T *row_at(const Heads &h, int64_t row, int head) { return (T *)h.data + row * h.tok + head * h.head; }

// Rows of no sequence (before `from`, from `to` on): all blocks together write them.
template <typename T, typename F>
__device__ __forceinline__ void fill_rest(const Heads &h, int heads, int dim, int n_tokens, int from, int to, T x, F store) {
  const int64_t count = (int64_t)(from + n_tokens - to) * heads * dim;
  for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < count; i += (int64_t)gridDim.x * blockDim.x) {
    const int64_t row = i / (heads * dim);
    const int in = (int)(i - row * heads * dim);
    store(row < from ? row : row - from + to, in / dim, in % dim, x);
  }
}
template <typename T> __device__ __forceinline__ void zero_rest(const Args &a, const Heads &h, int heads, int dim, const Stretch &s) {
  fill_rest(h, heads, dim, a.n_tokens, s.rest_from, s.rest_to, narrow<T>(0.f), [&](int64_t row, int head, int d, T x) { row_at<T>(h, row, head)[d] = x; });
}

// The 16 bytes at a source off the 16-byte grid.
template <typename T> __device__ __forceinline__ uint4 gather16(const T *from) {
  T e[8];
#pragma unroll
  for (int z = 0; z < 8; z++) e[z] = from[z];
  uint4 v;
  memcpy(&v, e, 16);
  return v;
}

// 16 columns of the warp's 32 rows
__device__ __forceinline__ void tc_ld16(uint32_t *r, uint32_t at) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
                 "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]) : "r"(at) : "memory");
}
__device__ __forceinline__ void tc_st16(uint32_t at, const uint32_t *r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};"
               ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
               "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(at) : "memory");
}

// Values of a row, two to a word: in pieces of 32 bytes where rows stand on that grid (half the accesses of 16, and whole sectors).
template <typename T, int N> __device__ __forceinline__ void store_piece(T *to, const uint32_t (&w)[N], bool aligned) {
  if (aligned) {
#pragma unroll
    for (int y = 0; y < N; y += 8)
      asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to + 2 * y), "r"(w[y]), "r"(w[y + 1]), "r"(w[y + 2]), "r"(w[y + 3]),
                   "r"(w[y + 4]), "r"(w[y + 5]), "r"(w[y + 6]), "r"(w[y + 7]) : "memory");
  } else {
#pragma unroll
    for (int y = 0; y < N; y++) {
      T e[2];
      memcpy(e, &w[y], 4);
      to[2 * y] = e[0], to[2 * y + 1] = e[1];
    }
  }
}
__device__ __forceinline__ bool rows_aligned(const Heads &h) { return (((uintptr_t)h.data >> 1 | h.tok | h.head) & 15) == 0; }   // to 32 bytes

// Two values of a word, and what their rounding took from them.
template <typename T> __device__ __forceinline__ float2 unpack(uint32_t two);
template <> __device__ __forceinline__ float2 unpack<__half>(uint32_t two) { return __half22float2(*(const __half2 *)&two); }
template <> __device__ __forceinline__ float2 unpack<__nv_bfloat16>(uint32_t two) { return make_float2(__uint_as_float(two << 16), __uint_as_float(two & 0xFFFF0000u)); }
template <typename T> __device__ __forceinline__ uint32_t pack_low(float x, float y) {
  const float2 z = unpack<T>(pack<T>(x, y));
  return pack<T>(x - z.x, y - z.y);
}

template <typename T> __device__ __forceinline__ void store4(T *to, const float4 &v, float f, bool aligned) {
  const uint32_t lo = pack<T>(v.x * f, v.y * f), hi = pack<T>(v.z * f, v.w * f);
  if (aligned) {
    *(uint2 *)to = make_uint2(lo, hi);
  } else {
    T e[4];
    memcpy(e, &lo, 4), memcpy(e + 2, &hi, 4);
#pragma unroll
    for (int i = 0; i < 4; i++) to[i] = e[i];
  }
}

// The row of a key, nullptr where its page is none of the cache's.
template <typename T>
__device__ __forceinline__ const T *key_row(const Args &a, const Heads &side, int64_t page_stride, int b, int first, int key, int kh) {
  if (!a.paged) return row_at<T>(side, first + key, kh);
  const int page = a.table[(int64_t)b * a.max_pages + key / a.in_page];
  if ((unsigned)page >= (unsigned)a.n_pages) {
    if (a.status) *a.status = GTS_ERR_INVALID_PARAMS;
    return nullptr;
  }
  return row_at<T>(side, key % a.in_page, kh) + page * page_stride;
}

// Tiles in shared memory: 64 columns after 64, each rows of 128 bytes, eight rows to a swizzled group.
template <int ROWS> __device__ __forceinline__ int tile_at(int row, int c) { return c / 8 * (ROWS * 128) + row * 128 + ((c % 8) ^ (row & 7)) * 16; }

// The top bit of each of two values that is infinite or NaN: all exponent bits are set.
template <typename T> __device__ __forceinline__ uint32_t not_finite(uint32_t two) {
  constexpr uint32_t ONES = std::is_same<T, __half>::value ? 0x7C007C00u : 0x7F807F80u, NEXT = std::is_same<T, __half>::value ? 0x04000400u : 0x00800080u;
  return ((two & ONES) + NEXT) & 0x80008000u;
}
template <typename T> __device__ __forceinline__ uint32_t finite_part(uint32_t two) {   // zero in place of the others
  const uint32_t x = not_finite<T>(two);
  return two & ~((x >> 15) * 0xFFFFu);
}

template <typename T> __device__ __forceinline__ uint32_t zero_times(uint32_t x, uint32_t sum);
template <> __device__ __forceinline__ uint32_t zero_times<__half>(uint32_t x, uint32_t sum) {
  asm("fma.rn.f16x2 %0, %1, %2, %0;" : "+r"(sum) : "r"(x), "r"(0));
  return sum;
}
template <> __device__ __forceinline__ uint32_t zero_times<__nv_bfloat16>(uint32_t x, uint32_t sum) {
  asm("fma.rn.bf16x2 %0, %1, %2, %0;" : "+r"(sum) : "r"(x), "r"(0));
  return sum;
}

// A tile's rows whose product is with weights of 0 where they are out of sight (one warp): 0 x infinity would be NaN.  Rows from
// `live` on are zeroed; where some rows are hidden from some, so are values that are not finite, and the numbers of their rows
// set in `bad`.
template <typename T, int D>
__device__ __forceinline__ void clean_tile(unsigned char *tile, int lane, int live, bool look, uint32_t (&bad)[4]) {
  constexpr int PER = D / 8;                           // 16-byte pieces of a row
#pragma unroll
  for (int i = 0; i < 4; i++) bad[i] = 0;
  for (int i = max(0, live) * PER + lane; i < TILE * PER; i += 32) *(uint4 *)(tile + tile_at<128>(i / PER, i % PER)) = make_uint4(0, 0, 0, 0);
  if (!look) return;
  // first whether there are any, in no order: 0 times each, added up, is NaN then
  uint32_t sum[4] = {0, 0, 0, 0};
  __syncwarp();
#pragma unroll 16
  for (int i = lane; i < TILE * PER; i += 32) {
    const uint4 v = *(const uint4 *)(tile + i * 16);
    sum[0] = zero_times<T>(v.x, sum[0]), sum[1] = zero_times<T>(v.y, sum[1]), sum[2] = zero_times<T>(v.z, sum[2]), sum[3] = zero_times<T>(v.w, sum[3]);
  }
  if (!__any_sync(~0u, not_finite<T>(sum[0]) | not_finite<T>(sum[1]) | not_finite<T>(sum[2]) | not_finite<T>(sum[3]))) return;
#pragma unroll 1
  for (int row = 0; row < TILE; row++) {
    bool some = false;
    if (lane < PER) {
      uint4 *const at = (uint4 *)(tile + tile_at<128>(row, lane));
      const uint4 v = *at;
      some = not_finite<T>(v.x) | not_finite<T>(v.y) | not_finite<T>(v.z) | not_finite<T>(v.w);
      if (some) *at = make_uint4(finite_part<T>(v.x), finite_part<T>(v.y), finite_part<T>(v.z), finite_part<T>(v.w));
    }
    const bool hit = __any_sync(~0u, some);
#pragma unroll
    for (int i = 0; i < 4; i++)
      if (hit && row / 32 == i) bad[i] |= 1u << row % 32;
  }
}

// ---------------------------------------------------------------- forward
// A block holds 2 x 128 rows of one key head - `queries / 2` queries of a sequence with all their heads in each half - and passes along
// its tiles of 128 keys:
//   warp 17 walks along the block's stretch, hands its items on through a short queue, and brings tiles of keys and values
//   (TMA where pages and strides allow it, else 16-byte copies or plain loads) into a ring;
//   warp 19 brings an item's queries, and cleans tiles of values in which some rows are out of sight;
//   warps 16 and 18 issue the products, each for one half: S = Q K^T to tensor memory, O += P V with P from tensor memory;
//   warps 0..7 and 8..15 take one half each, two threads to a row with 64 of a tile's keys each: maximum (of both, through shared
//   memory), weights, sum.  P overwrites S.
// The halves alternate: while one turns scores into weights, the tensor cores work for the other.  An item's first scores are
// worked out, and its queries brought, while the rows of the one before store their results.  The maximum that scores are taken against is
// raised, and what was summed rescaled, only when it has grown by more than 8 (in log 2).  Weights are rounded to the values'
// type for their product; the sum is of the unrounded ones, all else is in 32 bits.  In float16 both are held times 2^7, so that weights
// stay below 2^15 and lose 2^-32 of the largest one at most: many keys of little weight count (65536 of 2^-25.5 are 0.1%).
//
// A row's thread reads its scores twice, for the maximum and for the weights: 104 registers to a thread do not hold 64 scores (as it is,
// 240 bytes a thread are reloaded from spills at a head of 128, 308 at 64, over all paths).  The weights of the first 32 keys of both
// threads are multiplied while those of the others are made (1470 against 1605 us for 16384 tokens, causal, 32 heads on 8 of 128).
// At a head of 64 each of the two threads has sums and a maximum of its own, joined at the end
// (APART): no exchange for each tile, and four streams of scores for the tensor cores instead of two.  A thread with 128 keys of
// its own takes 1510 us there, but loses on short sequences; weights against the last tile's maximum, mended where it has grown,
// take 10% more at a head of 128.
//
// Bound by the chain of a tile from scores to weights to products, and on short sequences by the ends of items.  16384 tokens of 32
// heads on 8 of 128 without a mask: 2815 us, 1.56 PFLOP/s, 82% of the rate of a large matrix product; 2300 cycles for a tile of both
// halves against 2048 of products.  24 sequences of 1024: 289 us causal and 376 not, of which an item's begin and end take 6 of 19 us
// (both halves are at their ends at the same time; the stores themselves are 5%).  The tensor cores are busy for 35% of the causal time, and where
// items change so often rows wait for instructions as well as for scores.  A head of 64: 8192 tokens of 16 heads, causal, 160 us.
constexpr int ROW_WARPS = 16, ROW_THREADS = ROW_WARPS * 32, BLOCK_THREADS = ROW_THREADS + 128, FWD_THREADS = BLOCK_THREADS, QUEUE = 4;
constexpr float RAISE = 8.f;
template <typename T> constexpr float HELD = std::is_same<T, __half>::value ? 7.f : 0.f;   // weights and their sum: times 2^7
template <int D> struct Fwd {
  static constexpr bool APART = D == 64;               // sums of their own for either half of a tile's keys
  static constexpr int PIECE = APART ? 16 : 32;        // columns that a row's results are stored by (the other way round: 2% and 4% more)
  static constexpr int BESIDE = APART ? 3 : LEAD;      // what an item costs beside its tiles (2 at a head of 64: 184 against 166 us for
                                                       // 8192 tokens; 3 and 1 at 128: 2 and 14% more for ragged sequences)
  static constexpr int BYTES = TILE * D * 2, STAGES = D == 64 ? 8 : 5, Q = 2 * BYTES;
  static constexpr int BEHIND = 2816, SMEM = Q + STAGES * BYTES + BEHIND;
};

struct FwdMaps {
  Pages kv;
  CUtensorMap q;       // boxes of a key head's heads of the queries of a half
  int has_q;
};

// An item as one half of its rows sees it.
struct Half {
  int q0, queries, count;                              // its first query (of the sequence), how many it has, tiles of the block's stretch
  int seen;                                            // keys that its last query sees
};
__device__ __forceinline__ Half half_of(const Args &a, const Items<false> &items, const Item &i, int h) {
  Half x;
  const int per = items.q / 2;
  x.q0 = i.t * items.q + h * per;
  x.queries = max(0, min(per, i.n - x.q0));
  x.seen = a.causal ? max(0, i.keys - i.n + x.q0 + x.queries) : i.keys;
  x.count = x.queries ? max(0, min(i.tile1, max(1, (x.seen + TILE - 1) / TILE)) - i.tile0) : 0;
  return x;
}
// keys that the first query of a half sees: tiles that end after them hide keys from some row
__device__ __forceinline__ int seen_by_all(const Args &a, const Item &i, int q0) { return a.causal ? max(0, i.keys - i.n + q0 + 1) : i.keys; }

template <typename T, int D>
__global__ void __launch_bounds__(FWD_THREADS, 1) k_forward(const Args a, const Items<false> of_call, const Cut cut, const __grid_constant__ FwdMaps all_maps) {
  const Items<false> items = {of_call.q, of_call.causal, Fwd<D>::BESIDE};
  constexpr bool APART = Fwd<D>::APART;
  constexpr int PIECE = Fwd<D>::PIECE, BYTES = Fwd<D>::BYTES, STAGES = Fwd<D>::STAGES, COLUMNS = TILE * 128;   // bytes of 64 columns of a tile
  extern __shared__ __align__(1024) unsigned char smem[];
  unsigned char *const qs = smem, *const ring = qs + Fwd<D>::Q;
  uint64_t *const bars = (uint64_t *)(ring + STAGES * BYTES);
  constexpr int BARS = 8 + STAGES + 24 + 2 * QUEUE;
  Item *const queue = (Item *)(bars + BARS);
  uint32_t *const bad_rows = (uint32_t *)(queue + QUEUE);                               // [4][4]: of the last tiles of values
  float *const tops = (float *)(bad_rows + 16);                                         // [2][2][128]: each thread's maximum or sum
  uint32_t *const tmem_at = (uint32_t *)(tops + 512);
  volatile int *const dead = (volatile int *)(tmem_at + 1);
  void *const scratch = tops;                          // (done with before the first maximum)
  static_assert(BARS * 8 + QUEUE * sizeof(Item) + 16 * 4 + 2048 + 8 <= Fwd<D>::BEHIND && SCRATCH <= 2048 && QUEUE * sizeof(Item) % 8 == 0, "room behind the ring");
  const int tid = threadIdx.x, warp = __shfl_sync(~0u, tid / 32, 0), lane = tid % 32;
  const uint32_t bar0 = smem_u32(bars), q_at = smem_u32(qs), ring_at = smem_u32(ring);
  const Pages &maps = all_maps.kv;
  // a ring of barriers for keys and one for values: who waits for either sees each of its phases
  auto full = [&](int slot) { return bar0 + (slot % 2 * 4 + slot / 2 % 4) * 8; };
  auto empty = [&](int s) { return bar0 + (8 + s) * 8; };
  constexpr int B0 = 8 + STAGES;
  auto ready = [&](uint32_t v) { return bar0 + (B0 + v % 4) * 8; };                     // the v-th tile of values is clean
  auto q_full = [&](int h) { return bar0 + (B0 + 4 + h) * 8; };
  auto q_empty = [&](int h) { return bar0 + (B0 + 6 + h) * 8; };
  auto s_full = [&](int h, int y) { return bar0 + (B0 + 8 + (APART ? 2 * y : 0) + h) * 8; };   // (of half the keys, where those are apart)
  auto p_full = [&](int h, int x) { return bar0 + (B0 + 12 + h * 2 + x) * 8; };         // weights of half the keys of a tile
  auto o_full = [&](int h) { return bar0 + (B0 + 16 + h) * 8; };
  auto o_free = [&](int h) { return bar0 + (B0 + 18 + h) * 8; };
  auto my_turn = [&](int h) { return bar0 + (B0 + 20 + h) * 8; };
  auto given = [&](uint32_t i) { return bar0 + (B0 + 22 + i % QUEUE) * 8; };
  auto taken = [&](uint32_t i) { return bar0 + (B0 + 22 + QUEUE + i % QUEUE) * 8; };
  const uint32_t ended = bar0 + (B0 + 22 + 2 * QUEUE) * 8;

  dependents_may_start();
  Stretch line = find_stretch<false, FWD_THREADS>(a, items, cut.blocks, scratch);
  if (line.rest_from + a.n_tokens - line.rest_to > 0) {
    if (a.zero_rest & 1) zero_rest<T>(a, a.out, a.q_heads, D, line);
    if (a.zero_rest & 2 && a.lse)
      fill_rest(a.out, a.q_heads, 1, a.n_tokens, line.rest_from, line.rest_to, -INFINITY, [&](int64_t row, int head, int, float x) { a.lse[row * a.q_heads + head] = x; });
  }
  if (tid == 0) cut.ends[blockIdx.x] = make_int4(NOTHING, 0, 0, 0);
  if (line.x0 >= line.x1) return;
  if (tid == 0) {
    for (int s = 0; s < 8; s++) bar_init(full(s), 1);
    for (int s = 0; s < STAGES; s++) bar_init(empty(s), 2);
    for (int v = 0; v < 4; v++) bar_init(ready(v), 1);
    for (int h = 0; h < 2; h++) {
      bar_init(q_full(h), 1), bar_init(q_empty(h), 1), bar_init(s_full(h, 0), 1), bar_init(bar0 + (B0 + 10 + h) * 8, 1), bar_init(p_full(h, 0), APART ? 128 : 256), bar_init(p_full(h, 1), APART ? 128 : 256);
      bar_init(o_full(h), 1), bar_init(o_free(h), ROW_THREADS / 2), bar_init(my_turn(h), 1), bar_init(ended + 8 * h, 1);
    }
    for (int i = 0; i < QUEUE; i++) bar_init(given(i), 1), bar_init(taken(i), ROW_WARPS + 3);
    *dead = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == ROW_WARPS) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(tmem_at)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  }
  tc_before();
  __syncthreads();
  tc_after();
  const uint32_t tmem = __shfl_sync(~0u, *tmem_at, 0);
  auto scores = [&](int h) { return tmem + h * TILE; };
  auto sums = [&](int h) { return tmem + 256 + h * 128; };
  int copies = 0, asked[2] = {0, 0};                   // warp 17: tiles asked for by TMA; warp 19: halves of queries
  bool issues = false;                                 // the threads that issue products
  bool alive = true;
  auto need = [&](uint32_t bar, uint32_t parity) { alive = alive && bar_wait(bar, parity & 1, dead); };
  // the next item of the queue; false at the end
  uint32_t turn_of_queue = 0;
  auto next = [&](Item &i) {                           // (of one thread)
    need(given(turn_of_queue), turn_of_queue / QUEUE);
    if (alive) i = queue[turn_of_queue % QUEUE];
    return alive && i.tiles > 0;
  };
  auto need_all = [&](uint32_t bar, uint32_t parity) { alive = __all_sync(~0u, bar_wait(bar, parity & 1, dead)); };
  auto next_all = [&](Item &i) {                       // of a warp
    need_all(given(turn_of_queue), turn_of_queue / QUEUE);
    if (alive) i = queue[turn_of_queue % QUEUE];
    return alive && i.tiles > 0;
  };
  auto take = [&] { bar_arrive(taken(turn_of_queue++)); };

  if (warp >= ROW_WARPS) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
    if (warp == ROW_WARPS + 1) {
      // ---- the walk, keys and values
      const bool aligned = (((uintptr_t)a.k.data >> 1 | (uintptr_t)a.v.data >> 1 | a.k.tok | a.k.head | a.v.tok | a.v.head | (a.paged ? a.k_page | a.v_page : 0)) & 7) == 0;
      Stretch s = line;
      Seq q;
      Item i;
      i.b = -1;
      int slot = 0;
      for (uint32_t n = 0; alive; n++) {
        if (!next_item(a, items, s, q, i, lane == 0 ? cut.ends + blockIdx.x : nullptr)) i.tiles = 0;
        if (n >= QUEUE) need_all(taken(n), n / QUEUE - 1);
        if (!alive) break;
        if (lane == 0) queue[n % QUEUE] = i, bar_arrive(given(n));
        if (i.tiles == 0) break;
        if (maps.box) {
          // lane x brings the x-th box of tokens of a tile, 64 values after 64
          const int boxes = TILE / maps.box;
          auto look_up = [&](int t) {                      // this lane's page of tile t; -1: none
            const int key = t * TILE + lane * maps.box;
            return lane < boxes && key < i.keys ? a.paged ? page_number(a.table[(int64_t)i.b * a.max_pages + key / a.in_page]) : 0 : -1;
          };
          int page_next = look_up(i.tile0);
          for (int t = i.tile0; t < i.tile1 && alive; t++) {
            int page = page_next;
            const bool live = page >= 0;
            if (t + 1 < i.tile1) page_next = look_up(t + 1);
            if (page >= (a.paged ? a.n_pages : 1)) {
              page = a.n_pages;                            // outside the map: zeros
              if (a.status) *a.status = GTS_ERR_INVALID_PARAMS;
            }
            const int key = t * TILE + lane * maps.box, token = a.paged ? key % a.in_page : i.first + key;
            const uint32_t bytes = __popc(__ballot_sync(~0u, live)) * maps.box * D * 2;
            for (int kv = 0; kv < 2; kv++, copies++) {
              const int st = copies % STAGES;
              if (copies >= STAGES) need_all(empty(st), copies / STAGES - 1);
              if (!alive) break;
              if (lane == 0) bar_expect(full(copies), bytes);
              __syncwarp();
              if (live) {
                const bool heads_first = kv ? maps.v_heads_first : maps.k_heads_first;
#pragma unroll
                for (int x = 0; x < D / 64; x++)
                  tile_load(ring_at + st * BYTES + x * COLUMNS + lane * maps.box * 128, kv ? &maps.v : &maps.k, x * 64, heads_first ? i.kh : token,
                            heads_first ? token : i.kh, page, full(copies));
              }
            }
          }
        } else {
          // rows gathered: a tile's copies land while the next one's are asked for
          int landing = -1;
          auto landed = [&] {
            fence_async();
            __syncwarp();
            if (lane == 0) bar_arrive(full(landing));
          };
          for (int t = i.tile0; t < i.tile1 && alive; t++) {
            for (int kv = 0; kv < 2 && alive; kv++, slot++) {
              const int st = slot % STAGES;
              const T *rows[4];                            // of keys lane, lane + 32, ...
#pragma unroll
              for (int x = 0; x < 4; x++) {
                const int key = t * TILE + x * 32 + lane;
                rows[x] = key < i.keys ? key_row<T>(a, kv ? a.v : a.k, kv ? a.v_page : a.k_page, i.b, i.first, key, i.kh) : nullptr;
              }
              if (slot >= STAGES) need_all(empty(st), slot / STAGES - 1);
              if (!alive) break;
#pragma unroll
              for (int x = 0; x < 4; x++) {
#pragma unroll 4
                for (int y = 0; y < 32 * (D / 8); y += 32) {
                  const int r = (y + lane) / (D / 8), c = lane % (D / 8);
                  const T *from = (const T *)__shfl_sync(~0u, (unsigned long long)rows[x], r);
                  const int at = st * BYTES + tile_at<128>(x * 32 + r, c);
                  if (aligned) copy16(ring_at + at, from ? from + c * 8 : (const T *)a.k.data, from);
                  else *(uint4 *)(ring + at) = from ? gather16(from + c * 8) : make_uint4(0, 0, 0, 0);
                }
              }
              asm volatile("cp.async.commit_group;" ::: "memory");
              if (landing >= 0) {
                asm volatile("cp.async.wait_group 1;" ::: "memory");
                landed();
              }
              landing = slot;
            }
          }
          asm volatile("cp.async.wait_all;" ::: "memory");
          if (landing >= 0) landed();
        }
      }
    } else if (warp == ROW_WARPS + 3) {
      // ---- queries, and tiles of values made clean
      const bool aligned = (((uintptr_t)a.q.data >> 1 | a.q.tok | a.q.head) & 7) == 0;
      Item i;
      uint32_t tiles = 0, had[2] = {0, 0};
      while (next_all(i)) {
#pragma unroll 1
        for (int h = 0; h < 2; h++) {
          const Half x = half_of(a, items, i, h);
          if (x.count == 0) continue;
          if (had[h]) need_all(q_empty(h), had[h] - 1);
          had[h]++;
          if (!alive) break;
          if (all_maps.has_q) {
            if (lane == 0) {
              bar_expect(q_full(h), items.q / 2 * a.group * D * 2);
#pragma unroll
              for (int c = 0; c < D / 64; c++) tile_load(q_at + h * BYTES + c * COLUMNS, &all_maps.q, c * 64, i.kh * a.group, i.first + x.q0, 0, q_full(h));
            }
            asked[h]++;
            __syncwarp();
            continue;
          }
          const int rows = x.queries * a.group;
#pragma unroll 8
          for (int y = lane; y < rows * (D / 8); y += 32) {
            const int r = y / (D / 8), c = y % (D / 8), query = r / a.in_group;
            const T *from = row_at<const T>(a.q, i.first + x.q0 + query, i.kh * a.group + r - query * a.group) + c * 8;
            const int at = h * BYTES + tile_at<128>(r, c);
            if (aligned) copy16(q_at + at, from, true);
            else *(uint4 *)(qs + at) = gather16(from);
          }
          asm volatile("cp.async.wait_all;" ::: "memory");
          fence_async();
          __syncwarp();
          if (lane == 0) bar_arrive(q_full(h));
        }
        const int clear = seen_by_all(a, i, i.t * items.q);
        for (int t = i.tile0; t < i.tile1 && alive; t++, tiles++) {
          const int slot = 2 * tiles + 1, st = slot % STAGES;
          need_all(full(slot), slot / 8);
          if (!alive) break;
          uint32_t bad[4] = {0, 0, 0, 0};
          if ((t + 1) * TILE > clear) {
            clean_tile<T, D>(ring + st * BYTES, lane, i.keys - t * TILE, a.causal, bad);
            fence_async();
          }
          __syncwarp();
          if (lane < 4) bad_rows[tiles % 4 * 4 + lane] = bad[lane];
          __syncwarp();
          if (lane == 0) bar_arrive(ready(tiles));
        }
        __syncwarp();
        if (lane == 0) bar_arrive(taken(turn_of_queue));
        turn_of_queue++;
      }
    } else if (elected()) {
      // ---- products, from one thread for each half of the rows (one thread for both would set the time)
      issues = true;
      constexpr uint32_t TYPE = std::is_same<T, __nv_bfloat16>::value ? 1u : 0u;
      constexpr uint32_t COMMON = 1u << 4 | TYPE << 7 | TYPE << 10 | (128u >> 4) << 24;
      constexpr uint32_t QK = COMMON | ((APART ? TILE / 2 : TILE) >> 3) << 17, PV = COMMON | 1u << 16 | (D >> 3) << 17;
      const int h = warp == ROW_WARPS + 2;
      const uint32_t k_op = operand(ring_at, 16), v_op = operand(ring_at, COLUMNS), q_op = operand(q_at + h * BYTES, 16);
      const uint32_t s_at = scores(h), o_at = sums(h);
      uint32_t slot = 0, tiles = 0, items_done = 0, turn = 0, turns = 0;
      auto qk = [&](uint32_t sl, int y) {                // with all keys of a tile, or with those of half y
        const uint32_t st = sl % STAGES;
        uint32_t q = q_op, k = k_op + ((st * BYTES + (APART ? y * 64 * 128 : 0)) >> 4);
#pragma unroll
        for (int x = 0; x < D / 64; x++, q += COLUMNS >> 4, k += COLUMNS >> 4) {
#pragma unroll
          for (int z = 0; z < 4; z++) tc_mma(s_at + (APART ? y * 64 : 0), q + 2 * z, k + 2 * z, OPERAND_HI, QK, x + z > 0);
        }
        tc_commit(s_full(h, y));
        if (!APART || y) tc_commit(empty(st));
      };
      Item i;
      while (next(i)) {
        const Half x = half_of(a, items, i, h);
        const int both = min(x.count, half_of(a, items, i, !h).count), n = i.tile1 - i.tile0;
        take();
        if (x.count) {
          need(q_full(h), items_done);
          need(full(slot), slot / 8);
          if (!alive) break;
          tc_after();
          qk(slot, 0);
          if (APART) qk(slot, 1);
          slot++;
          if (x.count == 1) tc_commit(q_empty(h));
        }
        for (int j = 0; j < x.count && alive; j++, tiles++) {
          // this tile's values and the next one's keys, while the rows make their weights
          const uint32_t sv = slot++, sk = slot;
          const int seen = x.seen - (i.tile0 + j) * TILE;
          need(ready(tiles), tiles / 4);
          if (j + 1 < x.count) need(full(sk), sk / 8), slot++;
          if (j == 0 && items_done) need(o_free(h), items_done - 1);
          if (!alive) break;
          const uint32_t *const bad = bad_rows + tiles % 4 * 4;
          const bool add = j > 0 || (bad[0] | bad[1] | bad[2] | bad[3]);
          const uint32_t v = v_op + ((sv % STAGES * BYTES) >> 4);
#pragma unroll
          for (int y = 0; y < 2; y++) {
            need(p_full(h, y), turn);
            // The halves take turns, each with all its products for a tile: left alone they fall into step, and the tensor
            // cores wait while both make weights (four parts of scores to work on cover each other)
            if (!APART && y == 0 && j < both) need(my_turn(h), h ? turns : turns - 1), turns++;
            if (!alive) break;
            tc_after();
#pragma unroll
            for (int z = 0; z < 4; z++) {
              const int k = APART ? 4 * y + z : z / 2 * 4 + 2 * y + z % 2;   // the first or last 32 keys of either half, or a half's
              if (k == 0 || (APART && k == 4) || k * 16 < seen)
                tc_mma_t(o_at + (APART ? y * 64 : 0), s_at + k / 4 * 64 + k % 4 * 8, v + k * (2048 >> 4), OPERAND_HI, PV, add || (APART ? k % 4 : k) > 0);
            }
            if (APART && j + 1 < x.count) qk(sk, y);
          }
          turn++;
          if (!alive) break;
          tc_commit(empty(sv % STAGES));
          if (j + 1 < x.count) {
            if (!APART) qk(sk, 0);
            if (j + 2 == x.count) tc_commit(q_empty(h));
          } else {
            tc_commit(o_full(h));
          }
          if (!APART && j < both) bar_arrive(my_turn(!h));
        }
        if (x.count) items_done++;
        for (int j = x.count; j < n && alive; j++, tiles++) {          // tiles that are only the other half's pass by
          need(full(slot), slot / 8);
          if (alive) bar_arrive(empty(slot++ % STAGES));
          need(ready(tiles), tiles / 4);
          if (alive) bar_arrive(empty(slot++ % STAGES));
        }
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 104;");
    // ---- two threads to a row, y for the second 64 keys of a tile and the second half of the head's values
    const int h = warp / 8, y = warp / 4 % 2, r = tid % 128;
    const uint32_t lanes = (uint32_t)(warp % 4 * 32) << 16;
    const float sl2 = a.scale * 1.4426950408889634f;
    const bool aligned = rows_aligned(a.out), low_aligned = rows_aligned(a.low);
    const int in_half = r / a.in_group, head_in = r - in_half * a.group;
    float *const mine = tops + (h * 2 + y) * 128 + r, *const others = tops + (h * 2 + !y) * 128 + r;
    // The two warps of the same rows exchange a value each.  Their barrier has no limit of its own, so each also says whether a wait of
    // its ran out, and both go on or both leave: neither leaves on what it alone knows.  (A tile's exchange without its first barrier, as
    // scores come only after both have read the last one's, takes 1 to 2% less for 16384 tokens, but scores may also be given up.)
    auto meet = [&] { asm volatile("bar.sync %0, 64;" ::"r"(1 + h * 4 + warp % 4) : "memory"); };
    auto exchange = [&](float x, float ran_out = NAN) {  // (a value that x never has)
      meet();                                            // what was there has been read
      *mine = alive ? x : ran_out;
      meet();
      return *others;
    };
    auto wait = [&](uint32_t bar, uint32_t parity) { alive = __all_sync(~0u, bar_wait(bar, parity & 1, dead)) && alive; };
    uint32_t turn = 0, items_done = 0, tiles = 0;
    Item i;
    auto take_item = [&] {                               // the next one; both threads of a row go on with it, or neither
      wait(given(turn_of_queue), turn_of_queue / QUEUE);
      i = queue[turn_of_queue % QUEUE];
      const bool on = !isnan(exchange(0.f)) && alive && i.tiles > 0;
      if (lane == 0) bar_arrive(taken(turn_of_queue));
      turn_of_queue++;
      return on;
    };
    bool on = take_item();
    while (on) {
      const Half x = half_of(a, items, i, h);
      const int query = x.q0 + in_half, kh = i.kh;
      const bool valid = in_half < x.queries;
      const int64_t row = (int64_t)i.first + query;
      const int limit = a.causal ? min(i.keys, i.keys - i.n + query + 1) : i.keys, clear = seen_by_all(a, i, x.q0), clear_of_all = seen_by_all(a, i, i.t * items.q);
      const bool whole = i.tile0 == 0 && i.tile1 == i.tiles;
      float m = -INFINITY, l = 0.f;
      for (int j = 0; j < x.count; j++, turn++) {
        wait(s_full(h, y), turn);
        tc_after();
        const int t = i.tile0 + j, nv = limit - t * TILE - y * 64;
        const bool masked = (t + 1) * TILE > clear, cleaned = a.causal && (t + 1) * TILE > clear_of_all;
        // The maximum first, then weights, 32 scores at a time and read twice: more registers are not to be had.
        uint32_t s[32];
        auto fetch = [&](int c) {
          tc_ld(s, scores(h) + lanes + y * 64 + c);
          tc_ld_wait();
          if (masked) {
#pragma unroll
            for (int z = 0; z < 32; z++)
              if (c + z >= nv) s[z] = 0xFF800000u;         // -infinity
          }
        };
        float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
        for (int c = 0; c < 64; c += 32) {
          fetch(c);
#pragma unroll
          for (int z = 0; z < 32; z += 4) {
            top[0] = max3(top[0], __uint_as_float(s[z]), __uint_as_float(s[z + 1]));
            top[1] = max3(top[1], __uint_as_float(s[z + 2]), __uint_as_float(s[z + 3]));
          }
        }
        if (cleaned) wait(ready(tiles + j), (tiles + j) / 4);
        float big = fmaxf(top[0], top[1]);
        if (!APART) {
          const float theirs = exchange(big);
          alive = alive && !isnan(theirs);                 // (a maximum is none)
          big = fmaxf(big, theirs);
        }
        if (!alive) break;
        big *= sl2;
        const bool raise = big > m + RAISE || (m == -INFINITY && big > m);
        if (j == 0) {
          m = big;
        } else if (__any_sync(~0u, raise)) {
          const float to = raise ? big : m, f = raise ? exp2_fast(m - to) : 1.f;
          uint32_t o[16];
#pragma unroll 1
          for (int c = APART ? 0 : y * (D / 2); c < (APART ? D : (y + 1) * (D / 2)); c += 16) {
            const uint32_t at = sums(h) + (APART ? y * 64 : 0) + lanes + c;
            tc_ld16(o, at);
            tc_ld_wait();
#pragma unroll
            for (int z = 0; z < 16; z++) o[z] = __float_as_uint(__uint_as_float(o[z]) * f);
            tc_st16(at, o);
          }
          l *= f;
          m = to;
        }
        const float from = m == -INFINITY ? 0.f : m - HELD<T>;
        if (cleaned) {
          // values that are not finite: each for the rows that see it, before the products are added (the tile is clean: waited for
          // above, before both threads of a row agree to go on)
          const uint32_t *const bad = bad_rows + (tiles + j) % 4 * 4;
          if (bad[0] | bad[1] | bad[2] | bad[3]) {
            if (APART && j == 0 && items_done) {           // the other warp of these rows may still read sums of the item before
              wait(o_free(h), items_done - 1);
              if (!alive) break;
              tc_after();
            }
#pragma unroll 1
            for (int c = APART ? 0 : y * (D / 2); c < (APART ? D : (y + 1) * (D / 2)); c += 16) {
              uint32_t o[16];
              const uint32_t at = sums(h) + (APART ? y * 64 : 0) + lanes + c;
              if (j == 0) {
#pragma unroll
                for (int z = 0; z < 16; z++) o[z] = 0;
              } else {
                tc_ld16(o, at);
                tc_ld_wait();
              }
#pragma unroll 1
              for (int key = APART ? y * 64 : 0; key < (APART ? y * 64 + 64 : TILE); key++) {
                if (!(bad[key / 32] >> (key % 32) & 1)) continue;
                uint32_t score;
                asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];" : "=r"(score) : "r"(scores(h) + lanes + key) : "memory");
                tc_ld_wait();
                const T *value = key_row<T>(a, a.v, a.v_page, i.b, i.first, t * TILE + key, kh);
                if (key < limit - t * TILE && value) {
                  const float p = widen(narrow<T>(exp2_fast(__uint_as_float(score) * sl2 - from)));
#pragma unroll
                  for (int z = 0; z < 16; z++) {
                    const float v = widen(value[c + z]);
                    if (!isfinite(v)) o[z] = __float_as_uint(__uint_as_float(o[z]) + p * v);
                  }
                }
                __syncwarp();
              }
              tc_st16(at, o);
            }
            if (!APART) exchange(0.f);                     // both have read the scores before weights overwrite them
          }
        }
        const float2 scale2 = make_float2(sl2, sl2), from2 = make_float2(-from, -from);
        float2 part[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
        for (int c = 0; c < 64; c += 32) {                 // the products with the first 32 of both start under the others
          fetch(c);
#pragma unroll
          for (int z = 0; z < 32; z += 2) {
            float2 e = fma2(make_float2(__uint_as_float(s[z]), __uint_as_float(s[z + 1])), scale2, from2);
            e.x = exp2_fast(e.x), e.y = exp2_fast(e.y);
            part[z / 2 & 1] = add2(part[z / 2 & 1], e);
            s[z / 2] = pack<T>(e.x, e.y);
          }
          tc_st16(scores(h) + lanes + y * 64 + c / 2, s);
          if (!APART || c) {
            tc_st_wait();
            tc_before();
            bar_arrive(p_full(h, APART ? y : c / 32));
          }
        }
        const float2 sum = add2(part[0], part[1]);
        l += sum.x + sum.y;
      }
      // the row's sum: both threads', against one maximum
      float f0 = 1.f, f1 = 1.f;                            // of either half's sums
      if (APART) {
        const float m1 = exchange(m == -INFINITY ? -3e38f : m), l1 = exchange(l);
        alive = alive && !isnan(m1);
        if (!alive) break;                                 // (both: a maximum is no NaN)
        const float to = fmaxf(m, m1), against = to == -INFINITY || to == -3e38f ? 0.f : to;
        const float mine_f = exp2_fast(m - against), their_f = exp2_fast(m1 - against);
        l = l * mine_f + l1 * their_f, m = to == -3e38f ? -INFINITY : to;
        f0 = y ? their_f : mine_f, f1 = y ? mine_f : their_f;
      } else {
        const float l1 = exchange(l, -1.f);                // (a sum is not negative; it may be NaN)
        alive = alive && !(l1 < 0.f);
        if (!alive) break;                                 // (both)
        l += l1;
      }
      m -= HELD<T>;
      tiles += i.tile1 - i.tile0;
      const int64_t part = ((int64_t)blockIdx.x * 2 + (i.tile0 == 0)) * 256 + h * 128 + r;
      const float inv = l == 0.f ? 0.f : 1.f / l;
      T *const dst = row_at<T>(a.out, row, kh * a.group + head_in);
      float4 *const mid = cut.o + part / 256 * (D / 4) * 256 + part % 256;
      if (valid && y == 0) {
        if (!whole) cut.ml[part] = make_float2(m, l);
        else if (a.lse) a.lse[row * a.q_heads + kh * a.group + head_in] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
      }
      on = take_item();                                  // (while the last products are worked out)
      if (x.count) {
        wait(o_full(h), items_done);
        items_done++;
        tc_after();
#pragma unroll 1
        for (int c = y * (D / 2); c < (y + 1) * (D / 2) && alive; c += PIECE) {
          uint32_t o[PIECE];
          if constexpr (APART) {
            uint32_t o1[PIECE];
            tc_ld16(o, sums(h) + lanes + c);
            tc_ld16(o1, sums(h) + 64 + lanes + c);
            tc_ld_wait();
#pragma unroll
            for (int z = 0; z < PIECE; z++) o[z] = __float_as_uint(f0 * __uint_as_float(o[z]) + f1 * __uint_as_float(o1[z]));
          } else {
            tc_ld(o, sums(h) + lanes + c);
            tc_ld_wait();
          }
          if (valid && !whole) {
#pragma unroll
            for (int z = 0; z < PIECE; z += 4) *(uint4 *)(mid + (c + z) / 4 * 256) = make_uint4(o[z], o[z + 1], o[z + 2], o[z + 3]);
          } else if (valid) {
            uint32_t w[PIECE / 2];
#pragma unroll
            for (int z = 0; z < PIECE / 2; z++) w[z] = pack<T>(__uint_as_float(o[2 * z]) * inv, __uint_as_float(o[2 * z + 1]) * inv);
            store_piece<T>(dst + c, w, aligned);
            if (a.low.data) {
#pragma unroll
              for (int z = 0; z < PIECE / 2; z++) w[z] = pack_low<T>(__uint_as_float(o[2 * z]) * inv, __uint_as_float(o[2 * z + 1]) * inv);
              store_piece<T>(row_at<T>(a.low, row, kh * a.group + head_in) + c, w, low_aligned);
            }
          }
          __syncwarp();
        }
        tc_before();
        bar_arrive(o_free(h));
      }
    }
  }
  tc_before();
  __syncthreads();
  if (*dead) {
    // copies and products in flight end before the block does, whichever warp gave up
    const uint64_t from = now_ns();
    if (issues) {
      const uint32_t bar = ended + (warp == ROW_WARPS + 2 ? 8 : 0);
      tc_commit(bar);
      while (!bar_try(bar, 0) && now_ns() - from < DRAIN_NS) {}
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    if (warp == ROW_WARPS + 1) {
#pragma unroll 1
      for (int x = max(0, copies - STAGES); x < copies; x++)
        while (!bar_try(full(x), (x / 8) & 1) && now_ns() - from < DRAIN_NS) {}
    }
    if (warp == ROW_WARPS + 3) {
#pragma unroll 1
      for (int h = 0; h < 2; h++)
        while (asked[h] && !bar_try(q_full(h), (asked[h] - 1) & 1) && now_ns() - from < DRAIN_NS) {}
    }
    if (tid == 0 && a.status) *a.status = GTS_ERR_STEP_LIMIT;
    __syncthreads();
    // every result of the block's stretch is NaN
    Stretch s = line;
    Seq q;
    Item i;
    i.b = -1;
    while (next_item(a, items, s, q, i, tid == 0 ? cut.ends + blockIdx.x : nullptr)) {
      const bool whole = i.tile0 == 0 && i.tile1 == i.tiles;
      for (int r = tid; r < 256; r += FWD_THREADS) {
        const int in_half = r % 128 / a.in_group, query = i.t * items.q + r / 128 * (items.q / 2) + in_half;
        if (in_half >= items.q / 2 || query >= i.n) continue;
        const int head = i.kh * a.group + r % 128 - in_half * a.group;
        if (!whole) {
          cut.ml[((int64_t)blockIdx.x * 2 + (i.tile0 == 0)) * 256 + r] = make_float2(NAN, NAN);
        } else {
          for (int d = 0; d < D; d++) row_at<T>(a.out, i.first + query, head)[d] = narrow<T>(NAN);
          for (int d = 0; d < D && a.low.data; d++) row_at<T>(a.low, i.first + query, head)[d] = narrow<T>(NAN);
          if (a.lse) a.lse[((int64_t)i.first + query) * a.q_heads + head] = NAN;
        }
      }
    }
  }
  if (warp == ROW_WARPS) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
}

// Rows of the items that were cut, from the block where the item begins to that where it ends: a thread for a row and an eighth
// of its columns, so that loads of parts cover whole lines.
constexpr int JOIN_BLOCKS = 8, JOIN_THREADS = 256;      // thread blocks for an item of 256 rows
template <typename T, int D>
__global__ void __launch_bounds__(JOIN_THREADS) k_join(const Args a, const Items<false> items, const Cut cut) {
  wait_for_kernels_before();
  const int c = blockIdx.x / JOIN_BLOCKS, lane = threadIdx.x % 32, column = threadIdx.x / 32;
  const int4 end = cut.ends[c];
  if (end.x < 0) return;
  constexpr int E = D / 32;                             // fours of columns
  const int r = blockIdx.x % JOIN_BLOCKS * 32 + lane;
  const int in_half = r % 128 / a.in_group, query = end.z * items.q + r / 128 * (items.q / 2) + in_half;
  const Seq s = sequence(a, end.x);
  if (in_half >= items.q / 2 || query >= s.n) return;
  float m = -INFINITY, l = 0.f;
  float4 acc[E] = {};
  for (int x = 0; x <= end.w; x += 2) {
    float2 ml[2];
    float4 v[2][E];
#pragma unroll
    for (int k = 0; k < 2; k++) {
      if (x + k <= end.w) {
        const int64_t part = (int64_t)(c + x + k) * 2 + (x + k == 0);
        ml[k] = cut.ml[part * 256 + r];
#pragma unroll
        for (int e = 0; e < E; e++) v[k][e] = cut.o[(part * (D / 4) + column * E + e) * 256 + r];
      } else {
        ml[k] = make_float2(-INFINITY, 0.f);
      }
    }
    const float top = fmaxf(m, fmaxf(ml[0].x, ml[1].x)), from = top == -INFINITY ? 0.f : top, keep = exp2_fast(m - from);
    l *= keep, m = top;
#pragma unroll
    for (int e = 0; e < E; e++) acc[e].x *= keep, acc[e].y *= keep, acc[e].z *= keep, acc[e].w *= keep;
#pragma unroll
    for (int k = 0; k < 2; k++) {
      if (ml[k].x != -INFINITY || ml[k].y != 0.f) {     // (a part of no tiles has no values; one of NaN scores has a sum of NaN)
        const float f = exp2_fast(ml[k].x - from);
        l += f * ml[k].y;
#pragma unroll
        for (int e = 0; e < E; e++) acc[e].x += f * v[k][e].x, acc[e].y += f * v[k][e].y, acc[e].z += f * v[k][e].z, acc[e].w += f * v[k][e].w;
      }
    }
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  const int head = end.y * a.group + r % 128 - in_half * a.group;
  T *const dst = row_at<T>(a.out, (int64_t)s.first + query, head) + column * E * 4;
#pragma unroll
  for (int e = 0; e < E; e++) {
    store4(dst + 4 * e, acc[e], inv, rows_aligned(a.out));
    if (a.low.data) {
      const float4 x = acc[e];
      const float2 u = unpack<T>(pack<T>(x.x * inv, x.y * inv)), v = unpack<T>(pack<T>(x.z * inv, x.w * inv));
      store4(row_at<T>(a.low, (int64_t)s.first + query, head) + (column * E + e) * 4, make_float4(x.x * inv - u.x, x.y * inv - u.y, x.z * inv - v.x, x.w * inv - v.y), 1.f,
             rows_aligned(a.low));
    }
  }
  if (a.lse && column == 0) a.lse[((int64_t)s.first + query) * a.q_heads + head] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
}

// ---------------------------------------------------------------- gradients
// Two kernels, one for the gradients of keys and values (a block holds 128 keys and passes along the rows that see them) and one for
// those of the queries (a block holds 128 rows and passes along the keys they see).  Each works scores and weights out again, so
// there are seven products where one pass over both would have five, but every sum is taken in one order by one block, with
// no atomic adds, and nothing of the size of the scores is ever stored.  Weights p and ds are rounded to the inputs' type for
// their products; all else is in 32 bits.
//
// Bound by the rows' threads and the products of 128 weights, which want as much of shared memory as of the tensor cores: over 4096 tokens without
// a mask a tile of k_grad_kv takes 2960 cycles, ends of items included, against 2048 of its four products, one of k_grad_q 2460 against
// 1536 of its three.  k_grad_kv reloads 196 to 208 bytes a thread from spills, k_grad_q none in bfloat16 and 20 in float16.
// 32 heads on 8 of 128, causal: one sequence of 16384 tokens 5.4 ms (1.0 PFLOP/s of the five products, 1.4 of the seven that are done),
// 24 of 1024 775 us, 8 of 512 to 4096 1.30 ms.  The kernels start while the one before ends, and wait for it before they read what it
// wrote (1024 tokens: 66 us).
//
// float16 is short of numbers: weights are held times 2^10, and ds times the power of two that puts a bound of the call's |ds| between
// 2^14 and 2^15, below its largest number by a factor of two.  As p <= 1 and out is a mean of values, |ds_ij| = p_ij |dout_i . v_j - dout_i .
// out_i + dlse_i| <= 2 max |dout_i| max |v_j| + max |dlse_i|, with Euclidean norms of rows, over the rows of all sequences; what
// is lost is 2^-39 of that at most, below 2^-14.  bfloat16 has the range of 32 bits and needs neither.
constexpr int GRAD_THREADS = BLOCK_THREADS, DELTA_BLOCKS = 1216, DELTA_THREADS = 256;
template <typename T> constexpr float WEIGHT_SHIFT = std::is_same<T, __half>::value ? 10.f : 0.f;
template <typename T> constexpr float WEIGHT_UNIT = std::is_same<T, __half>::value ? 0x1p-10f : 1.f;

__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 y;
  asm("{\n.reg .b64 a, b;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %5};\nmul.rn.f32x2 a, a, b;\nmov.b64 {%0, %1}, a;\n}"
      : "=f"(y.x), "=f"(y.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return y;
}

// What the finite values of sequences' rows reach: squares of the norms of dout's and of v's rows, and |dlse|, the largest of each block.
struct Largest { float dout, v, dlse; };
__device__ __forceinline__ Largest most_of(const Largest &x, const Largest &y) { return {fmaxf(x.dout, y.dout), fmaxf(x.v, y.v), fmaxf(x.dlse, y.dlse)}; }
__device__ __forceinline__ Largest most_of_warp(Largest x) {
#pragma unroll
  for (int o = 16; o; o /= 2) x = most_of(x, {__shfl_xor_sync(~0u, x.dout, o), __shfl_xor_sync(~0u, x.v, o), __shfl_xor_sync(~0u, x.dlse, o)});
  return x;
}
// The power of two that ds is held times, as its exponent (at most 100, so that 32 bits hold it and what it multiplies).
__device__ __forceinline__ int ds_exponent(const Largest &x) {
  const float bound = fminf(2.f * sqrtf(x.dout) * sqrtf(x.v) + x.dlse, 0x1.fffffep127f);
  int e = 15;
  if (bound > 0.f) frexpf(bound, &e);                  // bound < 2^e
  return min(100, 15 - e);
}

// e_i = dout_i . out_i - dlse_i of the rows that belong to sequences, and in float16 what bounds ds.  Bound by memory.
template <typename T, int D>
__global__ void __launch_bounds__(DELTA_THREADS) k_delta(const Args a, Largest *largest) {
  constexpr int PER = D / 8;                           // lanes of a row
  constexpr bool HALF = std::is_same<T, __half>::value;
  __shared__ int ends[2];
  dependents_may_start();
  if (threadIdx.x == 0) ends[0] = a.n_tokens, ends[1] = 0;
  __syncthreads();
  for (int b = threadIdx.x; b < a.n_seqs; b += DELTA_THREADS) {
    const Seq s = sequence(a, b);
    if (s.n) atomicMin(&ends[0], s.first), atomicMax(&ends[1], s.first + s.n);
  }
  __syncthreads();
  const int from = ends[0], to = max(from, ends[1]);
  const bool aligned = (((uintptr_t)a.dout.data >> 1 | (uintptr_t)a.out.data >> 1 | (uintptr_t)a.low.data >> 1 | a.dout.tok | a.dout.head | a.out.tok | a.out.head |
                         a.low.tok | a.low.head) & 7) == 0;
  const int c = threadIdx.x % PER;
  Largest most = {0.f, 0.f, 0.f};
  const int64_t rows = (int64_t)(to - from) * a.q_heads;
  for (int64_t first = (int64_t)blockIdx.x * (DELTA_THREADS / PER); first < rows; first += (int64_t)gridDim.x * (DELTA_THREADS / PER)) {
    const int64_t r = first + threadIdx.x / PER;
    float sum = 0.f, square = 0.f;
    if (r < rows) {
      const int64_t token = quotient(r, a.q_heads) + from;
      const int head = (int)(r - (token - from) * a.q_heads);
      const T *x = row_at<const T>(a.dout, token, head) + c * 8, *y = row_at<const T>(a.out, token, head) + c * 8;
      const T *const z = a.low.data ? row_at<const T>(a.low, token, head) + c * 8 : nullptr;
      const uint4 u = aligned ? *(const uint4 *)x : gather16(x), v = aligned ? *(const uint4 *)y : gather16(y);
      uint4 l = make_uint4(0, 0, 0, 0);
      if (z) l = aligned ? *(const uint4 *)z : gather16(z);
      T e[8], f[8], g[8];
      memcpy(e, &u, 16), memcpy(f, &v, 16), memcpy(g, &l, 16);
#pragma unroll
      for (int i = 0; i < 8; i++) {
        const float w = widen(e[i]);
        sum += w * (widen(f[i]) + widen(g[i]));
        if (HALF && isfinite(w)) square += w * w;
      }
    }
#pragma unroll
    for (int o = PER / 2; o; o /= 2) {
      sum += __shfl_xor_sync(~0u, sum, o);
      if (HALF) square += __shfl_xor_sync(~0u, square, o);
    }
    if (HALF) most.dout = fmaxf(most.dout, square);
    if (r < rows && c == 0) {
      const int64_t at = (int64_t)from * a.q_heads + r;
      const float dl = a.dlse ? a.dlse[at] : 0.f;
      if (HALF && isfinite(dl)) most.dlse = fmaxf(most.dlse, fabsf(dl));
      a.delta[at] = sum - dl;
    }
  }
  if (HALF) {
    const bool v_aligned = (((uintptr_t)a.v.data >> 1 | a.v.tok | a.v.head) & 7) == 0;
    const int64_t v_rows = (int64_t)(to - from) * a.kv_heads;
    for (int64_t first = (int64_t)blockIdx.x * (DELTA_THREADS / PER); first < v_rows; first += (int64_t)gridDim.x * (DELTA_THREADS / PER)) {
      const int64_t r = first + threadIdx.x / PER;
      float square = 0.f;
      if (r < v_rows) {
        const int64_t token = quotient(r, a.kv_heads);
        const T *x = row_at<const T>(a.v, token + from, (int)(r - token * a.kv_heads)) + c * 8;
        const uint4 u = v_aligned ? *(const uint4 *)x : gather16(x);
        T e[8];
        memcpy(e, &u, 16);
#pragma unroll
        for (int i = 0; i < 8; i++) {
          const float w = widen(e[i]);
          if (isfinite(w)) square += w * w;
        }
      }
#pragma unroll
      for (int o = PER / 2; o; o /= 2) square += __shfl_xor_sync(~0u, square, o);
      most.v = fmaxf(most.v, square);
    }
    __shared__ Largest warps[DELTA_THREADS / 32];
    most = most_of_warp(most);
    if (threadIdx.x % 32 == 0) warps[threadIdx.x / 32] = most;
    __syncthreads();
    if (threadIdx.x == 0) {
      for (int w = 0; w < DELTA_THREADS / 32; w++) most = most_of(most, warps[w]);
      largest[blockIdx.x] = most;
    }
  }
}

// The factor of ds, from what bounds it: all threads of the block look.
template <typename T> __device__ __forceinline__ float ds_factor(const Largest *largest, void *scratch) {
  if (!std::is_same<T, __half>::value) return 1.f;
  static_assert(GRAD_THREADS / 32 * sizeof(Largest) <= SCRATCH, "room for the warps' largest");
  Largest *const warps = (Largest *)scratch;
  __syncthreads();
  Largest most = {0.f, 0.f, 0.f};
  for (int i = threadIdx.x; i < DELTA_BLOCKS; i += GRAD_THREADS) most = most_of(most, largest[i]);
  most = most_of_warp(most);
  if (threadIdx.x % 32 == 0) warps[threadIdx.x / 32] = most;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < GRAD_THREADS / 32; w++) most = most_of(most, warps[w]);
  return ldexpf(1.f, ds_exponent(most));
}

// Maps of the rows of queries (or of dout): a box is the `group` heads of a key head of `q` tokens; of keys and values.
struct GradMaps { CUtensorMap q, dout; Pages kv; };

// Columns of a row in tensor memory to a result, or as they are to a partial one.
template <typename T, int COLUMNS>
__device__ __forceinline__ void store_row(uint32_t at, T *dst, float4 *part, bool valid, bool aligned, float factor) {
#pragma unroll 1
  for (int c = 0; c < COLUMNS; c += 32) {
    uint32_t o[32];
    tc_ld(o, at + c);
    tc_ld_wait();
    if (valid && part) {
#pragma unroll
      for (int y = 0; y < 32; y += 4) *(uint4 *)(part + (c + y) / 4 * TILE) = make_uint4(o[y], o[y + 1], o[y + 2], o[y + 3]);
    } else if (valid) {
      uint32_t w[16];
#pragma unroll
      for (int y = 0; y < 16; y++) w[y] = pack<T>(__uint_as_float(o[2 * y]) * factor, __uint_as_float(o[2 * y + 1]) * factor);
      store_piece<T>(dst + c, w, aligned);
    }
    __syncwarp();
  }
}

// What the two kernels' threads that issue products need: shapes of S (or dP), 128 x 128 over a head, and of products with 128
// weights to a row, from tensor memory.  Quarter w of the threads writes its 32 weights to a row where its 32 scores were.
template <typename T, int D> struct Products {
  static constexpr uint32_t TYPE = std::is_same<T, __nv_bfloat16>::value ? 1u : 0u;
  static constexpr uint32_t COMMON = 1u << 4 | TYPE << 7 | TYPE << 10 | (128u >> 4) << 24;
  static constexpr uint32_t ROWS = COMMON | (TILE >> 3) << 17, SUMS = COMMON | 1u << 16 | (D >> 3) << 17;
  static constexpr uint32_t COLUMNS = TILE * 128 >> 4;
  static __device__ __forceinline__ void scores(uint32_t to, uint32_t x, uint32_t y) {
#pragma unroll
    for (int c = 0; c < D / 64; c++, x += COLUMNS, y += COLUMNS) {
#pragma unroll
      for (int k = 0; k < 4; k++) tc_mma(to, x + 2 * k, y + 2 * k, OPERAND_HI, ROWS, c + k > 0);
    }
  }
  static __device__ __forceinline__ void sums(uint32_t to, uint32_t weights, uint32_t y, bool add) {
#pragma unroll
    for (int k = 0; k < 8; k++) tc_mma_t(to, weights + k / 2 * 32 + k % 2 * 8, y + k * (2048 >> 4), OPERAND_HI, SUMS, add || k > 0);
  }
};

// Keys and values.  Warp 17 walks along the stretch and brings an item's keys and values and then its tiles of rows: queries and
// dout by TMA.  Warps 18 and 19 clean queries and dout where some are out of sight, and bring the rows' lse and e.  Warp 16 issues the products:
//   S^T = K Q^T, dP^T = V dout^T, dV += P^T dout, dK += dS^T Q
// in the order S, dP, (dV, next S, dK, next dP), ..., so that the tensor cores have the next scores to work out while rows turn the
// present ones into weights: nothing waits for a second buffer.  Warps 0..15: a thread for a key and a quarter of a tile's rows.
template <int D> struct GradKv {
  static constexpr int BYTES = TILE * D * 2, STAGES = D == 64 ? 8 : 5, STATS = 2;       // tiles of queries or dout; of lse and e
  static constexpr int BEHIND = D == 64 ? 1088 : 1024, SMEM = (2 + STAGES) * BYTES + STATS * 2 * TILE * 4 + BEHIND;
};

template <typename T, int D>
__global__ void __launch_bounds__(GRAD_THREADS, 1) k_grad_kv(const Args a, const Items<true> items, const Cut cut, const Largest *largest, const __grid_constant__ GradMaps maps) {
  constexpr int BYTES = GradKv<D>::BYTES, STAGES = GradKv<D>::STAGES, STATS = GradKv<D>::STATS, COLUMNS = TILE * 128;
  extern __shared__ __align__(1024) unsigned char smem[];
  unsigned char *const kv = smem, *const ring = kv + 2 * BYTES;
  float *const stats = (float *)(ring + STAGES * BYTES);                                // [STATS][2][128]: -lse (of log2 weights), -e
  uint64_t *const bars = (uint64_t *)(stats + STATS * 2 * TILE);
  constexpr int BARS = 16 + STAGES + STATS + 2 * QUEUE + 9;
  Item *const queue = (Item *)(bars + BARS);
  uint32_t *const bad_rows = (uint32_t *)(queue + QUEUE);                               // [STATS][4]: rows of dout with values that are not finite
  uint32_t *const tmem_at = bad_rows + 4 * STATS;
  volatile int *const dead = (volatile int *)(tmem_at + 1);
  void *const scratch = (void *)(tmem_at + 2);
  static_assert(BARS * 8 + QUEUE * sizeof(Item) + 16 * STATS + 8 + SCRATCH <= GradKv<D>::BEHIND && QUEUE * sizeof(Item) % 8 == 0, "room behind the ring, and its alignment");
  const int tid = threadIdx.x, warp = __shfl_sync(~0u, tid / 32, 0), lane = tid % 32;
  const uint32_t bar0 = smem_u32(bars), kv_at = smem_u32(kv), ring_at = smem_u32(ring);
  // slots of the ring: a tile's queries, its dout, the next one's queries, ...  Barriers are a ring for each kind, so that who waits for
  // one sees each of its phases
  auto full = [&](int slot) { return bar0 + (slot % 2 * 4 + slot / 2 % 4) * 8; };
  auto ready = [&](int slot) { return bar0 + (8 + slot % 2 * 4 + slot / 2 % 4) * 8; };
  auto empty = [&](int s) { return bar0 + (16 + s) * 8; };
  auto read = [&](int s) { return bar0 + (16 + STAGES + s) * 8; };                      // a tile's lse and e
  auto given = [&](uint32_t i) { return bar0 + (16 + STAGES + STATS + i % QUEUE) * 8; };
  auto taken = [&](uint32_t i) { return bar0 + (16 + STAGES + STATS + QUEUE + i % QUEUE) * 8; };
  const uint32_t rest = bar0 + (16 + STAGES + STATS + 2 * QUEUE) * 8;
  const uint32_t kv_full = rest, kv_empty = rest + 8, s_full = rest + 16, dp_full = rest + 24, p_full = rest + 32, ds_full = rest + 40,
                 o_full = rest + 48, o_free = rest + 56, ended = rest + 64;

  Stretch line = find_stretch<true, GRAD_THREADS>(a, items, cut.blocks, scratch);
  if (line.rest_from + a.n_tokens - line.rest_to > 0) {
    if (a.zero_rest & 2) zero_rest<T>(a, a.dk, a.kv_heads, D, line);
    if (a.zero_rest & 4) zero_rest<T>(a, a.dv, a.kv_heads, D, line);
  }
  if (tid == 0) cut.ends[blockIdx.x] = make_int4(NOTHING, 0, 0, 0);
  wait_for_kernels_before();                             // e; only then may the next kernel start, which wants it too
  dependents_may_start();
  if (line.x0 >= line.x1) return;
  const float factor = ds_factor<T>(largest, scratch);
  if (tid == 0) {
    for (int s = 0; s < 8; s++) bar_init(full(s), 1), bar_init(ready(s), 1);
    for (int s = 0; s < STAGES; s++) bar_init(empty(s), 1);
    for (int s = 0; s < STATS; s++) bar_init(read(s), ROW_WARPS);
    bar_init(kv_full, 1), bar_init(kv_empty, 1), bar_init(s_full, 1), bar_init(dp_full, 1), bar_init(p_full, ROW_THREADS), bar_init(ds_full, ROW_THREADS);
    bar_init(o_full, 1), bar_init(o_free, ROW_THREADS), bar_init(ended, 1);
    for (int i = 0; i < QUEUE; i++) bar_init(given(i), 1), bar_init(taken(i), ROW_WARPS + 3);
    *dead = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == ROW_WARPS) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(tmem_at)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  }
  // rows that no box reaches (where the group does not divide 128) stay zero
  const int box_rows = items.q * a.group;
  for (int y = tid; y < STAGES * (TILE - box_rows) * (D / 8); y += GRAD_THREADS) {
    const int c = y % (D / 8), r = y / (D / 8) % (TILE - box_rows) + box_rows, s = y / (D / 8) / (TILE - box_rows);
    *(uint4 *)(ring + s * BYTES + tile_at<128>(r, c)) = make_uint4(0, 0, 0, 0);
  }
  fence_async();
  tc_before();
  __syncthreads();
  tc_after();
  const uint32_t tmem = __shfl_sync(~0u, *tmem_at, 0), s_at = tmem, dp_at = tmem + 128, dv_at = tmem + 256, dk_at = tmem + 384;
  int copies = 0, kv_copies = 0;
  bool issues = false, alive = true;
  auto need = [&](uint32_t bar, uint32_t parity) { alive = alive && bar_wait(bar, parity & 1, dead); };
  uint32_t turn_of_queue = 0;
  auto next = [&](Item &i) {                           // (of one thread)
    need(given(turn_of_queue), turn_of_queue / QUEUE);
    if (alive) i = queue[turn_of_queue % QUEUE];
    return alive && i.tiles > 0;
  };
  auto need_all = [&](uint32_t bar, uint32_t parity) { alive = __all_sync(~0u, bar_wait(bar, parity & 1, dead)); };
  auto next_all = [&](Item &i) {                       // of a warp
    need_all(given(turn_of_queue), turn_of_queue / QUEUE);
    if (alive) i = queue[turn_of_queue % QUEUE];
    return alive && i.tiles > 0;
  };
  // the first query of a tile, and whether it hides keys from some of its rows
  auto first_query = [&](const Item &i, int tile) { return (items.first_tile(i.t) + tile) * items.q; };
  auto hides = [&](const Item &i, int q0) { return a.causal && q0 < min(i.t * TILE + TILE, i.keys) - 1; };

  if (warp >= ROW_WARPS) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
    if (warp == ROW_WARPS + 1) {
      Stretch s = line;
      Seq q;
      Item i;
      i.b = -1;
      for (uint32_t n = 0; alive; n++) {
        if (!next_item(a, items, s, q, i, lane == 0 ? cut.ends + blockIdx.x : nullptr)) i.tiles = 0;
        if (n >= QUEUE) need_all(taken(n), n / QUEUE - 1);
        if (!alive) break;
        if (lane == 0) queue[n % QUEUE] = i, bar_arrive(given(n));
        if (i.tiles == 0) break;
        if (n) need_all(kv_empty, n - 1);
        if (!alive) break;
        if (lane == 0) {
          bar_expect(kv_full, 2 * BYTES);
          const int token = i.first + i.t * TILE;
#pragma unroll
          for (int x = 0; x < D / 64; x++) {
            tile_load(kv_at + x * COLUMNS, &maps.kv.k, x * 64, maps.kv.k_heads_first ? i.kh : token, maps.kv.k_heads_first ? token : i.kh, 0, kv_full);
            tile_load(kv_at + BYTES + x * COLUMNS, &maps.kv.v, x * 64, maps.kv.v_heads_first ? i.kh : token, maps.kv.v_heads_first ? token : i.kh, 0, kv_full);
          }
        }
        kv_copies++;
        __syncwarp();
        for (int z = 2 * i.tile0; z < 2 * i.tile1; z++, copies++) {   // queries, dout, queries, ...
          const int st = copies % STAGES;
          if (copies >= STAGES) need_all(empty(st), copies / STAGES - 1);
          if (!alive) break;
          if (lane == 0) {
            bar_expect(full(copies), box_rows * D * 2);
            const int token = i.first + first_query(i, z / 2);
#pragma unroll
            for (int x = 0; x < D / 64; x++)
              tile_load(ring_at + st * BYTES + x * COLUMNS, z % 2 ? &maps.dout : &maps.q, x * 64, i.kh * a.group, token, 0, full(copies));
          }
          __syncwarp();
        }
      }
    } else if (warp >= ROW_WARPS + 2) {
      // ---- one cleans queries and brings lse, the other dout and e
      const int which = warp - ROW_WARPS - 2;
      const float *const src = which ? a.delta : a.lse;
      const float factor_of = which ? -factor * WEIGHT_UNIT<T> : -1.4426950408889634f, shift = which ? 0.f : WEIGHT_SHIFT<T>, none = which ? 0.f : -INFINITY;
      Item i;
      int tiles = 0;
      while (next_all(i)) {
        float x[4];
        bool odd = false;                              // the asked tile has rows with lse or e that is not finite
        auto ask = [&](int t) {                        // of rows lane, lane + 32, ... of a tile
          const int q0 = first_query(i, t), live = min(items.q, i.n - q0) * a.group;
#pragma unroll
          for (int k = 0; k < 4; k++) {
            const int r = lane + k * 32, query = r / a.in_group;
            x[k] = none;
            if (r < live) x[k] = src[((int64_t)i.first + q0 + query) * a.q_heads + i.kh * a.group + r - query * a.group];
          }
        };
        auto give = [&](int t, float *to) {            // to shared memory, in the units of the weights
          const int live = min(items.q, i.n - first_query(i, t)) * a.group;
          odd = false;
#pragma unroll
          for (int k = 0; k < 4; k++) {
            const bool there = lane + k * 32 < live;
            odd |= there && !isfinite(x[k]);
            to[lane + k * 32] = there ? x[k] * factor_of + shift : none;
          }
          odd = __any_sync(~0u, odd);
        };
        ask(i.tile0);
        for (int t = i.tile0; t < i.tile1 && alive; t++, tiles++) {
          const int slot = 2 * tiles + which, q0 = first_query(i, t), live = min(items.q, i.n - q0) * a.group;
          if (tiles >= STATS) need_all(read(tiles % STATS), tiles / STATS - 1);
          if (!alive) break;
          give(t, stats + (tiles % STATS * 2 + which) * TILE);
          const bool look = odd && hides(i, q0);       // a row with values that are not finite has such an lse (queries) or e (dout)
          if (t + 1 < i.tile1) ask(t + 1);
          need_all(full(slot), slot / 8);
          if (!alive) break;
          uint32_t bad[4] = {0, 0, 0, 0};
          if (look || live < box_rows) {
            clean_tile<T, D>(ring + slot % STAGES * BYTES, lane, live, look, bad);
            fence_async();
          }
          if (which && lane == 0) {
#pragma unroll
            for (int k = 0; k < 4; k++) bad_rows[tiles % STATS * 4 + k] = bad[k];
          }
          if (which && (bad[0] | bad[1] | bad[2] | bad[3])) {   // their ds is NaN, dv gets what the tile has lost at the item's end
#pragma unroll
            for (int k = 0; k < 4; k++)
              if (bad[k] >> lane & 1) stats[(tiles % STATS * 2 + 1) * TILE + lane + k * 32] = NAN;
          }
          __syncwarp();
          if (lane == 0) bar_arrive(ready(slot));
        }
        __syncwarp();
        if (lane == 0) bar_arrive(taken(turn_of_queue));
        turn_of_queue++;
      }
    } else if (elected()) {
      issues = true;
      using P = Products<T, D>;
      const uint32_t k_op = operand(kv_at, 16), v_op = operand(kv_at + BYTES, 16);
      const uint32_t rows_op = operand(ring_at, 16), sums_op = operand(ring_at, COLUMNS);
      auto stage = [&](int slot) { return (uint32_t)(slot % STAGES * BYTES) >> 4; };
      int tiles = 0;
      uint32_t done = 0;
      auto scores = [&](int tile) {
        need(ready(2 * tile), tile / 4);
        if (!alive) return;
        tc_after();
        P::scores(s_at, k_op, rows_op + stage(2 * tile));
        tc_commit(s_full);
      };
      auto dp = [&](int tile, bool last) {
        need(ready(2 * tile + 1), tile / 4);
        if (!alive) return;
        tc_after();
        P::scores(dp_at, v_op, rows_op + stage(2 * tile + 1));
        tc_commit(dp_full);
        if (last) tc_commit(kv_empty);
      };
      Item i;
      while (next(i)) {
        const int n = i.tile1 - i.tile0;
        bar_arrive(taken(turn_of_queue++));
        need(kv_full, done);
        if (alive) scores(tiles);
        if (alive) dp(tiles, n == 1);
        for (int j = 0; j < n && alive; j++, tiles++) {
          need(p_full, tiles);
          if (j == 0 && done) need(o_free, done - 1);
          if (!alive) break;
          tc_after();
          P::sums(dv_at, s_at, sums_op + stage(2 * tiles + 1), j > 0);
          tc_commit(empty((2 * tiles + 1) % STAGES));
          if (j + 1 < n) scores(tiles + 1);
          need(ds_full, tiles);
          if (!alive) break;
          tc_after();
          P::sums(dk_at, dp_at, sums_op + stage(2 * tiles), j > 0);
          tc_commit(empty(2 * tiles % STAGES));
          if (j + 1 < n) dp(tiles + 1, j + 2 == n);
          else tc_commit(o_full);
        }
        done++;
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 104;");
    const int w = warp / 4, r = tid % 128;
    const uint32_t lanes = (uint32_t)(warp % 4 * 32) << 16;
    const float sl2 = a.scale * 1.4426950408889634f, dp_scale = factor * WEIGHT_UNIT<T>;
    const Heads &to = w < 2 ? a.dv : a.dk;
    const bool aligned = rows_aligned(to);
    int tiles = 0;
    uint32_t done = 0;
    Item i;
    while (next_all(i)) {
      const int key = i.t * TILE + r;
      bool odd = false;                                         // whether dout's tiles have lost infinite and NaN values
      for (int t = i.tile0; t < i.tile1; t++, tiles++) {
        const int q0 = first_query(i, t);
        const bool masked = hides(i, q0);
        const int first_seen = (key - q0) * a.group - w * 32;   // columns before it are rows that do not see this key
        const float *const nl = stats + tiles % STATS * 2 * TILE + w * 32, *const ne = nl + TILE;
        need(ready(2 * tiles), tiles / 4);                      // (lse)
        need(s_full, tiles);
        alive = __all_sync(~0u, alive);
        if (!alive) break;
        tc_after();
        uint32_t p[32], pk[16];
        tc_ld(p, s_at + lanes + w * 32);
        tc_ld_wait();
        const float2 scale2 = make_float2(sl2, sl2);
#pragma unroll
        for (int c = 0; c < 32; c += 4) {
          const float4 l = *(const float4 *)(nl + c);
          const float2 x = fma2(make_float2(__uint_as_float(p[c]), __uint_as_float(p[c + 1])), scale2, make_float2(l.x, l.y));
          const float2 y = fma2(make_float2(__uint_as_float(p[c + 2]), __uint_as_float(p[c + 3])), scale2, make_float2(l.z, l.w));
          p[c] = __float_as_uint(exp2_fast(x.x)), p[c + 1] = __float_as_uint(exp2_fast(x.y));
          p[c + 2] = __float_as_uint(exp2_fast(y.x)), p[c + 3] = __float_as_uint(exp2_fast(y.y));
        }
        need(ready(2 * tiles + 1), tiles / 4);                  // (e)
        if (masked) {
          const uint32_t *const bad = bad_rows + tiles % STATS * 4;
          odd |= (bad[0] | bad[1] | bad[2] | bad[3]) != 0;
#pragma unroll
          for (int c = 0; c < 32; c++) p[c] = c < first_seen ? 0 : p[c];
        }
#pragma unroll
        for (int c = 0; c < 32; c += 2) pk[c / 2] = pack<T>(__uint_as_float(p[c]), __uint_as_float(p[c + 1]));
        __syncwarp();
        tc_st16(s_at + lanes + w * 32, pk);
        tc_st_wait();
        tc_before();
        bar_arrive(p_full);

        need(dp_full, tiles);
        alive = __all_sync(~0u, alive);
        if (!alive) break;
        tc_after();
        const float2 dp2 = make_float2(dp_scale, dp_scale);
        uint32_t d[32];
        tc_ld(d, dp_at + lanes + w * 32);
        tc_ld_wait();
#pragma unroll
        for (int c = 0; c < 32; c += 4) {
          const float4 e = *(const float4 *)(ne + c);
          const float2 x = fma2(make_float2(__uint_as_float(d[c]), __uint_as_float(d[c + 1])), dp2, make_float2(e.x, e.y));
          const float2 y = fma2(make_float2(__uint_as_float(d[c + 2]), __uint_as_float(d[c + 3])), dp2, make_float2(e.z, e.w));
          float2 u = mul2(make_float2(__uint_as_float(p[c]), __uint_as_float(p[c + 1])), x);
          float2 v = mul2(make_float2(__uint_as_float(p[c + 2]), __uint_as_float(p[c + 3])), y);
          if (masked) {
            u.x = c < first_seen ? 0.f : u.x, u.y = c + 1 < first_seen ? 0.f : u.y;
            v.x = c + 2 < first_seen ? 0.f : v.x, v.y = c + 3 < first_seen ? 0.f : v.y;
          }
          pk[c / 2] = pack<T>(u.x, u.y), pk[c / 2 + 1] = pack<T>(v.x, v.y);
        }
        tc_st16(dp_at + lanes + w * 32, pk);
        tc_st_wait();
        tc_before();
        bar_arrive(ds_full);
        __syncwarp();
        if (lane == 0) bar_arrive(read(tiles % STATS));
      }
      if (!alive) break;
      need_all(o_full, done);
      if (!alive) break;
      done++;
      tc_after();
      if (w < 2 && __any_sync(~0u, odd)) {
        // dout's values that are not finite, from tiles that hide rows from some keys: each for the keys that its row sees
#pragma unroll 1
        for (int c = 0; c < D / 2; c += 16) {
          uint32_t o[16];
          const uint32_t at = dv_at + lanes + w * (D / 2) + c;
          tc_ld16(o, at);
          tc_ld_wait();
#pragma unroll 1
          for (int t = i.tile0; t < i.tile1 && hides(i, first_query(i, t)); t++) {
            const int q0 = first_query(i, t), live = min(items.q, i.n - q0) * a.group;
#pragma unroll 1
            for (int x = 0; x < live; x++) {
              const int query = q0 + x / a.in_group, head = i.kh * a.group + x % a.in_group;
              if (query < key || isfinite(a.delta[((int64_t)i.first + query) * a.q_heads + head])) continue;
              const T *const from = row_at<const T>(a.dout, (int64_t)i.first + query, head) + w * (D / 2) + c;
#pragma unroll
              for (int z = 0; z < 16; z++) {
                const float v = widen(from[z]);
                if (!isfinite(v)) o[z] = __float_as_uint(__uint_as_float(o[z]) + v);
              }
            }
          }
          __syncwarp();
          tc_st16(at, o);
          tc_st_wait();
        }
      }
      const bool whole = i.tile0 == 0 && i.tile1 == i.tiles;
      float4 *const part = whole ? nullptr : cut.o + ((((int64_t)blockIdx.x * 2 + (i.tile0 == 0)) * 2 + w / 2) * (D / 4) + w % 2 * (D / 8)) * TILE + r;
      store_row<T, D / 2>((w < 2 ? dv_at : dk_at) + lanes + w % 2 * (D / 2), row_at<T>(to, (int64_t)i.first + key, i.kh) + w % 2 * (D / 2), part, key < i.keys,
                          aligned, w < 2 ? WEIGHT_UNIT<T> : a.scale / factor);
      tc_before();
      bar_arrive(o_free);
      __syncwarp();
      if (lane == 0) bar_arrive(taken(turn_of_queue));
      turn_of_queue++;
    }
  }
  tc_before();
  __syncthreads();
  if (*dead) {
    const uint64_t from = now_ns();
    if (issues) {
      tc_commit(ended);
      while (!bar_try(ended, 0) && now_ns() - from < DRAIN_NS) {}
    }
    if (warp == ROW_WARPS + 1) {
#pragma unroll 1
      for (int x = max(0, copies - STAGES); x < copies; x++)
        while (!bar_try(full(x), (x / 8) & 1) && now_ns() - from < DRAIN_NS) {}
      while (kv_copies && !bar_try(kv_full, (kv_copies - 1) & 1) && now_ns() - from < DRAIN_NS) {}
    }
    if (tid == 0 && a.status) *a.status = GTS_ERR_STEP_LIMIT;
    __syncthreads();
    Stretch s = line;
    Seq q;
    Item i;
    i.b = -1;
    while (next_item(a, items, s, q, i, tid == 0 ? cut.ends + blockIdx.x : nullptr)) {
      const bool whole = i.tile0 == 0 && i.tile1 == i.tiles;
      for (int x = tid; x < 2 * TILE * D; x += GRAD_THREADS) {
        const int w = x / (TILE * D), r = x / D % TILE, d = x % D, key = i.t * TILE + r;
        if (key >= i.keys) continue;
        if (whole) row_at<T>(w ? a.dk : a.dv, (int64_t)i.first + key, i.kh)[d] = narrow<T>(NAN);
        else if (d % 4 == 0) cut.o[((((int64_t)blockIdx.x * 2 + (i.tile0 == 0)) * 2 + w) * (D / 4) + d / 4) * TILE + r] = make_float4(NAN, NAN, NAN, NAN);
      }
    }
  }
  if (warp == ROW_WARPS) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
}

// Queries.  Warp 17 walks along the stretch and brings an item's queries and dout and then its tiles of keys and values; warp 18 cleans
// tiles of keys in which some are out of sight.  Warp 16 issues the products:
//   S = Q K^T (in two buffers), dP = dout V^T, dQ += dS K
// in the order (next dP, dQ, S of the tile after), so that the rows find their next scores and dP ready.  dS overwrites S.
// Warps 0..15: a thread for a row and a quarter of a tile's keys.
template <int D> struct GradQ {
  static constexpr int BYTES = TILE * D * 2, STAGES = D == 64 ? 8 : 5;
  static constexpr int BEHIND = 1152, SMEM = (2 + STAGES) * BYTES + BEHIND;
};

template <typename T, int D>
__global__ void __launch_bounds__(GRAD_THREADS, 1) k_grad_q(const Args a, const Items<false> items, const Cut cut, const Largest *largest, const __grid_constant__ GradMaps maps) {
  constexpr int BYTES = GradQ<D>::BYTES, STAGES = GradQ<D>::STAGES, COLUMNS = TILE * 128;
  extern __shared__ __align__(1024) unsigned char smem[];
  unsigned char *const rows = smem, *const ring = rows + 2 * BYTES;
  uint64_t *const bars = (uint64_t *)(ring + STAGES * BYTES);
  constexpr int BARS = 8 + STAGES + 2 * QUEUE + 14;
  Item *const queue = (Item *)(bars + BARS);
  uint32_t *const tmem_at = (uint32_t *)(queue + QUEUE);
  volatile int *const dead = (volatile int *)(tmem_at + 1);
  void *const scratch = (void *)(tmem_at + 2);
  static_assert(BARS * 8 + QUEUE * sizeof(Item) + 8 + SCRATCH <= GradQ<D>::BEHIND && QUEUE * sizeof(Item) % 8 == 0, "room behind the ring, and its alignment");
  const int tid = threadIdx.x, warp = __shfl_sync(~0u, tid / 32, 0), lane = tid % 32;
  const uint32_t bar0 = smem_u32(bars), rows_at = smem_u32(rows), ring_at = smem_u32(ring);
  // a ring of barriers for keys and one for values: who waits for either sees each of its phases
  auto full = [&](int slot) { return bar0 + (slot % 2 * 4 + slot / 2 % 4) * 8; };
  auto empty = [&](int s) { return bar0 + (8 + s) * 8; };
  auto given = [&](uint32_t i) { return bar0 + (8 + STAGES + i % QUEUE) * 8; };
  auto taken = [&](uint32_t i) { return bar0 + (8 + STAGES + QUEUE + i % QUEUE) * 8; };
  const uint32_t rest = bar0 + (8 + STAGES + 2 * QUEUE) * 8;
  const uint32_t q_full = rest, q_empty = rest + 8, dp_full = rest + 16, ds_full = rest + 24, o_full = rest + 32, o_free = rest + 40, ended = rest + 48;
  auto s_full = [&](int tile) { return rest + 56 + tile % 2 * 8; };
  auto ready = [&](int tile) { return rest + 72 + tile % 4 * 8; };                      // its keys are clean

  dependents_may_start();
  Stretch line = find_stretch<false, GRAD_THREADS>(a, items, cut.blocks, scratch);
  if (line.rest_from + a.n_tokens - line.rest_to > 0 && a.zero_rest & 1) zero_rest<T>(a, a.dq, a.q_heads, D, line);
  if (tid == 0) cut.ends[blockIdx.x] = make_int4(NOTHING, 0, 0, 0);
  // k_grad_kv has waited for e, but what lets this grid see it is a wait of its own.  Every thread waits here, before any wait that has a
  // limit (a block of k_grad_kv may take longer than another one by more than that), and every block does, so that the joining kernel
  // needs to wait for one kernel only.
  wait_for_kernels_before();
  if (line.x0 >= line.x1) return;
  const float factor = ds_factor<T>(largest, scratch);
  if (tid == 0) {
    for (int s = 0; s < 8; s++) bar_init(full(s), 1);
    for (int s = 0; s < STAGES; s++) bar_init(empty(s), 1);
    bar_init(q_full, 1), bar_init(q_empty, 1), bar_init(dp_full, 1), bar_init(ds_full, ROW_THREADS), bar_init(o_full, 1), bar_init(o_free, ROW_THREADS), bar_init(ended, 1);
    for (int s = 0; s < 2; s++) bar_init(s_full(s), 1);
    for (int s = 0; s < 4; s++) bar_init(ready(s), 1);
    for (int i = 0; i < QUEUE; i++) bar_init(given(i), 1), bar_init(taken(i), ROW_WARPS + 2);
    *dead = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == ROW_WARPS) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(tmem_at)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  }
  tc_before();
  __syncthreads();
  tc_after();
  const uint32_t tmem = __shfl_sync(~0u, *tmem_at, 0), dp_at = tmem + 256, dq_at = tmem + 384;
  auto s_at = [&](int tile) { return tmem + tile % 2 * 128; };
  int copies = 0, q_copies = 0;
  bool issues = false, alive = true;
  auto need = [&](uint32_t bar, uint32_t parity) { alive = alive && bar_wait(bar, parity & 1, dead); };
  uint32_t turn_of_queue = 0;
  auto next = [&](Item &i) {                           // (of one thread)
    need(given(turn_of_queue), turn_of_queue / QUEUE);
    if (alive) i = queue[turn_of_queue % QUEUE];
    return alive && i.tiles > 0;
  };
  auto need_all = [&](uint32_t bar, uint32_t parity) { alive = __all_sync(~0u, bar_wait(bar, parity & 1, dead)); };
  auto next_all = [&](Item &i) {                       // of a warp
    need_all(given(turn_of_queue), turn_of_queue / QUEUE);
    if (alive) i = queue[turn_of_queue % QUEUE];
    return alive && i.tiles > 0;
  };

  if (warp >= ROW_WARPS) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
    if (warp == ROW_WARPS + 1) {
      Stretch s = line;
      Seq q;
      Item i;
      i.b = -1;
      for (uint32_t n = 0; alive; n++) {
        if (!next_item(a, items, s, q, i, lane == 0 ? cut.ends + blockIdx.x : nullptr)) i.tiles = 0;
        if (n >= QUEUE) need_all(taken(n), n / QUEUE - 1);
        if (!alive) break;
        if (lane == 0) queue[n % QUEUE] = i, bar_arrive(given(n));
        if (i.tiles == 0) break;
        if (n) need_all(q_empty, n - 1);
        if (!alive) break;
        if (lane == 0) {
          bar_expect(q_full, 2 * items.q * a.group * D * 2);
          const int token = i.first + i.t * items.q;
#pragma unroll
          for (int x = 0; x < D / 64; x++) {
            tile_load(rows_at + x * COLUMNS, &maps.q, x * 64, i.kh * a.group, token, 0, q_full);
            tile_load(rows_at + BYTES + x * COLUMNS, &maps.dout, x * 64, i.kh * a.group, token, 0, q_full);
          }
        }
        q_copies++;
        __syncwarp();
        for (int x = 2 * i.tile0; x < 2 * i.tile1; x++, copies++) {   // keys, values, keys, ...
          const int st = copies % STAGES, token = i.first + x / 2 * TILE;
          if (copies >= STAGES) need_all(empty(st), copies / STAGES - 1);
          if (!alive) break;
          const bool heads_first = x % 2 ? maps.kv.v_heads_first : maps.kv.k_heads_first;
          if (lane == 0) {
            bar_expect(full(copies), BYTES);
#pragma unroll
            for (int c = 0; c < D / 64; c++)
              tile_load(ring_at + st * BYTES + c * COLUMNS, x % 2 ? &maps.kv.v : &maps.kv.k, c * 64, heads_first ? i.kh : token, heads_first ? token : i.kh, 0, full(copies));
          }
          __syncwarp();
        }
      }
    } else if (warp == ROW_WARPS + 2) {
      Item i;
      int tiles = 0;
      while (next_all(i)) {
        const int clear = seen_by_all(a, i, i.t * items.q);
        for (int t = i.tile0; t < i.tile1 && alive; t++, tiles++) {
          const int slot = 2 * tiles;
          need_all(full(slot), slot / 8);
          if (!alive) break;
          if ((t + 1) * TILE > clear) {
            uint32_t bad[4];
            clean_tile<T, D>(ring + slot % STAGES * BYTES, lane, i.keys - t * TILE, a.causal, bad);
            fence_async();
          }
          __syncwarp();
          if (lane == 0) bar_arrive(ready(tiles));
        }
        __syncwarp();
        if (lane == 0) bar_arrive(taken(turn_of_queue));
        turn_of_queue++;
      }
    } else if (warp == ROW_WARPS && elected()) {
      issues = true;
      using P = Products<T, D>;
      const uint32_t q_op = operand(rows_at, 16), do_op = operand(rows_at + BYTES, 16), rows_op = operand(ring_at, 16), sums_op = operand(ring_at, COLUMNS);
      auto stage = [&](int slot) { return (uint32_t)(slot % STAGES * BYTES) >> 4; };
      int tiles = 0;
      uint32_t done = 0;
      auto scores = [&](int tile) {
        need(ready(tile), tile / 4);
        if (!alive) return;
        tc_after();
        P::scores(s_at(tile), q_op, rows_op + stage(2 * tile));
        tc_commit(s_full(tile));
      };
      auto dp = [&](int tile, bool last) {
        need(full(2 * tile + 1), (2 * tile + 1) / 8);
        if (!alive) return;
        tc_after();
        P::scores(dp_at, do_op, rows_op + stage(2 * tile + 1));
        tc_commit(dp_full);
        tc_commit(empty((2 * tile + 1) % STAGES));
        if (last) tc_commit(q_empty);
      };
      Item i;
      while (next(i)) {
        const int n = i.tile1 - i.tile0;
        bar_arrive(taken(turn_of_queue++));
        need(q_full, done);
        if (alive) scores(tiles);
        if (alive) dp(tiles, n == 1);
        if (alive && n > 1) scores(tiles + 1);
        for (int j = 0; j < n && alive; j++, tiles++) {
          need(ds_full, tiles);
          if (j == 0 && done) need(o_free, done - 1);
          if (!alive) break;
          tc_after();
          if (j + 1 < n) dp(tiles + 1, j + 2 == n);
          if (!alive) break;
          P::sums(dq_at, s_at(tiles), sums_op + stage(2 * tiles), j > 0);
          tc_commit(empty(2 * tiles % STAGES));
          if (j + 2 < n) scores(tiles + 2);
          if (j + 1 == n) tc_commit(o_full);
        }
        done++;
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 104;");
    const int w = warp / 4, r = tid % 128, in_tile = r / a.in_group, head_in = r - in_tile * a.group;
    const uint32_t lanes = (uint32_t)(warp % 4 * 32) << 16;
    const float sl2 = a.scale * 1.4426950408889634f, dp_scale = factor * WEIGHT_UNIT<T>;
    const bool aligned = rows_aligned(a.dq);
    int tiles = 0;
    uint32_t done = 0;
    Item i = {};
    float nl = 0.f, ne = 0.f;
    auto ask = [&] {                                     // the item's lse and e of this row
      const int query = i.t * items.q + in_tile;
      if (in_tile < items.q && query < i.n) {
        const int64_t at = ((int64_t)i.first + query) * a.q_heads + i.kh * a.group + head_in;
        nl = a.lse[at], ne = a.delta[at];
      }
    };
    bool more = next_all(i);
    if (more) ask();
    while (more) {
      const int query = i.t * items.q + in_tile, limit = a.causal ? min(i.keys, query + 1) : i.keys, clear = seen_by_all(a, i, i.t * items.q);
      const bool valid = in_tile < items.q && query < i.n, whole = i.tile0 == 0 && i.tile1 == i.tiles;
      const int64_t row = (int64_t)i.first + query;
      const int head = i.kh * a.group + head_in, first_part = i.tile0 == 0;
      nl = WEIGHT_SHIFT<T> - nl * 1.4426950408889634f, ne = -ne * dp_scale;
      for (int t = i.tile0; t < i.tile1; t++, tiles++) {
        const bool masked = (t + 1) * TILE > clear;
        const int seen = limit - t * TILE - w * 32;
        need_all(s_full(tiles), tiles / 2);
        if (!alive) break;
        tc_after();
        const uint32_t at = s_at(tiles) + lanes + w * 32;
        uint32_t p[32], d[32], pk[16];
        tc_ld(p, at);
        tc_ld_wait();
        const float2 scale2 = make_float2(sl2, sl2), nl2 = make_float2(nl, nl);
#pragma unroll
        for (int c = 0; c < 32; c += 2) {
          const float2 x = fma2(make_float2(__uint_as_float(p[c]), __uint_as_float(p[c + 1])), scale2, nl2);
          p[c] = __float_as_uint(exp2_fast(x.x)), p[c + 1] = __float_as_uint(exp2_fast(x.y));
        }
        need_all(dp_full, tiles);
        if (!alive) break;
        tc_after();
        const float2 dp2 = make_float2(dp_scale, dp_scale), ne2 = make_float2(ne, ne);
        tc_ld(d, dp_at + lanes + w * 32);
        tc_ld_wait();
#pragma unroll
        for (int c = 0; c < 32; c += 2) {
          const float2 x = fma2(make_float2(__uint_as_float(d[c]), __uint_as_float(d[c + 1])), dp2, ne2);
          float2 u = mul2(make_float2(__uint_as_float(p[c]), __uint_as_float(p[c + 1])), x);
          if (masked) u.x = c < seen ? u.x : 0.f, u.y = c + 1 < seen ? u.y : 0.f;
          pk[c / 2] = pack<T>(u.x, u.y);
        }
        tc_st16(at, pk);
        tc_st_wait();
        tc_before();
        bar_arrive(ds_full);
      }
      if (!alive) break;
      __syncwarp();
      if (lane == 0) bar_arrive(taken(turn_of_queue));
      turn_of_queue++;
      more = next_all(i);                                // (given as soon as this item's tiles have been asked for)
      if (!alive) break;
      if (more) ask();                                   // arrives while the last products run and the results are stored
      need_all(o_full, done);
      if (!alive) break;
      done++;
      tc_after();
      if (w < D / 32) {
        float4 *const part = whole ? nullptr : cut.o + (((int64_t)blockIdx.x * 2 + first_part) * (D / 4) + w * 8) * TILE + r;
        store_row<T, 32>(dq_at + lanes + w * 32, row_at<T>(a.dq, row, head) + w * 32, part, valid, aligned, a.scale / factor);
      }
      tc_before();
      bar_arrive(o_free);
    }
  }
  tc_before();
  __syncthreads();
  if (*dead) {
    const uint64_t from = now_ns();
    if (issues) {
      tc_commit(ended);
      while (!bar_try(ended, 0) && now_ns() - from < DRAIN_NS) {}
    }
    if (warp == ROW_WARPS + 1) {
#pragma unroll 1
      for (int x = max(0, copies - STAGES); x < copies; x++)
        while (!bar_try(full(x), (x / 8) & 1) && now_ns() - from < DRAIN_NS) {}
      while (q_copies && !bar_try(q_full, (q_copies - 1) & 1) && now_ns() - from < DRAIN_NS) {}
    }
    if (tid == 0 && a.status) *a.status = GTS_ERR_STEP_LIMIT;
    __syncthreads();
    Stretch s = line;
    Seq q;
    Item i;
    i.b = -1;
    while (next_item(a, items, s, q, i, tid == 0 ? cut.ends + blockIdx.x : nullptr)) {
      const bool whole = i.tile0 == 0 && i.tile1 == i.tiles;
      for (int x = tid; x < TILE * D; x += GRAD_THREADS) {
        const int r = x / D, d = x % D, in_tile = r / a.in_group, query = i.t * items.q + in_tile;
        if (in_tile >= items.q || query >= i.n) continue;
        if (whole) row_at<T>(a.dq, (int64_t)i.first + query, i.kh * a.group + r - in_tile * a.group)[d] = narrow<T>(NAN);
        else if (d % 4 == 0) cut.o[(((int64_t)blockIdx.x * 2 + (i.tile0 == 0)) * (D / 4) + d / 4) * TILE + r] = make_float4(NAN, NAN, NAN, NAN);
      }
    }
  }
  if (warp == ROW_WARPS) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
}

// Sums of the parts of items that were cut, in their order: a thread for a row and an eighth of its columns.
template <typename T, int D, bool BY_KEYS>
__device__ __forceinline__ void join_grad(const Args &a, const Items<BY_KEYS> &items, const Cut &cut, const Largest *largest, int block) {
  constexpr int ROWS = BY_KEYS ? 2 * TILE : TILE, E = D / 32;   // (keys' gradients after values')
  const int c = block / (ROWS / 32), lane = threadIdx.x % 32, column = threadIdx.x / 32;
  const int4 end = cut.ends[c];
  if (end.x < 0) return;
  const Seq s = sequence(a, end.x);
  const int row = block % (ROWS / 32) * 32 + lane, which = row / TILE, r = row % TILE;
  float f = a.scale;
  if (BY_KEYS && which == 0) {
    f = WEIGHT_UNIT<T>;
  } else if (std::is_same<T, __half>::value) {
    Largest most = {0.f, 0.f, 0.f};
    for (int i = lane; i < DELTA_BLOCKS; i += 32) most = most_of(most, largest[i]);
    f = ldexpf(f, -ds_exponent(most_of_warp(most)));
  }
  const int in_tile = BY_KEYS ? 0 : r / a.in_group, at = BY_KEYS ? end.z * TILE + r : end.z * items.q + in_tile;
  if (at >= s.n || (!BY_KEYS && in_tile >= items.q)) return;
  const Heads &to = !BY_KEYS ? a.dq : which ? a.dk : a.dv;
  float4 acc[E] = {};
  for (int x = 0; x <= end.w; x += 2) {
    float4 v[2][E];
#pragma unroll
    for (int k = 0; k < 2; k++) {
      if (x + k <= end.w) {
#pragma unroll
        for (int e = 0; e < E; e++) v[k][e] = cut.o[((((int64_t)(c + x + k) * 2 + (x + k == 0)) * (ROWS / TILE) + which) * (D / 4) + column * E + e) * TILE + r];
      }
    }
#pragma unroll
    for (int k = 0; k < 2; k++) {
      if (x + k <= end.w) {
#pragma unroll
        for (int e = 0; e < E; e++) acc[e].x += v[k][e].x, acc[e].y += v[k][e].y, acc[e].z += v[k][e].z, acc[e].w += v[k][e].w;
      }
    }
  }
  T *const dst = row_at<T>(to, (int64_t)s.first + at, BY_KEYS ? end.y : end.y * a.group + r - in_tile * a.group) + column * E * 4;
#pragma unroll
  for (int e = 0; e < E; e++) store4(dst + 4 * e, acc[e], f, rows_aligned(to));
}

constexpr int JOIN_KV = SMS * (2 * TILE / 32), JOIN_Q = SMS * (TILE / 32);   // its blocks
template <typename T, int D>
__global__ void __launch_bounds__(JOIN_THREADS) k_join_grad(const Args a, const Items<true> by_keys, const Items<false> by_rows, const Cut kv, const Cut q, const Largest *largest) {
  wait_for_kernels_before();
  if (blockIdx.x < JOIN_KV) join_grad<T, D, true>(a, by_keys, kv, largest, blockIdx.x);
  else join_grad<T, D, false>(a, by_rows, q, largest, blockIdx.x - JOIN_KV);
}

// Rows that TMA cannot take as they lie, side by side.
template <typename T>
__global__ void __launch_bounds__(256) k_side_by_side(const Args a, const Heads from, T *to, int heads, int dim) {
  const int64_t all = (int64_t)a.n_tokens * heads * dim;
  for (int64_t x = (int64_t)blockIdx.x * 256 + threadIdx.x; x < all; x += (int64_t)gridDim.x * 256) {
    const int64_t row = x / (heads * dim);
    const int in = (int)(x - row * heads * dim);
    to[x] = row_at<const T>(from, row, in / dim)[in % dim];
  }
}

// ---------------------------------------------------------------- host side
// Maps of rows of queries: boxes of a key head's `group` heads of `queries` tokens.
bool rows_map(CUtensorMap &map, const Heads &h, int heads, int tokens, int dim, int group, int queries, bool bf16) {
  int64_t head = heads == 1 ? h.tok : h.head, tok = tokens == 1 ? head * heads : h.tok;
  if (heads == 1 && tokens == 1) head = tok = dim;
  if ((uintptr_t)h.data % 16 || head % 8 || head < dim || tok < head || tok % head || tok >= 1ll << 38) return false;
  const EncodeTiled encode = encode_tiled();
  if (!encode) return false;
  const cuuint64_t dims[4] = {(cuuint64_t)dim, (cuuint64_t)heads, (cuuint64_t)tokens, 1};
  const cuuint64_t strides[3] = {(cuuint64_t)head * 2, (cuuint64_t)tok * 2, (cuuint64_t)tok * 2 * (cuuint64_t)tokens};
  const cuuint32_t boxes[4] = {64, (cuuint32_t)group, (cuuint32_t)queries, 1}, ones[4] = {1, 1, 1, 1};
  return strides[2] < 1ull << 40 && encode(&map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, (void *)h.data, dims, strides, boxes, ones,
                                           CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                           CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The forward pass's workspace.
size_t plan(Cut &c, int dim, char *at) {
  size_t n = 0;
  auto take = [&](size_t bytes) {
    char *x = at ? at + n : nullptr;
    n += up(bytes);
    return x;
  };
  c.blocks = SMS;
  c.ends = (int4 *)take(SMS * sizeof(int4));
  c.ml = (float2 *)take((size_t)SMS * 2 * 256 * sizeof(float2));
  c.o = (float4 *)take((size_t)SMS * 2 * 256 * dim * sizeof(float));
  return n;
}

template <typename T, int D>
cudaError_t forward(const Args &a, const FwdMaps &maps, int64_t most_keys, char *workspace, cudaStream_t s) {
  static std::atomic<uint64_t> granted{0};
  cudaError_t e = grant(k_forward<T, D>, Fwd<D>::SMEM, granted);
  if (e != cudaSuccess) return e;
  Cut cut;
  const Items<false> items = {2 * (128 / a.group), a.causal};
  plan(cut, D, workspace);
  e = launch_kernel(k_forward<T, D>, cut.blocks, FWD_THREADS, Fwd<D>::SMEM, s, false, a, items, cut, maps);
  if (e != cudaSuccess || most_keys <= TILE) return e;   // (items of one tile are not cut)
  return launch_kernel(k_join<T, D>, cut.blocks * JOIN_BLOCKS, JOIN_THREADS, 0, s, true, a, items, cut);
}
cudaError_t run_forward(const Args &a, FwdMaps &maps, int32_t dtype, uint32_t dim, void *workspace, cudaStream_t s) {
  char *const w = (char *)workspace;
  maps.has_q = rows_map(maps.q, a.q, a.q_heads, a.n_tokens, (int)dim, a.group, TILE / a.group, dtype == GTS_BF16);
  const int64_t most = a.paged ? (int64_t)a.max_pages * a.page_size : a.n_tokens;   // keys of a sequence
  if (dtype == GTS_BF16) return dim == 64 ? forward<__nv_bfloat16, 64>(a, maps, most, w, s) : forward<__nv_bfloat16, 128>(a, maps, most, w, s);
  return dim == 64 ? forward<__half, 64>(a, maps, most, w, s) : forward<__half, 128>(a, maps, most, w, s);
}

// The gradients' workspace: e of every row, what bounds ds in float16, partial results, and q, dout, k, v where TMA cannot take
// them as they lie.
struct GradPlan {
  float *delta;
  Largest *largest;
  Cut kv, q;
  char *copy[4];
  size_t bytes;
};
GradPlan plan_grad(const gts_prompt_grad_desc &d, const bool (&copied)[4], char *at) {
  const gts_prompt_desc &f = d.forward;
  GradPlan p = {};
  auto take = [&](size_t bytes) {
    char *x = at ? at + p.bytes : nullptr;
    p.bytes += up(bytes);
    return x;
  };
  p.delta = (float *)take((size_t)f.n_tokens * f.q_heads * sizeof(float));
  p.largest = (Largest *)take(DELTA_BLOCKS * sizeof(Largest));
  p.kv.blocks = p.q.blocks = SMS;
  p.kv.ends = (int4 *)take(SMS * sizeof(int4)), p.q.ends = (int4 *)take(SMS * sizeof(int4));
  p.kv.o = (float4 *)take((size_t)SMS * 2 * 2 * TILE * f.head_dim * sizeof(float));
  p.q.o = (float4 *)take((size_t)SMS * 2 * TILE * f.head_dim * sizeof(float));
  for (int i = 0; i < 4; i++)
    if (copied[i]) p.copy[i] = take((size_t)f.n_tokens * (i < 2 ? f.q_heads : f.kv_heads) * f.head_dim * 2);
  return p;
}

void packed_maps(Pages &p, const gts_prompt_desc &d);

// The maps, and which of q, dout, k and v have to be copied for theirs.
void grad_maps(GradMaps &m, const gts_prompt_grad_desc &d, bool (&copied)[4]) {
  const gts_prompt_desc &f = d.forward;
  const int group = (int)(f.q_heads / f.kv_heads);
  const bool bf16 = f.dtype == GTS_BF16;
  auto rows = [&](CUtensorMap &map, const gts_heads &h) {
    return rows_map(map, {h.data, h.token_stride, h.head_stride}, (int)f.q_heads, (int)f.n_tokens, (int)f.head_dim, group, TILE / group, bf16);
  };
  copied[0] = !rows(m.q, f.q), copied[1] = !rows(m.dout, d.dout);
  packed_maps(m.kv, f);
  copied[2] = copied[3] = !m.kv.box;
}

template <typename T, int D>
cudaError_t backward(const Args &a, const GradPlan &p, const GradMaps &maps, cudaStream_t s) {
  static std::atomic<uint64_t> granted_kv{0}, granted_q{0};
  cudaError_t e = grant(k_grad_kv<T, D>, GradKv<D>::SMEM, granted_kv);
  if (e == cudaSuccess) e = grant(k_grad_q<T, D>, GradQ<D>::SMEM, granted_q);
  if (e != cudaSuccess) return e;
  const int queries = TILE / a.group;
  const Items<true> by_keys = {queries, a.causal};
  const Items<false> by_rows = {queries, a.causal};
  const Largest *const largest = p.largest;
  e = launch_kernel(k_delta<T, D>, DELTA_BLOCKS, DELTA_THREADS, 0, s, false, a, p.largest);
  // each may start while the one before it ends, and waits for all of it before it reads what that, or one before, has written
  if (e == cudaSuccess) e = launch_kernel(k_grad_kv<T, D>, SMS, GRAD_THREADS, GradKv<D>::SMEM, s, true, a, by_keys, p.kv, largest, maps);
  if (e == cudaSuccess) e = launch_kernel(k_grad_q<T, D>, SMS, GRAD_THREADS, GradQ<D>::SMEM, s, true, a, by_rows, p.q, largest, maps);
  if (e == cudaSuccess && a.n_tokens > queries)          // (else no item has more than a tile)
    e = launch_kernel(k_join_grad<T, D>, JOIN_KV + JOIN_Q, JOIN_THREADS, 0, s, true, a, by_keys, by_rows, p.kv, p.q, largest);
  return e;
}

template <typename T> cudaError_t side_by_side(const Args &a, Heads &h, int heads, int dim, char *to, cudaStream_t s) {
  const Heads from = h;
  const int64_t all = (int64_t)a.n_tokens * heads * dim;
  const cudaError_t e = launch_kernel(k_side_by_side<T>, (unsigned)std::min<int64_t>(SMS * 8, (all + 255) / 256), 256, 0, s, false, a, from, (T *)to, heads, dim);
  h = {to, (int64_t)heads * dim, dim};
  return e;
}

template <typename T>
cudaError_t run_grad(Args a, const GradPlan &p, GradMaps &maps, const gts_prompt_grad_desc &d, cudaStream_t s) {
  const int dim = (int)d.forward.head_dim;
  gts_prompt_grad_desc c = d;
  Heads *const from[4] = {&a.q, &a.dout, &a.k, &a.v};
  gts_heads *const to[4] = {&c.forward.q, &c.dout, &c.forward.k, &c.forward.v};
  bool any = false;
  for (int i = 0; i < 4; i++) {
    if (!p.copy[i]) continue;
    const cudaError_t e = side_by_side<T>(a, *from[i], i < 2 ? a.q_heads : a.kv_heads, dim, p.copy[i], s);
    if (e != cudaSuccess) return e;
    *to[i] = {(void *)from[i]->data, from[i]->tok, from[i]->head};
    any = true;
  }
  if (any) {
    bool copied[4];
    grad_maps(maps, c, copied);
    if (copied[0] || copied[1] || copied[2]) return cudaErrorInvalidValue;
  }
  return dim == 64 ? backward<T, 64>(a, p, maps, s) : backward<T, 128>(a, p, maps, s);
}

// What all of these calls refuse.
const char *refuse(uint32_t n_seqs, uint32_t n_tokens, uint32_t q_heads, uint32_t kv_heads, uint32_t head_dim, int32_t dtype) {
  if (dtype != GTS_BF16 && dtype != GTS_F16) return "attention: dtype must be GTS_BF16 or GTS_F16";
  if (head_dim != 64 && head_dim != 128) return "attention: head_dim must be 64 or 128";
  if (kv_heads < 1 || kv_heads > 1024 || q_heads < 1 || q_heads % kv_heads || q_heads / kv_heads > 128)
    return "attention: q_heads must be a multiple of kv_heads, at most 128 times it (1 <= kv_heads <= 1024)";
  if (n_seqs > 65535 || n_tokens > 1u << 28) return "attention: at most 65535 sequences and 2^28 tokens";
  if ((uint64_t)n_tokens * q_heads > 1u << 30) return "attention: more than 2^30 rows of queries";
  return nullptr;
}
bool misaligned(const gts_heads &h) { return (uintptr_t)h.data % 2; }
Heads heads(const gts_heads &h) { return {h.data, h.token_stride, h.head_stride}; }

const char *refuse_shape(const gts_prompt_desc &d) {
  if (const char *why = refuse(d.n_seqs, d.n_tokens, d.q_heads, d.kv_heads, d.head_dim, d.dtype)) return why;
  if (d.causal > 1 || d.zero_rest > 7) return "attention: causal is 0 or 1, zero_rest at most 7";
  return nullptr;
}
const char *refuse_call(const gts_prompt_desc &d, bool null_ok) {
  if (!(d.scale > 0.f) || std::isinf(d.scale)) return "attention: scale must be positive";
  if (!d.starts) return "attention: null starts";
  if (!null_ok && (!d.q.data || !d.k.data || !d.v.data || !d.out.data)) return "attention: null q, k, v or out";
  if (misaligned(d.q) || misaligned(d.k) || misaligned(d.v) || misaligned(d.out) || misaligned(d.low) ||
      ((uintptr_t)d.starts | (uintptr_t)d.lse | (uintptr_t)d.d_status) % 4)
    return "attention: tensor misaligned for its type";
  if (!d.workspace || (uintptr_t)d.workspace % 16) return "attention: null or misaligned workspace";
  return nullptr;
}
Args args(const gts_prompt_desc &d) {
  Args a = {};
  a.q = heads(d.q), a.k = heads(d.k), a.v = heads(d.v), a.out = heads(d.out);
  if (d.low.data) a.low = heads(d.low);
  a.lse = d.lse, a.starts = d.starts;
  a.n_seqs = (int)d.n_seqs, a.n_tokens = (int)d.n_tokens, a.q_heads = (int)d.q_heads, a.kv_heads = (int)d.kv_heads;
  a.group = a.q_heads / a.kv_heads, a.in_group = divisor(a.group), a.causal = (int)d.causal, a.zero_rest = (int)d.zero_rest;
  a.scale = d.scale, a.status = d.d_status;
  return a;
}

// Maps of packed keys and values: one page of all tokens.
void packed_maps(Pages &p, const gts_prompt_desc &d) {
  gts_cache c = {};
  c.n_pages = 1, c.page_size = d.n_tokens, c.kv_heads = d.kv_heads, c.head_dim = d.head_dim, c.dtype = d.dtype;
  p.box = TILE;
  if (!tile_map(p.k, p.k_heads_first, TILE, c, d.k.data, 0, d.k.token_stride, d.k.head_stride) ||
      !tile_map(p.v, p.v_heads_first, TILE, c, d.v.data, 0, d.v.token_stride, d.v.head_stride))
    p.box = 0;
}

const char *refuse_shape(const gts_chunk_desc &d) {
  const gts_cache &c = d.cache;
  if (const char *why = refuse(d.n_seqs, d.n_tokens, d.q_heads, c.kv_heads, c.head_dim, c.dtype)) return why;
  if (d.zero_rest > 3) return "attention: zero_rest is at most 3";
  if (c.page_size < 1 || c.page_size > 65536 || c.n_pages > 1u << 30 || d.max_pages > 1u << 30)
    return "attention: 1 <= page_size <= 65536, at most 2^30 pages";
  if ((uint64_t)d.max_pages * c.page_size > 1u << 30) return "attention: a sequence of more than 2^30 tokens";
  return nullptr;
}

}  // namespace

extern "C" size_t gts_prompt_workspace_bytes(const gts_prompt_desc *d) {
  Cut c;
  return !d || refuse_shape(*d) ? 0 : plan(c, (int)d->head_dim, nullptr);
}

extern "C" gts_status gts_prompt_attention(const gts_prompt_desc *d, void *stream) {
  gts::clear_error();
  if (!d) return gts::fail(GTS_ERR_INVALID_ARG, "attention: null desc");
  if (const char *why = refuse_shape(*d)) return gts::fail(GTS_ERR_INVALID_ARG, why);
  if (d->n_tokens == 0) return GTS_OK;
  if (const char *why = refuse_call(*d, false)) return gts::fail(GTS_ERR_INVALID_ARG, why);
  if (d->workspace_bytes < gts_prompt_workspace_bytes(d))
    return gts::fail(GTS_ERR_NOMEM, "attention: workspace smaller than gts_prompt_workspace_bytes");
  FwdMaps maps = {};
  packed_maps(maps.kv, *d);
  const cudaError_t e = run_forward(args(*d), maps, d->dtype, d->head_dim, d->workspace, (cudaStream_t)stream);
  return e == cudaSuccess ? GTS_OK : gts::cuda_fail(e, "attention: launch");
}

extern "C" size_t gts_prompt_grad_workspace_bytes(const gts_prompt_grad_desc *d) {
  if (!d || refuse_shape(d->forward)) return 0;
  GradMaps maps = {};
  bool copied[4];
  grad_maps(maps, *d, copied);
  return plan_grad(*d, copied, nullptr).bytes;
}

extern "C" gts_status gts_prompt_attention_grad(const gts_prompt_grad_desc *d, void *stream) {
  gts::clear_error();
  if (!d) return gts::fail(GTS_ERR_INVALID_ARG, "attention: null desc");
  const gts_prompt_desc &f = d->forward;
  if (const char *why = refuse_shape(f)) return gts::fail(GTS_ERR_INVALID_ARG, why);
  if (f.n_tokens == 0) return GTS_OK;
  if (const char *why = refuse_call(f, false)) return gts::fail(GTS_ERR_INVALID_ARG, why);
  if (!f.lse || !d->dout.data || !d->dq.data || !d->dk.data || !d->dv.data)
    return gts::fail(GTS_ERR_INVALID_ARG, "attention: null lse, dout, dq, dk or dv");
  if (misaligned(d->dout) || misaligned(d->dq) || misaligned(d->dk) || misaligned(d->dv) || (uintptr_t)d->dlse % 4)
    return gts::fail(GTS_ERR_INVALID_ARG, "attention: tensor misaligned for its type");
  GradMaps maps = {};
  bool copied[4];
  grad_maps(maps, *d, copied);
  const GradPlan p = plan_grad(*d, copied, (char *)f.workspace);
  if (f.workspace_bytes < p.bytes) return gts::fail(GTS_ERR_NOMEM, "attention: workspace smaller than gts_prompt_grad_workspace_bytes");
  Args a = args(f);
  a.dout = heads(d->dout), a.dq = heads(d->dq), a.dk = heads(d->dk), a.dv = heads(d->dv);
  a.dlse = d->dlse, a.delta = p.delta;
  const cudaError_t e = f.dtype == GTS_BF16 ? run_grad<__nv_bfloat16>(a, p, maps, *d, (cudaStream_t)stream) : run_grad<__half>(a, p, maps, *d, (cudaStream_t)stream);
  return e == cudaSuccess ? GTS_OK : gts::cuda_fail(e, "attention: launch");
}

extern "C" size_t gts_chunk_workspace_bytes(const gts_chunk_desc *d) {
  Cut c;
  return !d || refuse_shape(*d) ? 0 : plan(c, (int)d->cache.head_dim, nullptr);
}

extern "C" gts_status gts_chunk_attention(const gts_chunk_desc *d, void *stream) {
  gts::clear_error();
  if (!d) return gts::fail(GTS_ERR_INVALID_ARG, "attention: null desc");
  if (const char *why = refuse_shape(*d)) return gts::fail(GTS_ERR_INVALID_ARG, why);
  if (d->n_tokens == 0) return GTS_OK;
  const gts_cache &c = d->cache;
  if (!(d->scale > 0.f) || std::isinf(d->scale)) return gts::fail(GTS_ERR_INVALID_ARG, "attention: scale must be positive");
  if (!d->q.data || !d->out.data || !d->starts || (d->n_seqs && !d->lens)) return gts::fail(GTS_ERR_INVALID_ARG, "attention: null q, out, starts or lens");
  if (c.n_pages && (!c.k || !c.v)) return gts::fail(GTS_ERR_INVALID_ARG, "attention: null cache");
  if (d->max_pages && d->n_seqs && !d->page_table) return gts::fail(GTS_ERR_INVALID_ARG, "attention: null page_table");
  if (!d->workspace || (uintptr_t)d->workspace % 16) return gts::fail(GTS_ERR_INVALID_ARG, "attention: null or misaligned workspace");
  if (misaligned(d->q) || misaligned(d->out) || ((uintptr_t)c.k | (uintptr_t)c.v) % 2 ||
      ((uintptr_t)d->starts | (uintptr_t)d->lse | (uintptr_t)d->d_status | (uintptr_t)d->page_table | (uintptr_t)d->lens) % 4)
    return gts::fail(GTS_ERR_INVALID_ARG, "attention: tensor misaligned for its type");
  if (d->workspace_bytes < gts_chunk_workspace_bytes(d))
    return gts::fail(GTS_ERR_NOMEM, "attention: workspace smaller than gts_chunk_workspace_bytes");
  Args a = {};
  a.q = heads(d->q), a.out = heads(d->out);
  a.k = {c.k, c.k_token_stride, c.k_head_stride}, a.v = {c.v, c.v_token_stride, c.v_head_stride};
  a.k_page = c.k_page_stride, a.v_page = c.v_page_stride;
  a.lse = d->lse, a.starts = d->starts, a.lens = d->lens, a.table = d->page_table;
  a.n_seqs = (int)d->n_seqs, a.n_tokens = (int)d->n_tokens, a.q_heads = (int)d->q_heads, a.kv_heads = (int)c.kv_heads;
  a.group = a.q_heads / a.kv_heads, a.in_group = divisor(a.group), a.causal = 1, a.zero_rest = (int)d->zero_rest, a.paged = 1;
  a.n_pages = (int)c.n_pages, a.page_size = (int)c.page_size, a.max_pages = (int)d->max_pages, a.in_page = divisor(a.page_size);
  a.scale = d->scale, a.status = d->d_status;
  FwdMaps maps = {};
  tile_maps(maps.kv, c, TILE);
  const cudaError_t e = run_forward(a, maps, c.dtype, c.head_dim, d->workspace, (cudaStream_t)stream);
  return e == cudaSuccess ? GTS_OK : gts::cuda_fail(e, "attention: launch");
}
