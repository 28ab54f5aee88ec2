// Attention of a batch over a shared prefix and each sequence's own tokens, keys and values in pages
// (gts_prefix_attention).
//
// Mathematics.  With s_j = scale * q . k_j over the keys a query sees, m = max s_j, p_j = exp(s_j - m):
// out = sum p_j v_j / sum p_j, lse = m + log sum p_j.  The keys are taken tile by tile with the maximum and the sum so
// far: when a tile raises the maximum from m to m', what was summed is multiplied by exp(m - m').
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <atomic>
#include <cstring>
#include <type_traits>

#include "internal.h"

namespace {

// x / d for 0 <= x < 2^31 by a multiplication: m = floor(2^(31 + l) / d) + 1 with 2^(l-1) < d <= 2^l, so m d exceeds 2^(31 + l) by
// at most d <= 2^l, and x times that is below 2^(31 + l).
struct Divisor {
  uint32_t m;
  int shift;           // l - 1; -1 for d = 1
  int d;
};
Divisor divisor(int d) {
  int l = 0;
  while ((1ll << l) < d) l++;
  return {l ? (uint32_t)(((1ull << (31 + l)) / (uint32_t)d) + 1) : 0u, l - 1, d};
}
__device__ __forceinline__ int operator/(int x, const Divisor &d) { return d.shift < 0 ? x : (int)(__umulhi((uint32_t)x, d.m) >> d.shift); }
__device__ __forceinline__ int operator%(int x, const Divisor &d) { return x - x / d * d.d; }

struct Args {
  const void *q;
  void *out;
  float *lse;
  int64_t q_seq, q_tok, q_head, o_seq, o_tok, o_head;
  const void *k, *v;
  int64_t k_page, k_tok, k_head, v_page, v_tok, v_head;
  int n_seqs, n_new, q_heads, kv_heads, group;
  int n_pages, page_size, max_pages, prefix_len;
  Divisor in_page, in_group;   // by page_size, by group
  float scale;
  const int32_t *prefix_pages, *table, *lens;
  int32_t *status;
};

template <typename T> __device__ __forceinline__ float widen(T x);
template <> __device__ __forceinline__ float widen(__half x) { return __half2float(x); }
template <> __device__ __forceinline__ float widen(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T> __device__ __forceinline__ T narrow(float x);
template <> __device__ __forceinline__ __half narrow(float x) { return __float2half_rn(x); }
template <> __device__ __forceinline__ __nv_bfloat16 narrow(float x) { return __float2bfloat16_rn(x); }

// ---------------------------------------------------------------- pieces of PTX
__device__ __forceinline__ uint32_t smem_u32(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void copy16(uint32_t dst, const void *src, bool live) {  // zeros where not live
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(live ? 16 : 0) : "memory");
}
__device__ __forceinline__ void ldsm(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void ldsm_t(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
template <typename T> __device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1);
template <> __device__ __forceinline__ void mma<__nv_bfloat16>(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <> __device__ __forceinline__ void mma<__half>(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float exp2_fast(float x) {  // ex2.approx: 2 ulp, 0 for -infinity
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ void bar_init(uint32_t bar, int count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar) {
  asm volatile("{\n.reg .b64 t;\nmbarrier.arrive.shared::cta.b64 t, [%0];\n}" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("{\n.reg .b64 t;\nmbarrier.arrive.expect_tx.shared::cta.b64 t, [%0], %1;\n}" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}"
               : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  return ok;
}
// Every wait ends: after two seconds, or when another warp has given up, the block winds down with an error status.
__device__ __forceinline__ uint64_t now_ns() {
  uint64_t t;
  asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
  return t;
}
constexpr uint64_t LIMIT_NS = 2000000000ull, DRAIN_NS = 2000000000ull;   // of a wait; of what a block that winds down has in flight
constexpr int TRIES = 1024, BETWEEN = 64;   // before the timer is read first, and from then on (reading it takes longer than most waits)
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, volatile int *dead) {
  if (bar_try(bar, parity)) return true;   // (an unrolled loop around it would try several times before it looks)
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
__device__ __forceinline__ void tile_load(uint32_t dst, const CUtensorMap *map, int x, int y, int z, int page, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
               ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(page), "r"(bar) : "memory");
}
// the barrier's next arrival comes when this thread's copies so far have landed
__device__ __forceinline__ void bar_arrive_copies(uint32_t bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ float max3(float a, float b, float c) {
  float y;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
  return y;
}
// two 32-bit values in one instruction
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 y;
  asm("{\n.reg .b64 a, b, c;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %5};\nmov.b64 c, {%6, %7};\nfma.rn.f32x2 a, a, b, c;\nmov.b64 {%0, %1}, a;\n}"
      : "=f"(y.x), "=f"(y.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return y;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 y;
  asm("{\n.reg .b64 a, b;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %5};\nadd.rn.f32x2 a, a, b;\nmov.b64 {%0, %1}, a;\n}"
      : "=f"(y.x), "=f"(y.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return y;
}
template <typename T> __device__ __forceinline__ uint32_t pack(float lo, float hi);
template <> __device__ __forceinline__ uint32_t pack<__nv_bfloat16>(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
template <> __device__ __forceinline__ uint32_t pack<__half>(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// ---------------------------------------------------------------- how the work is cut
// A "pair" is a key head (or four of them) with a tile of up to ROWS query rows that see the same keys: of the prefix, rows of all
// sequences (row (b * n_new + i) * group + h of n_seqs * n_new * group); of a sequence's own keys, its n_new * group rows.
// A pair's keys come in tiles of KEYS, the unit of work.  All units stand in one line (prefix pairs, then the sequences'),
// and each block takes an equal stretch of it, so ragged lengths cost nothing and the cut needs no plan from the host.  Before a
// pair's first tile stand `lead` units for what it costs beside its tiles; a stretch that begins there begins with that tile.
// A pair that lies within one block's stretch leaves one result per row; one that is cut leaves a partial result per block,
// which k_join adds up in the order of the keys.
constexpr int SMS = 152;
constexpr int NOTHING = -1, GAVE_UP = -2;   // a block's record: no pair to be joined from it; its waits ran out, results are missing
constexpr int KEYS = 64;
constexpr int WARPS = 4, THREADS = 32 * WARPS;

struct Line {           // the units of one launch
  int has_prefix, has_own;
  int heads, rows, keys;  // key heads of a pair, rows of its tile (for each head), keys of a unit
  int beside_prefix;    // the tensor cores' kernel runs at the same time
  int side_by_side;     // that kernel's own: starts[n_seqs] row tiles at a time
  int prefix_tiles, own_tiles;   // row tiles of the prefix's rows, of a sequence's rows
  int blocks;
  int lead;             // units that stand for what a pair costs beside its tiles
  int64_t *starts;      // [n_seqs + 3]: first unit of each sequence, the units of all, units per block, before a pair's first tile
  float *cut_o;         // [blocks][2][heads][rows][D]: results of the first and last pair of a block that are cut
  float2 *cut_ml;       // [blocks][2][heads][rows]: maximum (of log2 scores) and sum
  int4 *ends;           // [blocks]: the pair that begins in a block and goes on in the next ones, see k_join_cut; x: its sequence,
                        // NOTHING or GAVE_UP
  float *whole_o[2];    // [rows of all][D], prefix and own: results of pairs that are not cut
  float2 *whole_ml[2];
};

__host__ __device__ __forceinline__ int tiles_of(int keys, int tile = KEYS) { return (keys + tile - 1) / tile; }

__device__ __forceinline__ int own_len(const Args &a, int b) {
  const int len = a.lens[b], most = a.max_pages * a.page_size;
  if (len > most && a.status) *a.status = GTS_ERR_INVALID_PARAMS;
  return max(0, min(len, most));
}

// A page number of a table: a negative one becomes the largest, which no cache has (-1 stands for "no page" in the kernels).
__device__ __forceinline__ int page_number(int32_t x) { return (int)min((uint32_t)x, 0x7FFFFFFFu); }

__device__ __forceinline__ int64_t quotient(int64_t x, int64_t y) {
  return ((x | y) >> 32) == 0 ? (int64_t)((uint32_t)x / (uint32_t)y) : x / y;
}

// The prefix's kernel is bound by the tensor cores and holds whole SMs, the sequences' own keys are bound by memory: both run
// at the same time, on SMs dealt out by the time each needs.  In units of an own tile's time on an SM (0.77 us measured at a
// head of 128, 0.42 at 64, 1.7 at 256, over all sizes of blocks): a tile of the prefix takes 2.2 (1.7 us), 3.3 (1.4 us) or 0.4
// (0.7 us), begin and end of its pair 8 or 4, the end of an own pair 3; own work with tiles of 16, 32 or 64 rows 0.8, 1.1 or 2.1
// times as long; and own tiles alone cannot go faster than memory brings them, 104 to that time.  Every block of the prefix takes
// the same whole number of tiles: of that number, one fewer and one more, the one with which the slower kernel is the fastest
// is taken, and no more SMs than it needs (64 sequences of 3 tokens over 8192 + 4096: 158 us without this choice, 139 with it; 64 of
// 16 over 8192 + 512 at a head of 256: 407 and 410).  Both kernels come to the same numbers from the lengths.
template <int D>
__device__ __forceinline__ int prefix_sms(const Args &a, const Line &prefix, int own_rows, int64_t own_tiles, int64_t own_pairs) {
  if (own_tiles == 0) return SMS;
  const int n = tiles_of(a.prefix_len, prefix.keys);
  const float tile = D == 64 ? 3.3f : D == 128 ? 2.2f : 0.4f, pair = D == 256 ? 4.f : 8.f;
  const float p = (tile * n + pair) * a.kv_heads * prefix.prefix_tiles;
  const float o = (own_tiles + 3.f * own_pairs) * (own_rows == 16 ? 0.8f : own_rows == 32 ? 1.1f : 2.1f), memory = own_tiles / 104.f;
  const int even = max(1, min(SMS - 1, (int)(p / fmaxf((p + o) / SMS, memory) + 0.5f)));
  const int side = even >= prefix.prefix_tiles ? prefix.prefix_tiles : 1;
  const int64_t units = (int64_t)n * a.kv_heads * (side == 1 ? prefix.prefix_tiles : 1), per = quotient(units + even / side - 1, even / side);
  int best = even;
  float least = INFINITY;
#pragma unroll 1
  for (int64_t x = max((int64_t)1, per - 1); x <= per + 1; x++) {
    const int64_t sms = quotient(units + x - 1, x) * side;
    if (sms >= SMS) continue;
    const float time = fmaxf((tile + pair / n) * x, fmaxf(o / (SMS - sms), memory));
    if (time < least) least = time, best = (int)sms;
  }
  return best;
}

__device__ __forceinline__ void dependents_may_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_kernels_before() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

struct Row { int b, i, h; };

// Row r of a pair's rows: prefix rows run over all sequences (b = -1), own rows over one.
__device__ __forceinline__ Row row_of(const Args &a, int b, int kh, int r) {
  const int per = a.n_new * a.group;
  Row x;
  x.b = b < 0 ? r / per : b;
  const int in = b < 0 ? r - x.b * per : r;
  x.i = in / a.in_group;
  x.h = kh * a.group + in - x.i * a.group;
  return x;
}

struct Pages {
  CUtensorMap k, v;    // pages x heads x tokens (or tokens x heads) x D, boxes of `box` tokens of a head x 64 values (0: no maps)
  int box, k_heads_first, v_heads_first;
};

// A place in the line of units: a tile of keys of a pair of a sequence (b = -1: the prefix).
struct Place { int b, len, n, pairs, pair, tile; };

// A block is 4 warps that compute and one that brings the data.  The fifth warp runs ahead along the block's stretch of the
// line, across the ends of pairs, and fills a ring of tiles: boxes of tokens by TMA where the pages allow it (see tile_map),
// else rows gathered by 16-byte copies, else (caches off the 16-byte grid) by plain loads.  A pair's queries come with its
// first tile.  (With four heads there are four such warps: issuing a tile's copies takes one of them 1600 cycles, the
// products 1000.  256 threads start with 128 registers each, 32768, and go on with 200 and 56.)
// Of the others, WM stand along the rows (16 each) and 4 / WM along a tile's keys; they meet only where a pair
// ends, to be joined in the stage just read.  Scores and weights stay in the fragments of m16n8k16 products, each warp with
// its own running maximum and sum.  Weights are rounded to the type of the values for their product with them (the sum is of
// the unrounded ones); everything else is in 32 bits.
//
// Bound by memory for long sequences: 128 of 1..4096 tokens, 1.08 GB, 178 us, 6.1 TB/s, 90% of the rate of a copy (187 us with the
// join); 256 of 1..1024, 537 MB, 94 us, 84% (105), where the ends of pairs and the first tiles' latencies count.  Tiles of 32 and
// 64 rows (5 and 16 new tokens) are bound by the latency of their products with two warps to a scheduler: 128 of 1..2048, 537 MB
// too, in 102 and 170 us (111 and 183).  Bytes spilled at a head of 128, a thread: 100 with 16 rows of one head, 32 by fours, 8
// and 96 with 32 and 64 rows; at 256, 0, 24 and 52; at 64, none, 8 and 60.
template <int D, int WM, int WH> struct Ring {
  static constexpr int STAGES = (D == 64 ? 4 : 3) - (WM > 1);   // as many as stream_per_sm blocks find room for
  static constexpr int TILE = KEYS * D * 2;                     // bytes of a tile of keys or of values
  static constexpr int QUERIES = WH > 1 ? 0 : 16 * WM * D * 2;  // with four heads they go straight to registers
  static constexpr int SMEM = 1024 /* alignment */ + STAGES * (2 * TILE + QUERIES) + 64 * (8 + 16) + (2 * STAGES + 1) * 8 + 56;
};
// (at a head of 64 one warp has half the copies to issue, and is enough)
__host__ __device__ constexpr int bringers(int D, int WH) { return D > 64 ? WH : 1; }
__host__ __device__ constexpr int stream_per_sm(int D) { return D == 64 ? 3 : D == 128 ? 2 : 1; }

template <typename T, int D, int WM, int WH>
__global__ void __launch_bounds__(THREADS + 32 * bringers(D, WH), stream_per_sm(D)) k_stream(const Args a, const Line w, const Line prefix, const __grid_constant__ Pages maps) {
  using R = Ring<D, WM, WH>;
  static_assert(WH == 1 || (WH == WARPS && WM == 1), "a warp for each head, or all for one");
  constexpr int WK = WARPS / WM / WH, ROWS = 16 * WM, KU = KEYS / WH, KW = KU / WK, STAGES = R::STAGES, TILE = R::TILE;
  constexpr int CH = D / 8, HALF = KEYS * 128, QHALF = ROWS * 128;  // a tile's and the queries' 64 columns: rows of 128 bytes
  extern __shared__ unsigned char smem_raw[];
  unsigned char *const ring = (unsigned char *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  unsigned char *const qs = ring + STAGES * 2 * TILE;
  float2 *const stat = (float2 *)(qs + STAGES * R::QUERIES);        // [64]: maximum and sum of each warp's rows
  longlong2 *const place = (longlong2 *)(stat + 64);                // [64]: of each row in the output, and its number
  uint64_t *const bars = (uint64_t *)(place + 64);
  int64_t *const found = (int64_t *)(bars + 2 * STAGES + 1);        // [4]
  int *const nonempty = (int *)(found + 4);                         // [4]
  volatile int *const dead = (volatile int *)(nonempty + 4);
  const int tid = threadIdx.x, warp = __shfl_sync(~0u, tid / 32, 0), lane = tid % 32;
  const uint32_t ring_at = smem_u32(ring), q_at = smem_u32(qs), bar0 = smem_u32(bars);
  auto full = [&](int s) { return bar0 + s * 8; };
  auto empty = [&](int s) { return bar0 + (STAGES + s) * 8; };
  const uint32_t together = bar0 + 2 * STAGES * 8;
  if (tid == 0) {
    for (int s = 0; s < STAGES; s++) bar_init(full(s), 33 * bringers(D, WH)), bar_init(empty(s), WARPS);
    bar_init(together, WARPS);
    *dead = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }

  // the line of units, and this block's stretch of it
  const int n_prefix = w.has_prefix ? tiles_of(a.prefix_len, KU) : 0, head_groups = a.kv_heads / WH;
  const int prefix_pairs = n_prefix ? head_groups * w.prefix_tiles : 0;
  const int own_pairs = head_groups * w.own_tiles;
  const int each = w.has_own && tid < THREADS ? (a.n_seqs + THREADS - 1) / THREADS : 0;
  const int b_first = min(a.n_seqs, tid * each), b_last = min(a.n_seqs, (tid + 1) * each);
  int64_t mine = 0;
  int some = 0;                                        // sequences with keys of their own
  for (int b = b_first; b < b_last; b++) {
    const int n = tiles_of(own_len(a, b), KU);
    mine += (int64_t)n * own_pairs;
    some += n > 0;
  }
  int64_t upto = mine;
  int some_upto = some;
  for (int o = 1; o < 32; o *= 2) {
    const int64_t x = __shfl_up_sync(~0u, upto, o);
    const int y = __shfl_up_sync(~0u, some_upto, o);
    if (lane >= o) upto += x, some_upto += y;
  }
  if (lane == 31 && warp < WARPS) found[warp] = upto, nonempty[warp] = some_upto;
  __syncthreads();
  int64_t before = upto - mine, pairs_before = some_upto - some, own_tiles = 0, pairs = 0;
  for (int x = 0; x < WARPS; x++) {
    if (x < warp) before += found[x], pairs_before += nonempty[x];
    own_tiles += found[x], pairs += nonempty[x];
  }
  pairs_before *= own_pairs, pairs *= own_pairs;
  int blocks = w.blocks;
  if (w.beside_prefix) blocks = max(1, min(blocks, stream_per_sm(D) * (SMS - prefix_sms<D>(a, prefix, ROWS, own_tiles, pairs))));
  // what a pair costs beside its tiles counts as units before its first (with few tiles to a block, each goes to its own)
  const int lead = own_tiles + (int64_t)n_prefix * prefix_pairs >= 4 * blocks ? w.lead : 0;
  auto own_units = [&](int b) {
    const int n = tiles_of(own_len(a, b), KU);
    return n ? (int64_t)(n + lead) * own_pairs : 0;
  };
  const int64_t prefix_units = (int64_t)(n_prefix + lead) * prefix_pairs, total = prefix_units + own_tiles + lead * pairs;
  const int64_t base = prefix_units + before + lead * pairs_before;   // first unit of sequence b_first
  mine += (int64_t)lead * some * own_pairs;
  const int64_t per = quotient(total + blocks - 1, blocks);
  const int64_t u0 = per * blockIdx.x, u1 = min(total, u0 + per);
  __syncthreads();
  if (blockIdx.x == 0 && tid < THREADS) {
    int64_t at = base;
    for (int b = b_first; b < b_last; b++) {
      w.starts[b] = at;
      at += own_units(b);
    }
    if (tid == 0) w.starts[a.n_seqs] = total, w.starts[a.n_seqs + 1] = per, w.starts[a.n_seqs + 2] = lead;
  }
  auto nothing_here = [&] {
    // the kernel after this one waits for this one alone: so this one ends after the one before it
    if (tid == 0) w.ends[blockIdx.x] = make_int4(NOTHING, 0, 0, 0);
    if (blockIdx.x == 0) wait_for_kernels_before();
  };
  if (u0 >= u1) {
    nothing_here();
    return;
  }
  if (u0 >= prefix_units && u0 >= base && u0 < base + mine) {
    int64_t at = base;
    int b = b_first;
    for (;; b++) {
      const int64_t n = own_units(b);
      if (u0 < at + n) break;
      at += n;
    }
    found[0] = b, found[1] = u0 - at;
  }
  __syncthreads();
  Place now;                                           // the tile whose turn it is
  int left = (int)(u1 - u0);                           // units from it to the end of the stretch
  bool inside;                                         // the stretch begins with a pair's first tile or a later one
  {
    const bool in_prefix = u0 < prefix_units;
    const int64_t in = in_prefix ? u0 : found[1];
    now.b = in_prefix ? -1 : (int)found[0];
    now.len = in_prefix ? a.prefix_len : own_len(a, now.b);
    now.n = tiles_of(now.len, KU);
    now.pairs = in_prefix ? head_groups * w.prefix_tiles : own_pairs;
    now.pair = (int)quotient(in, now.n + lead);
    const int unit = (int)(in - (int64_t)now.pair * (now.n + lead));
    inside = unit >= lead;
    now.tile = max(0, unit - lead);
    left -= max(0, lead - unit);
  }
  if (left <= 0) {
    nothing_here();
    return;
  }
  auto units_to_next = [&](const Place &p) { return p.tile == p.n - 1 ? 1 + lead : 1; };
  auto advance = [&](Place &p) {                       // only ever to units of this block
    if (++p.tile < p.n) return;
    p.tile = 0;
    if (++p.pair < p.pairs) return;
    p.pair = 0, p.pairs = own_pairs;
    do {
      p.len = own_len(a, ++p.b);
      p.n = tiles_of(p.len, KU);
    } while (p.n == 0);
  };
  auto row_tiles = [&](const Place &p) { return p.b < 0 ? w.prefix_tiles : w.own_tiles; };
  bool alive = true;
  int stage = 0;
  uint32_t lap = 0;
  auto next = [&] {
    if (++stage == STAGES) stage = 0, lap++;
  };

  if (warp >= WARPS) {
    // ---- the warp that brings the data (of one head: with four, there are four)
    constexpr int HB = WH / bringers(D, WH), RB = HB * KU;   // its heads, and rows of a tile
    if constexpr (bringers(D, WH) > 1) asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
    const bool aligned = ((((uintptr_t)a.k | (uintptr_t)a.v) >> 1 | a.k_page | a.k_tok | a.k_head | a.v_page | a.v_tok | a.v_head) & 7) == 0;
    const bool q_aligned = (((uintptr_t)a.q >> 1 | a.q_seq | a.q_tok | a.q_head) & 7) == 0;
    const int box = maps.box, boxes = box ? KU / box : 0;
    const int hh = (warp - WARPS) * HB + (box ? lane / boxes : 0), at_box = box ? lane % boxes : 0;  // this lane's box and its head
    int page[2];                                       // of this lane's box, or of its two rows; -1: none
    auto look_up = [&](const Place &p) {
      const int32_t *pages = p.b < 0 ? a.prefix_pages : a.table + (int64_t)p.b * a.max_pages;
      page[0] = page[1] = -1;
      if (box) {
        const int j = p.tile * KU + at_box * box;
        if (lane < boxes * HB && j < p.len) page[0] = page_number(pages[j / a.in_page]);
      } else {
#pragma unroll
        for (int x = 0; x < 2; x++) {
          const int j = p.tile * KU + (lane + 32 * x) % KU;
          if (lane + 32 * x < RB && j < p.len) page[x] = page_number(pages[j / a.in_page]);
        }
      }
    };
    Place ahead = now;
    look_up(ahead);
    int seg = -1;
    for (int unit = 0; left > 0; unit++) {
      const Place at = ahead;
      int to_load[2] = {page[0], page[1]};
      left -= units_to_next(at);
      if (left > 0) {                                  // the next tile's page numbers are fetched while this one waits
        advance(ahead);
        look_up(ahead);
      }
      if (unit >= STAGES) alive = __all_sync(~0u, bar_wait(empty(stage), (lap - 1) & 1, dead));
      if (!alive) break;
      const int tiles = row_tiles(at), group = tiles == 1 ? at.pair : at.pair / tiles;
#pragma unroll
      for (int x = 0; x < 2; x++) {
        if (to_load[x] >= a.n_pages) {                 // (a negative number among them, see page_number)
          to_load[x] = box ? a.n_pages : -1;           // outside the map: the box is filled with zeros
          if (a.status) *a.status = GTS_ERR_INVALID_PARAMS;
        }
      }
      const uint32_t to = ring_at + stage * 2 * TILE;
      uint32_t bytes = 0;
      if (box) {
        const bool live = to_load[0] >= 0;
        bytes = __popc(__ballot_sync(~0u, live)) * box * D * 4;
        if (lane == 0) bar_expect(full(stage), bytes);
        __syncwarp();
        if (live) {
          const int token = (at.tile * KU + at_box * box) % a.in_page, kh = group * WH + hh;
          const int k_y = maps.k_heads_first ? kh : token, k_z = maps.k_heads_first ? token : kh;
          const int v_y = maps.v_heads_first ? kh : token, v_z = maps.v_heads_first ? token : kh;
          const uint32_t dst = to + (hh * KU + at_box * box) * 128;
#pragma unroll
          for (int x = 0; x < D / 64; x++) {
            tile_load(dst + x * HALF, &maps.k, x * 64, k_y, k_z, to_load[0], full(stage));
            tile_load(dst + TILE + x * HALF, &maps.v, x * 64, v_y, v_z, to_load[0], full(stage));
          }
        }
      } else {
        if (lane == 0) bar_expect(full(stage), 0);
        int64_t k_off[2], v_off[2];                    // this lane's two rows
#pragma unroll
        for (int x = 0; x < 2; x++) {
          const int in = (at.tile * KU + (lane + 32 * x) % KU) % a.in_page, kh = group * WH + hh + (lane + 32 * x) / KU;
          k_off[x] = to_load[x] < 0 ? -1 : to_load[x] * a.k_page + in * a.k_tok + kh * a.k_head;
          v_off[x] = to_load[x] < 0 ? -1 : to_load[x] * a.v_page + in * a.v_tok + kh * a.v_head;
        }
#pragma unroll
        for (int x = 0; x < (RB + 31) / 32; x++) {
#pragma unroll 4
          for (int y = 0; y < min(32, RB); y++) {      // lanes along the row: D / 8 pieces of keys, then of values
            const int r = hh * KU + x * 32 + y;
            const int64_t k = __shfl_sync(~0u, k_off[x], y), v = __shfl_sync(~0u, v_off[x], y);
#pragma unroll
            for (int z = 0; z < 2 * CH; z += 32) {
              const int c = (z + lane) % CH;
              const bool is_k = z + lane < CH, live = k >= 0;
              if (z + lane >= 2 * CH) continue;
              const T *src = (const T *)(is_k ? a.k : a.v) + (live ? (is_k ? k : v) + c * 8 : 0);
              const uint32_t dst = stage * 2 * TILE + (is_k ? 0 : TILE) + c / 8 * HALF + r * 128 + ((c % 8) ^ (r & 7)) * 16;
              if (aligned) {
                copy16(ring_at + dst, src, live);
              } else {
                T e[8];
#pragma unroll
                for (int j = 0; j < 8; j++) e[j] = live ? src[j] : narrow<T>(0.f);
                memcpy(ring + dst, e, 16);
              }
            }
          }
        }
      }
      if (WH == 1 && (unit == 0 || at.tile == 0)) {    // a pair begins: its queries, zeros beyond the last row
        seg = seg + 1 == STAGES ? 0 : seg + 1;
        const int kh = group, row0 = (at.pair - kh * tiles) * ROWS, rows = (at.b < 0 ? a.n_seqs : 1) * a.n_new * a.group - row0;
#pragma unroll
        for (int x = 0; x < (ROWS + 31) / 32; x++) {   // a lane finds where a row is, then lanes along the rows
          const Row p = row_of(a, at.b, kh, row0 + min(x * 32 + lane, rows - 1));
          const unsigned long long row = (unsigned long long)((const T *)a.q + p.b * a.q_seq + p.i * a.q_tok + p.h * a.q_head);
#pragma unroll 4
          for (int y = 0; y < min(32, ROWS) * CH; y += 32) {
            const int in = (y + lane) / CH, r = x * 32 + in, c = lane % CH;
            const uint32_t dst = seg * R::QUERIES + c / 8 * QHALF + r * 128 + ((c % 8) ^ (r & 7)) * 16;
            const T *src = (const T *)__shfl_sync(~0u, row, in) + c * 8;
            if (q_aligned) {
              copy16(q_at + dst, src, r < rows);
            } else {
              T e[8];
#pragma unroll
              for (int j = 0; j < 8; j++) e[j] = r < rows ? src[j] : narrow<T>(0.f);
              memcpy(qs + dst, e, 16);
            }
          }
        }
      }
      // every lane's arrival: when its copies have landed; plain stores are ordered by a plain one after them
      if ((WH == 1 && !q_aligned) || (!box && !aligned)) {
        asm volatile("cp.async.wait_all;" ::: "memory");
        bar_arrive(full(stage));
      } else {
        bar_arrive_copies(full(stage));
      }
      next();
    }
  } else {
    // ---- the warps that compute
    if constexpr (bringers(D, WH) > 1) asm volatile("setmaxnreg.inc.sync.aligned.u32 200;");
    const int wm = warp % WM, wk = warp / WM, wh = WH > 1 ? warp : 0, quad = lane / 4, t4 = lane % 4, mi = lane / 8, mr = lane % 8;
    const bool o_aligned = (((uintptr_t)a.out >> 1 | a.o_seq | a.o_tok | a.o_head) & 3) == 0;
    const float sl2 = a.scale * 1.4426950408889634f;   // scores in units of log 2
    constexpr bool KEEP_Q = WH > 1 || (D <= 128 && WM == 1);       // the queries' fragments stay in registers
    // where this lane's rows of a fragment start; column d * 16 of the 64 is reached by turning bits 5 and 6
    const uint32_t k_lane = (wk * KW + (mi >> 1) * 8 + mr) * 128 + ((mi & 1) ^ mr) * 16;
    const uint32_t v_lane = (wk * KW + (mi & 1) * 8 + mr) * 128 + ((mi >> 1) ^ mr) * 16;
    const uint32_t q_lane = (wm * 16 + (mi & 1) * 8 + mr) * 128 + ((mi >> 1) ^ mr) * 16;
    uint32_t meetings = 0;
    auto meet = [&] {
      __syncwarp();
      if (lane == 0) bar_arrive(together);
      alive = __all_sync(~0u, bar_wait(together, meetings++ & 1, dead));
    };
    int seg = -1, tile0 = 0, kh = 0, row0 = 0, rows = 0, limit[2] = {0, 0}, seen_by_all = 0;
    bool first_slot = inside;                          // where a cut pair's part goes: k_join works it out from the units
    float o[D / 8][4], m[2], l[2];
    uint32_t qf[KEEP_Q ? D / 16 : 1][4];
    // Four heads: the next pair's queries are brought to L2 while this one's keys are worked on (from memory, while it is busy,
    // a load takes up to 5 us)
    auto ask_for_queries = [&](int b, int kh, int row0, int rows) {
      constexpr int LINES = D / 64;                    // of a row
      for (int x = lane; x < rows * LINES; x += 32) {
        const Row p = row_of(a, b, kh, row0 + x / LINES);
        const T *src = (const T *)a.q + p.b * a.q_seq + p.i * a.q_tok + p.h * a.q_head + x % LINES * 64;
        asm volatile("prefetch.global.L2 [%0];" ::"l"(src));
      }
    };
    int after = WH > 1 && now.b + 1 < a.n_seqs ? a.lens[now.b + 1] : 0, after_b = now.b;   // the next sequence's length, ahead of time
    for (int unit = 0; left > 0; unit++) {
      const int then = left - units_to_next(now);      // units left at the next tile
      const bool begins = unit == 0 || now.tile == 0;
      if (begins) {                                    // a pair begins
        const int tiles = row_tiles(now);
        seg = seg + 1 == STAGES ? 0 : seg + 1;
        tile0 = now.tile;
        kh = tiles == 1 ? now.pair : now.pair / tiles, row0 = (now.pair - kh * tiles) * ROWS;
        kh = kh * WH + wh;
        rows = min(ROWS, (now.b < 0 ? a.n_seqs : 1) * a.n_new * a.group - row0);
        seen_by_all = now.b < 0 ? now.len : now.len - (a.n_new - 1);
        if constexpr (WH > 1) {
          // straight to the fragments' places
          const bool q_aligned = (((uintptr_t)a.q >> 1 | a.q_seq | a.q_tok | a.q_head) & 1) == 0;
#pragma unroll
          for (int x = 0; x < 2; x++) {
            const Row p = row_of(a, now.b, kh, row0 + min(quad + 8 * x, rows - 1));
            const T *src = (const T *)a.q + p.b * a.q_seq + p.i * a.q_tok + p.h * a.q_head + t4 * 2;
#pragma unroll
            for (int d = 0; d < D / 16; d++) {
#pragma unroll
              for (int y = 0; y < 2; y++) {
                uint32_t v = 0;
                if (quad + 8 * x < rows) {
                  if (q_aligned) {
                    v = *(const uint32_t *)(src + d * 16 + y * 8);
                  } else {
                    const T e[2] = {src[d * 16 + y * 8], src[d * 16 + y * 8 + 1]};
                    memcpy(&v, e, 4);
                  }
                }
                qf[d][x + 2 * y] = v;
              }
            }
          }
        }
      }
      alive = __all_sync(~0u, bar_wait(full(stage), lap & 1, dead));
      if (!alive) break;
      if (begins) {
#pragma unroll
        for (int x = 0; x < 2; x++) {                  // keys that the rows of this thread's fragments see
          const int r = row0 + wm * 16 + quad + 8 * x;
          limit[x] = now.b < 0 ? now.len : now.len - (a.n_new - 1 - min(r / a.in_group, a.n_new - 1));
          m[x] = -INFINITY, l[x] = 0.f;
        }
#pragma unroll
        for (int x = 0; x < D / 8; x++) o[x][0] = o[x][1] = o[x][2] = o[x][3] = 0.f;
        if constexpr (KEEP_Q && WH == 1) {
#pragma unroll
          for (int d = 0; d < D / 16; d++) ldsm(qf[d], q_at + seg * R::QUERIES + (q_lane ^ d % 4 * 32) + d / 4 * QHALF);
        }
      }
      uint32_t k_at[4], v_at[4], q_from[4];
#pragma unroll
      for (int x = 0; x < 4; x++) {
        k_at[x] = ring_at + stage * 2 * TILE + (k_lane ^ x * 32);
        v_at[x] = ring_at + stage * 2 * TILE + (v_lane ^ x * 32);
        q_from[x] = q_at + seg * R::QUERIES + (q_lane ^ x * 32);
      }
      const int key0 = now.tile * KU + (WH > 1 ? 0 : wk * KW);
      const bool mask = key0 + KW > seen_by_all;       // some row does not see some key of this warp's
      auto attend = [&](auto is_masked) {
        constexpr bool masked = decltype(is_masked)::value;
        uint64_t bad = 0;                                // keys of this warp with values that are not finite, see below
        if constexpr (masked) {
          // value rows past the end are zeros: what the pages hold there may be NaN, and 0 * NaN is not 0
          const int end = now.len - key0;
          for (int x = lane; x < (KW - max(0, min(KW, end))) * CH; x += 32) {
            const int r = KW - 1 - x / CH, c = x % CH;
            *(uint4 *)(ring + stage * 2 * TILE + TILE + c / 8 * HALF + (wk * KW + r) * 128 + c % 8 * 16) = make_uint4(0, 0, 0, 0);
          }
          // and so for a value that some rows see and others do not: not finite, it is kept out of the products
          for (int r = max(0, seen_by_all - key0) + lane / CH; r < min(KW, end); r += 32 / CH) {
            const int c = lane % CH;
            const uint4 v = *(const uint4 *)(ring + stage * 2 * TILE + TILE + c / 8 * HALF + (wk * KW + r) * 128 + c % 8 * 16);
            const uint32_t e = std::is_same<T, __half>::value ? 0x7C00u : 0x7F80u, w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int x = 0; x < 4; x++)
              if ((w[x] & e) == e || (w[x] >> 16 & e) == e) bad |= 1ull << r;
          }
          bad = (uint64_t)__reduce_or_sync(~0u, (uint32_t)(bad >> 32)) << 32 | __reduce_or_sync(~0u, (uint32_t)bad);
          __syncwarp();
        }
        float s[KW / 8][4];
#pragma unroll
        for (int x = 0; x < KW / 8; x++) s[x][0] = s[x][1] = s[x][2] = s[x][3] = 0.f;
#pragma unroll
        for (int d = 0; d < D / 16; d++) {
          if constexpr (!KEEP_Q) ldsm(qf[0], q_from[d % 4] + d / 4 * QHALF);
#pragma unroll
          for (int x = 0; x < KW / 16; x++) {
            uint32_t kf[4];
            ldsm(kf, k_at[d % 4] + d / 4 * HALF + x * 16 * 128);
            mma<T>(s[2 * x], qf[KEEP_Q ? d : 0], kf[0], kf[1]);
            mma<T>(s[2 * x + 1], qf[KEEP_Q ? d : 0], kf[2], kf[3]);
          }
        }
        float top[2] = {m[0], m[1]};
#pragma unroll
        for (int x = 0; x < KW / 8; x++) {
#pragma unroll
          for (int c = 0; c < 4; c++) {
            s[x][c] *= sl2;
            if (masked && key0 + x * 8 + t4 * 2 + (c & 1) >= limit[c >> 1]) s[x][c] = -INFINITY;
            top[c >> 1] = fmaxf(top[c >> 1], s[x][c]);
          }
        }
        float keep[2], from[2];
#pragma unroll
        for (int x = 0; x < 2; x++) {
          top[x] = fmaxf(top[x], __shfl_xor_sync(~0u, top[x], 1));
          top[x] = fmaxf(top[x], __shfl_xor_sync(~0u, top[x], 2));
          from[x] = top[x] == -INFINITY ? 0.f : top[x];  // nothing seen so far
          keep[x] = exp2_fast(m[x] - from[x]);
          m[x] = top[x];
          l[x] *= keep[x];
        }
        if (__any_sync(~0u, keep[0] != 1.f || keep[1] != 1.f)) {
#pragma unroll
          for (int x = 0; x < D / 8; x++) {
            o[x][0] *= keep[0], o[x][1] *= keep[0];
            o[x][2] *= keep[1], o[x][3] *= keep[1];
          }
        }
        uint32_t pf[KW / 16][4];
#pragma unroll
        for (int x = 0; x < KW / 8; x++) {
#pragma unroll
          for (int c = 0; c < 4; c++) {
            s[x][c] = exp2_fast(s[x][c] - from[c >> 1]);
            l[c >> 1] += s[x][c];
          }
          pf[x / 2][(x & 1) * 2] = pack<T>(s[x][0], s[x][1]);
          pf[x / 2][(x & 1) * 2 + 1] = pack<T>(s[x][2], s[x][3]);
        }
#pragma unroll
        for (int x = 0; x < KW / 16; x++) {
          uint32_t stay[2] = {~0u, ~0u};                 // of the fragment's keys 2 t4, 2 t4 + 1 and the same + 8
          if (masked && bad) {
#pragma unroll
            for (int y = 0; y < 2; y++) {
              const uint32_t two = (uint32_t)(bad >> (x * 16 + y * 8 + t4 * 2)) & 3;
              stay[y] = (two & 1 ? 0 : 0xFFFFu) | (two & 2 ? 0 : 0xFFFF0000u);
            }
          }
#pragma unroll
          for (int d = 0; d < D / 16; d++) {
            uint32_t vf[4];
            ldsm_t(vf, v_at[d % 4] + TILE + d / 4 * HALF + x * 16 * 128);
            mma<T>(o[2 * d], pf[x], vf[0] & stay[0], vf[1] & stay[1]);
            mma<T>(o[2 * d + 1], pf[x], vf[2] & stay[0], vf[3] & stay[1]);
          }
        }
        if (masked && bad) {
          // each such key alone, for the rows that see it
#pragma unroll
          for (int x = 0; x < KW / 8; x++) {
#pragma unroll 1
            for (int k = 0; k < 8; k++) {
              if (!(bad >> (x * 8 + k) & 1)) continue;
              const int r = wk * KW + x * 8 + k, key = key0 + x * 8 + k;
              const unsigned char *row = ring + stage * 2 * TILE + TILE + r * 128;
              T two[2];
              float weight[2];
#pragma unroll
              for (int y = 0; y < 2; y++) {
                const uint32_t both = __shfl_sync(~0u, pf[x / 2][(x & 1) * 2 + y], quad * 4 + k / 2);
                memcpy(two, &both, 4);
                weight[y] = widen(k & 1 ? two[1] : two[0]);
              }
#pragma unroll
              for (int d = 0; d < D / 8; d++) {
                memcpy(two, row + d / 8 * HALF + ((d % 8) ^ (r & 7)) * 16 + t4 * 4, 4);
#pragma unroll
                for (int c = 0; c < 2; c++) {
                  if (key < limit[0]) o[d][c] += weight[0] * widen(two[c]);
                  if (key < limit[1]) o[d][2 + c] += weight[1] * widen(two[c]);
                }
              }
            }
          }
        }
      };
      if (mask) attend(std::true_type());
      else attend(std::false_type());

      if constexpr (WH > 1) {
        if (now.tile == tile0 && now.n - now.tile + lead < left) {
          const int tiles = row_tiles(now), pair = now.pair + 1 < now.pairs ? now.pair + 1 : 0;
          const bool same = now.pair + 1 < now.pairs;
          if (same || after > 0) {                     // (with an empty sequence in between: no matter)
            const int b = same ? now.b : now.b + 1, t = same ? tiles : w.own_tiles;
            const int group = t == 1 ? pair : pair / t, first = (pair - group * t) * ROWS;
            ask_for_queries(b, group * WH + wh, first, min(ROWS, (b < 0 ? a.n_seqs : 1) * a.n_new * a.group - first));
          }
        }
      }
      if (now.tile == now.n - 1 || then <= 0) {
        const bool whole = tile0 == 0 && now.tile == now.n - 1;
        if (tid == 0 && then <= 0)
          w.ends[blockIdx.x] = tile0 > 0 || whole ? make_int4(NOTHING, 0, 0, 0)
                                                  : make_int4(now.b, now.pair, (int)quotient(now.n - 2 - now.tile + per, per), !first_slot);
        const bool final = whole && now.b >= 0 && a.prefix_len == 0;
        if constexpr (WH > 1) {
          // a pair ends here, and each warp has its head's rows
#pragma unroll
          for (int x = 0; x < 2; x++) {
            l[x] += __shfl_xor_sync(~0u, l[x], 1);
            l[x] += __shfl_xor_sync(~0u, l[x], 2);
            const int r = quad + 8 * x;
            if (r >= rows) continue;
            const Row p = row_of(a, now.b, kh, row0 + r);
            const int64_t row = ((int64_t)p.b * a.n_new + p.i) * a.q_heads + p.h;
            if (final) {
              const float inv = l[x] == 0.f ? 0.f : 1.f / l[x];
              T *dst = (T *)a.out + p.b * a.o_seq + p.i * a.o_tok + p.h * a.o_head + t4 * 2;
#pragma unroll
              for (int d = 0; d < D / 8; d++) {
                const uint32_t v = pack<T>(o[d][2 * x] * inv, o[d][2 * x + 1] * inv);
                if (o_aligned) {
                  *(uint32_t *)(dst + d * 8) = v;
                } else {
                  T e[2];
                  memcpy(e, &v, 4);
                  dst[d * 8] = e[0], dst[d * 8 + 1] = e[1];
                }
              }
              if (t4 == 0 && a.lse) a.lse[row] = l[x] == 0.f ? -INFINITY : (m[x] + log2f(l[x])) * 0.6931471805599453f;
            } else {
              const int64_t at = whole ? row : (((int64_t)blockIdx.x * 2 + !first_slot) * WH + wh) * ROWS + r;
              float *dst = (whole ? w.whole_o[now.b >= 0] : w.cut_o) + at * D + t4 * 2;
#pragma unroll
              for (int d = 0; d < D / 8; d++) *(float2 *)(dst + d * 8) = make_float2(o[d][2 * x], o[d][2 * x + 1]);
              if (t4 == 0) (whole ? w.whole_ml[now.b >= 0] : w.cut_ml)[at] = make_float2(m[x], l[x]);
            }
          }
          if (mask) fence_async();
        } else {
          // a pair ends here: the warps along the keys are joined in the stage just read, and its rows written
          const Row goes = row_of(a, now.b, kh, row0 + min(tid, rows - 1));
          meet();                                      // (all are done with the rows of the pair before)
          if (!alive) break;
          if (tid < rows)
            place[tid] = make_longlong2(goes.b * a.o_seq + goes.i * a.o_tok + goes.h * a.o_head, ((int64_t)goes.b * a.n_new + goes.i) * a.q_heads + goes.h);
          float *acc = (float *)(ring + stage * 2 * TILE);   // [4 warps][16][D], columns of row r turned by 8 (r mod 4)
#pragma unroll
          for (int x = 0; x < 2; x++) {
            l[x] += __shfl_xor_sync(~0u, l[x], 1);
            l[x] += __shfl_xor_sync(~0u, l[x], 2);
            const int r = warp * 16 + quad + 8 * x;
            if (t4 == 0) stat[r] = make_float2(m[x], l[x]);
#pragma unroll
            for (int d = 0; d < D / 8; d++)
              *(float2 *)(acc + r * D + ((d * 8 + t4 * 2) ^ (r & 3) * 8)) = make_float2(o[d][2 * x], o[d][2 * x + 1]);
          }
          meet();
          if (!alive) break;
          for (int x = tid; x < rows * (D / 4); x += THREADS) {
            const int r = x / (D / 4), c = x % (D / 4) * 4;
            float best = -INFINITY;
#pragma unroll
            for (int k = 0; k < WK; k++) best = fmaxf(best, stat[(k * WM + r / 16) * 16 + r % 16].x);
            const float against = best == -INFINITY ? 0.f : best;
            float sum = 0.f;
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int k = 0; k < WK; k++) {
              const int at = (k * WM + r / 16) * 16 + r % 16;
              const float f = exp2_fast(stat[at].x - against);
              const float4 y = *(const float4 *)(acc + at * D + (c ^ (at & 3) * 8));
              sum += f * stat[at].y;
              v.x += f * y.x, v.y += f * y.y, v.z += f * y.z, v.w += f * y.w;
            }
            const int64_t row = place[r].y;
            if (final) {
              const float inv = sum == 0.f ? 0.f : 1.f / sum;
              T *dst = (T *)a.out + place[r].x + c;
              const uint32_t lo = pack<T>(v.x * inv, v.y * inv), hi = pack<T>(v.z * inv, v.w * inv);
              if (o_aligned) {
                *(uint2 *)dst = make_uint2(lo, hi);
              } else {
                T e[4];
                memcpy(e, &lo, 4), memcpy(e + 2, &hi, 4);
                for (int j = 0; j < 4; j++) dst[j] = e[j];
              }
              if (c == 0 && a.lse) a.lse[row] = sum == 0.f ? -INFINITY : (best + log2f(sum)) * 0.6931471805599453f;
            } else {
              // whole pairs by row, cut ones by block: its first (0) or its last (1)
              const int64_t at = whole ? row : ((int64_t)blockIdx.x * 2 + !first_slot) * ROWS + r;
              *(float4 *)((whole ? w.whole_o[now.b >= 0] : w.cut_o) + at * D + c) = v;
              if (c == 0) (whole ? w.whole_ml[now.b >= 0] : w.cut_ml)[at] = make_float2(best, sum);
            }
          }
          fence_async();                               // the stage was written here and is next written by TMA
        }
        first_slot = false;
      } else if (mask) {
        fence_async();
      }
      __syncwarp();
      if (lane == 0) bar_arrive(empty(stage));
      left = then;
      if (left > 0) advance(now);
      if (WH > 1 && now.b != after_b) {
        after_b = now.b;
        after = now.b + 1 < a.n_seqs ? a.lens[now.b + 1] : 0;
      }
      next();
    }
  }
  dependents_may_start();
  __syncthreads();
  if (*dead) {
    // copies in flight end before the block does, whichever warp gave up
    if (warp >= WARPS) {
      asm volatile("cp.async.wait_all;" ::: "memory");
      const uint64_t from = now_ns();
#pragma unroll 1
      for (int s = 0; s < STAGES; s++)
        while (!bar_try(full(s), (s < stage ? lap : lap - 1) & 1) && now_ns() - from < DRAIN_NS) {}
    }
    if (tid == 0) {
      w.ends[blockIdx.x] = make_int4(GAVE_UP, 0, 0, 0);
      if (a.status) *a.status = GTS_ERR_STEP_LIMIT;
    }
  }
  if (blockIdx.x == 0) wait_for_kernels_before();
}

// ---------------------------------------------------------------- the prefix on the tensor cores
__device__ __forceinline__ void tc_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tc_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
// d [128 rows][N] (+)= a [128][16] b [16][N]; a from shared memory, or from tensor memory.  Operands in shared memory are
// described by two words; the upper one is the same for all of them here.
__device__ __forceinline__ void tc_mma(uint32_t d, uint32_t a, uint32_t b, uint32_t hi, uint32_t shape, bool add) {
  asm volatile("{\n.reg .pred p;\n.reg .b64 x, y;\nmov.b64 x, {%1, %3};\nmov.b64 y, {%2, %3};\nsetp.ne.u32 p, %5, 0;\n"
               "tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %4, p;\n}"
               ::"r"(d), "r"(a), "r"(b), "r"(hi), "r"(shape), "r"((uint32_t)add) : "memory");
}
__device__ __forceinline__ void tc_mma_t(uint32_t d, uint32_t a, uint32_t b, uint32_t hi, uint32_t shape, bool add) {
  asm volatile("{\n.reg .pred p;\n.reg .b64 y;\nmov.b64 y, {%2, %3};\nsetp.ne.u32 p, %5, 0;\n"
               "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], y, %4, p;\n}"
               ::"r"(d), "r"(a), "r"(b), "r"(hi), "r"(shape), "r"((uint32_t)add) : "memory");
}
__device__ __forceinline__ bool elected() {  // one lane of a converged warp
  uint32_t is;
  asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(is));
  return is;
}
#define R8(r, i) "=r"(r[i]), "=r"(r[i + 1]), "=r"(r[i + 2]), "=r"(r[i + 3]), "=r"(r[i + 4]), "=r"(r[i + 5]), "=r"(r[i + 6]), "=r"(r[i + 7])
#define W8(r, i) "r"(r[i]), "r"(r[i + 1]), "r"(r[i + 2]), "r"(r[i + 3]), "r"(r[i + 4]), "r"(r[i + 5]), "r"(r[i + 6]), "r"(r[i + 7])
// 32 columns of the warp's 32 rows, one row a lane
__device__ __forceinline__ void tc_ld(uint32_t *r, uint32_t at) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
               "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
               : R8(r, 0), R8(r, 8), R8(r, 16), R8(r, 24) : "r"(at) : "memory");
}
__device__ __forceinline__ void tc_st(uint32_t at, const uint32_t *r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
               "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};"
               ::W8(r, 0), W8(r, 8), W8(r, 16), W8(r, 24), "r"(at) : "memory");
}
#undef R8
#undef W8
__device__ __forceinline__ void tc_ld_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Operands in shared memory are rows of 128 bytes, eight rows to a swizzled group of 1024 bytes, groups one after the other.
// Lower word: address, and the bytes from one 128-byte column of groups to the next (for operands that are wider and not
// summed over); upper word: bytes from group to group, version, swizzle.
__device__ __forceinline__ uint32_t operand(uint32_t at, uint32_t blocks) { return at >> 4 | (blocks >> 4) << 16; }
constexpr uint32_t OPERAND_HI = 1024 >> 4 | 1u << 14 | 2u << 29;

// The rows of all sequences against the prefix.  A block holds 2 x 128 rows of one key head and passes along its stretch of
// the keys in tiles of 128, each read once for all rows:
//   warp 9 brings tiles of keys and values from their pages by TMA into a ring;
//   warps 8 and 10 issue the products, each for one half of the rows: scores S = Q K^T to tensor memory, O += P V with P
//   from tensor memory;
//   warps 0..3 and 4..7 take one half of the rows each, one row a thread: maximum, weights, sum.  P overwrites S.
// The halves alternate: while one turns scores into weights, the tensor cores work for the other.  The maximum that scores
// are taken against is raised, and what was summed rescaled, only when it has grown by more than 8 (in log 2): weights stay
// below 2^8, sums are exact in the same way, and the result is the same up to rounding.
// Weights are rounded to the values' type for their product; the sum is of the unrounded ones, all else is in 32 bits.
//
// Bound by the chain of a half: products 1024 cycles, scores to weights 1250, handing over 330, so 2600 cycles for a tile of
// 256 x 128 x 128 whose products take 2048.  What was tried: scores in pieces of 32 (shorter code, but a longer chain: 3200),
// all 128 scores in registers (spills), one issuing thread for both halves (3200), no turns (3300), turns from the second part
// of the weights on (7% slower), tiles of 64 keys with scores a tile ahead as at a head of 256 (8% slower: products of 64
// columns wait for shared memory).  128 x 4 rows over 131072 keys on 142 SMs: 187 us, 1.47 PFLOP/s, 82% of cuBLAS's burst rate on
// as many; 256 x 4 rows over 32768 on 84, beside the own keys' kernel: 156 us, 0.88, 83%.  Bytes spilled a thread: 104 at a head of
// 128, 56 at 64, 176 at 256.
//
// A head of 256 has room for one half in tensor memory (256 columns of sums): 128 rows, tiles of 64 keys, and two buffers of
// scores, so that the products of the next tile's scores run while the rows make their weights.
constexpr int TC_THREADS = 352;
constexpr float RAISE = 8.f;
template <int D> struct Tc {
  static constexpr bool SINGLE = D == 256;
  static constexpr int KEYS = SINGLE ? 64 : 128, ROWS = SINGLE ? 128 : 256;
  static constexpr int TILE = KEYS * D * 2, STAGES = D == 64 ? 8 : 5, Q = ROWS * D * 2;
  static constexpr int SMEM = Q + STAGES * TILE + 1024 /* alignment */ + 256 /* barriers */;
};

template <typename T, int D>
__global__ void __launch_bounds__(TC_THREADS, 1) k_prefix(const Args a, const Line w, const Line own_line, const __grid_constant__ Pages maps, const uint32_t flip) {
  constexpr bool SINGLE = Tc<D>::SINGLE;
  constexpr int TC_KEYS = Tc<D>::KEYS, TILE = Tc<D>::TILE, STAGES = Tc<D>::STAGES;
  constexpr int HALF = TC_KEYS * 128, QHALF = 128 * 128;       // 64 columns of a tile, of a half's queries
  extern __shared__ unsigned char smem_raw[];
  unsigned char *const smem = (unsigned char *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  unsigned char *const qs = smem, *const ring = smem + Tc<D>::Q;
  uint64_t *const bars = (uint64_t *)(ring + STAGES * TILE);
  uint32_t *const tmem_at = (uint32_t *)(bars + 2 * STAGES + 13);
  volatile int *const dead = (volatile int *)(tmem_at + 1);
  const int tid = threadIdx.x, warp = __shfl_sync(~0u, tid / 32, 0), lane = tid % 32;
  const uint32_t bar0 = smem_u32(bars), q_at = smem_u32(qs), ring_at = smem_u32(ring);
  auto full = [&](int s) { return bar0 + s * 8; };
  auto empty = [&](int s) { return bar0 + (STAGES + s) * 8; };
  auto q_full = [&](int h) { return bar0 + (2 * STAGES + h) * 8; };
  auto s_full = [&](int h) { return bar0 + (2 * STAGES + 2 + h) * 8; };
  auto p_full = [&](int h, int q) { return bar0 + (2 * STAGES + 4 + h * 2 + q) * 8; };  // of half the keys
  const uint32_t ended = bar0 + (2 * STAGES + 8) * 8;
  auto my_turn = [&](int h) { return bar0 + (2 * STAGES + 10 + h) * 8; };
  const uint32_t o_full = bar0 + (2 * STAGES + 12) * 8;
  dependents_may_start();                              // the sequences' own keys need nothing from here
  __shared__ int own[TC_THREADS / 32][2];              // of each warp: sequences' tiles, sequences that have any
  int tiles = 0, some = 0;
  for (int b = tid; b < a.n_seqs; b += TC_THREADS) {
    const int x = tiles_of(own_len(a, b), own_line.keys);
    tiles += x;
    some += x > 0;
  }
  tiles = __reduce_add_sync(~0u, tiles), some = __reduce_add_sync(~0u, some);
  if (lane == 0) own[warp][0] = tiles, own[warp][1] = some;
  __syncthreads();
  int64_t own_tiles = 0, own_pairs = 0;
  for (int x = 0; x < TC_THREADS / 32; x++) own_tiles += own[x][0], own_pairs += own[x][1];
  const int pairs_each = a.kv_heads / own_line.heads * own_line.own_tiles;
  const int blocks = prefix_sms<D>(a, w, own_line.rows, own_tiles * pairs_each, own_pairs * pairs_each);
  // Row tiles that see the same keys go side by side, in blocks next to each other: each stretch of the keys is then read from
  // memory once and found in L2 by the others.  (With more row tiles than blocks, all of them follow each other instead.)
  const int side = blocks >= w.prefix_tiles ? w.prefix_tiles : 1, behind = side == 1 ? w.prefix_tiles : 1;
  const int n = tiles_of(a.prefix_len, TC_KEYS), stretches = blocks / side;
  const int64_t units = (int64_t)n * a.kv_heads * behind, per = quotient(units + stretches - 1, stretches);
  const int64_t u0 = per * (blockIdx.x / side), u1 = min(units, u0 + per);
  const int my_tile = blockIdx.x % side;
  auto head_of = [&](int pair) { return pair / behind; };
  auto first_row = [&](int pair) { return (side == 1 ? pair % behind : my_tile) * Tc<D>::ROWS; };
  if (blockIdx.x == 0 && tid == 0) w.starts[a.n_seqs] = side, w.starts[a.n_seqs + 1] = per, w.starts[a.n_seqs + 2] = 0;
  if (u0 >= u1) return;
  if (tid == 0) {
    for (int s = 0; s < STAGES; s++) bar_init(full(s), 1), bar_init(empty(s), SINGLE ? 1 : 2);
    bar_init(o_full, 1);
    for (int h = 0; h < 2; h++) bar_init(ended + 8 * h, 1), bar_init(my_turn(h), 1), bar_init(q_full(h), 128), bar_init(s_full(h), 1), bar_init(p_full(h, 0), 128), bar_init(p_full(h, 1), 128);
    *dead = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 8) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(tmem_at)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  }
  tc_before();
  __syncthreads();
  tc_after();
  const uint32_t tmem = __shfl_sync(~0u, *tmem_at, 0);
  auto scores = [&](int h) { return tmem + h * TC_KEYS; };       // of a half, or a buffer
  auto sums = [&](int h) { return tmem + 256 + h * 128; };

  const int all = a.n_seqs * a.n_new * a.group;
  int copies = 0;                                      // warp 9: tiles of keys or values asked for
  bool issues = false;                                 // the threads that issue products

  if (warp >= 8) {
    if (warp == 9) {
      // ---- keys and values: lane x brings the x-th box of tokens of a tile, both of its 64-value halves
      const int boxes = TC_KEYS / maps.box;
      bool alive = true;
      int pair = (int)quotient(u0, n), tile = (int)(u0 - (int64_t)pair * n), kh = head_of(pair);
      auto look_up = [&](int t) {                          // this lane's page of tile t; -1: none
        const int key = t * TC_KEYS + lane * maps.box;
        return lane < boxes && key < a.prefix_len ? page_number(a.prefix_pages[key / a.in_page]) : -1;
      };
      int page_next = look_up(tile);
      for (int64_t u = u0; u < u1 && alive; u++) {
        const int key = tile * TC_KEYS + lane * maps.box, head = kh;
        int page = page_next;
        const bool live = page >= 0;
        if (++tile == n) tile = 0, kh = head_of(++pair);
        if (u + 1 < u1) page_next = look_up(tile);         // arrives while this tile waits for room
        if (page >= a.n_pages) {                           // (a negative number among them, see page_number)
          page = a.n_pages;                                // outside the map: the box is filled with zeros
          if (a.status) *a.status = GTS_ERR_INVALID_PARAMS;
        }
        const uint32_t bytes = __popc(__ballot_sync(~0u, live)) * maps.box * D * 2;
        for (int kv = 0; kv < 2; kv++, copies++) {
          const int s = copies % STAGES;
          if (copies >= STAGES && !bar_wait(empty(s), (copies / STAGES - 1) & 1, dead)) alive = false;
          alive = __all_sync(~0u, alive);
          if (!alive) break;
          if (lane == 0) bar_expect(full(s), bytes);
          __syncwarp();
          if (live) {
            const bool heads_first = kv ? maps.v_heads_first : maps.k_heads_first;
            const int token = key % a.in_page;
#pragma unroll
            for (int x = 0; x < D / 64; x++)
              tile_load(ring_at + s * TILE + x * HALF + lane * maps.box * 128, kv ? &maps.v : &maps.k, x * 64, heads_first ? head : token,
                        heads_first ? token : head, page, full(s));
          }
        }
      }
    } else if (SINGLE && warp == 8 && elected()) {
      // ---- products of the one half: scores a tile ahead, in two buffers
      issues = true;
      constexpr uint32_t TYPE = std::is_same<T, __nv_bfloat16>::value ? 1u : 0u;
      constexpr uint32_t COMMON = 1u << 4 | TYPE << 7 | TYPE << 10 | (128u >> 4) << 24;
      constexpr uint32_t QK = COMMON | (TC_KEYS >> 3) << 17, PV = COMMON | 1u << 16 | (D >> 3) << 17;
      const uint32_t k_op = operand(ring_at, 16), v_op = operand(ring_at, HALF), q_op = operand(q_at, 16);
      uint32_t seg = 0, turn = 0, made[2] = {0, 0};        // pairs, tiles (and ends of pairs), weights in each buffer so far
      uint32_t at = 0;                                     // place in the ring: a tile's keys, then its values
      bool alive = true;
      auto need = [&](uint32_t bar, uint32_t parity) { alive = alive && bar_wait(bar, parity & 1, dead); };
      auto qk = [&](uint32_t place, uint32_t t) {
        const int s = place % STAGES;
        need(full(s), place / STAGES);
        if (!alive) return;
        tc_after();
        uint32_t q = q_op, k = k_op + ((s * TILE) >> 4);
        const uint32_t to = scores(t & 1);
#pragma unroll 1
        for (int x = 0; x < D / 64; x++, q += QHALF >> 4, k += HALF >> 4) {
#pragma unroll
          for (int y = 0; y < 4; y++) tc_mma(to, q + 2 * y, k + 2 * y, OPERAND_HI, QK, x + y > 0);
        }
        tc_commit(s_full(t & 1));
        tc_commit(empty(s));
      };
      for (int64_t u = u0; u < u1 && alive;) {
        const int pair = (int)(u / n), tile0 = (int)(u - (int64_t)pair * n), count = (int)min((int64_t)(n - tile0), u1 - u);
        u += count;
        need(q_full(0), seg++);
        if (!alive) break;
        qk(at, turn);
        if (count > 1 && alive) qk(at + 2, turn + 1);
        for (int j = 0; j < count && alive; j++, turn++, at += 2) {
          const int sv = (at + 1) % STAGES, b = turn & 1, nv = a.prefix_len - (tile0 + j) * TC_KEYS;
          need(full(sv), (at + 1) / STAGES);
          if (nv < TC_KEYS && nv % 16 && alive) {          // value rows past the end, in the last 16 that count: zeros
            for (int x = 0; x < (16 - nv % 16) * (D / 8); x++) {
              const int r = nv + x / (D / 8), c = x % (D / 8);
              *(uint4 *)(ring + sv * TILE + c / 8 * HALF + r * 128 + c % 8 * 16) = make_uint4(0, 0, 0, 0);
            }
            fence_async();
          }
          need(p_full(b, 0), b ? made[1]++ : made[0]++);
          if (!alive) break;
          tc_after();
          const uint32_t v = v_op + ((sv * TILE) >> 4), w_at = scores(b);
#pragma unroll
          for (int k = 0; k < TC_KEYS / 16; k++)
            if (k * 16 < nv) tc_mma_t(sums(0), w_at + k * 8, v + k * (2048 >> 4), OPERAND_HI, PV, j + k > 0);
          tc_commit(o_full);
          tc_commit(empty(sv));
          if (j + 2 < count) qk(at + 4, turn + 2);
        }
        if (!alive) break;
        tc_commit(s_full(turn & 1));                       // the pair's sums are complete
        turn++;
      }
    } else if (!SINGLE && warp != 9 && elected()) {
      // ---- products, from one thread for each half of the rows (one thread for both would set the time)
      issues = true;
      constexpr uint32_t TYPE = std::is_same<T, __nv_bfloat16>::value ? 1u : 0u;
      constexpr uint32_t COMMON = 1u << 4 | TYPE << 7 | TYPE << 10 | (128u >> 4) << 24;
      constexpr uint32_t QK = COMMON | (TC_KEYS >> 3) << 17, PV = COMMON | 1u << 16 | (D >> 3) << 17;
      const int h = warp == 10;
      const uint32_t k_op = operand(ring_at, 16), v_op = operand(ring_at, HALF), q_op = operand(q_at + h * (Tc<D>::Q / 2), 16);
      const uint32_t s_at = scores(h), o_at = sums(h);
      int stage = 0;                                       // of the ring
      uint32_t lap = 0, seg = 0, turn = 0, turns = 0;      // laps of the ring; this half's pairs and tiles so far, and turns
      bool alive = true;
      auto need = [&](uint32_t bar, uint32_t parity) { alive = alive && bar_wait(bar, parity & 1, dead); };
      auto next = [&] {
        if (++stage == STAGES) stage = 0, lap++;
      };
      auto qk = [&](int s) {
        uint32_t q = q_op, k = k_op + ((s * TILE) >> 4);
#pragma unroll
        for (int x = 0; x < D / 64; x++, q += QHALF >> 4, k += HALF >> 4) {
#pragma unroll
          for (int y = 0; y < 4; y++) tc_mma(s_at, q + 2 * y, k + 2 * y, OPERAND_HI, QK, x + y > 0);
        }
        tc_commit(s_full(h));
        tc_commit(empty(s));
      };
      for (int64_t u = u0; u < u1 && alive;) {
        const int pair = (int)(u / n), tile0 = (int)(u - (int64_t)pair * n), count = (int)min((int64_t)(n - tile0), u1 - u);
        u += count;
        if (all - first_row(pair) <= h * 128) {              // no rows for this half: the tiles pass by
          for (int x = 0; x < 2 * count && alive; x++, next()) {
            need(full(stage), lap);
            bar_arrive(empty(stage));
          }
          continue;
        }
        const bool both = all - first_row(pair) > 128;
        need(q_full(h), seg++);
        need(full(stage), lap);
        if (!alive) break;
        tc_after();
        qk(stage);
        next();
        for (int j = 0; j < count; j++) {
          // this tile's values and the next one's keys, while the rows make their weights
          const int sv = stage, nv = a.prefix_len - (tile0 + j) * TC_KEYS;
          need(full(sv), lap);
          next();
          const int sk = stage;
          if (j + 1 < count) {
            need(full(sk), lap);
            next();
          }
          if (nv < TC_KEYS && nv % 16 && alive) {          // value rows past the end, in the last 16 that count: zeros
            for (int x = 0; x < (16 - nv % 16) * (D / 8); x++) {
              const int r = nv + x / (D / 8), c = x % (D / 8);
              *(uint4 *)(ring + sv * TILE + c / 8 * HALF + r * 128 + c % 8 * 16) = make_uint4(0, 0, 0, 0);
            }
            fence_async();
          }
          const uint32_t v = v_op + ((sv * TILE) >> 4);
#pragma unroll
          for (int q = 0; q < 2; q++) {
            need(p_full(h, q), turn);
            // The halves take turns, each with all its products for a tile: left alone they fall into step, and the tensor
            // cores wait while both make weights (3300 against 2600 cycles a tile)
            if (q == 0 && both) need(my_turn(h), h ? turns : turns - 1), turns++;
            if (!alive) break;
            tc_after();
#pragma unroll
            for (int k = 4 * q; k < 4 * q + 4; k++)
              if (k * 16 < nv) tc_mma_t(o_at, s_at + k * 8, v + k * (2048 >> 4), OPERAND_HI, PV, j + k > 0);
          }
          turn++;
          if (!alive) break;
          tc_commit(empty(sv));
          if (j + 1 < count) qk(sk);
          else tc_commit(s_full(h));                       // the pair's sums are complete
          if (both) bar_arrive(my_turn(!h));
        }
      }
    }
  } else if (!SINGLE || warp < 4) {
    // ---- one row a thread
    const int h = warp / 4, r = tid % 128;
    const uint32_t lanes = (uint32_t)(warp % 4 * 32) << 16;
    const float sl2 = fabsf(a.scale) * 1.4426950408889634f;
    const bool q_aligned = (((uintptr_t)a.q >> 1 | a.q_seq | a.q_tok | a.q_head) & 7) == 0;
    uint32_t turn = 0, tiles_done = 0;                   // phases of s_full: a pair's tiles, then its sums
    bool alive = true;
    for (int64_t u = u0; u < u1 && alive;) {
      const int pair = (int)(u / n), tile0 = (int)(u - (int64_t)pair * n), count = (int)min((int64_t)(n - tile0), u1 - u);
      const int kh = head_of(pair), row = first_row(pair) + h * 128 + r;
      if (all - first_row(pair) <= h * 128) {              // no rows for this half: the phases of its barriers stand still
        u += count;
        continue;
      }
      const Row p = row_of(a, -1, kh, row);
      // queries: the warp takes its 32 rows together, lanes along them
      const unsigned long long src = row < all ? (unsigned long long)((const T *)a.q + p.b * a.q_seq + p.i * a.q_tok + p.h * a.q_head) : 0;
      uint4 v[D / 8];
#pragma unroll
      for (int x = 0; x < D / 8; x++) {                  // all loads first
        const T *from = (const T *)__shfl_sync(~0u, src, (x * 32 + lane) / (D / 8));
        v[x] = make_uint4(0, 0, 0, 0);
        if (from) {
          from += lane % (D / 8) * 8;
          if (q_aligned) {
            v[x] = *(const uint4 *)from;
          } else {
            T e[8];
#pragma unroll
            for (int z = 0; z < 8; z++) e[z] = from[z];
            memcpy(&v[x], e, 16);
          }
        }
      }
#pragma unroll
      for (int x = 0; x < D / 8; x++) {
        const int c = lane % (D / 8), at = warp % 4 * 32 + (x * 32 + lane) / (D / 8);
        v[x].x ^= flip, v[x].y ^= flip, v[x].z ^= flip, v[x].w ^= flip;   // a negative scale: its sign goes to the queries
        *(uint4 *)(qs + h * (Tc<D>::Q / 2) + c / 8 * QHALF + at * 128 + ((c % 8) ^ (at & 7)) * 16) = v[x];
      }
      fence_async();
      bar_arrive(q_full(h));

      float m = -INFINITY, l = 0.f;
      for (int j = 0; j < count; j++, turn++, tiles_done++) {
        const int b = SINGLE ? turn & 1 : h;               // the buffer of scores
        alive = __all_sync(~0u, bar_wait(s_full(b), (SINGLE ? turn >> 1 : turn) & 1, dead));
        if (!alive) break;
        tc_after();
        const int nv = a.prefix_len - (tile0 + j) * TC_KEYS;
        // Half of the scores at a time, and tensor memory read again for the weights: all 128 in registers would spill, and
        // shorter pieces add their latencies.
        uint32_t s[64];
        auto fetch = [&](int c) {
          tc_ld(s, scores(b) + lanes + c);
          tc_ld(s + 32, scores(b) + lanes + c + 32);
          tc_ld_wait();
          if (c + 64 > nv) {
#pragma unroll
            for (int x = 0; x < 64; x++)
              if (c + x >= nv) s[x] = 0xFF800000u;       // -infinity
          }
        };
        float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int q = 0; q < TC_KEYS / 64; q++) {
          fetch(q * 64);
#pragma unroll
          for (int c = 0; c < 64; c += 8) {
#pragma unroll
            for (int x = 0; x < 4; x++) top[x] = max3(top[x], __uint_as_float(s[c + 2 * x]), __uint_as_float(s[c + 2 * x + 1]));
          }
        }
        const float big = fmaxf(max3(top[0], top[1], top[2]), top[3]) * sl2;
        const bool raise = big > m + RAISE || (m == -INFINITY && big > m);
        if (j == 0) {
          m = big;
        } else if (__any_sync(~0u, raise)) {
          const float to = raise ? big : m, f = raise ? exp2_fast(m - to) : 1.f;
          if (SINGLE) {                                    // the scores were ahead: the last product with values may not be done
            alive = __all_sync(~0u, bar_wait(o_full, (tiles_done - 1) & 1, dead));
            if (!alive) break;
            tc_after();
          }
          uint32_t o[32];
#pragma unroll 1
          for (int c = 0; c < D / 32; c++) {
            tc_ld(o, sums(h) + lanes + c * 32);
            tc_ld_wait();
#pragma unroll
            for (int x = 0; x < 32; x++) o[x] = __float_as_uint(__uint_as_float(o[x]) * f);
            tc_st(sums(h) + lanes + c * 32, o);
          }
          l *= f;
          m = to;
        }
        const float from = m == -INFINITY ? 0.f : m;
        const float2 scale2 = make_float2(sl2, sl2), from2 = make_float2(-from, -from);
        float2 part[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
        for (int q = 0; q < TC_KEYS / 64; q++) {         // the products with the first 64 weights start under the others
          uint32_t pk[32];
          if (!SINGLE) fetch(q * 64);
#pragma unroll
          for (int c = 0; c < 64; c += 2) {
            float2 x = fma2(make_float2(__uint_as_float(s[c]), __uint_as_float(s[c + 1])), scale2, from2);
            x.x = exp2_fast(x.x), x.y = exp2_fast(x.y);
            part[c / 2 & 1] = add2(part[c / 2 & 1], x);
            pk[c / 2] = pack<T>(x.x, x.y);
          }
          tc_st(scores(b) + lanes + q * 32, pk);
          tc_st_wait();
          tc_before();
          bar_arrive(p_full(b, q));
        }
        const float2 both = add2(part[0], part[1]);
        l += both.x + both.y;
      }
      if (!alive) break;
      alive = __all_sync(~0u, SINGLE ? bar_wait(s_full(turn & 1), turn >> 1 & 1, dead) : bar_wait(s_full(h), turn & 1, dead));
      turn++;
      if (!alive) break;
      tc_after();
      const bool whole = count == n;
      const int64_t at = whole ? ((int64_t)p.b * a.n_new + p.i) * a.q_heads + p.h
                               : ((int64_t)blockIdx.x * 2 + (u > u0)) * Tc<D>::ROWS + h * 128 + r;
      // the sums, 32 columns at a time, through the warp's part of the queries' room (all products with them are done), so
      // that a store covers whole lines
      const unsigned long long to = row < all ? (unsigned long long)((whole ? w.whole_o[0] : w.cut_o) + at * D) : 0;
      unsigned char *const room = qs + h * (Tc<D>::Q / 2) + warp % 4 * 4096;
#pragma unroll 1
      for (int c = 0; c < D / 32; c++) {
        uint32_t o[32];
        tc_ld(o, sums(h) + lanes + c * 32);
        tc_ld_wait();
#pragma unroll
        for (int x = 0; x < 8; x++)
          *(uint4 *)(room + lane * 128 + (x ^ (lane & 7)) * 16) = make_uint4(o[4 * x], o[4 * x + 1], o[4 * x + 2], o[4 * x + 3]);
        __syncwarp();
#pragma unroll
        for (int x = 0; x < 8; x++) {
          const int y = x * 4 + lane / 8;
          float *dst = (float *)__shfl_sync(~0u, to, y);
          const uint4 v = *(const uint4 *)(room + y * 128 + ((lane % 8) ^ (y & 7)) * 16);
          if (dst) *(uint4 *)(dst + c * 32 + lane % 8 * 4) = v;
        }
        __syncwarp();
      }
      if (row < all) (whole ? w.whole_ml[0] : w.cut_ml)[at] = make_float2(m, l);
      tc_before();
      u += count;
    }
  }
  tc_before();
  __syncthreads();
  if (tid == 0) w.ends[blockIdx.x] = make_int4(*dead ? GAVE_UP : NOTHING, 0, 0, 0);
  if (*dead) {
    // copies and products in flight end before the block does, whichever warp gave up
    const uint64_t from = now_ns();
    if (issues) {
      const uint32_t bar = ended + (warp == 10 ? 8 : 0);
      tc_commit(bar);
      while (!bar_try(bar, 0) && now_ns() - from < DRAIN_NS) {}
    }
    if (warp == 9) {
#pragma unroll 1
      for (int x = max(0, copies - STAGES); x < copies; x++)
        while (!bar_try(full(x % STAGES), (x / STAGES) & 1) && now_ns() - from < DRAIN_NS) {}
    }
    if (tid == 0 && a.status) *a.status = GTS_ERR_STEP_LIMIT;
    __syncthreads();
  }
  if (warp == 8) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
}

// Every block with work leaves a record, so the joins know the parts that a block whose waits ran out has left unwritten: rows that
// miss one are NaN, whether or not the caller looks at a status.
__device__ __forceinline__ bool gave_up(const Line &w, int64_t block) { return w.ends[block].x == GAVE_UP; }
__device__ __forceinline__ float2 missing() { return make_float2(NAN, NAN); }

// The result of a row from its parts, in their order: one warp.  Up to 32 parts at a time, a lane takes the maximum and sum of
// one; then all lanes add up the parts' values, several loads in flight.
struct Part {
  const float *o;
  float2 ml;
};
template <typename T, int D, typename F>
__device__ __forceinline__ void join_row(const Args &a, int lane, int b, int i, int h, int total, F part) {
  constexpr int E = D / 32;
  using V = typename std::conditional<E == 2, float2, float4>::type;
  constexpr int NV = E * 4 / sizeof(V);
  float m = -INFINITY, l = 0.f, acc[E] = {};
  for (int first = 0; first < total; first += 32) {
    const int x = first + lane;
    const float *o = nullptr;
    float2 ml = make_float2(-INFINITY, 0.f);
    if (x < total) {
      const auto p = part(x);
      o = p.o, ml = p.ml;
    }
    float top = fmaxf(m, ml.x);
#pragma unroll
    for (int k = 16; k; k >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, k));
    const float from = top == -INFINITY ? 0.f : top, keep = exp2_fast(m - from);
    const float f = exp2_fast(ml.x - from);
    float sum = f * ml.y;
#pragma unroll
    for (int k = 16; k; k >>= 1) sum += __shfl_xor_sync(~0u, sum, k);
    l = l * keep + sum;
    m = top;
#pragma unroll
    for (int e = 0; e < E; e++) acc[e] *= keep;
    const int count = min(32, total - first);
    for (int y = 0; y < count; y += 4) {
      V v[4][NV];
      float g[4];
#pragma unroll
      for (int k = 0; k < 4; k++) {
        const float *from_o = (const float *)__shfl_sync(~0u, (unsigned long long)o, y + k);
        g[k] = __shfl_sync(~0u, f, y + k);
        if (y + k < count) {
#pragma unroll
          for (int e = 0; e < NV; e++) v[k][e] = ((const V *)from_o)[lane * NV + e];
        }
      }
#pragma unroll
      for (int k = 0; k < 4; k++) {
        if (y + k < count) {
#pragma unroll
          for (int e = 0; e < E; e++) acc[e] += g[k] * ((const float *)v[k])[e];
        }
      }
    }
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  T *dst = (T *)a.out + b * a.o_seq + i * a.o_tok + h * a.o_head + lane * E;
  uint32_t packed[E / 2];
#pragma unroll
  for (int e = 0; e < E; e += 2) packed[e / 2] = pack<T>(acc[e] * inv, acc[e + 1] * inv);
  if ((((uintptr_t)a.out >> 1 | a.o_seq | a.o_tok | a.o_head) & (E - 1)) == 0) {
    if constexpr (E == 2) *(uint32_t *)dst = packed[0];
    else if constexpr (E == 4) *(uint2 *)dst = make_uint2(packed[0], packed[1]);
    else *(uint4 *)dst = make_uint4(packed[0], packed[1], packed[2], packed[3]);
  } else {
    T e[E];
    memcpy(e, packed, sizeof(e));
#pragma unroll
    for (int k = 0; k < E; k++) dst[k] = e[k];
  }
  if (a.lse && lane == 0) a.lse[((int64_t)b * a.n_new + i) * a.q_heads + h] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
}

// With a prefix: every row, from the parts of its prefix pair and then of its sequence's own.  Bound by L2: 8192 rows of 128 with
// about 4 parts each, 22 MB, 5 us.
template <typename T, int D>
__global__ void __launch_bounds__(THREADS) k_join(const Args a, const Line lp, const Line lo) {
  const int lane = threadIdx.x % 32;
  const int64_t row = (int64_t)blockIdx.x * WARPS + threadIdx.x / 32;
  if (row >= (int64_t)a.n_seqs * a.n_new * a.q_heads) return;
  wait_for_kernels_before();
  const int64_t token = quotient(row, a.q_heads), seq = quotient(token, a.n_new);
  const int h = (int)(row - token * a.q_heads), i = (int)(token - seq * a.n_new), b = (int)seq;
  const int kh = h / a.in_group;
  // a pair's parts: its blocks c0 .. c0 + count - 1, or one result of its own
  struct Parts { int64_t u0, c0, per; int count, r, side, lane; bool whole; };
  auto parts = [&](const Line &w, int r, int tiles, int64_t start, int n, int side) {
    Parts p = {0, 0, 0, 0, 0, side, 0, false};
    if (n) {
      const int tile = r / w.rows;
      p.per = w.starts[a.n_seqs + 1];
      p.lane = side > 1 ? tile : 0;                    // of `side` row tiles side by side
      const int lead = (int)w.starts[a.n_seqs + 2];
      p.u0 = start + (int64_t)(side > 1 ? kh : kh / w.heads * tiles + tile) * (n + lead) + lead;
      p.r = kh % w.heads * w.rows + r % w.rows;
      p.c0 = quotient(p.u0, p.per);
      p.count = (int)(quotient(p.u0 + n - 1, p.per) - p.c0) + 1;
      p.whole = p.count == 1;
    }
    return p;
  };
  const int in = h - kh * a.group, n = tiles_of(own_len(a, b), lo.keys);
  const Parts pre = parts(lp, (b * a.n_new + i) * a.group + in, lp.prefix_tiles, 0, tiles_of(a.prefix_len, lp.keys),
                          lp.side_by_side ? (int)lp.starts[a.n_seqs] : 1);
  const Parts own = parts(lo, i * a.group + in, lo.own_tiles, n ? lo.starts[b] : 0, n, 1);
  join_row<T, D>(a, lane, b, i, h, pre.count + own.count, [&](int x) {
    const bool mine = x >= pre.count;
    const bool whole = mine ? own.whole : pre.whole;
    const int64_t c = mine ? own.c0 + x - pre.count : pre.c0 + x;
    const bool last = mine ? own.u0 > c * own.per : pre.u0 > c * pre.per;
    const int64_t block = mine ? c : c * pre.side + pre.lane;
    const int64_t at = whole ? row : (block * 2 + last) * (mine ? lo.heads * lo.rows : lp.heads * lp.rows) + (mine ? own.r : pre.r);
    const float *o = (whole ? mine ? lo.whole_o[1] : lp.whole_o[0] : mine ? lo.cut_o : lp.cut_o) + at * D;
    const float2 ml = (whole ? mine ? lo.whole_ml[1] : lp.whole_ml[0] : mine ? lo.cut_ml : lp.cut_ml)[at];
    return Part{o, gave_up(mine ? lo : lp, block) ? missing() : ml};
  });
}

// Without one: the rows of the pairs that are cut, each from the block where it begins (Line::ends) to that where it ends,
// the rows of sequences without keys, and those of pairs that a block which gave up had a part of; the others are done.
template <typename T, int D>
__global__ void __launch_bounds__(THREADS) k_join_cut(const Args a, const Line w, const int cut_blocks) {
  const int lane = threadIdx.x % 32, rows = w.heads * w.rows;
  wait_for_kernels_before();
  if ((int)blockIdx.x >= cut_blocks) {
    const int b = (blockIdx.x - cut_blocks) * WARPS + threadIdx.x / 32;
    if (b >= a.n_seqs) return;
    const int n = tiles_of(own_len(a, b), w.keys);
    const int64_t per = w.starts[a.n_seqs + 1], lead = w.starts[a.n_seqs + 2], start = n ? w.starts[b] : 0;
    auto any_gave_up = [&](int64_t first, int64_t last) {  // of the blocks of these units
      bool any = false;
      for (int64_t c = quotient(first, per) + lane, end = quotient(last, per); c <= end; c += 32) any |= gave_up(w, c);
      return __any_sync(~0u, any);
    };
    if (n && !any_gave_up(start, start + (n + lead) * (a.kv_heads / w.heads * w.own_tiles) - 1)) return;
    for (int x = 0; x < a.n_new * a.q_heads; x++) {
      const int i = x / a.q_heads, h = x % a.q_heads, kh = h / a.in_group;
      if (n) {
        const int64_t pair = kh / w.heads * w.own_tiles + (i * a.group + h - kh * a.group) / w.rows, u0 = start + pair * (n + lead) + lead;
        if (!any_gave_up(u0, u0 + n - 1)) continue;
      }
      join_row<T, D>(a, lane, b, i, h, n ? 1 : 0, [&](int) { return Part{w.cut_o, missing()}; });
    }
    return;
  }
  const int x = blockIdx.x * WARPS + threadIdx.x / 32, c = x / rows, r = x % rows;
  if (c >= w.blocks) return;
  const int4 end = w.ends[c];                          // sequence, pair, blocks after this one, 1 if it is not this block's first
  if (end.x < 0) return;
  const int group = end.y / w.own_tiles, row = (end.y - group * w.own_tiles) * w.rows + r % w.rows;
  if (row >= a.n_new * a.group) return;
  const Row p = row_of(a, end.x, group * w.heads + r / w.rows, row);
  join_row<T, D>(a, lane, p.b, p.i, p.h, 1 + end.z, [&](int y) {
    const int64_t at = ((int64_t)(c + y) * 2 + (y ? 0 : end.w)) * rows + r;
    return Part{w.cut_o + at * D, gave_up(w, c + y) ? missing() : w.cut_ml[at]};
  });
}

// ---------------------------------------------------------------- host side
// A kernel's shared memory above 48 KB is granted once per device.
template <typename K> cudaError_t grant(K kernel, int bytes, std::atomic<uint64_t> &granted) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess || (dev < 64 && (granted.load(std::memory_order_relaxed) >> dev & 1))) return e;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == cudaSuccess && dev < 64) granted.fetch_or(1ull << dev, std::memory_order_relaxed);
  return e;
}

size_t up(size_t x) { return (x + 255) / 256 * 256; }

// How a call is run.  The prefix's rows (of all sequences) go to the tensor cores' kernel where its boxes fit the pages; else to
// the streaming kernel, in the launch of the sequences' own keys or, with many rows, in one of its own with tiles of 64 rows.
enum Way { TOGETHER, APART, TENSOR };
struct Plan {
  Way way;
  Line prefix, own;
  size_t bytes;
};

constexpr int64_t APART_ROWS = 64;

int box_of(int page_size, int most) {  // tokens of a TMA box: the largest power of two that divides both the page and a tile
  int box = 1;
  while (box < most && page_size % (box * 2) == 0) box *= 2;
  return box;
}

int stream_blocks(int D) { return SMS * stream_per_sm(D); }

Plan make_plan(const gts_attention_desc &d, bool tensor, char *at) {
  const int D = (int)d.cache.head_dim, group = (int)(d.q_heads / d.cache.kv_heads);
  const int64_t own_rows = (int64_t)d.n_new * group, all = own_rows * d.n_seqs;
  Plan p = {};
  // On the tensor cores even few rows of the prefix go faster (4 rows of one key head over 8192 keys 28 us on the GPU, in the streaming
  // kernel 34; of eight key heads 28 and 40; 512 over 256 29 and 33), except over the shortest prefixes, where a launch more costs what
  // it gains.  At a head of 256, with smaller tiles, from 32 rows on (16 over 8192 keys take 43 us here and 31 there, 256 over 512 53
  // and 48, 512 over 32768 198 and 459).
  tensor &= d.prefix_len >= 256 && d.prefix_len * (uint64_t)std::max<int64_t>(all, 16) >= 16384 && (D < 256 || all >= 32);
  p.way = tensor ? TENSOR : d.prefix_len && all > APART_ROWS && own_rows <= 32 ? APART : TOGETHER;
  size_t n = 0;
  auto take = [&](size_t bytes) {
    char *x = at ? at + n : nullptr;
    n += up(bytes);
    return x;
  };
  // A pair's begin and end (first loads, queries, the join of its warps, its results) in units of its tiles.  Without them blocks
  // with many short pairs end last: 128 sequences of 16 tokens over 1..2048 take 280 us without and 183 with 7 (4: 184, 12: 192);
  // of 5, 150 and 111 with 5 (4: 110, 12: 117); 256 of one over 1..1024, by fours, 118 and 105 with 8 (4: 109, 12: 105); 128 of one
  // over 1..4096 208 and 187 with 2 (4: 184, 12: 183).
  auto line = [&](Line &w, int heads, int rows, int keys, int blocks, bool has_prefix, bool has_own) {
    w.has_prefix = has_prefix, w.has_own = has_own, w.heads = heads, w.rows = rows, w.keys = keys, w.blocks = blocks, w.lead = heads > 1 ? 8 : rows == 16 ? 2 : rows == 32 ? 5 : 7;
    w.prefix_tiles = (int)((all + rows - 1) / rows), w.own_tiles = (int)((own_rows + rows - 1) / rows);
    w.starts = (int64_t *)take(((size_t)d.n_seqs + 3) * 8);
    w.ends = (int4 *)take((size_t)blocks * 16);
    w.cut_ml = (float2 *)take((size_t)blocks * 2 * heads * rows * 8);
    w.cut_o = (float *)take((size_t)blocks * 2 * heads * rows * D * 4);
  };
  const int own_tile = own_rows <= 16 ? 16 : own_rows <= 32 ? 32 : 64;
  // Few rows: a warp to each of four heads, which have nothing to join at a pair's end, where the heads can be had by fours.
  // Long sequences seldom end, and their tiles of 64 keys of one head come in larger boxes.  The table's width stands for the lengths,
  // which only the device knows: 256 of 1..1024 tokens take 105 us by fours and 114 by ones (which is what a wide table gets), 128 of
  // 1..2048 103 and 109.  At 128 of 1..4096 the kernel of one head has lost its lead to its spills: 187, by fours 180.
  const bool fours = own_tile == 16 && D <= 128 && d.cache.kv_heads % WARPS == 0 && (uint64_t)d.max_pages * d.cache.page_size <= 2048;
  const int heads = fours ? WARPS : 1;
  line(p.own, heads, own_tile, KEYS / heads, stream_blocks(D), p.way == TOGETHER && d.prefix_len, true);
  if (p.way == APART) line(p.prefix, 1, 64, KEYS, stream_blocks(D), true, false);
  if (p.way == TENSOR) {
    line(p.prefix, 1, D == 256 ? Tc<256>::ROWS : Tc<128>::ROWS, D == 256 ? Tc<256>::KEYS : Tc<128>::KEYS, SMS, true, false);
    p.own.beside_prefix = 1, p.prefix.side_by_side = 1;
  }
  if (p.way == TOGETHER) p.prefix = p.own;
  if (d.prefix_len) {
    const size_t rows = (size_t)d.n_seqs * d.n_new * d.q_heads;
    for (int k = 0; k < 2; k++) {
      p.prefix.whole_ml[k] = p.own.whole_ml[k] = (float2 *)take(rows * 8);
      p.prefix.whole_o[k] = p.own.whole_o[k] = (float *)take(rows * D * 4);
    }
  }
  p.bytes = n;
  return p;
}


typedef CUresult (*EncodeTiled)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiled encode_tiled() {
  static std::atomic<void *> found{nullptr};
  void *f = found.load(std::memory_order_relaxed);
  if (!f) {
    cudaDriverEntryPointQueryResult got;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &got) != cudaSuccess ||
        got != cudaDriverEntryPointSuccess)
      return nullptr;
    found.store(f, std::memory_order_relaxed);
  }
  return (EncodeTiled)f;
}

// A map of the cache's pages for the tensor cores' kernel.  False where strides or alignment do not fit one: each dimension's
// stride has to be a multiple of 16 bytes and of the one before it.
bool tile_map(CUtensorMap &map, int &heads_first, int box, const gts_cache &c, void *base, int64_t page, int64_t token, int64_t head) {
  const int64_t D = c.head_dim;
  heads_first = c.page_size > 1 && (c.kv_heads == 1 || head < token);
  if (c.kv_heads == 1) head = heads_first ? D : token * c.page_size;
  if (c.page_size == 1) token = D;
  const int64_t lo = heads_first ? head : token, hi = heads_first ? token : head;
  if (c.n_pages == 1) page = hi * (heads_first ? c.page_size : c.kv_heads);
  if ((uintptr_t)base % 16 || lo % 8 || lo < D || hi < lo || hi % lo || page < hi || page % hi || page >= 1ll << 38) return false;
  const EncodeTiled encode = encode_tiled();
  if (!encode) return false;
  const cuuint64_t dims[4] = {(cuuint64_t)D, heads_first ? c.kv_heads : c.page_size, heads_first ? c.page_size : c.kv_heads, c.n_pages};
  const cuuint64_t strides[3] = {(cuuint64_t)lo * 2, (cuuint64_t)hi * 2, (cuuint64_t)page * 2};
  const cuuint32_t boxes[4] = {64, heads_first ? 1u : (cuuint32_t)box, heads_first ? (cuuint32_t)box : 1u, 1}, ones[4] = {1, 1, 1, 1};
  return encode(&map, c.dtype == GTS_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, base, dims, strides,
                boxes, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool tile_maps(Pages &p, const gts_cache &c, int most) {
  const int box = box_of((int)c.page_size, most);
  if (box < 8 || !c.n_pages) return false;   // a box is whole groups of eight rows
  p.box = box;
  const bool ok = tile_map(p.k, p.k_heads_first, p.box, c, c.k, c.k_page_stride, c.k_token_stride, c.k_head_stride) &&
                  tile_map(p.v, p.v_heads_first, p.box, c, c.v, c.v_page_stride, c.v_token_stride, c.v_head_stride);
  if (!ok) p.box = 0;
  return ok;
}

// A launch that may start as soon as the kernel before it allows (`early`): the kernels above wait for each other themselves.
template <typename... P, typename... A>
cudaError_t launch_kernel(void (*kernel)(P...), unsigned blocks, unsigned threads, int shared, cudaStream_t s, bool early, const A &...args) {
  cudaLaunchAttribute attr = {};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t c = {};
  c.gridDim = dim3(blocks), c.blockDim = dim3(threads), c.dynamicSmemBytes = (size_t)shared, c.stream = s;
  c.attrs = &attr, c.numAttrs = early ? 1 : 0;
  return cudaLaunchKernelEx(&c, kernel, args...);
}

template <typename T, int D, int WM, int WH>
cudaError_t stream(const Args &a, const Line &w, const Line &prefix, const Pages &maps, bool early, cudaStream_t s) {
  static std::atomic<uint64_t> granted{0};
  const cudaError_t e = grant(k_stream<T, D, WM, WH>, Ring<D, WM, WH>::SMEM, granted);
  return e != cudaSuccess ? e : launch_kernel(k_stream<T, D, WM, WH>, w.blocks, THREADS + 32 * bringers(D, WH), Ring<D, WM, WH>::SMEM, s, early, a, w, prefix, maps);
}

template <typename T, int D>
cudaError_t tensor(const Args &a, const Line &w, const Line &own, const Pages &maps, cudaStream_t s) {
  static std::atomic<uint64_t> granted{0};
  const cudaError_t e = grant(k_prefix<T, D>, Tc<D>::SMEM, granted);
  return e != cudaSuccess ? e : launch_kernel(k_prefix<T, D>, w.blocks, TC_THREADS, Tc<D>::SMEM, s, false, a, w, own, maps, a.scale < 0 ? 0x80008000u : 0u);
}

template <typename T, int D>
cudaError_t run(const Args &a, const Plan &p, const Pages &maps, const Pages &own_maps, cudaStream_t s) {
  cudaError_t e = cudaSuccess;
  if (p.way == APART) e = stream<T, D, 4, 1>(a, p.prefix, p.prefix, own_maps, false, s);
  if (p.way == TENSOR) e = tensor<T, D>(a, p.prefix, p.own, maps, s);
  if (e != cudaSuccess) return e;
  const bool early = p.way != TOGETHER;
  if constexpr (D <= 128) {
    if (p.own.heads > 1) e = stream<T, D, 1, WARPS>(a, p.own, p.prefix, own_maps, early, s);
  }
  if (p.own.heads == 1)
    e = p.own.rows == 16 ? stream<T, D, 1, 1>(a, p.own, p.prefix, own_maps, early, s)
        : p.own.rows == 32 ? stream<T, D, 2, 1>(a, p.own, p.prefix, own_maps, early, s)
                           : stream<T, D, 4, 1>(a, p.own, p.prefix, own_maps, early, s);
  if (e != cudaSuccess) return e;
  if (a.prefix_len == 0) {
    const int cut_blocks = (p.own.blocks * p.own.heads * p.own.rows + WARPS - 1) / WARPS, empty = (a.n_seqs + WARPS - 1) / WARPS;
    return launch_kernel(k_join_cut<T, D>, (unsigned)(cut_blocks + empty), THREADS, 0, s, true, a, p.own, cut_blocks);
  }
  const int64_t rows = (int64_t)a.n_seqs * a.n_new * a.q_heads;
  return launch_kernel(k_join<T, D>, (unsigned)((rows + WARPS - 1) / WARPS), THREADS, 0, s, true, a, p.prefix, p.own);
}

template <typename T>
cudaError_t launch(const Args &a, const Plan &p, const Pages &maps, const Pages &own_maps, int head_dim, cudaStream_t s) {
  return head_dim == 64    ? run<T, 64>(a, p, maps, own_maps, s)
         : head_dim == 128 ? run<T, 128>(a, p, maps, own_maps, s)
                           : run<T, 256>(a, p, maps, own_maps, s);
}

const char *refuse_shape(const gts_attention_desc &d) {
  const gts_cache &c = d.cache;
  if (c.dtype != GTS_BF16 && c.dtype != GTS_F16) return "attention: dtype must be GTS_BF16 or GTS_F16";
  if (c.head_dim != 64 && c.head_dim != 128 && c.head_dim != 256) return "attention: head_dim must be 64, 128 or 256";
  if (c.kv_heads < 1 || c.kv_heads > 1024 || d.q_heads < 1 || d.q_heads > 65536 || d.q_heads % c.kv_heads)
    return "attention: q_heads must be a multiple of kv_heads (1 <= kv_heads <= 1024)";
  if (c.page_size < 1 || c.page_size > 65536 || c.n_pages > 1u << 30 || d.max_pages > 1u << 30)
    return "attention: 1 <= page_size <= 65536, at most 2^30 pages";
  if ((uint64_t)d.n_seqs * d.n_new > 65535 || d.n_seqs > 65535 || d.n_new > 65535)
    return "attention: n_seqs * n_new must be at most 65535";
  if ((uint64_t)d.n_seqs * d.n_new * d.q_heads > 1u << 30) return "attention: more than 2^30 rows of queries";
  if (d.prefix_len > 1u << 30 || (uint64_t)d.max_pages * c.page_size > 1u << 30)
    return "attention: a prefix or a sequence of more than 2^30 tokens";
  return nullptr;
}

}  // namespace

extern "C" size_t gts_attention_workspace_bytes(const gts_attention_desc *d) {
  if (!d || refuse_shape(*d)) return 0;
  return std::max(make_plan(*d, false, nullptr).bytes, make_plan(*d, true, nullptr).bytes);
}

extern "C" gts_status gts_prefix_attention(const gts_attention_desc *d, void *stream) {
  gts::clear_error();
  if (!d) return gts::fail(GTS_ERR_INVALID_ARG, "attention: null desc");
  if (const char *why = refuse_shape(*d)) return gts::fail(GTS_ERR_INVALID_ARG, why);
  if (d->n_seqs == 0 || d->n_new == 0) return GTS_OK;
  const gts_cache &c = d->cache;
  if (!d->q || !d->out || !d->lens) return gts::fail(GTS_ERR_INVALID_ARG, "attention: null q, out or lens");
  if (c.n_pages && (!c.k || !c.v)) return gts::fail(GTS_ERR_INVALID_ARG, "attention: null cache");
  if (d->prefix_len && !d->prefix_pages) return gts::fail(GTS_ERR_INVALID_ARG, "attention: null prefix_pages");
  if (d->max_pages && !d->page_table) return gts::fail(GTS_ERR_INVALID_ARG, "attention: null page_table");
  if (!d->workspace || (uintptr_t)d->workspace % 16)
    return gts::fail(GTS_ERR_INVALID_ARG, "attention: null or misaligned workspace");
  Args a = {};
  a.q = d->q;
  a.out = d->out;
  a.lse = d->lse;
  a.q_seq = d->q_seq_stride, a.q_tok = d->q_token_stride, a.q_head = d->q_head_stride;
  a.o_seq = d->out_seq_stride, a.o_tok = d->out_token_stride, a.o_head = d->out_head_stride;
  a.k = c.k, a.v = c.v;
  a.k_page = c.k_page_stride, a.k_tok = c.k_token_stride, a.k_head = c.k_head_stride;
  a.v_page = c.v_page_stride, a.v_tok = c.v_token_stride, a.v_head = c.v_head_stride;
  a.n_seqs = (int)d->n_seqs, a.n_new = (int)d->n_new, a.q_heads = (int)d->q_heads, a.kv_heads = (int)c.kv_heads;
  a.group = a.q_heads / a.kv_heads;
  a.n_pages = (int)c.n_pages, a.page_size = (int)c.page_size, a.max_pages = (int)d->max_pages;
  a.prefix_len = (int)d->prefix_len;
  a.in_page = divisor(a.page_size), a.in_group = divisor(a.group);
  a.scale = d->scale;
  a.prefix_pages = d->prefix_pages, a.table = d->page_table, a.lens = d->lens;
  a.status = d->d_status;
  if (((uintptr_t)d->q | (uintptr_t)d->out | (uintptr_t)c.k | (uintptr_t)c.v) % 2 ||
      ((uintptr_t)d->lse | (uintptr_t)d->prefix_pages | (uintptr_t)d->page_table | (uintptr_t)d->lens | (uintptr_t)d->d_status) % 4)
    return gts::fail(GTS_ERR_INVALID_ARG, "attention: tensor misaligned for its type");
  if (d->workspace_bytes < gts_attention_workspace_bytes(d))
    return gts::fail(GTS_ERR_NOMEM, "attention: workspace smaller than gts_attention_workspace_bytes");
  Pages maps = {}, own_maps = {};
  // (a scale of 0 would turn the -infinity of masked scores into NaN on the tensor cores)
  const bool mapped = tile_maps(maps, c, c.head_dim == 256 ? Tc<256>::KEYS : Tc<128>::KEYS);
  const Plan p = make_plan(*d, mapped && d->scale != 0.f, (char *)d->workspace);
  if (mapped) tile_maps(own_maps, c, p.own.keys);
  const cudaError_t e = c.dtype == GTS_BF16 ? launch<__nv_bfloat16>(a, p, maps, own_maps, c.head_dim, (cudaStream_t)stream)
                                            : launch<__half>(a, p, maps, own_maps, c.head_dim, (cudaStream_t)stream);
  return e == cudaSuccess ? GTS_OK : gts::cuda_fail(e, "attention: launch");
}
