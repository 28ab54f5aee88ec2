// Attention of a batch over a shared prefix and each sequence's own tokens, keys and values in pages
// (gts_prefix_attention).
//
// Mathematics.  With s_j = scale * q . k_j over the keys a query sees, m = max s_j, p_j = exp(s_j - m):
// out = sum p_j v_j / sum p_j, lse = m + log sum p_j.  The keys are taken tile by tile with the maximum and the sum so
// far: when a tile raises the maximum from m to m', what was summed is multiplied by exp(m - m').
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <atomic>
#include <cstring>
#include <string>

#include "internal.h"

namespace {

struct Args {
  const void *q;
  void *out;
  float *lse;
  int64_t q_seq, q_tok, q_head, o_seq, o_tok, o_head;
  const void *k, *v;
  int64_t k_page, k_tok, k_head, v_page, v_tok, v_head;
  int n_seqs, n_new, q_heads, kv_heads, group;
  int n_pages, page_size, max_pages, prefix_len;
  float scale;
  const int32_t *prefix_pages, *table, *lens;
  int32_t *status;
};

template <typename T> __device__ __forceinline__ T narrow(float x);
template <> __device__ __forceinline__ __half narrow(float x) { return __float2half_rn(x); }
template <> __device__ __forceinline__ __nv_bfloat16 narrow(float x) { return __float2bfloat16_rn(x); }

// ---------------------------------------------------------------- pieces of PTX
__device__ __forceinline__ uint32_t smem_u32(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void copy16(uint32_t dst, const void *src, bool live) {  // zeros where not live
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(live ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
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
// A "pair" is a key head with a tile of up to ROWS query rows that see the same keys: of the prefix, rows of all
// sequences (row (b * n_new + i) * group + h of n_seqs * n_new * group); of a sequence's own keys, its n_new * group rows.
// A pair's keys come in tiles of KEYS, the unit of work.  All units stand in one line (prefix pairs, then the sequences'),
// and each block takes an equal stretch of it, so ragged lengths cost nothing and the cut needs no plan from the host.
// A pair that lies within one block's stretch leaves one result per row; one that is cut leaves a partial result per block,
// which k_join adds up in the order of the keys.
constexpr int KEYS = 64;
constexpr int WARPS = 4, THREADS = 32 * WARPS;

struct Line {           // the units of one launch
  int has_prefix, has_own;
  int rows;             // of a pair's tile
  int prefix_tiles, own_tiles;   // row tiles of the prefix's rows, of a sequence's rows
  int blocks;
  int64_t *starts;      // [n_seqs + 2]: first unit of each sequence, the units of all, units per block
  float *cut_o;         // [blocks][2][rows][D]: results of the first and last pair of a block that are cut
  float2 *cut_ml;       // [blocks][2][rows]: maximum (of log2 scores) and sum
  float *whole_o[2];    // [rows of all][D], prefix and own: results of pairs that are not cut
  float2 *whole_ml[2];
};

__device__ __forceinline__ int tiles_of(int keys) { return (keys + KEYS - 1) / KEYS; }

__device__ __forceinline__ int own_len(const Args &a, int b) {
  const int len = a.lens[b], most = a.max_pages * a.page_size;
  if (len > most && a.status) *a.status = GTS_ERR_INVALID_PARAMS;
  return max(0, min(len, most));
}

struct Row { int b, i, h; };

// Row r of a pair's rows: prefix rows run over all sequences (b = -1), own rows over one.
__device__ __forceinline__ Row row_of(const Args &a, int b, int kh, int r) {
  const int per = a.n_new * a.group;
  Row x;
  x.b = b < 0 ? r / per : b;
  const int in = b < 0 ? r - x.b * per : r;
  x.i = in / a.group;
  x.h = kh * a.group + in - x.i * a.group;
  return x;
}

// One block of 4 warps: WM of them along the rows (16 each), 4 / WM along a tile's keys.  Keys and values stream through
// a ring of tiles in shared memory by 16-byte asynchronous copies, gathered row by row from their pages.  Scores and
// weights stay in the fragments of m16n8k16 products; each warp keeps its own running maximum and sum, and the warps
// along the keys are joined at the end of a pair.  Weights are rounded to the type of the values for their product with
// them (the sum is of the unrounded ones); everything else is in 32 bits.
template <int D> struct Ring {
  static constexpr int STAGES = D == 64 ? 4 : 3;
  static constexpr int TILE = KEYS * D * 2;            // bytes of a tile of keys or of values
};
template <int D, int WM> constexpr int stream_smem() {
  return Ring<D>::STAGES * 2 * Ring<D>::TILE + 16 * WM * D * 2 + 2 * KEYS * 2 * 8 + 64 * 8 + 64;
}

template <typename T, int D, int WM>
__global__ void __launch_bounds__(THREADS) k_stream(const Args a, const Line w) {
  constexpr int WK = WARPS / WM, ROWS = 16 * WM, KW = KEYS / WK, STAGES = Ring<D>::STAGES, TILE = Ring<D>::TILE;
  constexpr int CH = D / 8, PITCH = D * 2, OPITCH = D + 8;
  static_assert(64 * OPITCH * 4 <= STAGES * 2 * TILE, "the joined result fits the ring");
  extern __shared__ __align__(128) unsigned char smem[];
  unsigned char *ring = smem, *qs = smem + STAGES * 2 * TILE;
  int64_t *offs = (int64_t *)(qs + ROWS * PITCH);      // [2][KEYS][2]: where the rows of the next tile to load start
  float2 *stat = (float2 *)(offs + 2 * KEYS * 2);      // [64]: maximum and sum of each warp's rows
  int64_t *found = (int64_t *)(stat + 64);             // [4]
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
  const int wm = warp % WM, wk = warp / WM, quad = lane / 4, t4 = lane % 4;
  const uint32_t ring_at = smem_u32(ring), q_at = smem_u32(qs);
  const bool aligned = ((((uintptr_t)a.k | (uintptr_t)a.v) >> 1 | a.k_page | a.k_tok | a.k_head | a.v_page | a.v_tok | a.v_head) & 7) == 0;
  const bool q_aligned = (((uintptr_t)a.q >> 1 | a.q_seq | a.q_tok | a.q_head) & 7) == 0;
  const bool o_aligned = (((uintptr_t)a.out >> 1 | a.o_seq | a.o_tok | a.o_head) & 3) == 0;
  const float sl2 = a.scale * 1.4426950408889634f;     // scores in units of log 2

  // the line of units, and this block's stretch of it
  const int n_prefix = w.has_prefix ? tiles_of(a.prefix_len) : 0;
  const int64_t prefix_units = (int64_t)n_prefix * a.kv_heads * w.prefix_tiles;
  const int own_pairs = a.kv_heads * w.own_tiles;
  const int each = w.has_own ? (a.n_seqs + THREADS - 1) / THREADS : 0;
  const int b_first = min(a.n_seqs, tid * each), b_last = min(a.n_seqs, (tid + 1) * each);
  int64_t mine = 0;
  for (int b = b_first; b < b_last; b++) mine += (int64_t)tiles_of(own_len(a, b)) * own_pairs;
  int64_t upto = mine;
  for (int o = 1; o < 32; o *= 2) {
    const int64_t x = __shfl_up_sync(~0u, upto, o);
    if (lane >= o) upto += x;
  }
  if (lane == 31) found[warp] = upto;
  __syncthreads();
  int64_t base = prefix_units, total = prefix_units;
  for (int x = 0; x < WARPS; x++) {
    if (x < warp) base += found[x];
    total += found[x];
  }
  base += upto - mine;                                 // first unit of sequence b_first
  const int64_t per = (total + w.blocks - 1) / w.blocks;
  int64_t u = per * blockIdx.x;
  const int64_t u_end = min(total, u + per);
  __syncthreads();
  if (blockIdx.x == 0) {
    int64_t at = base;
    for (int b = b_first; b < b_last; b++) {
      w.starts[b] = at;
      at += (int64_t)tiles_of(own_len(a, b)) * own_pairs;
    }
    if (tid == 0) w.starts[a.n_seqs] = total, w.starts[a.n_seqs + 1] = per;
  }
  if (u >= u_end) return;
  if (u >= prefix_units && u >= base && u < base + mine) {
    int64_t at = base;
    int b = b_first;
    for (;; b++) {
      const int64_t n = (int64_t)tiles_of(own_len(a, b)) * own_pairs;
      if (u < at + n) break;
      at += n;
    }
    found[0] = b, found[1] = at;
  }
  __syncthreads();
  int b = u >= prefix_units ? (int)found[0] : -1;
  int64_t b_start = u >= prefix_units ? found[1] : 0;
  int len = b < 0 ? a.prefix_len : own_len(a, b);
  __syncthreads();

  while (u < u_end) {
    int64_t n = tiles_of(len), units = n * (b < 0 ? (int64_t)a.kv_heads * w.prefix_tiles : own_pairs);
    while (u >= b_start + units) {                     // the next sequence that has keys of its own
      b_start += units;
      len = own_len(a, ++b);
      n = tiles_of(len);
      units = n * own_pairs;
    }
    const int pair = (int)((u - b_start) / n), tiles = b < 0 ? w.prefix_tiles : w.own_tiles;
    const int tile0 = (int)((u - b_start) - pair * n), tile1 = (int)min((int64_t)n, tile0 + (u_end - u));
    const int kh = pair / tiles, row0 = (pair - kh * tiles) * ROWS;
    const int rows = min(ROWS, (b < 0 ? a.n_seqs : 1) * a.n_new * a.group - row0);
    const bool whole = tile0 == 0 && tile1 == n;
    const int32_t *pages = b < 0 ? a.prefix_pages : a.table + (int64_t)b * a.max_pages;

    // queries: rows beyond the last are zeros
    for (int x = tid; x < ROWS * CH; x += THREADS) {
      const int r = x / CH, c = x % CH;
      const uint32_t at = r * PITCH + ((c ^ (r & 7)) * 16);
      uint4 v = make_uint4(0, 0, 0, 0);
      if (r < rows) {
        const Row p = row_of(a, b, kh, row0 + r);
        const T *src = (const T *)a.q + p.b * a.q_seq + p.i * a.q_tok + p.h * a.q_head + c * 8;
        if (q_aligned) {
          v = *(const uint4 *)src;
        } else {
          T e[8];
#pragma unroll
          for (int j = 0; j < 8; j++) e[j] = src[j];
          memcpy(&v, e, 16);
        }
      }
      *(uint4 *)(qs + at) = v;
    }
    // own keys that the rows of this thread's fragments see
    int limit[2];
#pragma unroll
    for (int x = 0; x < 2; x++) {
      const int r = row0 + wm * 16 + quad + 8 * x;
      limit[x] = b < 0 ? len : len - (a.n_new - 1 - min(r / a.group, a.n_new - 1));
    }
    const int seen_by_all = b < 0 ? len : len - (a.n_new - 1);

    // page numbers are fetched two tiles ahead, places one tile ahead of the copies
    int page_next = 0;
    auto fetch = [&](int tile) {
      const int j = tile * KEYS + tid;
      if (tid < KEYS && tile < tile1 && j < len) page_next = pages[j / a.page_size];
    };
    auto place = [&](int tile) {
      if (tid >= KEYS || tile >= tile1) return;
      const int j = tile * KEYS + tid;
      int64_t k_off = -1, v_off = 0;
      if (j < len) {
        if (page_next < 0 || page_next >= a.n_pages) {
          if (a.status) *a.status = GTS_ERR_INVALID_PARAMS;
        } else {
          const int in = j % a.page_size;
          k_off = page_next * a.k_page + in * a.k_tok + kh * a.k_head;
          v_off = page_next * a.v_page + in * a.v_tok + kh * a.v_head;
        }
      }
      int64_t *to = offs + ((tile & 1) * KEYS + tid) * 2;
      to[0] = k_off, to[1] = v_off;
    };
    auto load = [&](int tile) {
      if (tile < tile1) {
        const uint32_t at = ring_at + (tile % STAGES) * 2 * TILE;
        for (int x = tid; x < KEYS * CH; x += THREADS) {
          const int r = x / CH, c = x % CH;
          const int64_t *from = offs + ((tile & 1) * KEYS + r) * 2;
          const bool live = from[0] >= 0;
          const T *k = (const T *)a.k + (live ? from[0] + c * 8 : 0), *v = (const T *)a.v + (live ? from[1] + c * 8 : 0);
          const uint32_t to = at + r * PITCH + ((c ^ (r & 7)) * 16);
          if (aligned) {
            copy16(to, k, live);
            copy16(to + TILE, v, live);
          } else {
            T e[8], f[8];
#pragma unroll
            for (int j = 0; j < 8; j++) e[j] = live ? k[j] : narrow<T>(0.f), f[j] = live ? v[j] : narrow<T>(0.f);
            memcpy(ring + (to - ring_at), e, 16);
            memcpy(ring + (to - ring_at) + TILE, f, 16);
          }
        }
      }
      copies_commit();
    };
    fetch(tile0);
    place(tile0);
    fetch(tile0 + 1);
    __syncthreads();
#pragma unroll
    for (int x = 0; x < STAGES - 1; x++) {
      load(tile0 + x);
      place(tile0 + x + 1);
      fetch(tile0 + x + 2);
      __syncthreads();
    }

    float o[D / 8][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
    for (int x = 0; x < D / 8; x++) o[x][0] = o[x][1] = o[x][2] = o[x][3] = 0.f;

    for (int tile = tile0; tile < tile1; tile++) {
      copies_wait<STAGES - 2>();
      __syncthreads();
      load(tile + STAGES - 1);
      place(tile + STAGES);
      fetch(tile + STAGES + 1);
      const uint32_t k_at = ring_at + (tile % STAGES) * 2 * TILE, v_at = k_at + TILE;
      const int mi = lane / 8, mr = lane % 8;
      float s[KW / 8][4];
#pragma unroll
      for (int x = 0; x < KW / 8; x++) s[x][0] = s[x][1] = s[x][2] = s[x][3] = 0.f;
#pragma unroll
      for (int d = 0; d < D / 16; d++) {
        uint32_t qf[4];
        const int r = wm * 16 + (mi & 1) * 8 + mr;
        ldsm(qf, q_at + r * PITCH + (((d * 2 + (mi >> 1)) ^ (r & 7)) * 16));
#pragma unroll
        for (int x = 0; x < KW / 16; x++) {
          uint32_t kf[4];
          const int key = wk * KW + x * 16 + (mi >> 1) * 8 + mr;
          ldsm(kf, k_at + key * PITCH + (((d * 2 + (mi & 1)) ^ (key & 7)) * 16));
          mma<T>(s[2 * x], qf, kf[0], kf[1]);
          mma<T>(s[2 * x + 1], qf, kf[2], kf[3]);
        }
      }
      const int key0 = tile * KEYS + wk * KW;
      const bool masked = key0 + KW > seen_by_all;
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
        const int key = wk * KW + x * 16 + (mi & 1) * 8 + mr;
#pragma unroll
        for (int d = 0; d < D / 16; d++) {
          uint32_t vf[4];
          ldsm_t(vf, v_at + key * PITCH + (((d * 2 + (mi >> 1)) ^ (key & 7)) * 16));
          mma<T>(o[2 * d], pf[x], vf[0], vf[1]);
          mma<T>(o[2 * d + 1], pf[x], vf[2], vf[3]);
        }
      }
    }

    // join the warps along the keys, in shared memory, and write the pair's rows
    copies_wait<0>();
    __syncthreads();
    float *acc = (float *)ring;                        // [4 warps][16][OPITCH]
#pragma unroll
    for (int x = 0; x < 2; x++) {
      l[x] += __shfl_xor_sync(~0u, l[x], 1);
      l[x] += __shfl_xor_sync(~0u, l[x], 2);
      const int r = warp * 16 + quad + 8 * x;
      if (t4 == 0) stat[r] = make_float2(m[x], l[x]);
#pragma unroll
      for (int d = 0; d < D / 8; d++) *(float2 *)(acc + r * OPITCH + d * 8 + t4 * 2) = make_float2(o[d][2 * x], o[d][2 * x + 1]);
    }
    __syncthreads();
    const bool final = whole && b >= 0 && a.prefix_len == 0;
    const int side = u > per * blockIdx.x;             // 0: the block's first pair
    for (int x = tid; x < rows * (D / 4); x += THREADS) {
      const int r = x / (D / 4), c = x % (D / 4) * 4;
      float top = -INFINITY;
#pragma unroll
      for (int k = 0; k < WK; k++) top = fmaxf(top, stat[(k * WM + r / 16) * 16 + r % 16].x);
      const float from = top == -INFINITY ? 0.f : top;
      float sum = 0.f;
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int k = 0; k < WK; k++) {
        const int at = (k * WM + r / 16) * 16 + r % 16;
        const float f = exp2_fast(stat[at].x - from);
        const float4 y = *(const float4 *)(acc + at * OPITCH + c);
        sum += f * stat[at].y;
        v.x += f * y.x, v.y += f * y.y, v.z += f * y.z, v.w += f * y.w;
      }
      if (final) {
        const Row p = row_of(a, b, kh, row0 + r);
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        T *dst = (T *)a.out + p.b * a.o_seq + p.i * a.o_tok + p.h * a.o_head + c;
        const uint32_t lo = pack<T>(v.x * inv, v.y * inv), hi = pack<T>(v.z * inv, v.w * inv);
        if (o_aligned) {
          *(uint2 *)dst = make_uint2(lo, hi);
        } else {
          T e[4];
          memcpy(e, &lo, 4), memcpy(e + 2, &hi, 4);
          for (int j = 0; j < 4; j++) dst[j] = e[j];
        }
        if (c == 0 && a.lse)
          a.lse[((int64_t)p.b * a.n_new + p.i) * a.q_heads + p.h] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * 0.6931471805599453f;
      } else if (whole) {
        const Row p = row_of(a, b, kh, row0 + r);
        const int64_t at = ((int64_t)p.b * a.n_new + p.i) * a.q_heads + p.h;
        *(float4 *)(w.whole_o[b >= 0] + at * D + c) = v;
        if (c == 0) w.whole_ml[b >= 0][at] = make_float2(top, sum);
      } else {
        const int64_t at = ((int64_t)blockIdx.x * 2 + side) * ROWS + r;
        *(float4 *)(w.cut_o + at * D + c) = v;
        if (c == 0) w.cut_ml[at] = make_float2(top, sum);
      }
    }
    __syncthreads();
    u += tile1 - tile0;
  }
}

// Joins what a row's pairs left, prefix first, then the sequence's own keys, each in the order of its blocks: one warp a
// row.  A row whose one pair was written whole, with no prefix, is done already.
template <typename T, int D>
__global__ void __launch_bounds__(THREADS) k_join(const Args a, const Line lp, const Line lo) {
  constexpr int E = D / 32;
  const int lane = threadIdx.x % 32;
  const int64_t row = (int64_t)blockIdx.x * WARPS + threadIdx.x / 32;
  if (row >= (int64_t)a.n_seqs * a.n_new * a.q_heads) return;
  const int h = (int)(row % a.q_heads), i = (int)(row / a.q_heads % a.n_new), b = (int)(row / a.q_heads / a.n_new);
  const int kh = h / a.group;
  float m = -INFINITY, l = 0.f, acc[E] = {};
  auto add = [&](const float *o, float2 ml) {
    const float top = fmaxf(m, ml.x), from = top == -INFINITY ? 0.f : top;
    const float f = exp2_fast(m - from), g = exp2_fast(ml.x - from);
#pragma unroll
    for (int e = 0; e < E; e++) acc[e] = acc[e] * f + o[lane * E + e] * g;
    l = l * f + ml.y * g;
    m = top;
  };
  auto gather = [&](const Line &w, bool own, int r, int tiles, int64_t start, int64_t n) {
    const int pair = kh * tiles + r / w.rows;
    const int64_t u0 = start + pair * n, per = w.starts[a.n_seqs + 1], c0 = u0 / per, c1 = (u0 + n - 1) / per;
    if (c0 == c1) {
      if (own && a.prefix_len == 0) return true;
      add(w.whole_o[own] + row * D, w.whole_ml[own][row]);
    } else {
      for (int64_t c = c0; c <= c1; c++) {
        const int64_t at = (c * 2 + (u0 > c * per)) * w.rows + r % w.rows;
        add(w.cut_o + at * D, w.cut_ml[at]);
      }
    }
    return false;
  };
  if (a.prefix_len) gather(lp, false, (b * a.n_new + i) * a.group + h - kh * a.group, lp.prefix_tiles, 0, tiles_of(a.prefix_len));
  const int n = tiles_of(own_len(a, b));
  if (n && gather(lo, true, i * a.group + h - kh * a.group, lo.own_tiles, lo.starts[b], n)) return;
  const float inv = l == 0.f ? 0.f : 1.f / l;
  T *dst = (T *)a.out + b * a.o_seq + i * a.o_tok + h * a.o_head + lane * E;
#pragma unroll
  for (int e = 0; e < E; e++) dst[e] = narrow<T>(acc[e] * inv);
  if (a.lse && lane == 0) a.lse[row] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
}

// ---------------------------------------------------------------- host side
constexpr int SMS = 152;

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

struct Plan {
  int wm;              // warps along the rows
  int blocks;
  Line line;
  size_t bytes;
};

// rows of a sequence's own pairs decide the shape: 16, 32 or 64 of them to a tile
Plan make_plan(const gts_attention_desc &d, char *at) {
  const int D = (int)d.cache.head_dim, group = (int)(d.q_heads / d.cache.kv_heads);
  const int64_t own_rows = (int64_t)d.n_new * group, all = own_rows * d.n_seqs;
  Plan p = {};
  p.wm = own_rows <= 16 ? 1 : own_rows <= 32 ? 2 : 4;
  const int rows = 16 * p.wm;
  p.blocks = SMS * (D == 64 ? 3 : D == 128 ? 2 : 1);
  Line &w = p.line;
  w.has_prefix = d.prefix_len > 0, w.has_own = 1, w.rows = rows;
  w.prefix_tiles = (int)((all + rows - 1) / rows), w.own_tiles = (int)((own_rows + rows - 1) / rows);
  w.blocks = p.blocks;
  size_t n = 0;
  auto take = [&](size_t bytes) {
    char *x = at ? at + n : nullptr;
    n += up(bytes);
    return x;
  };
  const size_t total_rows = (size_t)d.n_seqs * d.n_new * d.q_heads, cut = (size_t)p.blocks * 2 * rows;
  w.starts = (int64_t *)take(((size_t)d.n_seqs + 2) * 8);
  w.cut_ml = (float2 *)take(cut * 8);
  w.cut_o = (float *)take(cut * D * 4);
  if (d.prefix_len) {
    for (int k = 0; k < 2; k++) {
      w.whole_ml[k] = (float2 *)take(total_rows * 8);
      w.whole_o[k] = (float *)take(total_rows * D * 4);
    }
  }
  p.bytes = n;
  return p;
}

template <typename T, int D, int WM>
cudaError_t stream(const Args &a, const Line &w, cudaStream_t s) {
  constexpr int bytes = stream_smem<D, WM>();
  static std::atomic<uint64_t> granted{0};
  const cudaError_t e = grant(k_stream<T, D, WM>, bytes, granted);
  if (e != cudaSuccess) return e;
  k_stream<T, D, WM><<<w.blocks, THREADS, bytes, s>>>(a, w);
  return cudaGetLastError();
}

template <typename T, int D>
cudaError_t run(const Args &a, const Plan &p, cudaStream_t s) {
  cudaError_t e = p.wm == 1 ? stream<T, D, 1>(a, p.line, s) : p.wm == 2 ? stream<T, D, 2>(a, p.line, s) : stream<T, D, 4>(a, p.line, s);
  if (e != cudaSuccess) return e;
  const int64_t rows = (int64_t)a.n_seqs * a.n_new * a.q_heads;
  k_join<T, D><<<(unsigned)((rows + WARPS - 1) / WARPS), THREADS, 0, s>>>(a, p.line, p.line);
  return cudaGetLastError();
}

template <typename T>
cudaError_t launch(const Args &a, const Plan &p, int head_dim, cudaStream_t s) {
  return head_dim == 64 ? run<T, 64>(a, p, s) : head_dim == 128 ? run<T, 128>(a, p, s) : run<T, 256>(a, p, s);
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
  if (d.prefix_len > 1u << 30 || (uint64_t)d.max_pages * c.page_size > 1u << 30)
    return "attention: a prefix or a sequence of more than 2^30 tokens";
  return nullptr;
}

}  // namespace

extern "C" size_t gts_attention_workspace_bytes(const gts_attention_desc *d) {
  if (!d || refuse_shape(*d)) return 0;
  return make_plan(*d, nullptr).bytes;
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
  a.scale = d->scale;
  a.prefix_pages = d->prefix_pages, a.table = d->page_table, a.lens = d->lens;
  a.status = d->d_status;
  const Plan p = make_plan(*d, (char *)d->workspace);
  if (d->workspace_bytes < p.bytes)
    return gts::fail(GTS_ERR_NOMEM, ("attention: workspace too small: need " + std::to_string(p.bytes) + " bytes").c_str());
  const cudaError_t e = c.dtype == GTS_BF16 ? launch<__nv_bfloat16>(a, p, c.head_dim, (cudaStream_t)stream)
                                            : launch<__half>(a, p, c.head_dim, (cudaStream_t)stream);
  return e == cudaSuccess ? GTS_OK : gts::cuda_fail(e, "attention: launch");
}
