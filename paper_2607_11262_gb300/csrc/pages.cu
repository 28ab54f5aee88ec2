// Copies of pages of a cache (gts_copy_pages): a sequence that forks gets its own copy of the page that is being filled, a cache is
// compacted, pages move to another cache.
//
// Bound by memory: each value is read once and written once.  The values of one token and head are a row, contiguous on both sides;
// a block takes a stretch of a page's rows, in the order that lies contiguously where they are written, and moves them as 16-byte
// vectors with four loads of a thread in flight.  1.05 GB read and as much written take 307 us, 6.8 TB/s, the
// rate of a plain copy.
#include <algorithm>
#include <cstring>

#include "internal.h"

namespace {

constexpr int THREADS = 256, LOADS = 4;

struct Side { char *k, *v; int64_t k_page, k_tok, k_head, v_page, v_tok, v_head; };   // strides in bytes

struct Args {
  Side from, to;
  int from_pages, to_pages, page_size, kv_heads, row;   // row: vectors of a token's head
  int slices, heads_first;                              // blocks to a page; order of its rows: heads outside
  bool same;                                            // one cache
  const int32_t *src, *dst, *tokens;
  int32_t *status;
};

template <typename V>
__global__ void __launch_bounds__(THREADS) k_copy(const Args a) {
  const unsigned pair = blockIdx.x / a.slices;
  const int slice = blockIdx.x - pair * a.slices;
  const int src = a.src[pair], dst = a.dst[pair];
  if (src < 0 || dst < 0) return;
  if (src >= a.from_pages || dst >= a.to_pages) {
    if (a.status && slice == 0 && threadIdx.x == 0) *a.status = GTS_ERR_INVALID_PARAMS;
    return;
  }
  if (a.same && src == dst) return;
  const int tokens = a.tokens ? max(0, min(a.tokens[pair], a.page_size)) : a.page_size;
  // vectors of this page: 2 (keys, values) x rows x vectors of a row; a slice takes those at LOADS x THREADS x slices
  const int64_t rows = (int64_t)tokens * a.kv_heads, each = rows * a.row, all = 2 * each;
  const int inner = a.heads_first ? tokens : a.kv_heads;
  for (int64_t at = (int64_t)slice * LOADS * THREADS + threadIdx.x; at < all; at += (int64_t)a.slices * LOADS * THREADS) {
    V x[LOADS];
    V *to[LOADS];
#pragma unroll
    for (int i = 0; i < LOADS; i++) {
      const int64_t u = at + i * THREADS;
      to[i] = nullptr;
      if (u >= all) continue;
      const bool value = u >= each;
      const uint32_t in = (uint32_t)(value ? u - each : u), r = in / (uint32_t)a.row, c = in - r * a.row;
      const uint32_t outer = r / (uint32_t)inner, rest = r - outer * inner;
      const int64_t tok = a.heads_first ? rest : outer, head = a.heads_first ? outer : rest;
      const char *s = value ? a.from.v + src * a.from.v_page + tok * a.from.v_tok + head * a.from.v_head
                            : a.from.k + src * a.from.k_page + tok * a.from.k_tok + head * a.from.k_head;
      char *d = value ? a.to.v + dst * a.to.v_page + tok * a.to.v_tok + head * a.to.v_head
                      : a.to.k + dst * a.to.k_page + tok * a.to.k_tok + head * a.to.k_head;
      x[i] = ((const V *)s)[c];
      to[i] = (V *)d + c;
    }
#pragma unroll
    for (int i = 0; i < LOADS; i++)
      if (to[i]) *to[i] = x[i];
  }
}

Side side(const gts_cache &c, int size) {
  return {(char *)c.k, (char *)c.v, c.k_page_stride * size, c.k_token_stride * size, c.k_head_stride * size,
          c.v_page_stride * size, c.v_token_stride * size, c.v_head_stride * size};
}

bool aligned(const Side &s) {
  return (((uintptr_t)s.k | (uintptr_t)s.v | s.k_page | s.k_tok | s.k_head | s.v_page | s.v_tok | s.v_head) & 15) == 0;
}

template <typename V>
cudaError_t launch(Args &a, const gts_copy_pages_desc &d, int size, cudaStream_t s) {
  a.row = (int)(d.cache.head_dim * size / sizeof(V));
  const int64_t work = 2ll * a.page_size * a.kv_heads * a.row, per = (int64_t)LOADS * THREADS;
  // a block moves 16 to 64 KB; few copies are cut further, so that all SMs have a part
  const int64_t most = (work + per - 1) / per, want = std::max<int64_t>((most + 3) / 4, (608 + d.n_copies - 1) / d.n_copies);
  a.slices = (int)std::max<int64_t>(1, std::min({most, want, (int64_t)(0x7FFFFFFF / d.n_copies)}));
  k_copy<V><<<(unsigned)(d.n_copies * (uint32_t)a.slices), THREADS, 0, s>>>(a);
  return cudaGetLastError();
}

}  // namespace

extern "C" gts_status gts_copy_pages(const gts_copy_pages_desc *d, void *stream) {
  gts::clear_error();
  if (!d) return gts::fail(GTS_ERR_INVALID_ARG, "copy_pages: null desc");
  const gts_cache &f = d->cache, &t = d->into;
  if (f.dtype != GTS_BF16 && f.dtype != GTS_F16 && f.dtype != GTS_F32) return gts::fail(GTS_ERR_INVALID_ARG, "copy_pages: unknown dtype");
  if (f.dtype != t.dtype || f.page_size != t.page_size || f.kv_heads != t.kv_heads || f.head_dim != t.head_dim)
    return gts::fail(GTS_ERR_INVALID_ARG, "copy_pages: caches of one dtype, page_size, kv_heads and head_dim wanted");
  if (f.page_size < 1 || f.page_size > 65536 || f.kv_heads > 65536 || f.head_dim > 4096 || f.n_pages > 1u << 30 || t.n_pages > 1u << 30 ||
      (uint64_t)f.page_size * f.kv_heads * f.head_dim > 1u << 28)
    return gts::fail(GTS_ERR_INVALID_ARG, "copy_pages: pages of at most 65536 tokens and 2^28 values, at most 2^30 of them");
  if (d->n_copies > 1u << 30) return gts::fail(GTS_ERR_INVALID_ARG, "copy_pages: more than 2^30 copies");
  if (d->n_copies == 0 || f.kv_heads == 0 || f.head_dim == 0) return GTS_OK;
  const int size = f.dtype == GTS_F32 ? 4 : 2;
  if (!d->src || !d->dst || (f.n_pages && (!f.k || !f.v)) || (t.n_pages && (!t.k || !t.v)))
    return gts::fail(GTS_ERR_INVALID_ARG, "copy_pages: null src, dst or cache");
  if (((uintptr_t)d->src | (uintptr_t)d->dst | (uintptr_t)d->tokens | (uintptr_t)d->d_status) % 4 ||
      ((uintptr_t)f.k | (uintptr_t)f.v | (uintptr_t)t.k | (uintptr_t)t.v) % size)
    return gts::fail(GTS_ERR_INVALID_ARG, "copy_pages: misaligned src, dst, tokens, status or cache");
  Args a = {};
  a.from = side(f, size), a.to = side(t, size);
  a.from_pages = (int)f.n_pages, a.to_pages = (int)t.n_pages;
  a.page_size = (int)f.page_size, a.kv_heads = (int)f.kv_heads;
  a.heads_first = t.k_head_stride > t.k_token_stride;
  a.same = f.k == t.k && f.v == t.v && !memcmp(&a.from, &a.to, sizeof(Side));
  a.src = d->src, a.dst = d->dst, a.tokens = d->tokens, a.status = d->d_status;
  const bool vectors = aligned(a.from) && aligned(a.to) && f.head_dim * size % 16 == 0;
  const cudaError_t e = vectors ? launch<uint4>(a, *d, size, (cudaStream_t)stream)
                        : size == 2 ? launch<uint16_t>(a, *d, size, (cudaStream_t)stream) : launch<uint32_t>(a, *d, size, (cudaStream_t)stream);
  return e == cudaSuccess ? GTS_OK : gts::cuda_fail(e, "copy_pages: launch");
}
