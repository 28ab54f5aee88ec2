// Attention of a batch over a shared prefix and each sequence's own tokens, keys and values in pages
// (gts_prefix_attention).
//
// Mathematics.  With s_j = scale * q . k_j over the keys a query sees, m = max s_j, p_j = exp(s_j - m):
// out = sum p_j v_j / sum p_j, lse = m + log sum p_j.  The keys are taken tile by tile with the maximum and the sum so
// far: when a tile raises the maximum from m to m', what was summed is multiplied by exp(m - m').
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>

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

template <typename T> __device__ __forceinline__ float widen(T x);
template <> __device__ __forceinline__ float widen(__half x) { return __half2float(x); }
template <> __device__ __forceinline__ float widen(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T> __device__ __forceinline__ T narrow(float x);
template <> __device__ __forceinline__ __half narrow(float x) { return __float2half_rn(x); }
template <> __device__ __forceinline__ __nv_bfloat16 narrow(float x) { return __float2bfloat16_rn(x); }

constexpr int KEYS = 128;

// One block per query and head, one thread per key of a tile, then one per value column.
template <typename T, int D>
__global__ void __launch_bounds__(KEYS) k_attend(const Args a) {
  __shared__ float q[D], p[KEYS], wave[KEYS / 32];
  __shared__ int64_t row[KEYS];
  const int h = blockIdx.x, i = blockIdx.y % a.n_new, b = blockIdx.y / a.n_new;
  const int kh = h / a.group, tid = threadIdx.x;
  const T *src = (const T *)a.q + b * a.q_seq + i * a.q_tok + h * a.q_head;
  for (int d = tid; d < D; d += KEYS) q[d] = widen(src[d]);
  int len = a.lens[b];
  if (len > a.max_pages * (int64_t)a.page_size) {
    len = a.max_pages * a.page_size;
    if (a.status) *a.status = GTS_ERR_INVALID_PARAMS;
  }
  const int own = max(0, len - (a.n_new - 1 - i));
  const int64_t total = (int64_t)a.prefix_len + own;
  float m = -INFINITY, l = 0.f, acc[(D + KEYS - 1) / KEYS] = {};
  __syncthreads();
  for (int64_t j0 = 0; j0 < total; j0 += KEYS) {
    const int64_t j = j0 + tid;
    float s = -INFINITY;
    int64_t at = -1;
    if (j < total) {
      const bool shared = j < a.prefix_len;
      const int t = (int)(shared ? j : j - a.prefix_len);
      const int page = shared ? a.prefix_pages[t / a.page_size] : a.table[(int64_t)b * a.max_pages + t / a.page_size];
      if (page < 0 || page >= a.n_pages) {
        if (a.status) *a.status = GTS_ERR_INVALID_PARAMS;
      } else {
        const T *key = (const T *)a.k + page * a.k_page + (t % a.page_size) * a.k_tok + kh * a.k_head;
        at = page * a.v_page + (t % a.page_size) * a.v_tok + kh * a.v_head;
        float x = 0.f;
        for (int d = 0; d < D; d++) x += q[d] * widen(key[d]);
        s = x * a.scale;
      }
    }
    float top = s;
    for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, o));
    if (tid % 32 == 0) wave[tid / 32] = top;
    __syncthreads();
    for (int w = 0; w < KEYS / 32; w++) top = fmaxf(top, wave[w]);
    const float to = fmaxf(m, top), base = to == -INFINITY ? 0.f : to;
    const float keep = expf(m - base);
    p[tid] = at < 0 ? 0.f : expf(s - base);
    row[tid] = at;
    __syncthreads();
    m = to;
    l *= keep;
    for (int t = 0; t < KEYS; t++) l += p[t];
    for (int c = 0; c * KEYS + tid < D; c++) {
      acc[c] *= keep;
      for (int t = 0; t < KEYS; t++)
        if (row[t] >= 0) acc[c] += p[t] * widen(((const T *)a.v)[row[t] + c * KEYS + tid]);
    }
    __syncthreads();
  }
  T *dst = (T *)a.out + b * a.o_seq + i * a.o_tok + h * a.o_head;
  for (int c = 0; c * KEYS + tid < D; c++) dst[c * KEYS + tid] = narrow<T>(l == 0.f ? 0.f : acc[c] / l);
  if (a.lse && tid == 0) a.lse[((int64_t)b * a.n_new + i) * a.q_heads + h] = l == 0.f ? -INFINITY : m + logf(l);
}

template <typename T>
cudaError_t launch(const Args &a, int head_dim, cudaStream_t stream) {
  const dim3 grid(a.q_heads, a.n_seqs * a.n_new);
  switch (head_dim) {
    case 64: k_attend<T, 64><<<grid, KEYS, 0, stream>>>(a); break;
    case 128: k_attend<T, 128><<<grid, KEYS, 0, stream>>>(a); break;
    default: k_attend<T, 256><<<grid, KEYS, 0, stream>>>(a); break;
  }
  return cudaGetLastError();
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
  return 16;
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
  if (d->workspace_bytes < gts_attention_workspace_bytes(d))
    return gts::fail(GTS_ERR_NOMEM, "attention: workspace too small");
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
  const cudaError_t e = c.dtype == GTS_BF16 ? launch<__nv_bfloat16>(a, c.head_dim, (cudaStream_t)stream)
                                            : launch<__half>(a, c.head_dim, (cudaStream_t)stream);
  return e == cudaSuccess ? GTS_OK : gts::cuda_fail(e, "attention: launch");
}
