// Attention of packed sequences over themselves with its gradient (gts_prompt_attention, gts_prompt_attention_grad), and of chunks of
// new tokens over a paged cache (gts_chunk_attention).
//
// Mathematics.  Query i of a sequence with n queries and m keys sees the keys j <= i + m - n (causal) or all.  With s_ij = scale *
// q_i . k_j, out_i = sum_j exp(s_ij - max) v_j / sum_j exp(s_ij - max), taken with the maximum and the sum so far.  Backward: with
// p_ij = exp(s_ij - lse_i), e_i = dout_i . out_i - dlse_i and ds_ij = p_ij (dout_i . v_j - e_i): dv_j = sum p_ij dout_i,
// dq_i = scale sum ds_ij k_j, dk_j = scale sum ds_ij q_i.
//
// The simplest form: a warp for each row of a result, the head's values along its lanes, everything in 32 bits.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <cmath>

#include "internal.h"

namespace {

constexpr int WARPS = 8;

struct Heads { const void *data; int64_t tok, head; };

struct Args {
  Heads q, k, v, out, dout, dq, dk, dv;
  float *lse, *delta;
  const float *dlse;
  const int32_t *starts, *lens, *table;
  int64_t k_page, v_page;
  int n_seqs, n_tokens, q_heads, kv_heads, group, causal, zero_rest, paged;
  int n_pages, page_size, max_pages;
  float scale;
  int32_t *status;
};

template <typename T> __device__ __forceinline__ float widen(T x);
template <> __device__ __forceinline__ float widen(__half x) { return __half2float(x); }
template <> __device__ __forceinline__ float widen(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T> __device__ __forceinline__ T narrow(float x);
template <> __device__ __forceinline__ __half narrow(float x) { return __float2half_rn(x); }
template <> __device__ __forceinline__ __nv_bfloat16 narrow(float x) { return __float2bfloat16_rn(x); }

struct Seq { int first, n, keys; };  // rows of the queries, and keys

__device__ __forceinline__ Seq sequence(const Args &a, int b) {
  const int from = a.starts[b], to = a.starts[b + 1];
  Seq s;
  s.first = max(0, min(from, a.n_tokens));
  s.n = max(0, min(to, a.n_tokens) - s.first);
  bool bad = from != s.first || to != s.first + s.n;
  s.keys = s.n;
  if (a.paged) {
    const int most = a.max_pages * a.page_size;
    s.keys = max(0, min(a.lens[b], most));
    bad |= a.lens[b] > most;
  }
  if (bad && a.status) *a.status = GTS_ERR_INVALID_PARAMS;
  return s;
}

// The sequence of a row, -1: none.
__device__ __forceinline__ int sequence_of(const Args &a, int row) {
  for (int b = 0; b < a.n_seqs; b++)
    if (a.starts[b] <= row && row < a.starts[b + 1]) return b;
  return -1;
}

template <typename T, int E> __device__ __forceinline__ void load(float (&x)[E], const T *p) {
#pragma unroll
  for (int e = 0; e < E; e++) x[e] = widen(p[e * 32]);
}
template <typename T, int E> __device__ __forceinline__ void store(T *p, const float (&x)[E], float f) {
#pragma unroll
  for (int e = 0; e < E; e++) p[e * 32] = narrow<T>(x[e] * f);
}
template <int E> __device__ __forceinline__ float dot(const float (&x)[E], const float (&y)[E]) {
  float s = 0.f;
#pragma unroll
  for (int e = 0; e < E; e++) s += x[e] * y[e];
#pragma unroll
  for (int o = 16; o; o /= 2) s += __shfl_xor_sync(~0u, s, o);
  return s;
}
template <typename T> __device__ __forceinline__ const T *at(const Heads &h, int64_t row, int head) { return (const T *)h.data + row * h.tok + head * h.head; }

// The rows of a key and its value: false where the page table has no such page.
template <typename T>
__device__ __forceinline__ bool key_rows(const Args &a, int b, const Seq &s, int j, int kh, const T *&k, const T *&v) {
  if (!a.paged) {
    k = at<T>(a.k, s.first + j, kh), v = at<T>(a.v, s.first + j, kh);
    return true;
  }
  const int page = a.table[(int64_t)b * a.max_pages + j / a.page_size];
  if ((unsigned)page >= (unsigned)a.n_pages) {
    if (a.status) *a.status = GTS_ERR_INVALID_PARAMS;
    return false;
  }
  k = at<T>(a.k, j % a.page_size, kh) + page * a.k_page;
  v = at<T>(a.v, j % a.page_size, kh) + page * a.v_page;
  return true;
}

template <typename T, int D>
__global__ void __launch_bounds__(WARPS * 32) k_forward(const Args a) {
  const int64_t w = (int64_t)blockIdx.x * WARPS + threadIdx.x / 32;
  const int lane = threadIdx.x % 32;
  if (blockIdx.x == 0)
    for (int b = threadIdx.x; b < a.n_seqs; b += WARPS * 32) sequence(a, b);   // reports those out of range
  if (w >= (int64_t)a.n_tokens * a.q_heads) return;
  const int row = (int)(w / a.q_heads), h = (int)(w % a.q_heads), b = sequence_of(a, row);
  float o[D / 32] = {}, q[D / 32], k[D / 32], v[D / 32], m = -INFINITY, l = 0.f;
  if (b >= 0) {
    const Seq s = sequence(a, b);
    const int seen = a.causal ? min(s.keys, s.keys - s.n + (row - s.first) + 1) : s.keys;
    load(q, at<T>(a.q, row, h) + lane);
    for (int j = 0; j < seen; j++) {
      const T *kp, *vp;
      if (!key_rows(a, b, s, j, h / a.group, kp, vp)) continue;
      load(k, kp + lane), load(v, vp + lane);
      const float x = dot(q, k) * a.scale, top = fmaxf(m, x), keep = m == -INFINITY ? 0.f : __expf(m - top), p = __expf(x - top);
      l = l * keep + p, m = top;
#pragma unroll
      for (int e = 0; e < D / 32; e++) o[e] = o[e] * keep + p * v[e];
    }
  }
  if (b >= 0 || a.zero_rest & 1) store((T *)at<T>(a.out, row, h) + lane, o, l == 0.f ? 0.f : 1.f / l);
  if ((b >= 0 || a.zero_rest & 2) && a.lse && lane == 0) a.lse[w] = l == 0.f ? -INFINITY : m + logf(l);
}

template <typename T, int D>
__global__ void __launch_bounds__(WARPS * 32) k_grad_q(const Args a) {
  const int64_t w = (int64_t)blockIdx.x * WARPS + threadIdx.x / 32;
  const int lane = threadIdx.x % 32;
  if (blockIdx.x == 0)
    for (int b = threadIdx.x; b < a.n_seqs; b += WARPS * 32) sequence(a, b);
  if (w >= (int64_t)a.n_tokens * a.q_heads) return;
  const int row = (int)(w / a.q_heads), h = (int)(w % a.q_heads), b = sequence_of(a, row);
  float g[D / 32] = {}, q[D / 32], k[D / 32], v[D / 32], y[D / 32];
  if (b >= 0) {
    const Seq s = sequence(a, b);
    const int seen = a.causal ? row - s.first + 1 : s.keys;
    load(q, at<T>(a.q, row, h) + lane), load(y, at<T>(a.dout, row, h) + lane), load(v, at<T>(a.out, row, h) + lane);
    const float delta = dot(y, v) - (a.dlse ? a.dlse[w] : 0.f), lse = a.lse[w];
    if (lane == 0) a.delta[w] = delta;
    for (int j = 0; j < seen; j++) {
      const T *kp, *vp;
      key_rows(a, b, s, j, h / a.group, kp, vp);
      load(k, kp + lane), load(v, vp + lane);
      const float ds = __expf(dot(q, k) * a.scale - lse) * (dot(y, v) - delta);
#pragma unroll
      for (int e = 0; e < D / 32; e++) g[e] += ds * k[e];
    }
  }
  if (b >= 0 || a.zero_rest & 1) store((T *)at<T>(a.dq, row, h) + lane, g, a.scale);
}

template <typename T, int D>
__global__ void __launch_bounds__(WARPS * 32) k_grad_kv(const Args a) {
  const int64_t w = (int64_t)blockIdx.x * WARPS + threadIdx.x / 32;
  const int lane = threadIdx.x % 32;
  if (w >= (int64_t)a.n_tokens * a.kv_heads) return;
  const int row = (int)(w / a.kv_heads), kh = (int)(w % a.kv_heads), b = sequence_of(a, row);
  float gk[D / 32] = {}, gv[D / 32] = {}, q[D / 32], k[D / 32], v[D / 32], y[D / 32];
  if (b >= 0) {
    const Seq s = sequence(a, b);
    load(k, at<T>(a.k, row, kh) + lane), load(v, at<T>(a.v, row, kh) + lane);
    for (int x = a.causal ? row : s.first; x < s.first + s.n; x++) {
      for (int h = kh * a.group; h < (kh + 1) * a.group; h++) {
        load(q, at<T>(a.q, x, h) + lane), load(y, at<T>(a.dout, x, h) + lane);
        const int64_t r = (int64_t)x * a.q_heads + h;
        const float p = __expf(dot(q, k) * a.scale - a.lse[r]), ds = p * (dot(y, v) - a.delta[r]);
#pragma unroll
        for (int e = 0; e < D / 32; e++) gk[e] += ds * q[e], gv[e] += p * y[e];
      }
    }
  }
  if (b >= 0 || a.zero_rest & 2) store((T *)at<T>(a.dk, row, kh) + lane, gk, a.scale);
  if (b >= 0 || a.zero_rest & 4) store((T *)at<T>(a.dv, row, kh) + lane, gv, 1.f);
}

// ---------------------------------------------------------------- host side
unsigned blocks_for(int64_t rows) { return (unsigned)((rows + WARPS - 1) / WARPS); }

template <typename T, int D> void forward(const Args &a, cudaStream_t s) {
  k_forward<T, D><<<blocks_for((int64_t)a.n_tokens * a.q_heads), WARPS * 32, 0, s>>>(a);
}
template <typename T, int D> void backward(const Args &a, cudaStream_t s) {
  k_grad_q<T, D><<<blocks_for((int64_t)a.n_tokens * a.q_heads), WARPS * 32, 0, s>>>(a);
  k_grad_kv<T, D><<<blocks_for((int64_t)a.n_tokens * a.kv_heads), WARPS * 32, 0, s>>>(a);
}
cudaError_t run(const Args &a, int32_t dtype, uint32_t dim, bool grad, cudaStream_t s) {
  if (dtype == GTS_BF16) {
    if (dim == 64) grad ? backward<__nv_bfloat16, 64>(a, s) : forward<__nv_bfloat16, 64>(a, s);
    else grad ? backward<__nv_bfloat16, 128>(a, s) : forward<__nv_bfloat16, 128>(a, s);
  } else {
    if (dim == 64) grad ? backward<__half, 64>(a, s) : forward<__half, 64>(a, s);
    else grad ? backward<__half, 128>(a, s) : forward<__half, 128>(a, s);
  }
  return cudaGetLastError();
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
  if (misaligned(d.q) || misaligned(d.k) || misaligned(d.v) || misaligned(d.out) ||
      ((uintptr_t)d.starts | (uintptr_t)d.lse | (uintptr_t)d.d_status) % 4)
    return "attention: tensor misaligned for its type";
  if (!d.workspace || (uintptr_t)d.workspace % 16) return "attention: null or misaligned workspace";
  return nullptr;
}
Args args(const gts_prompt_desc &d) {
  Args a = {};
  a.q = heads(d.q), a.k = heads(d.k), a.v = heads(d.v), a.out = heads(d.out);
  a.lse = d.lse, a.starts = d.starts;
  a.n_seqs = (int)d.n_seqs, a.n_tokens = (int)d.n_tokens, a.q_heads = (int)d.q_heads, a.kv_heads = (int)d.kv_heads;
  a.group = a.q_heads / a.kv_heads, a.causal = (int)d.causal, a.zero_rest = (int)d.zero_rest;
  a.scale = d.scale, a.status = d.d_status;
  return a;
}
size_t up(size_t x) { return (x + 255) / 256 * 256; }

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

extern "C" size_t gts_prompt_workspace_bytes(const gts_prompt_desc *d) { return !d || refuse_shape(*d) ? 0 : 256; }

extern "C" gts_status gts_prompt_attention(const gts_prompt_desc *d, void *stream) {
  gts::clear_error();
  if (!d) return gts::fail(GTS_ERR_INVALID_ARG, "attention: null desc");
  if (const char *why = refuse_shape(*d)) return gts::fail(GTS_ERR_INVALID_ARG, why);
  if (d->n_tokens == 0) return GTS_OK;
  if (const char *why = refuse_call(*d, false)) return gts::fail(GTS_ERR_INVALID_ARG, why);
  if (d->workspace_bytes < gts_prompt_workspace_bytes(d))
    return gts::fail(GTS_ERR_NOMEM, "attention: workspace smaller than gts_prompt_workspace_bytes");
  const cudaError_t e = run(args(*d), d->dtype, d->head_dim, false, (cudaStream_t)stream);
  return e == cudaSuccess ? GTS_OK : gts::cuda_fail(e, "attention: launch");
}

extern "C" size_t gts_prompt_grad_workspace_bytes(const gts_prompt_grad_desc *d) {
  return !d || refuse_shape(d->forward) ? 0 : up((size_t)d->forward.n_tokens * d->forward.q_heads * 4) + 256;
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
  if (f.workspace_bytes < gts_prompt_grad_workspace_bytes(d))
    return gts::fail(GTS_ERR_NOMEM, "attention: workspace smaller than gts_prompt_grad_workspace_bytes");
  Args a = args(f);
  a.dout = heads(d->dout), a.dq = heads(d->dq), a.dk = heads(d->dk), a.dv = heads(d->dv);
  a.dlse = d->dlse, a.delta = (float *)f.workspace;
  const cudaError_t e = run(a, f.dtype, f.head_dim, true, (cudaStream_t)stream);
  return e == cudaSuccess ? GTS_OK : gts::cuda_fail(e, "attention: launch");
}

extern "C" size_t gts_chunk_workspace_bytes(const gts_chunk_desc *d) { return !d || refuse_shape(*d) ? 0 : 256; }

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
  a.group = a.q_heads / a.kv_heads, a.causal = 1, a.zero_rest = (int)d->zero_rest, a.paged = 1;
  a.n_pages = (int)c.n_pages, a.page_size = (int)c.page_size, a.max_pages = (int)d->max_pages;
  a.scale = d->scale, a.status = d->d_status;
  const cudaError_t e = run(a, c.dtype, c.head_dim, false, (cudaStream_t)stream);
  return e == cudaSuccess ? GTS_OK : gts::cuda_fail(e, "attention: launch");
}
