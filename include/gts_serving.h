/*
 * gts_serving.h -- C ABI of libgts's operators of a decode step: rotary
 * positions, appending keys and values to a paged cache, and attention of a
 * batch over a prefix that all its sequences share and each sequence's own
 * tokens; and of prompts: attention of packed sequences with its gradient,
 * attention of chunks of new tokens over a paged cache, and copies of pages.
 *
 * They are the work whose tile graphs the simulator takes (attention and the
 * kernels around it), as kernels that run on the machine itself, so that a
 * graph's cycles can be set beside a measured time.
 *
 * Conventions are those of gts.h: the caller owns every buffer and the stream,
 * the library allocates no device memory, calls enqueue work on `stream` and
 * return without waiting, host-side errors come back as a status with a
 * message in gts_last_error(), and no call throws, traps or spins without
 * bound.  All pointers are device pointers on the current device.  Strides are
 * in elements; the innermost dimension of every tensor is contiguous.  Outputs
 * may not overlap inputs, except that a rotation may write each value over the
 * one it came from (same pointer and strides).
 *
 * Values on the device that the host cannot check (slots, page numbers,
 * lengths) are checked by the kernels: an index outside its range is never
 * followed, and GTS_ERR_INVALID_PARAMS is stored to *d_status where that is
 * given; what it would have contributed to a result is then unspecified.
 * *d_status is never cleared by the library.  Waits inside the attention
 * kernels end after two seconds: GTS_ERR_STEP_LIMIT is then stored to *d_status
 * where that is given, and rows of out and lse that miss a part are NaN.
 */
#ifndef GTS_SERVING_H
#define GTS_SERVING_H

#include "gts.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types. */
#define GTS_BF16 0
#define GTS_F16  1
#define GTS_F32  2

/* How a head's first rot_dim values form the rot_dim / 2 pairs that are turned. */
#define GTS_ROTARY_HALF        0  /* pair i: values i and i + rot_dim / 2 */
#define GTS_ROTARY_INTERLEAVED 1  /* pair i: values 2 i and 2 i + 1 */

/* A [tokens][heads][head_dim] tensor. */
typedef struct {
  void *data;
  int64_t token_stride, head_stride;
} gts_heads;

/* A paged cache: keys and values, each [pages][page_size][kv_heads][head_dim]. */
typedef struct {
  void *k, *v;
  int64_t k_page_stride, k_token_stride, k_head_stride;
  int64_t v_page_stride, v_token_stride, v_head_stride;
  uint32_t n_pages, page_size, kv_heads, head_dim;
  int32_t dtype; /* GTS_BF16, GTS_F16 or GTS_F32 */
} gts_cache;

/* The rotation of a position p: pair i turns by the angle a = 2 pi * (p * units[i] mod 2^64) / 2^64, and both values
 * are multiplied by factor:  (x, y) -> factor * (x cos a - y sin a, y cos a + x sin a).
 * units[i] is the pair's turns a position times 2^64, rounded, so that the phase of any position is exact. */
typedef struct {
  const uint64_t *units; /* [rot_dim / 2] */
  uint32_t rot_dim;      /* even, 0 <= rot_dim <= head_dim; the values after it are copied */
  int32_t layout;        /* GTS_ROTARY_* */
  float factor;
  uint32_t transposed;   /* 1: by -a, the transposed map: what a gradient of the rotated values goes through */
} gts_rotary;

/* q_out = rotated q, k_out = rotated k; one angle per token from positions[tokens].
 * k.data may be NULL (then kv_heads is 0 and k is skipped). */
typedef struct {
  uint32_t n_tokens, q_heads, kv_heads, head_dim;
  int32_t dtype; /* GTS_BF16, GTS_F16 or GTS_F32 */
  const int32_t *positions;
  gts_rotary rotary;
  gts_heads q, k, q_out, k_out;
} gts_rope_desc;
gts_status gts_rope(const gts_rope_desc *desc, void *stream);

/* Rotated k and plain v of every token go to the cache, rotated q to q_out.  Token t's place is slots[t] =
 * page * page_size + index within the page; a negative slot writes nothing to the cache (a padding row; its q is
 * rotated all the same).  Two tokens of a call may not have the same slot. */
typedef struct {
  uint32_t n_tokens, q_heads;
  const int32_t *positions;
  const int64_t *slots;
  gts_rotary rotary;       /* transposed must be 0 */
  gts_heads q, k, v, q_out; /* k, v: kv_heads and head_dim of the cache */
  gts_cache cache;
  int32_t *d_status;       /* optional */
} gts_append_desc;
gts_status gts_append_kv(const gts_append_desc *desc, void *stream);

/* Attention of n_seqs x n_new queries.  Query i of sequence b sees the first prefix_len tokens of the pages in
 * prefix_pages, and of its own pages (page_table row b) the tokens j with j < lens[b] - (n_new - 1 - i): lens[b] counts
 * the sequence's own tokens with the n_new newest, which are the queries' own (a value below 0 counts as none).  With
 * s_j = scale * q . k_j over the keys it sees and m = max s_j:
 *   out = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m),   lse = m + log sum_j exp(s_j - m);
 * a query that sees no key gets out = 0 and lse = -infinity.  Query head h uses key head h / (q_heads / kv_heads).
 * Cache values that no query sees (the rest of a page) may be anything, NaN included.
 * Types: GTS_BF16 or GTS_F16; head_dim 64, 128 or 256; q_heads a multiple of kv_heads.  Products are summed in 32 bits.
 */
typedef struct {
  uint32_t n_seqs, n_new, q_heads;
  float scale;
  const void *q; /* [n_seqs][n_new][q_heads][head_dim] */
  int64_t q_seq_stride, q_token_stride, q_head_stride;
  void *out;     /* as q */
  int64_t out_seq_stride, out_token_stride, out_head_stride;
  float *lse;    /* [n_seqs][n_new][q_heads], contiguous; may be NULL */
  gts_cache cache;
  const int32_t *prefix_pages; /* [ceil(prefix_len / page_size)] */
  uint32_t prefix_len;
  const int32_t *page_table;   /* [n_seqs][max_pages] */
  uint32_t max_pages;
  const int32_t *lens;         /* [n_seqs] */
  void *workspace;             /* gts_attention_workspace_bytes, 16-byte aligned; contents need not be kept */
  size_t workspace_bytes;
  int32_t *d_status;           /* optional */
} gts_attention_desc;
gts_status gts_prefix_attention(const gts_attention_desc *desc, void *stream);

/* Bytes of workspace gts_prefix_attention wants for the shape in desc (its pointers are not looked at); 0 where the
 * shape is refused. */
size_t gts_attention_workspace_bytes(const gts_attention_desc *desc);

/* Attention of packed sequences over themselves.  Sequence b's tokens are the rows starts[b] .. starts[b + 1] - 1 of q, k, v and
 * out; its query i sees its keys j <= i (causal) or all of them.  With s_j = scale * q_i . k_j over the keys seen and m = max s_j:
 *   out = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m),   lse = m + log sum_j exp(s_j - m).
 * Query head h uses key head h / (q_heads / kv_heads).  Rows of no sequence (before starts[0], from starts[n_seqs] on) are left as
 * they are, or get out = 0 (zero_rest bit 0) and lse = -infinity (bit 1); what they hold in q, k and v is not looked at.  starts
 * has to rise from 0 or more to n_tokens at most: other values are clamped to that (d_status, see above).  A row whose scores are all
 * -infinity counts as one that sees no key: out = 0, lse = -infinity; one with a score of +infinity or NaN is NaN.  Results may not
 * overlap what the call reads.
 * Types: GTS_BF16 or GTS_F16; head_dim 64 or 128; q_heads a multiple of kv_heads, at most 128 times it; scale positive.  Products
 * are summed in 32 bits. */
typedef struct {
  uint32_t n_seqs, n_tokens, q_heads, kv_heads, head_dim;
  int32_t dtype;
  uint32_t causal, zero_rest;   /* 0 or 1; bits */
  float scale;
  const int32_t *starts;        /* [n_seqs + 1] */
  gts_heads q, k, v, out;
  gts_heads low;                /* as out; data may be NULL: what rounding took from out, for the gradients */
  float *lse;                   /* [n_tokens][q_heads], contiguous; may be NULL */
  void *workspace;              /* gts_prompt_workspace_bytes, 16-byte aligned; contents need not be kept */
  size_t workspace_bytes;
  int32_t *d_status;            /* optional */
} gts_prompt_desc;
gts_status gts_prompt_attention(const gts_prompt_desc *desc, void *stream);

/* Bytes of workspace for the shape in desc (pointers and strides are not looked at); 0 where the shape is refused. */
size_t gts_prompt_workspace_bytes(const gts_prompt_desc *desc);

/* The gradients of gts_prompt_attention: forward is its desc, with out, lse and, where given, low as it left them (they are read;
 * its workspace is this call's).  Without low, e_i below has the rounding of out in it, of all its errors the one that adds up.
 * With p_ij = exp(s_ij - lse_i), e_i = sum_d dout_id (out_id + low_id) - dlse_i and ds_ij = p_ij (dout_i . v_j - e_i):
 *   dv_j = sum_i p_ij dout_i,   dq_i = scale sum_j ds_ij k_j,   dk_j = scale sum_i ds_ij q_i,
 * those of a key head summed over its query heads.  Rows of no sequence are left as they are, or get 0: dq, dk, dv with
 * bits 0, 1, 2 of forward.zero_rest.
 * Every sum has one order: results repeat bit for bit.  GTS_F16 holds ds to 2^-39 of 2 max |dout_i| max |v_j| + max |dlse_i| (norms of
 * rows, over the call).  Results may not overlap what the call reads. */
typedef struct {
  gts_prompt_desc forward;
  gts_heads dout;
  const float *dlse;            /* as lse; may be NULL: zero */
  gts_heads dq, dk, dv;
} gts_prompt_grad_desc;
gts_status gts_prompt_attention_grad(const gts_prompt_grad_desc *desc, void *stream);

/* Bytes of workspace; addresses and strides of q, k, v and dout count: those off the 16-byte grid, or with heads further apart than
 * tokens, are laid side by side there. */
size_t gts_prompt_grad_workspace_bytes(const gts_prompt_grad_desc *desc);

/* Attention of chunks of new tokens over a paged cache that holds them already.  Sequence b's queries are the rows starts[b] ..
 * starts[b + 1] - 1 of q, its keys the first lens[b] tokens of its pages (page_table row b; none where lens[b] is negative); the last query sees all of them,
 * and query i those j < lens[b] - (n - 1 - i), n its sequence's queries.  A query that sees no key gets out = 0 and lse =
 * -infinity.  Otherwise as gts_prompt_attention; cache values that no query sees may be anything, NaN included. */
typedef struct {
  uint32_t n_seqs, n_tokens, q_heads, zero_rest;
  float scale;
  const int32_t *starts;        /* [n_seqs + 1] */
  gts_heads q, out;
  float *lse;                   /* [n_tokens][q_heads], contiguous; may be NULL */
  gts_cache cache;
  const int32_t *page_table;    /* [n_seqs][max_pages] */
  uint32_t max_pages;
  const int32_t *lens;          /* [n_seqs] */
  void *workspace;
  size_t workspace_bytes;
  int32_t *d_status;
} gts_chunk_desc;
gts_status gts_chunk_attention(const gts_chunk_desc *desc, void *stream);
size_t gts_chunk_workspace_bytes(const gts_chunk_desc *desc);

/* The first tokens[i] tokens (NULL: all) of page src[i] of one cache, keys and values, go to page dst[i] of another one, or of the
 * same.  The caches have the same page_size, kv_heads, head_dim and dtype, and strides of their own.  A negative src or dst
 * copies nothing, nor does a page onto itself; tokens is clamped to 0 .. page_size.  A page may be copied to several others, but
 * what a page holds that is written twice, or read and written, in one call is unspecified. */
typedef struct {
  uint32_t n_copies;
  const int32_t *src, *dst;     /* [n_copies] */
  const int32_t *tokens;        /* [n_copies] or NULL */
  gts_cache cache, into;
  int32_t *d_status;            /* optional */
} gts_copy_pages_desc;
gts_status gts_copy_pages(const gts_copy_pages_desc *desc, void *stream);

#ifdef __cplusplus
}
#endif
#endif
