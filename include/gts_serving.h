/*
 * gts_serving.h -- C ABI of libgts's operators of a decode step: rotary
 * positions, appending keys and values to a paged cache, and attention of a
 * batch over a prefix that all its sequences share and each sequence's own
 * tokens.
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

#ifdef __cplusplus
}
#endif
#endif
