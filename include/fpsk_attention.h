/*
 * fpsk_attention.h - the attention operators that follow a verified projection.
 *
 * The QKV projection of a transformer layer is a GEMM whose FP32 accumulator C is delivered un-narrowed so that
 * fpsk_probe can check it.  What a fused epilogue would have done to C before narrowing it is done here, after the
 * check: the norms and the position rotation of queries and keys, the writes of keys and values to a paged cache,
 * and the attention of the new tokens over that cache.
 *
 * The conventions of fpsk.h hold: the caller owns every buffer, nothing is allocated, every call is asynchronous on
 * `stream` without a host synchronisation, errors are return codes, nothing throws.  Strides are in ELEMENTS; the
 * head_dim channels of one head are contiguous.  What only the device can see (a position beyond the tables, a page
 * number outside the cache, a device-side wait that gave up) is reported through d_status: a device int32 or NULL, to
 * which the kernels only ever write an fpsk_status other than FPSK_OK (zero it before, read it when convenient).
 */
#ifndef FPSK_ATTENTION_H
#define FPSK_ATTENTION_H

#include "fpsk.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { FPSK_ELEM_FP16 = 0, FPSK_ELEM_BF16 = 1, FPSK_ELEM_FP32 = 2 } fpsk_elem;

#define FPSK_MAX_HEAD_DIM 256

/* Position rotation.  Channels are paired, (i, i + rot_dim / 2) or, interleaved, (2 i, 2 i + 1), for i < rot_dim / 2; a
 * pair (a, b) of a token at position p becomes (a c - b s, b c + a s) with c = cos[p][i], s = sin[p][i].  Channels from
 * rot_dim on are not rotated; rot_dim = 0 rotates nothing (the tables may then be NULL).  rot_dim % 8 == 0. */
typedef struct {
    const float *cos, *sin;      /* device, n_pos x rot_dim / 2, contiguous                            */
    const int32_t *positions;    /* device, one per token; NULL: see the entry point                    */
    int64_t n_pos;
    int32_t rot_dim;
    int32_t interleaved;
} fpsk_rotary;

/* The heads of one kind (queries, keys or values): element (token t, head h, channel c) at
 * t * token_stride + h * head_stride + c. */
typedef struct {
    const void *in;              /* device, in_type                                                    */
    void *out;                   /* device, out_type                                                   */
    const void *weight;          /* device, head_dim values of weight_type; NULL: this kind is not normed */
    int64_t in_token_stride, in_head_stride, out_token_stride, out_head_stride;
    int32_t n_heads;
    int32_t weight_type;         /* fpsk_elem                                                          */
} fpsk_heads;

/* Norm and rotation of queries and keys in one pass: z = x rsqrt(mean(x^2) + eps) w over the channels of a head (where
 * a weight is given), rotated by the token's position, rounded once to out_type.  Sums in FP32.
 *   q, k       either may be NULL or have n_heads = 0
 *   rot        rot->positions is required when rot_dim > 0.  A position outside [0, n_pos) makes the token's rows NaN
 *              and sets *d_status to FPSK_ERR_PARAM.
 * head_dim: a multiple of 8 up to FPSK_MAX_HEAD_DIM.  n_tokens = 0 does nothing.  Loads and stores are 4 elements wide
 * where pointers and strides allow it, otherwise single elements, with the same arithmetic. */
fpsk_status fpsk_qk_norm_rope(const fpsk_heads *q, const fpsk_heads *k, int64_t n_tokens, int32_t head_dim,
                              fpsk_elem in_type, fpsk_elem out_type, const fpsk_rotary *rot, float eps,
                              int32_t *d_status, void *stream);

/* Gradients of one kind of heads. */
typedef struct {
    const void *in;              /* the forward pass's input, in_type                                  */
    const void *dout;            /* gradient of its output, grad_type                                  */
    void *din;                   /* receives the gradient of the input, grad_type                      */
    const void *weight;          /* as in the forward pass; NULL: not normed                           */
    float *dweight;              /* device, head_dim floats, overwritten; NULL when weight is NULL      */
    int64_t in_token_stride, in_head_stride, dout_token_stride, dout_head_stride, din_token_stride, din_head_stride;
    int32_t n_heads;
    int32_t weight_type;
} fpsk_heads_grad;

/* Backward pass of fpsk_qk_norm_rope.  With u = R^T dout, n = x r, r = rsqrt(mean(x^2) + eps) (recomputed from x):
 *   din = r (u w - n mean(u w n)),   dweight = sum over tokens and heads of u n
 * (without a weight: din = u).  FP32 sums in a fixed order: bit-identical from call to call on one device.
 * The workspace is zeroed once by fpsk_attention_workspace_init and serves one call at a time. */
size_t fpsk_norm_rope_workspace_bytes(int32_t head_dim);
fpsk_status fpsk_qk_norm_rope_backward(const fpsk_heads_grad *q, const fpsk_heads_grad *k, int64_t n_tokens,
                                       int32_t head_dim, fpsk_elem in_type, fpsk_elem grad_type,
                                       const fpsk_rotary *rot, float eps, void *workspace, size_t ws_bytes,
                                       int32_t *d_status, void *stream);

/* A paged cache of keys and values: element (page g, token s of the page, key head h, channel c) of K at
 * k + g k_page_stride + s k_token_stride + h k_head_stride + c (either order of token and head), V likewise. */
typedef struct {
    void *k, *v;                 /* device                                                             */
    int64_t k_page_stride, k_token_stride, k_head_stride;
    int64_t v_page_stride, v_token_stride, v_head_stride;
    int64_t n_pages;
    int32_t page_size, n_heads, head_dim;
    int32_t type;                /* FPSK_ELEM_FP16 or FPSK_ELEM_BF16                                   */
} fpsk_paged_cache;

/* The sequences of one step.  Sequence b has the new tokens cu_q[b] .. cu_q[b+1] - 1 of the packed token axis and
 * kv_len[b] keys, the new tokens' own ones last: token t sits at p = kv_len[b] - (cu_q[b+1] - t), in slot p % page_size
 * of page block_table[b][p / page_size].  New tokens beyond kv_len (p < 0) have no place: they are not written and
 * attend to nothing.  Lengths of zero are allowed.  Rows of the token axis behind cu_q[n_seqs] belong to no sequence. */
typedef struct {
    const int32_t *cu_q;         /* device, n_seqs + 1, ascending from 0                               */
    const int32_t *kv_len;       /* device, n_seqs                                                     */
    const int32_t *block_table;  /* device, n_seqs rows of max_pages page numbers                      */
    int64_t table_stride;
    int64_t n_tokens;            /* rows of the packed token axis                                      */
    int32_t n_seqs, max_pages;
} fpsk_paged_batch;

/* Writes the new tokens' keys (normed where k->weight is given, rotated) and values to their pages, and, where q is
 * given, the queries, normed and rotated, to q->out: one launch.  k->out and the weights and outputs of v are ignored.
 * in_type: any; what is written has the cache's type, rounded once.  rot->positions = NULL rotates by p.
 * A page number outside [0, n_pages) is skipped and sets *d_status to FPSK_ERR_PARAM, as do positions outside the
 * tables (the rows become NaN).  Queries of tokens without a place, rotated by p, become zero. */
fpsk_status fpsk_paged_append(const fpsk_paged_cache *cache, const fpsk_paged_batch *batch, const fpsk_heads *k,
                              const fpsk_heads *v, const fpsk_heads *q, fpsk_elem in_type, const fpsk_rotary *rot,
                              float eps, int32_t *d_status, void *stream);

/* Attention of the new tokens over their sequences' pages:
 *   out_t = sum_j softmax_j(scale q_t . k_j) v_j over the keys j that token t (at position p) may see:
 *   j < kv_len[b];  j <= p when causal;  j >= p - window when window >= 0.
 * A token that may see nothing gets zeros and lse = -inf.  A page number outside [0, n_pages), or a key behind the last column of the
 * table, reads as zeros (a score of 0) and sets *d_status to FPSK_ERR_PARAM.  Query head h reads key head h / (n_heads_q / cache->n_heads).
 * Keys that no token of a sequence may see are never used, whatever the memory holds (table entries behind the last page,
 * NaN).  A NaN or infinite value among keys that some tokens see and others do not can reach the others.  Rows that belong to no
 * sequence are left alone.  Scores, softmax and sums are FP32; on the tensor cores each weight exp(s - m) is rounded to
 * cache->type, half a unit at most, before it multiplies its value (the sum that divides is not rounded).
 *   q, out     device, cache->type, (token, head) strides; lse: device FP32 n_tokens x n_heads_q, or NULL
 *   max_q_len, max_kv_len   upper bounds of the lengths, known to the host: they choose tiles and grid (a bound that is
 *              too small costs time only)
 *   workspace  fpsk_paged_attention_workspace_bytes() for the current device, 256-byte aligned, initialised once by
 *              fpsk_attention_workspace_init (and again after a FPSK_ERR_TIMEOUT); one call at a time
 * head_dim: a multiple of 8 up to FPSK_MAX_HEAD_DIM.  Heads of up to 128 channels, up to 128 query heads to a key head and 16-byte
 * aligned rows run on the tensor cores (fastest in pages of a multiple of 8 tokens); the rest on a plain kernel. */
typedef struct {
    const void *q;
    void *out;
    float *lse;
    int64_t q_token_stride, q_head_stride, out_token_stride, out_head_stride;
    int32_t n_heads;
    int32_t causal;
    int32_t window;              /* -1: none                                                           */
    int32_t max_q_len, max_kv_len;
    float scale;                 /* 0: 1 / sqrt(head_dim)                                              */
} fpsk_attention;

size_t fpsk_paged_attention_workspace_bytes(void);
fpsk_status fpsk_paged_attention(const fpsk_paged_cache *cache, const fpsk_paged_batch *batch, const fpsk_attention *a,
                                 void *workspace, size_t ws_bytes, int32_t *d_status, void *stream);

/* Zeroes the synchronisation words of a workspace (async on `stream`): once after allocating it. */
fpsk_status fpsk_attention_workspace_init(void *workspace, size_t ws_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* FPSK_ATTENTION_H */
