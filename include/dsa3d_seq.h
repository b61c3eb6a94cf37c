/*
 * Attention of packed token sequences, C ABI (gfx950 HIP kernels, MFMA): whole prompts forward
 * and backward, with an optional learned relative position bias, and the newest tokens of each
 * request over keys and values kept in pages.
 *
 * Video tokens stand on a grid (dsa3d.h, dsa3d_win.h); the prompts that condition them are
 * sequences of different lengths.  The sequences of a batch lie one behind the other: sequence b
 * has the rows cu[b] .. cu[b + 1] - 1 of a packed tensor, cu[0] = 0.  For sequence b with n
 * queries and m keys, query i stands at position p = m - n + i among the keys (the newest query
 * at the newest key), and head h reads the keys of head h / (heads / kv_heads):
 *
 *   t_ij = scale <q_i, k_j> + table[bucket(j - p)][h],   visible: every j, or j <= p if causal
 *   alpha = softmax over the visible keys,  out = sum alpha v,  lse = logsumexp t
 *
 * A query that sees no key gets out = 0 and lse = -inf, and takes part in no gradient.  Rows
 * behind the last sequence are treated as such queries (and such keys get zero gradients), so
 * every element of every output is written.
 *
 * The bias (rel_buckets > 0): bucket(d) = map[clamp(d, rel_min, rel_min + rel_span - 1) -
 * rel_min], an int32 device array of rel_span entries; table is float32 [rel_buckets][heads].
 * An entry outside [0, rel_buckets) adds no bias and takes no gradient.  A value of -1e30 or
 * less (-inf and the lowest float are) hides the keys at its distances, as a mask does.
 * dsa3d_relative_buckets fills the usual map.
 *
 * Conventions are those of dsa3d.h (plain device pointers, work enqueued on `stream`, host
 * validation first, no allocation, no synchronisation).  float32 and bf16 storage; logits,
 * softmax statistics and sums are float32.  With bf16, alpha and dS enter their second products
 * rounded to bf16 (half a unit in the last place each, as the output's own rounding), unless
 * out_res is asked for.  float32 products are made of bf16 parts to 2^-24 of a product, and an
 * infinity (or 3.39e38 and more) in a float32 tensor becomes NaN.  What is hidden has weight 0,
 * and 0 times what is not finite is NaN: a NaN or an infinity among the keys or values of a
 * sequence, in the backward also among its queries or upstream gradients (those of a query that
 * sees no key among them), can make NaN of rows of that sequence that it is hidden from, but never
 * of another sequence's, and what lies behind a sequence's end is never used.
 *
 * Values in device memory cannot be checked on the host.  cu must not decrease; entries outside
 * [0, rows] are clamped to it, so that a wrong one gives wrong results but no access outside the
 * tensors.
 *
 * Layouts (row-major; 16-byte aligned, lse and the bias arrays 4-byte aligned):
 *   q            [total_q] rows, q_stride elements apart, of [heads][head_dim]
 *   k, v         [total_k] rows, k_stride / v_stride apart, of [kv_heads][head_dim]
 *   out, out_res, dout, dq   [total_q][heads][head_dim]
 *   dk, dv       [total_k][kv_heads][head_dim]
 *   lse          [total_q][heads]   float32
 */
#ifndef DSA3D_SEQ_H
#define DSA3D_SEQ_H

#include <stddef.h>
#include <stdint.h>

#include "dsa3d.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Most distances a bias tells apart (rel_span), and most buckets. */
#define DSA3D_SEQ_MAX_SPAN 2048
#define DSA3D_SEQ_MAX_BUCKETS 256

/* Index range: total_q * heads and total_k * kv_heads below 2^31, batch below 2^24, and the
 * workgroups of a launch, heads * (total_q / 128 + batch + 1) of queries and kv_heads *
 * (total_k / 128 + batch + 1) of keys, at most 2^31 - 2^22 (up to 16 times as many of keys where
 * kv_heads * total_k is below 2^17). */
typedef struct {
  int32_t batch;                       /* sequences, at least 1                               */
  int32_t total_q, total_k;            /* rows of q and of k, v (0 is allowed)                */
  int32_t heads, kv_heads, head_dim;   /* heads a multiple of kv_heads; head_dim 64 or 128    */
  int32_t causal;                      /* 0: every key of the sequence, 1: keys j <= p        */
  int32_t rel_min, rel_span;           /* the distances the bias tells apart                  */
  int32_t rel_buckets;                 /* rows of the bias table, 0: no bias                  */
  float scale;                         /* logit scale > 0; 0 selects 1/sqrt(head_dim)         */
  dsa3d_dtype dtype;                   /* type of q, k, v, out, dout and the gradients        */
  int64_t q_stride, k_stride, v_stride;/* elements from one token's row to the next's, at least
                                          a row, a multiple of 16 bytes and below 16 MiB; 0: a
                                          row                                                 */
} dsa3d_seq_desc;

/* out and, when not NULL, lse and out_res.  out_res (bf16 only, else it must be NULL) is the
 * rounding residual bf16(O - out), with alpha carried to 16 significant bits in its product:
 * out + out_res then has O to about 16 bits, which the backward needs for a bias gradient
 * that is off by no more than some 2^-17 of its size.  cu_k NULL: the keys' sequences are the
 * queries' (total_k = total_q).
 * bias_table and bias_map may be NULL when rel_buckets is 0.
 * Errors: NULL desc, cu_q, or a tensor with rows -> DSA3D_ERR_NULL_POINTER; a size outside the
 * ranges above, heads not a multiple of kv_heads, total_k != total_q without cu_k, a negative or
 * non-finite scale, a stride below a row or not a multiple of 16 bytes -> DSA3D_ERR_INVALID_SHAPE;
 * a dtype or head_dim not built in, rel_span above DSA3D_SEQ_MAX_SPAN or rel_buckets above
 * DSA3D_SEQ_MAX_BUCKETS -> DSA3D_ERR_UNSUPPORTED; a broken alignment -> DSA3D_ERR_MISALIGNED; an
 * output overlapping an input or another output -> DSA3D_ERR_ALIAS. */
dsa3d_status dsa3d_seq_forward(const dsa3d_seq_desc* desc, const void* q, const void* k,
                               const void* v, const int32_t* cu_q, const int32_t* cu_k,
                               const float* bias_table, const int32_t* bias_map, void* out,
                               void* out_res, float* lse, hipStream_t stream);

/* Workspace bytes dsa3d_seq_backward needs (0 for a descriptor it would reject): 8 per query
 * row and head, with a bias 4 rel_buckets per head and tile of 128 queries (total_q / 128 +
 * batch + 1 tiles), and where there are few keys float32 parts of dk and dv, up to 16 of them. */
size_t dsa3d_seq_backward_workspace_size(const dsa3d_seq_desc* desc);

/* Backward for upstream gradient dout, alpha recomputed from lse:
 *   dP = <dout, v_j>,  Delta = <dout, O>,  dS = alpha (dP - Delta)
 *   dq = scale sum_j dS k_j,   dk_j = scale sum dS q,   dv_j = sum alpha dout
 *   d_table[c][h] = sum of dS over the pairs whose distance has bucket c
 * The sums of dk and dv run over the queries of every head that reads the key's head.  O is out
 * + out_res, or out alone when out_res is NULL.  lse, out and out_res may be those of more keys
 * than the call has (a sequence's keys in several calls, their statistics joined): the gradients
 * are then sums over the call's keys.  dq, dk, dv are in the descriptor's dtype, the table's
 * gradient is float32 and may be NULL (then it is not formed); in it a query's sum of dS that is
 * no larger than the rounding of its Delta (2^-16 of the root of <dout^2, O^2>, with out_res or in
 * float32) counts as 0.  Every element is written once and sums have a fixed order: repeated calls
 * give the same bits.  The workspace (256-byte aligned) must not overlap any argument.
 * Errors as for the forward, plus: lse, dout or a gradient NULL -> DSA3D_ERR_NULL_POINTER; a
 * workspace missing or too small -> DSA3D_ERR_WORKSPACE. */
dsa3d_status dsa3d_seq_backward(const dsa3d_seq_desc* desc, const void* q, const void* k,
                                const void* v, const int32_t* cu_q, const int32_t* cu_k,
                                const float* bias_table, const int32_t* bias_map, const void* out,
                                const void* out_res, const float* lse, const void* dout, void* dq,
                                void* dk, void* dv, float* d_table, void* workspace,
                                size_t workspace_bytes, hipStream_t stream);

/* The map (a HOST array) of the distances rel_min .. rel_min + rel_span - 1 for `buckets` buckets
 * up to max_distance: the distances behind the query, 0 .. max_distance, get buckets
 * 0 .. s - 1, s = buckets, or s = buckets / 2 when both directions are told apart, the distances
 * ahead of it then s .. 2 s - 1.  The first e = s / 2 distances have a bucket each; distance n >=
 * e has e + floor((s - e) log(n / e) / log(max_distance / e)), at most s - 1.  A distance on the
 * border of two buckets falls to the farther one.  Without `both`, distances ahead take bucket
 * 0 and rel_min .. 0 is told apart.  Writes rel_min and rel_span (max_distance + 1, or twice
 * max_distance plus 1); map may be NULL to ask for these alone.
 * Errors: a NULL rel_min or rel_span -> DSA3D_ERR_NULL_POINTER; s < 2, buckets odd with `both`,
 * or max_distance <= e -> DSA3D_ERR_INVALID_SHAPE; a span or a number of buckets above the
 * limits -> DSA3D_ERR_UNSUPPORTED. */
dsa3d_status dsa3d_relative_buckets(int32_t buckets, int32_t max_distance, int32_t both,
                                    int32_t* map, int32_t* rel_min, int32_t* rel_span);

/* ------------------------------------------------------------------------ a paged cache
 *
 * Token j of request b lies in row j % page_size of page pages[b][j / page_size] of two tensors
 * k_pages, v_pages [num_pages][page_size][kv_heads][head_dim]; pages is int32
 * [batch][max_pages], kv_lens int32 [batch] counts a request's tokens, the new ones included.
 * The new tokens of the requests are packed as above (cu_q): with n new and m held tokens, new
 * token i stands at position m - n + i.  A page number outside [0, num_pages) holds no tokens: it
 * is neither read nor written, and its tokens are hidden from every query. */
typedef struct {
  int32_t batch, total_q;              /* requests and new tokens of all of them; workgroups as
                                          above, kv_heads * (total_q * heads / kv_heads / 32 +
                                          batch + 1) of queries (times the parts)             */
  int32_t heads, kv_heads, head_dim;   /* as dsa3d_seq_desc (heads is not used by the append) */
  int32_t num_pages, page_size;        /* num_pages * page_size below 2^31                    */
  int32_t max_pages;                   /* columns of the page table                           */
  int32_t max_kv;                      /* no request holds more tokens than this; 0 selects
                                          max_pages * page_size.  Tokens from max_kv on are not
                                          attended to.  The smaller of the two is at most 2^30
                                          for dsa3d_paged_forward.                            */
  int32_t causal;
  int32_t rel_min, rel_span, rel_buckets;
  float scale;
  dsa3d_dtype dtype;
  int64_t q_stride;                    /* as above, for q                                     */
  int64_t k_stride, v_stride;          /* for the append's k, v                               */
} dsa3d_paged_desc;

/* Writes rows k, v [total_q][kv_heads][head_dim] (k_stride, v_stride apart) to the new tokens'
 * places in the pages.  Nothing else in the pages is touched; new tokens without a place (a
 * position below 0 or behind the page table, a page number outside the tensors, a row behind the
 * last request) are dropped.  Of two tokens with the same place, each 16 bytes are from either.
 * Errors as for dsa3d_seq_forward. */
dsa3d_status dsa3d_paged_append(const dsa3d_paged_desc* desc, const void* k, const void* v,
                                const int32_t* cu_q, const int32_t* kv_lens, const int32_t* pages,
                                void* k_pages, void* v_pages, hipStream_t stream);

/* Workspace bytes dsa3d_paged_forward needs; may be 0.  Long caches are read in parts by several
 * workgroups, whose float32 results and log-sum-exps are joined by a second kernel. */
size_t dsa3d_paged_forward_workspace_size(const dsa3d_paged_desc* desc);

/* Attention of the new tokens over the pages: out [total_q][heads][head_dim] and, when not NULL,
 * lse.  With a bias, (heads / kv_heads) * rel_span must not exceed DSA3D_PAGED_MAX_BIAS
 * (DSA3D_ERR_UNSUPPORTED).  Errors as for dsa3d_seq_forward, plus DSA3D_ERR_WORKSPACE. */
#define DSA3D_PAGED_MAX_BIAS 6144
dsa3d_status dsa3d_paged_forward(const dsa3d_paged_desc* desc, const void* q, const void* k_pages,
                                 const void* v_pages, const int32_t* pages,
                                 const int32_t* kv_lens, const int32_t* cu_q,
                                 const float* bias_table, const int32_t* bias_map, void* out,
                                 float* lse, void* workspace, size_t workspace_bytes,
                                 hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* DSA3D_SEQ_H */
