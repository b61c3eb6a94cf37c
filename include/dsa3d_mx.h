/*
 * A paged cache of keys and values held in 8 or 4 bits, C ABI (gfx950 HIP kernels): the write of
 * new tokens, their reading back, and the newest tokens' attention over the pages.
 *
 * Requests, new tokens, positions, masks, biases and the page table are those of the paged cache
 * of dsa3d_seq.h; what differs is how a token's key and value are held.  The 32 channels 32 i ..
 * 32 i + 31 of one token and key head are a block: 32 elements and a power of two that they share.
 *
 *   elements  8 bits: 4 exponent and 3 mantissa bits, bias 7, largest 448, 0x7f and 0xff NaN
 *             4 bits: 2 exponent and 1 mantissa bit, bias 1, largest 6; channel 2 i in the lower
 *             half of a byte, channel 2 i + 1 in the upper
 *   scale     a byte s: 2^(s - 127), or NaN for 255
 *
 * The write takes the least power of two of 2^-117 and more (s >= 10) that holds the block's
 * largest magnitude without saturating, and the nearest element of each channel's quotient (of two
 * as near the one with an even code), so that a channel is off by at most 2^-4 of itself in 8 bits
 * and 2^-2 in 4, or half the least element, 2^-10 and 2^-2 of the power.  A block that holds a NaN
 * or an infinity, or a value whose rounding would reach 2^128, gets s = 255 and elements 0, and
 * reads as NaN throughout.  A value read back has at most 4 significant bits and no exponent below
 * -126: bf16 and float32 hold it exactly (where s < 10, which the write does not leave, values
 * below 2^-126 may read as 0).
 */
#ifndef DSA3D_MX_H
#define DSA3D_MX_H

#include <stddef.h>
#include <stdint.h>

#include "dsa3d_seq.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Token j of request b lies in row j % page_size of page pages[b][j / page_size] of
 *   k, v                [num_pages][kv_heads][page_size][head_dim * bits / 8]
 *   k_scales, v_scales  [num_pages][kv_heads][page_size][head_dim / 32]
 * (one head's rows of a page lie together, as they are read; 16-byte aligned). */
typedef struct {
  uint8_t *k, *v, *k_scales, *v_scales;
  int32_t bits;                        /* 8 or 4                                              */
} dsa3d_mx_cache;

/* Descriptors and errors are those of the calls of dsa3d_seq.h without _mx, the dtype being that of
 * k, v, q and out; besides, a NULL cache -> DSA3D_ERR_NULL_POINTER and other bits ->
 * DSA3D_ERR_UNSUPPORTED. */

/* Writes rows k, v [total_q][kv_heads][head_dim] (k_stride, v_stride apart) to the new tokens'
 * places, rounded as above.  Nothing else in the pages is touched; new tokens without a place are
 * dropped.  Of two tokens with the same place, each 4 bytes of elements and each scale are from
 * either. */
dsa3d_status dsa3d_paged_append_mx(const dsa3d_paged_desc* desc, const void* k, const void* v,
                                   const int32_t* cu_q, const int32_t* kv_lens,
                                   const int32_t* pages, const dsa3d_mx_cache* cache,
                                   hipStream_t stream);

/* Reads the newest tokens back as rows k, v [total_q][kv_heads][head_dim] (k_stride, v_stride
 * apart; the one's rows must not lie between the other's, or DSA3D_ERR_ALIAS): cu_q[b + 1] - cu_q[b]
 * tokens of request b, the last of its kv_lens[b].  Tokens without a place and rows behind the last
 * request read as 0.  max_kv is not used. */
dsa3d_status dsa3d_paged_read_mx(const dsa3d_paged_desc* desc, const dsa3d_mx_cache* cache,
                                 const int32_t* pages, const int32_t* kv_lens,
                                 const int32_t* cu_q, void* k, void* v, hipStream_t stream);

/* Workspace bytes dsa3d_paged_forward_mx needs; may be 0.  With up to 64 requests it does not grow
 * with the longest cache that the descriptor allows: 16 bytes per row and head of out, and float32
 * results of the parts that long caches are read in, some hundreds of 16 to 128 rows each. */
size_t dsa3d_paged_forward_mx_workspace_size(const dsa3d_paged_desc* desc, int32_t bits);

/* Attention of the new tokens over the pages: out [total_q][heads][head_dim] and, when not NULL,
 * lse.  Keys and values enter the products as the bf16 numbers that they are; float32 queries and
 * alpha are made of bf16 parts, to 2^-24 of a product.  With bf16 queries alpha is made of two, to
 * 2^-17 of itself. */
dsa3d_status dsa3d_paged_forward_mx(const dsa3d_paged_desc* desc, const void* q,
                                    const dsa3d_mx_cache* cache, const int32_t* pages,
                                    const int32_t* kv_lens, const int32_t* cu_q,
                                    const float* bias_table, const int32_t* bias_map, void* out,
                                    float* lse, void* workspace, size_t workspace_bytes,
                                    hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* DSA3D_MX_H */
