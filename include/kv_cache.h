/*
 * kv_cache.h -- C ABI of the quantized paged cache: keys and values (or any per-token, per-head vectors) stored as int8 or
 * MXFP4 when they are written and read back as bf16. Conventions on pointers, streams and status codes as in
 * w8a8_linear.h. The calls allocate nothing, only enqueue, and can be captured in a CUDA graph.
 *
 * A cache is num_pages pages of page_size tokens; a token's place is its slot = page * page_size + offset. Per side:
 *     KV_CACHE_INT8   codes int8  [slots, heads, dim]      scales fp32  [slots, heads]
 *                     s = amax > 0 ? amax / 127 : 1;  q = clamp(rne(x / s), -127, 127);  value = bf16(q * s)
 *                     (fp32 division, quotient and product, each rounded once: the arithmetic of the int8 linear)
 *     KV_CACHE_MXFP4  codes uint8 [slots, heads, dim / 2]  scales uint8 [slots, heads, ceil(dim / 32)]
 *                     the MXFP4 format of mxfp4_linear.h in blocks of 32 along dim (the last may be shorter)
 * A head vector (int8) or block (MXFP4) that holds an Inf or a NaN gets a NaN scale and codes 0 and reads back as NaN.
 * dim % 8 == 0, dim <= KV_CACHE_MAX_DIM, heads * dim <= KV_CACHE_MAX_WIDTH. Codes, inputs and outputs 16-byte aligned; token and head strides in elements,
 * multiples of 8 (inputs may be slices of a fused projection); a head's elements are contiguous. A NULL v (write) or
 * v_out (read) leaves the value side out, for caches that keep one vector a head.
 */
#ifndef KV_CACHE_H_
#define KV_CACHE_H_

#include "w8a8_linear.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { KV_CACHE_INT8 = 0, KV_CACHE_MXFP4 = 1 };
enum { KV_CACHE_ZERO_REST = 0x100 }; /* or'd into the fmt of a read */
#define KV_CACHE_MAX_DIM 256
#define KV_CACHE_MAX_WIDTH 65536 /* heads * dim */

/*
 * Quantizes `tokens` tokens into their slots. slots: int64 [tokens], device; one outside [0, num_slots) is skipped (-1 for
 * padding tokens). Slots of one call must be distinct. No tokens and a cache of no slots are valid calls; their pointers may be NULL.
 */
int kv_cache_write(int fmt, const void* k, int64_t k_token_stride, int64_t k_head_stride, const void* v, int64_t v_token_stride,
                   int64_t v_head_stride, const int64_t* slots, int64_t tokens, int64_t heads, int64_t dim, void* k_codes, void* k_scales,
                   void* v_codes, void* v_scales, int64_t num_slots, void* stream);

/*
 * Reads `seqs` sequences back, one after another: output token t belongs to sequence b with cu_seqlens[b] <= t <
 * cu_seqlens[b + 1] and is the sequence's token p = t - cu_seqlens[b] + (starts ? starts[b] : 0), kept in page
 * table[b * table_stride + p / page_size].
 *   table       int32 [seqs, max_pages]; a page outside [0, num_pages), or a token past max_pages, reads as zeros
 *   cu_seqlens  int32 [seqs + 1], not decreasing; empty sequences are fine
 *   starts      int32 [seqs] or NULL: the first token to read of each sequence (a window's)
 *   total       rows of the outputs (<= 2^31 - 1); rows that belong to no sequence (before cu_seqlens[0], from cu_seqlens[seqs]
 *               on) are left as they are, or written as zeros with KV_CACHE_ZERO_REST
 *   k_out, v_out  bf16 [total, heads, dim] with their strides
 * No rows, no sequences and a cache of no pages are valid calls; pointers to what has no elements may be NULL.
 */
int kv_cache_read(int fmt, const void* k_codes, const void* k_scales, const void* v_codes, const void* v_scales, int64_t num_pages, int64_t page_size,
                  int64_t heads, int64_t dim, const int32_t* table, int64_t table_stride, int64_t max_pages, const int32_t* cu_seqlens,
                  const int32_t* starts, int64_t seqs, int64_t total, void* k_out, int64_t k_token_stride, int64_t k_head_stride, void* v_out,
                  int64_t v_token_stride, int64_t v_head_stride, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* KV_CACHE_H_ */
