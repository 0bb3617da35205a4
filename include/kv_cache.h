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
#define KV_CACHE_MAX_AXES 8

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

/*
 * Appends new tokens: rotates queries and keys by their positions, quantizes keys and values into the cache's slots, in one launch.
 * Pairs of elements of a head turn by an angle that the token's position on the pair's axis gives (one axis for text; time, height and width
 * for images and video):
 *     p = positions[axis of pair i][token],  c = cos_sin[p][i],  s = cos_sin[p][rot / 2 + i]
 *     a' = a * c - b * s,  b' = b * c + a * s           fp32: two products and a sum, each rounded once
 * of the elements (a, b) = (2i, 2i + 1) if interleaved, else (i, i + rot / 2); elements from rot on stay as they are.
 *   q_out = bf16(q'), the cache gets k' (not rounded to bf16 in between) and v as kv_cache_write would store them.
 *   q, q_out    bf16 [tokens, q_heads, dim] with their strides; both NULL for none; q_out may be q itself (with its strides)
 *   cos_sin     fp32 [num_positions, rot] dense, 16-byte aligned, or NULL: nothing is rotated (positions and axes are not read)
 *   rot         a multiple of 8, at most dim
 *   positions   int64 [axes, tokens], rows position_stride apart; a position outside the table makes its pairs NaN
 *   axis_of     uint8 [rot / 2]: the axis of each pair, or NULL with one axis; one that is not below `axes` makes its pair NaN
 * Everything else as for kv_cache_write; a token whose slot is outside the cache still gets its queries.
 */
int kv_cache_append(int fmt, const void* q, int64_t q_token_stride, int64_t q_head_stride, int64_t q_heads, void* q_out, int64_t q_out_token_stride,
                    int64_t q_out_head_stride, const void* k, int64_t k_token_stride, int64_t k_head_stride, const void* v, int64_t v_token_stride,
                    int64_t v_head_stride, const float* cos_sin, int64_t num_positions, int64_t rot, int interleaved, const int64_t* positions,
                    int64_t position_stride, int64_t axes, const uint8_t* axis_of, const int64_t* slots, int64_t tokens, int64_t heads, int64_t dim,
                    void* k_codes, void* k_scales, void* v_codes, void* v_scales, int64_t num_slots, void* stream);

/*
 * The table that kv_cache_append reads: cos and sin of (first + p) * inv_freq[i], times `scale`, worked out in 64 bits and rounded once.
 *   inv_freq  fp64 [pairs], device;  cos_sin  fp32 [num_positions, 2 * pairs]
 */
int kv_cache_rope_table(const double* inv_freq, int64_t pairs, int64_t first, int64_t num_positions, double scale, float* cos_sin, void* stream);

/*
 * Attention of new tokens over the cache, on the codes: nothing is expanded in memory.
 *     o = sum_p softmax_p(scale * q . k_p) v_p             over the tokens p that the query sees; k, v: what the codes stand for, unrounded
 * Sequence b holds lens[b] tokens in its pages. The last n_b = cu_q[b + 1] - cu_q[b] of them are its new ones, appended before the call;
 * query i of them (row cu_q[b] + i of q) sees, of the tokens from starts[b] on, those that come before the new ones, and of the new ones
 *   tree == NULL  those up to and with itself (one token a sequence, or a chain)
 *   else          token j where bit j % 64 of tree[(cu_q[b] + i) * tree_words + j / 64] is set: a tree of drafted tokens, each of which sees its
 *                 ancestors (and itself, where its own bit is set); new tokens from 64 * tree_words on are not seen
 * starts[b] is one for all new tokens of a sequence, and hides those of them that come before it, too: a window that moves on with each of several new tokens is not one of its uses.
 * Query head h reads the keys and values of head h / (q_heads / heads). A query that sees nothing gets zeros and a logarithm of -inf. A token whose page
 * is outside the cache or past the table is not seen. NaN keys and values (their scale is NaN) reach the queries that see them, and no others.
 *   q, out      bf16 [total_q, q_heads, dim] with their strides; rows of no sequence as for kv_cache_read (KV_CACHE_ZERO_REST); out and lse overlap no input (a
 *               row of queries is read by several CTAs, at different times; out over q is refused, and so are two that reach into one another with different strides)
 *   lse         fp32 [total_q, q_heads]: log(sum_p exp(scale * q . k_p)), or NULL
 *   table       int32 [seqs, max_pages];  lens, starts int32 [seqs] (starts may be NULL: from the first);  cu_q int32 [seqs + 1], not decreasing
 *   tree        int64 [total_q, tree_words] or NULL
 *   workspace   device scratch of kv_cache_attention_workspace_bytes(), 256-byte aligned; its first kv_cache_attention_zeroed_bytes() bytes must be zero
 *               before the first call that uses it, and each call leaves them zero. One workspace, given with its whole size, serves calls with fewer
 *               sequences and rows too, in any order, if what the largest needs to be zero was; one that needs more counters than it has is refused. Two calls that may overlap on the device need distinct workspaces.
 *               A wait that runs out shows in its first word (int8_check_status) and in the sticky status.
 * The cache must have both sides, scales that are not negative and 4-byte aligned; num_pages * page_size <= 2^31 - 1, max_pages * page_size <= 2^31 - 4096; q_heads a
 * multiple of heads. Scores, softmax
 * and sums are fp32; for the product with the values, probability times the token's value scale (MXFP4: that of its largest block) is rounded to fp16, relative to the
 * row's own size; with many rows of queries (more than 32 a sequence and head on average, heads of at most 128 elements), it is the probability that is, and values are
 * rounded to fp16 relative to the sequence's largest scale. Repeated calls give the same bits. What lies far below its neighbours may count as zero: elements of a query 2^-38 below its largest, MXFP4 blocks
 * 2^-27 below the largest of their head and token, tokens whose probability is 2^-110, or whose product with the value's scale is 2^-31, of the row's largest
 * (many rows: elements of a query 2^-30 below its largest, MXFP4 blocks of keys 2^-37 below the largest of 128 tokens, tokens whose probability is 2^-31, or whose value's scale 2^-32 of the sequence's largest).
 */
size_t kv_cache_attention_workspace_bytes(int64_t seqs, int64_t total_q, int64_t q_heads, int64_t heads, int64_t dim);
size_t kv_cache_attention_zeroed_bytes(int64_t seqs, int64_t total_q, int64_t q_heads, int64_t heads, int64_t dim);
int kv_cache_attention(int fmt, const void* k_codes, const void* k_scales, const void* v_codes, const void* v_scales, int64_t num_pages, int64_t page_size,
                       int64_t heads, int64_t dim, const int32_t* table, int64_t table_stride, int64_t max_pages, const int32_t* lens, const int32_t* starts,
                       const int32_t* cu_q, int64_t seqs, const void* q, int64_t q_token_stride, int64_t q_head_stride, int64_t q_heads, int64_t total_q,
                       const int64_t* tree, int64_t tree_words, float scale, void* out, int64_t out_token_stride, int64_t out_head_stride, float* lse,
                       void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* KV_CACHE_H_ */
