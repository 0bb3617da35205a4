/*
 * mxfp4_linear.h -- C ABI of the B200 (sm_100a) 4-bit linear layer: MXFP4 weights, activations quantized to MXFP4
 * inside the call, fp32 accumulation on the block-scaled tensor cores, bias added in the epilogue, bf16 out. The
 * 4-bit counterpart of w8a8_linear.h; its conventions on pointers, streams, chaining, capture and status codes hold
 * here too. Every operand, the weights among them, is read after the work ahead of the call on its stream is complete: a
 * quantizer, a copy or any other kernel may write them directly before the call.
 *
 * The format (OCP Microscaling v1.0, MXFP4): 32 consecutive elements of a row share a power-of-two scale.
 *     amax  = max |x| of the block
 *     e     = max(floor(log2(amax)) - 2, -127), -127 for an all-zero block;  scale byte (E8M0) = e + 127
 *     code  = x * 2^-e rounded to the nearest of 0 .5 1 1.5 2 3 4 6 (E2M1, ties to the even code, saturating), sign in bit 3
 *     value = (-1)^sign * magnitude(code) * 2^e
 * A block that holds an Inf or a NaN is written as scale byte 255 (NaN) and codes 0: it reads back as NaN, and the
 * linear gives NaN in every output of that row. Blocks with finite inputs are not affected by their neighbours.
 *     out[m,n] = bf16(sum_k value(A)[m,k] * value(W)[n,k] + bias[n])
 * Products are exact; the sum is accumulated in fp32 in an order that depends on the sizes only (a call repeated on
 * the same inputs gives the same bits); one rounding to bf16.
 *
 * Layout: codes are [rows, K/2] bytes, row-major, element 2i in the low nibble of byte i. Scales are tiles of 512
 * bytes, one for 128 rows x 4 blocks, tiles row by row ([ceil(rows/128)][ceil(K/128)][512]); inside a tile the scale
 * of row r, block c is byte 16 * (r % 32) + 4 * (r / 32) + c. Bytes for rows or blocks past the end are 0.
 *
 * Sizes: K % 32 == 0, N % 8 == 0, 1 <= M, N <= 2^30, 1 <= K <= MXFP4_K_MAX. Pointers 16-byte aligned, row strides
 * multiples of 16 bytes.
 */
#ifndef MXFP4_LINEAR_H_
#define MXFP4_LINEAR_H_

#include "w8a8_linear.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { MXFP4_BF16 = 0, MXFP4_FP32 = 1, MXFP4_CODES = 2 };
#define MXFP4_K_MAX (1 << 24)

/* Bytes of the scale tiles of a [rows, K] matrix (0 on invalid sizes). */
size_t mxfp4_scale_bytes(int64_t rows, int64_t K);

/*
 * x [M,K] to codes and scale tiles (weights at load time, or activations that feed several linears).
 *   x       in   dtype MXFP4_BF16 or MXFP4_FP32, row stride ldx elements
 *   codes   out  [M,K/2] dense           scales  out  mxfp4_scale_bytes(M, K) bytes
 */
int mxfp4_quantize(const void* x, int dtype, int64_t M, int64_t K, int64_t ldx, uint8_t* codes, uint8_t* scales, void* stream);

/* The values of codes and scale tiles, exactly, as bf16 or fp32 (out: row stride ldo elements). */
int mxfp4_dequantize(const uint8_t* codes, const uint8_t* scales, int64_t M, int64_t K, void* out, int dtype, int64_t ldo, void* stream);

/*
 * Device workspace of mxfp4_linear_fused (256-byte aligned, no initialisation; 0 on invalid sizes): a 256-byte status
 * block, then scratch for the scale tiles and the codes of the activations. With a_dtype MXFP4_CODES 256 bytes are enough.
 */
size_t mxfp4_linear_workspace_bytes(int64_t M, int64_t N, int64_t K);

/*
 *   A         in   a_dtype MXFP4_BF16: [M,K], row stride lda elements, quantized inside the call;
 *                  MXFP4_CODES: [M,K/2] packed codes, row stride lda bytes, with a_scales (else a_scales is NULL)
 *   qw, sw    in   weight codes [N,K/2] dense and scale tiles
 *   bias      in   fp32 [N] or NULL
 *   out       out  bf16 [M,N], row stride ldo elements
 * int8_check_status and int8_sticky_status report a bounded device-side wait that ran out, as for the int8 linear.
 */
int mxfp4_linear_fused(const void* A, int a_dtype, int64_t lda, const uint8_t* a_scales, const uint8_t* qw, const uint8_t* sw, const float* bias,
                       void* out, int64_t ldo, int64_t M, int64_t N, int64_t K, void* workspace, size_t workspace_bytes, void* stream);

/*
 * For sweeps and tests: the kernel configuration of the following linears of this process. -1 (default) chooses from the
 * sizes; 0, 1, 2 are the tiled GEMM with 256 x 256 and 256 x 192 tiles on CTA pairs and 128 x 128 tiles on single CTAs, 3 the
 * kernel for at most 64 tokens. Another id, or 3 with more tokens, makes mxfp4_linear_fused return W8A8_ERR_INVALID_ARG.
 * Returns the previous value.
 */
int mxfp4_linear_force_config(int config_id);

#ifdef __cplusplus
}
#endif
#endif /* MXFP4_LINEAR_H_ */
