/*
 * int8_norm.h -- C ABI of the root-mean-square norm with the residual's addition, in front of a quantized linear: int8 codes with
 * a scale a token (what int8_linear_fused takes as W8A8_ACT_INT8), or bf16 (what mxfp4_linear_fused takes). Conventions on pointers,
 * streams and status codes as in w8a8_linear.h. The call allocates nothing, only enqueues, and can be captured in a CUDA graph.
 *
 *     h[m,k] = bf16(x[m,k] + residual[m,k])                  (x itself without a residual; fp32 addition)
 *     u[m,k] = h[m,k] * weight[k]                            fp32, rounded once
 *     r[m]   = 1 / sqrt(sum_k h[m,k]^2 / K + eps)            fp32 sum
 *     int8:    t = max_k |u[m,k]|;  c = t > 0 ? t / 127 : 1;  q = clamp(rne(u / c), -127, 127);  s_tok = t > 0 ? c * r : 1
 *     bf16:    y = bf16(u * r)
 * The norm is one factor of a whole row: the codes do not depend on it (so not on the order of the sum), the scale carries it. c, u / c
 * and c * r are fp32 and rounded once each, as in int8_quantize_act_per_token. A row that holds an Inf or a NaN, or whose squares sum to more
 * than fp32 holds, gets codes 0 with a NaN scale, and NaN in y; other rows are not touched by it.
 */
#ifndef INT8_NORM_H_
#define INT8_NORM_H_

#include "w8a8_linear.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { INT8_NORM_FP32 = 0, INT8_NORM_BF16 = 1 }; /* type of the weight */
#define INT8_NORM_K_MAX (1 << 24)

/*
 *   x          in   bf16 [M,K], row stride ldx
 *   residual   in   bf16 [M,K], row stride ldr, or NULL
 *   weight     in   fp32 or bf16 [K] (weight_dtype)
 *   sum_out    out  bf16 [M,K], row stride lds: h; may be x or residual itself (same address and stride); NULL if not wanted
 *   qa, s_tok  out  int8 [M,K] dense and fp32 [M], or both NULL
 *   y          out  bf16 [M,K], row stride ldy, or NULL; one of qa and y is needed, both are fine
 * Outputs overlap neither one another nor, but for sum_out, an input.
 * Strides in elements, multiples of 8, at least K; K % 8 == 0 (the int8 linear wants K % 16 == 0), 0 < K <= INT8_NORM_K_MAX; x, residual,
 * weight, sum_out, qa and y 16-byte aligned; eps > 0 and finite. M == 0 is a valid call.
 */
int int8_rmsnorm(const void* x, int64_t ldx, const void* residual, int64_t ldr, const void* weight, int weight_dtype, float eps, int64_t M, int64_t K,
                 void* sum_out, int64_t lds, int8_t* qa, float* s_tok, void* y, int64_t ldy, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* INT8_NORM_H_ */
