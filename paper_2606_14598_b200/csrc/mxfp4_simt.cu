// MXFP4 linear on the CUDA cores: out[m,n] = bf16(sum_b 2^(ea + ew) * sum_{k in b} qa * qw + bias[n]).
// Each warp owns one output channel and MB tokens; a lane takes whole blocks of 32 along K.
#include "internal.h"
#include "mxfp4_math.cuh"
#include "ptx.cuh"

namespace w8a8 {
namespace {

constexpr int MB = 4;
constexpr int kWarps = 8;

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ float block_scale(uint32_t byte) { return __uint_as_float(mx_scale_bf16(byte) << 16); }

__device__ __forceinline__ float dot8(uint32_t a, uint32_t b) {
    const uint2 a0 = e2m1x4_to_bf16(a), a1 = e2m1x4_to_bf16(a >> 16), b0 = e2m1x4_to_bf16(b), b1 = e2m1x4_to_bf16(b >> 16);
    float s = bf16_lo(a0.x) * bf16_lo(b0.x);
    s = fmaf(bf16_hi(a0.x), bf16_hi(b0.x), s);
    s = fmaf(bf16_lo(a0.y), bf16_lo(b0.y), s);
    s = fmaf(bf16_hi(a0.y), bf16_hi(b0.y), s);
    s = fmaf(bf16_lo(a1.x), bf16_lo(b1.x), s);
    s = fmaf(bf16_hi(a1.x), bf16_hi(b1.x), s);
    s = fmaf(bf16_lo(a1.y), bf16_lo(b1.y), s);
    return fmaf(bf16_hi(a1.y), bf16_hi(b1.y), s);
}

__global__ void __launch_bounds__(kWarps * 32)
mx_linear_simt_kernel(const uint8_t* qa, int64_t ldqa, const uint8_t* sa, const uint8_t* __restrict__ qw, const uint8_t* __restrict__ sw,
                      const float* __restrict__ bias, __nv_bfloat16* __restrict__ out, int64_t ldo, int M, int N, int K, int* status) {
    grid_dep_wait();
    if (status != nullptr && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *status = 0;
    const int lane = threadIdx.x & 31, n = blockIdx.x * kWarps + (threadIdx.x >> 5);
    if (n >= N) return;
    const int kb = K / kMxBlock, ktiles = (kb + kScaleTileBlocks - 1) / kScaleTileBlocks;
    auto scale = [&](const uint8_t* s, int row, int b) {
        return block_scale(__ldcg(s + (static_cast<int64_t>(row / kScaleTileRows) * ktiles + b / kScaleTileBlocks) * kScaleTileBytes +
                                  scale_in_tile(row % kScaleTileRows, b % kScaleTileBlocks)));
    };
    for (int m0 = blockIdx.y * MB; m0 < M; m0 += gridDim.y * MB) {
        float acc[MB] = {};
        for (int b = lane; b < kb; b += 32) {
            const uint4 w = __ldcg(reinterpret_cast<const uint4*>(qw + static_cast<int64_t>(n) * (K / 2)) + b);
            const float ws = scale(sw, n, b);
#pragma unroll
            for (int i = 0; i < MB; ++i) {
                const int m = min(m0 + i, M - 1);
                const uint4 a = __ldcg(reinterpret_cast<const uint4*>(qa + m * ldqa) + b);
                const float d = (dot8(a.x, w.x) + dot8(a.y, w.y)) + (dot8(a.z, w.z) + dot8(a.w, w.w));   // exact: below 2^11 quarters
                acc[i] = fmaf(d * ws, scale(sa, m, b), acc[i]);
            }
        }
#pragma unroll
        for (int i = 0; i < MB; ++i) {
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) acc[i] += __shfl_xor_sync(0xffffffffu, acc[i], o);
            if (lane == 0 && m0 + i < M) out[static_cast<int64_t>(m0 + i) * ldo + n] = __float2bfloat16_rn(bias != nullptr ? acc[i] + bias[n] : acc[i]);
        }
    }
}

} // namespace

cudaError_t launch_mx_linear_simt(const MxLinearArgs& a, cudaStream_t st) {
    const int rows = (a.M + MB - 1) / MB;
    const dim3 grid((a.N + kWarps - 1) / kWarps, rows < 65535 ? rows : 65535);
    mx_linear_simt_kernel<<<grid, kWarps * 32, 0, st>>>(a.qa, a.ldqa, a.sa, a.qw, a.sw, a.bias, static_cast<__nv_bfloat16*>(a.out), a.ldo, a.M, a.N, a.K,
                                                        a.after_quantizer ? nullptr : a.status);
    return cudaGetLastError();
}

} // namespace w8a8
