// Root-mean-square norm with the residual's addition, written as int8 codes with a scale a row, as bf16, or both.
//
//   h = bf16(x + residual)    u = h * weight    r = 1 / sqrt(mean(h^2) + eps)
//   int8: t = max |u|, c = t / 127, q = rne(u / c), s = c * r          bf16: y = bf16(u * r)
//
// The norm is one factor of the row, so it cancels out of the codes: the sum of squares and the largest |u| are found in one pass over
// the row, which then sits in registers as u and is written from there. One trip through HBM: 4 bytes an element in, 3 or 4 out, which is what bounds it: 8221 rows
// of 12288 in bf16 take 131 to 141 us (123 at the copy's rate; the clock falls to 1740 MHz under the power limit where calls follow one another), 4110 of 4608 in int8 28 us (20, at
// 1965 MHz; 4.6 waves of six CTAs an SM; what holds them at 4.7 TB/s is not known), one row of 4608 3.3 us.
#include "../../include/int8_norm.h"
#include "internal.h"
#include "mxfp4_math.cuh"
#include "ptx.cuh"
#include "quant_math.cuh"

#include <cmath>

namespace w8a8 {
namespace {

struct NormArgs {
    const __nv_bfloat16 *x, *residual;
    const void* weight;
    __nv_bfloat16 *sum, *y;
    int8_t* qa;
    float* s_tok;
    int64_t ldx, ldr, lds, ldy, M;
    int K;
    float eps;
};

constexpr int kMaxThreads = 1024;

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&p);
}

// h of eight elements, packed
template <bool RES>
__device__ __forceinline__ uint4 add8(const uint4& x, const uint4& r) {
    if (!RES) return x;
    float a[8], b[8];
    unpack_bf16x8(x, a);
    unpack_bf16x8(r, b);
    return make_uint4(pack_bf16(a[0] + b[0], a[1] + b[1]), pack_bf16(a[2] + b[2], a[3] + b[3]), pack_bf16(a[4] + b[4], a[5] + b[5]),
                      pack_bf16(a[6] + b[6], a[7] + b[7]));
}
// (plain loads, which L1 keeps for the CTAs to come; the read-only path is not for memory that work ahead may still be writing)
template <bool W16>
__device__ __forceinline__ void weight8(const void* w, int k, float (&f)[8]) {
    if (W16) {
        unpack_bf16x8(*reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(w) + k), f);
    } else {
        const float4* p = reinterpret_cast<const float4*>(static_cast<const float*>(w) + k);
        const float4 a = p[0], b = p[1];
        f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
        f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
    }
}
// u of eight elements; their squares and largest magnitude are added to the row's
template <bool W16>
__device__ __forceinline__ void scale8(const uint4& h, const void* w, int k, float (&u)[8], float& squares, uint32_t& top) {
    float f[8], g[8];
    unpack_bf16x8(h, f);
    weight8<W16>(w, k, g);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        squares = __fmaf_rn(f[i], f[i], squares);
        u[i] = __fmul_rn(f[i], g[i]);
        top = max(top, __float_as_uint(u[i]) & 0x7fffffffu);           // patterns of magnitudes order like them, Inf and NaN on top
    }
}

// Sum and maximum over the threads of a row (whole warps, `warps` of them, the row's part of `share` being theirs)
__device__ __forceinline__ void reduce_row(float& squares, uint32_t& top, float2* share, int warps) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        squares += __shfl_xor_sync(0xffffffffu, squares, o);
        top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
    }
    if (warps == 1) return;
    const int lane = threadIdx.x & 31;
    if (lane == 0) share[threadIdx.x >> 5] = make_float2(squares, __uint_as_float(top));
    __syncthreads();
    float2 v = lane < warps ? share[(threadIdx.x >> 5) / warps * warps + lane] : make_float2(0.f, 0.f);
    squares = v.x;
    top = __float_as_uint(v.y);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        squares += __shfl_xor_sync(0xffffffffu, squares, o);
        top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
    }
}

struct RowNorm {
    RowScale c;          // what the codes are divided by
    RowScale2 c2;
    float r, s;          // the norm's factor, the row's scale
    bool fine;           // finite
};
__device__ __forceinline__ RowNorm row_norm(float squares, uint32_t top, int K, float eps) {
    RowNorm n;
    n.fine = top < 0x7f800000u && squares < INFINITY;
    n.c = head_scale(n.fine ? __uint_as_float(top) : 0.f);
    n.c2 = head_scale2(n.c);
    n.r = n.fine ? __frsqrt_rn(__fadd_rn(__fdiv_rn(squares, static_cast<float>(K)), eps)) : __uint_as_float(0x7fc00000u);
    n.s = !n.fine ? n.r : top == 0u ? 1.f : __fmul_rn(n.c.s, n.r);
    return n;
}
__device__ __forceinline__ void write8(const NormArgs& a, int64_t row, int k, const float (&u)[8], const RowNorm& n) {
    if (a.qa != nullptr) {
        const uint2 c = n.fine ? make_uint2(quant4f(u[0], u[1], u[2], u[3], n.c, n.c2), quant4f(u[4], u[5], u[6], u[7], n.c, n.c2)) : make_uint2(0, 0);
        *reinterpret_cast<uint2*>(a.qa + row * a.K + k) = c;
    }
    if (a.y != nullptr)
        *reinterpret_cast<uint4*>(a.y + row * a.ldy + k) = make_uint4(pack_bf16(u[0] * n.r, u[1] * n.r), pack_bf16(u[2] * n.r, u[3] * n.r),
                                                                       pack_bf16(u[4] * n.r, u[5] * n.r), pack_bf16(u[6] * n.r, u[7] * n.r));
}

// Rows of up to per_row * VPT * 8 elements: per_row threads a row (whole warps), blockDim.x / per_row rows a CTA.
template <int VPT, bool RES, bool W16>
__global__ void __launch_bounds__(kMaxThreads) norm_kernel(const NormArgs a, int per_row) {
    __shared__ float2 share[kMaxThreads / 32];
    grid_dep_wait();
    grid_dep_launch_dependents();
    const int rows = blockDim.x / per_row, mine = threadIdx.x / per_row, at = threadIdx.x - mine * per_row, vecs = a.K / 8;
    const int64_t row = static_cast<int64_t>(blockIdx.x) * rows + mine;
    const bool live = row < a.M;
    uint4 x[VPT], r[VPT];
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
        const int v = at + j * per_row;
        x[j] = r[j] = make_uint4(0, 0, 0, 0);
        if (live && v < vecs) {
            x[j] = __ldcg(reinterpret_cast<const uint4*>(a.x + row * a.ldx + v * 8));
            if (RES) r[j] = __ldcg(reinterpret_cast<const uint4*>(a.residual + row * a.ldr + v * 8));
        }
    }
    float u[VPT][8], squares = 0.f;
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
        const int v = at + j * per_row;
        if (!live || v >= vecs) continue;
        const uint4 h = add8<RES>(x[j], r[j]);
        if (a.sum != nullptr) *reinterpret_cast<uint4*>(a.sum + row * a.lds + v * 8) = h;
        scale8<W16>(h, a.weight, v * 8, u[j], squares, top);
    }
    reduce_row(squares, top, share, per_row / 32);
    const RowNorm n = row_norm(squares, top, a.K, a.eps);
    if (!live) return;
    if (at == 0 && a.s_tok != nullptr) a.s_tok[row] = n.s;
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
        const int v = at + j * per_row;
        if (v < vecs) write8(a, row, v * 8, u[j], n);
    }
}

// Longer rows: a CTA a row, read twice (the second time mostly out of L2). h comes back from sum_out where that is written: it may be x
// or the residual. Every thread reads again only what it wrote.
template <bool RES, bool W16>
__global__ void __launch_bounds__(kMaxThreads) norm_long_kernel(const NormArgs a) {
    __shared__ float2 share[kMaxThreads / 32];
    grid_dep_wait();
    grid_dep_launch_dependents();
    const int vecs = a.K / 8;
    const int64_t row = blockIdx.x;
    float u[8], squares = 0.f;
    uint32_t top = 0;
    const uint4 none = make_uint4(0, 0, 0, 0);
    auto load = [&](int v) {
        const uint4 x = __ldcg(reinterpret_cast<const uint4*>(a.x + row * a.ldx + static_cast<int64_t>(v) * 8));
        return add8<RES>(x, RES ? __ldcg(reinterpret_cast<const uint4*>(a.residual + row * a.ldr + static_cast<int64_t>(v) * 8)) : none);
    };
    for (int v = threadIdx.x; v < vecs; v += blockDim.x) {
        const uint4 h = load(v);
        if (a.sum != nullptr) *reinterpret_cast<uint4*>(a.sum + row * a.lds + static_cast<int64_t>(v) * 8) = h;
        scale8<W16>(h, a.weight, v * 8, u, squares, top);
    }
    reduce_row(squares, top, share, blockDim.x / 32);
    const RowNorm n = row_norm(squares, top, a.K, a.eps);
    if (threadIdx.x == 0 && a.s_tok != nullptr) a.s_tok[row] = n.s;
    for (int v = threadIdx.x; v < vecs; v += blockDim.x) {
        const uint4 h = a.sum != nullptr ? __ldcg(reinterpret_cast<const uint4*>(a.sum + row * a.lds + static_cast<int64_t>(v) * 8)) : load(v);
        scale8<W16>(h, a.weight, v * 8, u, squares, top);
        write8(a, row, v * 8, u, n);
    }
}

template <int VPT>
auto norm_variant(bool res, bool w16) {
    return res ? (w16 ? norm_kernel<VPT, true, true> : norm_kernel<VPT, true, false>) : (w16 ? norm_kernel<VPT, false, true> : norm_kernel<VPT, false, false>);
}

int run_norm(const NormArgs& a, bool w16, cudaStream_t st) {
    const bool res = a.residual != nullptr;
    const int vecs = a.K / 8;
    cudaError_t e;
    if (vecs > 3 * kMaxThreads) {
        const auto kern = res ? (w16 ? norm_long_kernel<true, true> : norm_long_kernel<true, false>) : (w16 ? norm_long_kernel<false, true> : norm_long_kernel<false, false>);
        e = launch_pdl(kern, dim3(static_cast<unsigned>(a.M)), kMaxThreads, st, a);
    } else {
        // three vectors a thread, all on their way at once, are the best of 1, 2, 3, 4 and 6 in long rows (4110 rows of 4608: 36, 30, 28, 29 and 31 us; of
        // 12288: 99, 99, 69, 71 and 67), two up to 256 vectors (of 2048: 16.6, 15.7, 16.1). Between them, three and two, 20000 rows: of 2064 elements 56 and 62 us, of 2304 57 and 63,
        // of 2560 71 and 67 (a sixth of three vectors' places idle), of 2816 74 and 81, of 3328 84 and 96, of 3584 90 and 100. (One row: 3.3 and 2.9.)
        const int vpt = vecs <= 256 ? 2 : 3;
        const int per_row = ((vecs + vpt - 1) / vpt + 31) / 32 * 32, rows = per_row >= 256 ? 1 : 256 / per_row;
        const auto kern = vpt == 2 ? norm_variant<2>(res, w16) : norm_variant<3>(res, w16);
        e = launch_pdl(kern, dim3(static_cast<unsigned>((a.M + rows - 1) / rows)), rows * per_row, st, a, per_row);
    }
    return e == cudaSuccess ? W8A8_OK : W8A8_ERR_CUDA;
}

bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

} // namespace
} // namespace w8a8

extern "C" int int8_rmsnorm(const void* x, int64_t ldx, const void* residual, int64_t ldr, const void* weight, int weight_dtype, float eps, int64_t M, int64_t K,
                            void* sum_out, int64_t lds, int8_t* qa, float* s_tok, void* y, int64_t ldy, void* stream) {
    using namespace w8a8;
    if (M < 0 || M > INT32_MAX || K <= 0 || K > INT8_NORM_K_MAX || weight == nullptr || (weight_dtype != INT8_NORM_FP32 && weight_dtype != INT8_NORM_BF16) ||
        !(eps > 0.f) || !std::isfinite(eps) || (M > 0 && (x == nullptr || (qa == nullptr && y == nullptr))) || (qa == nullptr) != (s_tok == nullptr))
        return W8A8_ERR_INVALID_ARG;
    if (ldx < K || (residual != nullptr && ldr < K) || (sum_out != nullptr && lds < K) || (y != nullptr && ldy < K)) return W8A8_ERR_INVALID_ARG;
    // (in place is fine, shifted is not: a thread writes only what it has read)
    if (M > 1 && sum_out != nullptr && ((sum_out == x && lds != ldx) || (sum_out == residual && lds != ldr))) return W8A8_ERR_INVALID_ARG;
    if (K % 8 != 0 || ldx % 8 != 0 || !aligned(x, 16) || !aligned(weight, 16) || !aligned(s_tok, 4) || !aligned(qa, 16)) return W8A8_ERR_ALIGNMENT;
    if (residual != nullptr && (ldr % 8 != 0 || !aligned(residual, 16))) return W8A8_ERR_ALIGNMENT;
    if (sum_out != nullptr && (lds % 8 != 0 || !aligned(sum_out, 16))) return W8A8_ERR_ALIGNMENT;
    if (y != nullptr && (ldy % 8 != 0 || !aligned(y, 16))) return W8A8_ERR_ALIGNMENT;
    if (int e = check_arch()) return e;
    if (M == 0) return W8A8_OK;
    NormArgs a{};
    a.x = static_cast<const __nv_bfloat16*>(x);
    a.residual = static_cast<const __nv_bfloat16*>(residual);
    a.weight = weight;
    a.sum = static_cast<__nv_bfloat16*>(sum_out);
    a.y = static_cast<__nv_bfloat16*>(y);
    a.qa = qa;
    a.s_tok = s_tok;
    a.ldx = ldx;
    a.ldr = ldr;
    a.lds = lds;
    a.ldy = ldy;
    a.M = M;
    a.K = static_cast<int>(K);
    a.eps = eps;
    return run_norm(a, weight_dtype == INT8_NORM_BF16, static_cast<cudaStream_t>(stream));
}
