// C ABI of the MXFP4 linear: argument validation, workspace layout, dispatch.
#include "../../include/mxfp4_linear.h"
#include "internal.h"
#include "mxfp4_math.cuh"

#include <nvtx3/nvToolsExt.h>

#include <atomic>

namespace {

using namespace w8a8;

constexpr size_t kStatusBlock = 256;
std::atomic<int> g_forced_config{-1};
// Tokens up to which the few-token kernel quantizes them itself. GPU time of 8 x 4608 -> 4608 8.5 us that way, of 14 tokens with a
// quantizer ahead 8.4 us, which costs the host a second launch (3 us); 8 x 4608 -> 13824 12.3 us, 16 tokens with a quantizer 12.1 us
// (12 tokens quantized inside 14.6, ahead 12.1 us).
constexpr int kQuantizeInside = 8;
constexpr int64_t kMaxRows = int64_t(1) << 30;

struct Range {
    explicit Range(const char* name) { nvtxRangePushA(name); }
    ~Range() { nvtxRangePop(); }
};

inline size_t round_up(size_t v, size_t a) { return (v + a - 1) / a * a; }
inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

int check_matrix(int64_t rows, int64_t K) {
    if (rows <= 0 || K <= 0 || rows > kMaxRows || K > MXFP4_K_MAX) return W8A8_ERR_INVALID_ARG;
    return K % kMxBlock == 0 ? W8A8_OK : W8A8_ERR_ALIGNMENT;
}

} // namespace

extern "C" {

size_t mxfp4_scale_bytes(int64_t rows, int64_t K) {
    if (check_matrix(rows, K) != W8A8_OK) return 0;
    const size_t mt = (static_cast<size_t>(rows) + kScaleTileRows - 1) / kScaleTileRows;
    const size_t kt = (static_cast<size_t>(K) + kScaleTileBlocks * kMxBlock - 1) / (kScaleTileBlocks * kMxBlock);
    return mt * kt * kScaleTileBytes;
}

int mxfp4_quantize(const void* x, int dtype, int64_t M, int64_t K, int64_t ldx, uint8_t* codes, uint8_t* scales, void* stream) {
    const Range range("mxfp4 quantize");
    if (x == nullptr || codes == nullptr || scales == nullptr || (dtype != MXFP4_BF16 && dtype != MXFP4_FP32)) return W8A8_ERR_INVALID_ARG;
    if (int e = check_matrix(M, K)) return e;
    if (ldx < K) return W8A8_ERR_INVALID_ARG;
    if (ldx % (dtype == MXFP4_BF16 ? 8 : 4) != 0 || !aligned16(x) || !aligned16(codes) || !aligned16(scales)) return W8A8_ERR_ALIGNMENT;
    if (int e = check_arch()) return e;
    return launch_mx_quantize(x, dtype == MXFP4_FP32, ldx, static_cast<int>(M), static_cast<int>(K), codes, scales, nullptr, false,
                              static_cast<cudaStream_t>(stream)) == cudaSuccess ? W8A8_OK : W8A8_ERR_CUDA;
}

int mxfp4_dequantize(const uint8_t* codes, const uint8_t* scales, int64_t M, int64_t K, void* out, int dtype, int64_t ldo, void* stream) {
    const Range range("mxfp4 dequantize");
    if (codes == nullptr || scales == nullptr || out == nullptr || (dtype != MXFP4_BF16 && dtype != MXFP4_FP32)) return W8A8_ERR_INVALID_ARG;
    if (int e = check_matrix(M, K)) return e;
    if (ldo < K) return W8A8_ERR_INVALID_ARG;
    if (ldo % (dtype == MXFP4_BF16 ? 8 : 4) != 0 || !aligned16(codes) || !aligned16(scales) || !aligned16(out)) return W8A8_ERR_ALIGNMENT;
    if (int e = check_arch()) return e;
    return launch_mx_dequantize(codes, scales, static_cast<int>(M), static_cast<int>(K), out, dtype == MXFP4_FP32, ldo,
                                static_cast<cudaStream_t>(stream)) == cudaSuccess ? W8A8_OK : W8A8_ERR_CUDA;
}

int mxfp4_linear_force_config(int config_id) { return g_forced_config.exchange(config_id); }

size_t mxfp4_linear_workspace_bytes(int64_t M, int64_t N, int64_t K) {
    if (check_matrix(M, K) != W8A8_OK || N <= 0 || N > kMaxRows) return 0;
    return kStatusBlock + mxfp4_scale_bytes(M, K) + round_up(static_cast<size_t>(M) * static_cast<size_t>(K / 2), 256);
}

int mxfp4_linear_fused(const void* A, int a_dtype, int64_t lda, const uint8_t* a_scales, const uint8_t* qw, const uint8_t* sw, const float* bias,
                       void* out, int64_t ldo, int64_t M, int64_t N, int64_t K, void* workspace, size_t workspace_bytes, void* stream) {
    const Range range("mxfp4 linear fused");
    if (A == nullptr || qw == nullptr || sw == nullptr || out == nullptr || (a_dtype != MXFP4_BF16 && a_dtype != MXFP4_CODES))
        return W8A8_ERR_INVALID_ARG;
    if ((a_dtype == MXFP4_CODES) != (a_scales != nullptr)) return W8A8_ERR_INVALID_ARG;
    if (int e = check_matrix(M, K)) return e;
    if (N <= 0 || N > kMaxRows || lda < (a_dtype == MXFP4_BF16 ? K : K / 2) || ldo < N) return W8A8_ERR_INVALID_ARG;
    if (N % 8 != 0 || ldo % 8 != 0 || lda % (a_dtype == MXFP4_BF16 ? 8 : 16) != 0) return W8A8_ERR_ALIGNMENT;
    if (!aligned16(A) || !aligned16(a_scales) || !aligned16(qw) || !aligned16(sw) || !aligned16(out) || !aligned16(bias)) return W8A8_ERR_ALIGNMENT;
    const size_t need = a_dtype == MXFP4_BF16 ? mxfp4_linear_workspace_bytes(M, N, K) : kStatusBlock;
    if (workspace == nullptr || (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0 || workspace_bytes < need) return W8A8_ERR_WORKSPACE;
    const int forced = g_forced_config.load();
    if (forced < -1 || forced > kMxGemmConfigs || (forced == kMxGemmConfigs && !mx_skinny_fits(static_cast<int>(M)))) return W8A8_ERR_INVALID_ARG;
    if (int e = check_arch()) return e;

    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    MxLinearArgs g{};
    g.qw = qw; g.sw = sw; g.bias = bias; g.out = out; g.ldo = ldo;
    g.M = static_cast<int>(M); g.N = static_cast<int>(N); g.K = static_cast<int>(K);
    g.status = reinterpret_cast<int*>(ws);
    const bool skinny = forced == kMxGemmConfigs || (forced < 0 && mx_skinny_preferred(g.M, g.K));
    if (skinny && a_dtype == MXFP4_BF16 && g.M <= kQuantizeInside) return launch_mx_skinny_bf16(g, A, lda, st);
    if (a_dtype == MXFP4_BF16) {
        uint8_t* sa = ws + kStatusBlock;
        uint8_t* qa = sa + mxfp4_scale_bytes(M, K);
        if (launch_mx_quantize(A, false, lda, g.M, g.K, qa, sa, g.status, true, st) != cudaSuccess) return W8A8_ERR_CUDA;
        g.qa = qa; g.sa = sa; g.ldqa = K / 2; g.after_quantizer = true;
    } else {
        g.qa = static_cast<const uint8_t*>(A); g.sa = a_scales; g.ldqa = lda; g.after_quantizer = false;
    }
    if (skinny) return launch_mx_skinny_codes(g, st);
    return launch_mx_gemm(g, forced >= 0 ? forced : choose_mx_config(g.M, g.N, g.K), st);
}

} // extern "C"
