// MXFP4 quantizer and its inverse: rows of bf16 or fp32 to packed E2M1 codes and tiles of E8M0 scales, and back.
// Both move bytes and compute next to nothing (a conversion and a multiply an element): HBM is the bound, 2.53 bytes an
// element for bf16, 4.53 for fp32.
//
// A lane holds 8 consecutive elements of a row (16 bytes of bf16), four neighbouring lanes one block of 32, a warp one
// segment of 256 elements: loads and stores are contiguous across the warp, the block's maximum takes two shuffles, and
// a segment's eight scale bytes leave as two 4-byte words (one for each tile of four blocks that the segment crosses).
#include "internal.h"
#include "mxfp4_math.cuh"
#include "ptx.cuh"

namespace w8a8 {
namespace {

constexpr int kWarps = 8;
constexpr int kSegment = 256;        // elements of a row a warp takes at a time
constexpr int kUnroll = 4;           // segments whose loads are in flight together

__device__ __forceinline__ void load8(const __nv_bfloat16* p, float (&x)[8], uint32_t& amax) {
    const uint4 v = __ldcg(reinterpret_cast<const uint4*>(p));
    amax = absmax_bits8(v);
    unpack_bf16x8(v, x);
}
__device__ __forceinline__ void load8(const float* p, float (&x)[8], uint32_t& amax) {
    const float4 a = __ldcg(reinterpret_cast<const float4*>(p)), b = __ldcg(reinterpret_cast<const float4*>(p) + 1);
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
    x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    amax = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) amax = max(amax, __float_as_uint(x[i]) & 0x7fffffffu);
}

// Work: tasks of kUnroll segments of one row, row by row; rows up to the end of the last scale tile (rows past M get
// zero scales, so that a scale tensor's contents depend on nothing but x).
template <typename T>
__global__ void __launch_bounds__(kWarps * 32)
mx_quantize_kernel(const T* __restrict__ x, int64_t ldx, int M, int K, uint8_t* __restrict__ codes, uint8_t* __restrict__ scales,
                   int tasks_per_row, int64_t num_tasks, int* status_to_clear, int early) {
    if (early) grid_dep_launch_dependents();
    grid_dep_wait();
    if (status_to_clear != nullptr && blockIdx.x == 0 && threadIdx.x == 0) *status_to_clear = 0;
    const int lane = threadIdx.x & 31;
    const int ktiles = (K + kScaleTileBlocks * kMxBlock - 1) / (kScaleTileBlocks * kMxBlock);
    for (int64_t task = static_cast<int64_t>(blockIdx.x) * kWarps + (threadIdx.x >> 5); task < num_tasks;
         task += static_cast<int64_t>(gridDim.x) * kWarps) {
        const int row = static_cast<int>(task / tasks_per_row);
        const int k0 = static_cast<int>(task - static_cast<int64_t>(row) * tasks_per_row) * (kUnroll * kSegment) + lane * 8;
        float v[kUnroll][8];
        uint32_t amax[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int k = k0 + u * kSegment;
            if (row < M && k < K) {
                load8(x + row * ldx + k, v[u], amax[u]);
            } else {
                amax[u] = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) v[u][i] = 0.f;
            }
        }
        uint8_t* tile_row = scales + static_cast<int64_t>(row / kScaleTileRows) * ktiles * kScaleTileBytes + scale_in_tile(row % kScaleTileRows, 0);
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int k = k0 + u * kSegment;
            uint32_t m = amax[u];
            m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
            m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
            const uint32_t byte = mx_scale_byte(m);
            if (row < M && k < K) *reinterpret_cast<uint32_t*>(codes + static_cast<int64_t>(row) * (K / 2) + k / 2) = mx_codes8(v[u], byte);
            // the four blocks of a tile sit in 16 lanes: two shuffles bring their bytes into one word
            uint32_t word = byte << (((lane >> 2) & 3) * 8);
            word |= __shfl_xor_sync(0xffffffffu, word, 4);
            word |= __shfl_xor_sync(0xffffffffu, word, 8);
            const int kt = k / (kScaleTileBlocks * kMxBlock);
            if ((lane & 15) == 0 && kt < ktiles) *reinterpret_cast<uint32_t*>(tile_row + static_cast<int64_t>(kt) * kScaleTileBytes) = word;
        }
    }
}

__device__ __forceinline__ void store8(__nv_bfloat16* p, const uint4& v) { *reinterpret_cast<uint4*>(p) = v; }
__device__ __forceinline__ void store8(float* p, const uint4& v) {
    float f[8];
    unpack_bf16x8(v, f);
    reinterpret_cast<float4*>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
}

template <typename T>
__global__ void __launch_bounds__(kWarps * 32)
mx_dequantize_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, int M, int K, T* __restrict__ out, int64_t ldo,
                     int tasks_per_row, int64_t num_tasks) {
    grid_dep_wait();
    const int lane = threadIdx.x & 31;
    const int ktiles = (K + kScaleTileBlocks * kMxBlock - 1) / (kScaleTileBlocks * kMxBlock);
    for (int64_t task = static_cast<int64_t>(blockIdx.x) * kWarps + (threadIdx.x >> 5); task < num_tasks;
         task += static_cast<int64_t>(gridDim.x) * kWarps) {
        const int row = static_cast<int>(task / tasks_per_row);
        const int k0 = static_cast<int>(task - static_cast<int64_t>(row) * tasks_per_row) * (kUnroll * kSegment) + lane * 8;
        const uint8_t* tile_row = scales + static_cast<int64_t>(row / kScaleTileRows) * ktiles * kScaleTileBytes + scale_in_tile(row % kScaleTileRows, 0);
        uint32_t c[kUnroll], s[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int k = k0 + u * kSegment, b = k / kMxBlock;
            c[u] = s[u] = 0;
            if (k < K) {
                c[u] = __ldcg(reinterpret_cast<const uint32_t*>(codes + static_cast<int64_t>(row) * (K / 2) + k / 2));
                s[u] = __ldcg(tile_row + static_cast<int64_t>(b / kScaleTileBlocks) * kScaleTileBytes + b % kScaleTileBlocks);
            }
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int k = k0 + u * kSegment;
            if (k < K) store8(out + row * ldo + k, mx_values8(c[u], s[u]));
        }
    }
}

// Launched so that it may be set up while the kernel ahead of it on the stream is finishing; it waits for that kernel
// before it touches global memory.
template <typename... P, typename... A>
cudaError_t launch_pdl(void (*kern)(P...), int grid, int threads, cudaStream_t st, A... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(threads);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kern, P(args)...);
}

int grid_for(int64_t num_tasks) {
    const int64_t ctas = (num_tasks + kWarps - 1) / kWarps, most = static_cast<int64_t>(sm_count()) * 8;
    return static_cast<int>(ctas < most ? ctas : most);
}

} // namespace

cudaError_t launch_mx_quantize(const void* x, bool fp32, int64_t ldx, int M, int K, uint8_t* codes, uint8_t* scales, int* status_to_clear,
                               bool early, cudaStream_t st) {
    const int tasks_per_row = (K + kUnroll * kSegment - 1) / (kUnroll * kSegment);
    const int64_t rows = (static_cast<int64_t>(M) + kScaleTileRows - 1) / kScaleTileRows * kScaleTileRows;
    const int64_t tasks = rows * tasks_per_row;
    if (fp32)
        return launch_pdl(mx_quantize_kernel<float>, grid_for(tasks), kWarps * 32, st, static_cast<const float*>(x), ldx, M, K, codes, scales,
                          tasks_per_row, tasks, status_to_clear, early ? 1 : 0);
    return launch_pdl(mx_quantize_kernel<__nv_bfloat16>, grid_for(tasks), kWarps * 32, st, static_cast<const __nv_bfloat16*>(x), ldx, M, K, codes,
                      scales, tasks_per_row, tasks, status_to_clear, early ? 1 : 0);
}

cudaError_t launch_mx_dequantize(const uint8_t* codes, const uint8_t* scales, int M, int K, void* out, bool fp32, int64_t ldo, cudaStream_t st) {
    const int tasks_per_row = (K + kUnroll * kSegment - 1) / (kUnroll * kSegment);
    const int64_t tasks = static_cast<int64_t>(M) * tasks_per_row;
    if (fp32)
        return launch_pdl(mx_dequantize_kernel<float>, grid_for(tasks), kWarps * 32, st, codes, scales, M, K, static_cast<float*>(out), ldo,
                          tasks_per_row, tasks);
    return launch_pdl(mx_dequantize_kernel<__nv_bfloat16>, grid_for(tasks), kWarps * 32, st, codes, scales, M, K,
                      static_cast<__nv_bfloat16*>(out), ldo, tasks_per_row, tasks);
}

} // namespace w8a8
