// MXFP4 quantizer and its inverse: rows of bf16 or fp32 to packed E2M1 codes and tiles of E8M0 scales, and back.
// Both move bytes and compute next to nothing (a conversion and a multiply an element): HBM is the bound, 2.53 bytes an
// element for bf16, 4.53 for fp32.
//
// A lane holds 16 consecutive elements of a row, two neighbouring lanes one block of 32, a warp one segment of 512: codes
// leave as 8 bytes a lane, the block's maximum takes one shuffle, and a segment's 16 scale bytes leave as four 4-byte
// words (one for each tile of four blocks that the segment crosses). Where the rows allow it a lane moves 32 bytes at
// a time, so that every memory sector is touched by one instruction.
//
// Measured: 13824 x 4608 fp32 42.3 us to codes and 44.4 us back (6.8 and 6.5 TB/s; the copy that gives 6.5 TB/s writes half of its bytes,
// the quantizer a ninth, and what it wrote last is still in L2 when it ends); 4110 x 12288 bf16 21.7 and 21.7 us (5.9 TB/s;
// 24.1 and 21.9 us when every segment worked out its own addresses, 12 instructions an element); 77 x 4608 1.9 and 1.9 us, launch.
#include "internal.h"
#include "mxfp4_math.cuh"
#include "ptx.cuh"

namespace w8a8 {
namespace {

constexpr int kWarps = 8;
constexpr int kLane = 16;            // elements a lane takes at a time
constexpr int kSegment = 32 * kLane;
// Rows whose segments a warp takes together: divisors of the 32 rows that lie 16 bytes apart in a scale tile. (Twice as many, with
// four CTAs an SM: 20.4 against 21.1 us for 4110 x 12288 bf16, but 2.1 against 1.7 us for 77 x 4608 and 9.6 against 9.4 us for 4110 x 4608.)
template <typename T> constexpr int quantize_rows = sizeof(T) == 2 ? 2 : 1;
constexpr int kDequantizeRows = 2;

// N 16-byte words at p: WIDE = p is 32-byte aligned. Coherent loads past L1: the kernel may be resident while the one ahead writes.
template <int N, bool WIDE>
__device__ __forceinline__ void load_words(const void* p, uint32_t (&r)[4 * N]) {
    if (WIDE) {
#pragma unroll
        for (int i = 0; i < N / 2; ++i) ldcg_32(static_cast<const uint8_t*>(p) + 32 * i, r + 8 * i);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint4 v = __ldcg(static_cast<const uint4*>(p) + i);
            r[4 * i] = v.x; r[4 * i + 1] = v.y; r[4 * i + 2] = v.z; r[4 * i + 3] = v.w;
        }
    }
}
template <int N, bool WIDE>
__device__ __forceinline__ void store_words(void* p, const uint32_t (&r)[4 * N]) {
    if (WIDE) {
#pragma unroll
        for (int i = 0; i < N / 2; ++i) st_32(static_cast<uint8_t*>(p) + 32 * i, r + 8 * i);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) static_cast<uint4*>(p)[i] = make_uint4(r[4 * i], r[4 * i + 1], r[4 * i + 2], r[4 * i + 3]);
    }
}

// bit pattern of the largest magnitude of 16 elements, as binary32
__device__ __forceinline__ uint32_t absmax_bits(const uint32_t (&r)[8]) {
    uint32_t m = r[0] & 0x7fff7fffu;
#pragma unroll
    for (int i = 1; i < 8; ++i) m = __vmaxu2(m, r[i] & 0x7fff7fffu);
    return max(m >> 16, m & 0xffffu) << 16;
}
__device__ __forceinline__ uint32_t absmax_bits(const uint32_t (&r)[16]) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) m = max(m, r[i] & 0x7fffffffu);
    return m;
}
// codes of 16 elements whose block has this scale byte
__device__ __forceinline__ uint2 codes_of(const uint32_t (&r)[8], uint32_t byte) {
    return make_uint2(mx_codes8(make_uint4(r[0], r[1], r[2], r[3]), byte), mx_codes8(make_uint4(r[4], r[5], r[6], r[7]), byte));
}
__device__ __forceinline__ uint2 codes_of(const uint32_t (&r)[16], uint32_t byte) {
    if (byte == 255u) return make_uint2(0, 0);
    const float inv = mx_inverse_scale(byte);
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = __uint_as_float(r[i]) * inv;
    const uint32_t lo = e2m1x8(y);
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = __uint_as_float(r[8 + i]) * inv;
    return make_uint2(lo, e2m1x8(y));
}

// A warp's task: the same segment of ROWS consecutive rows, so that what addresses take is worked out once for all of them.
struct Task {
    int row, k;
};
__device__ __forceinline__ Task task_of(int64_t task, int per_row, int rows) {
    // 32-bit division wherever the numbers allow it
    const int64_t group = task <= 0xffffffffll ? static_cast<uint32_t>(task) / static_cast<uint32_t>(per_row) : task / per_row;
    return Task{static_cast<int>(group) * rows, static_cast<int>(task - group * per_row) * kSegment + static_cast<int>(threadIdx.x & 31) * kLane};
}
// Scale tiles of a row's k-th element: the row's four bytes in the tile. Rows of a task share a tile and are 16 bytes apart.
__device__ __forceinline__ int64_t scale_offset(int row, int k, int ktiles) {
    return (static_cast<int64_t>(row / kScaleTileRows) * ktiles + k / (kScaleTileBlocks * kMxBlock)) * kScaleTileBytes + scale_in_tile(row % kScaleTileRows, 0);
}

// Rows go up to the end of the last scale tile: rows past M get zero scales, so that a scale tensor's contents depend on nothing but x.
template <typename T, bool WIDE>
__global__ void __launch_bounds__(kWarps * 32, 6)
mx_quantize_kernel(const T* x, int64_t ldx, int M, int K, uint8_t* __restrict__ codes, uint8_t* __restrict__ scales, int per_row, int64_t num_tasks,
                   int* status_to_clear, int early) {
    constexpr int WORDS = kLane * sizeof(T) / 4, ROWS = quantize_rows<T>;
    if (early) grid_dep_launch_dependents();
    grid_dep_wait();
    if (status_to_clear != nullptr && blockIdx.x == 0 && threadIdx.x == 0) *status_to_clear = 0;
    const int lane = threadIdx.x & 31;
    const int ktiles = (K + kScaleTileBlocks * kMxBlock - 1) / (kScaleTileBlocks * kMxBlock);
    const int64_t step = static_cast<int64_t>(gridDim.x) * kWarps;
    for (int64_t task = static_cast<int64_t>(blockIdx.x) * kWarps + (threadIdx.x >> 5); task < num_tasks; task += step) {
        const Task at = task_of(task, per_row, ROWS);
        const T* src = x + at.row * ldx + at.k;
        uint32_t r[ROWS][WORDS];
#pragma unroll
        for (int u = 0; u < ROWS; ++u) {
            if (at.row + u < M && at.k < K) {
                load_words<WORDS / 4, WIDE>(src + u * ldx, r[u]);
            } else {
#pragma unroll
                for (int i = 0; i < WORDS; ++i) r[u][i] = 0;
            }
        }
        uint8_t* dst = codes + static_cast<int64_t>(at.row) * (K / 2) + at.k / 2;
        uint8_t* sdst = scales + scale_offset(at.row, at.k, ktiles);
        const bool writes_scales = (lane & 7) == 0 && at.k / (kScaleTileBlocks * kMxBlock) < ktiles;
#pragma unroll
        for (int u = 0; u < ROWS; ++u) {
            uint32_t m = absmax_bits(r[u]);
            m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
            const uint32_t byte = mx_scale_byte(m);
            const uint2 c = codes_of(r[u], byte);
            // the four blocks of a tile sit in 8 lanes: two shuffles bring their bytes into one word
            uint32_t word = byte << (((lane >> 1) & 3) * 8);
            word |= __shfl_xor_sync(0xffffffffu, word, 2);
            word |= __shfl_xor_sync(0xffffffffu, word, 4);
            if (at.row + u < M && at.k < K) *reinterpret_cast<uint2*>(dst + u * static_cast<int64_t>(K / 2)) = c;
            if (writes_scales) *reinterpret_cast<uint32_t*>(sdst + 16 * u) = word;
        }
    }
}

template <typename T, bool WIDE>
__global__ void __launch_bounds__(kWarps * 32, 6)
mx_dequantize_kernel(const uint8_t* codes, const uint8_t* scales, int M, int K, T* __restrict__ out, int64_t ldo, int per_row, int64_t num_tasks) {
    constexpr int ROWS = kDequantizeRows;
    grid_dep_wait();
    const int ktiles = (K + kScaleTileBlocks * kMxBlock - 1) / (kScaleTileBlocks * kMxBlock);
    const int64_t step = static_cast<int64_t>(gridDim.x) * kWarps;
    for (int64_t task = static_cast<int64_t>(blockIdx.x) * kWarps + (threadIdx.x >> 5); task < num_tasks; task += step) {
        const Task at = task_of(task, per_row, ROWS);
        if (at.k >= K) continue;
        const uint8_t* src = codes + static_cast<int64_t>(at.row) * (K / 2) + at.k / 2;
        const uint8_t* ssrc = scales + scale_offset(at.row, at.k, ktiles) + at.k / kMxBlock % kScaleTileBlocks;
        T* dst = out + at.row * ldo + at.k;
        uint2 c[ROWS];
        uint32_t b[ROWS];
#pragma unroll
        for (int u = 0; u < ROWS; ++u) {
            c[u] = make_uint2(0, 0);
            b[u] = 0;
            if (at.row + u < M) {
                c[u] = __ldcg(reinterpret_cast<const uint2*>(src + u * static_cast<int64_t>(K / 2)));
                b[u] = __ldcg(ssrc + 16 * u);
            }
        }
#pragma unroll
        for (int u = 0; u < ROWS; ++u) {
            if (at.row + u < M) {
                const uint4 lo = mx_values8(c[u].x, b[u]), hi = mx_values8(c[u].y, b[u]);
                const uint32_t v[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
                if (sizeof(T) == 2) {
                    store_words<2, WIDE>(dst + u * ldo, v);
                } else {
                    uint32_t f[16];
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        f[2 * i] = v[i] << 16;
                        f[2 * i + 1] = v[i] & 0xffff0000u;
                    }
                    store_words<4, WIDE>(dst + u * ldo, f);
                }
            }
        }
    }
}

// One task a warp up to 64 CTAs an SM. (Twice the bytes a warp and CTAs that walk over the rest, 8 an SM, before tasks were rows: 25.1
// against 24.2 us to quantize 4110 x 12288 bf16, 47.9 against 42.3 us for 13824 x 4608 fp32, 2.5 against 1.9 us for 77 x 4608.)
int grid_for(int64_t num_tasks) {
    const int64_t ctas = (num_tasks + kWarps - 1) / kWarps, most = static_cast<int64_t>(sm_count()) * 64;
    return static_cast<int>(ctas < most ? ctas : most);
}

bool aligned32(const void* p, int64_t row_bytes) { return ((reinterpret_cast<uintptr_t>(p) | static_cast<uintptr_t>(row_bytes)) & 31u) == 0; }

template <typename T, bool WIDE>
cudaError_t quantize(const void* x, int64_t ldx, int M, int K, uint8_t* codes, uint8_t* scales, int* status_to_clear, bool early, cudaStream_t st) {
    const int per_row = (K + kSegment - 1) / kSegment;
    const int64_t rows = (static_cast<int64_t>(M) + kScaleTileRows - 1) / kScaleTileRows * kScaleTileRows, tasks = rows / quantize_rows<T> * per_row;
    return launch_pdl(mx_quantize_kernel<T, WIDE>, dim3(grid_for(tasks)), kWarps * 32, st, static_cast<const T*>(x), ldx, M, K, codes, scales, per_row, tasks,
                      status_to_clear, early ? 1 : 0);
}
template <typename T, bool WIDE>
cudaError_t dequantize(const uint8_t* codes, const uint8_t* scales, int M, int K, void* out, int64_t ldo, cudaStream_t st) {
    const int per_row = (K + kSegment - 1) / kSegment;
    const int64_t tasks = (static_cast<int64_t>(M) + kDequantizeRows - 1) / kDequantizeRows * per_row;
    return launch_pdl(mx_dequantize_kernel<T, WIDE>, dim3(grid_for(tasks)), kWarps * 32, st, codes, scales, M, K, static_cast<T*>(out), ldo, per_row, tasks);
}

} // namespace

cudaError_t launch_mx_quantize(const void* x, bool fp32, int64_t ldx, int M, int K, uint8_t* codes, uint8_t* scales, int* status_to_clear,
                               bool early, cudaStream_t st) {
    const bool wide = aligned32(x, ldx * (fp32 ? 4 : 2));
    if (fp32)
        return wide ? quantize<float, true>(x, ldx, M, K, codes, scales, status_to_clear, early, st)
                    : quantize<float, false>(x, ldx, M, K, codes, scales, status_to_clear, early, st);
    return wide ? quantize<__nv_bfloat16, true>(x, ldx, M, K, codes, scales, status_to_clear, early, st)
                : quantize<__nv_bfloat16, false>(x, ldx, M, K, codes, scales, status_to_clear, early, st);
}

cudaError_t launch_mx_dequantize(const uint8_t* codes, const uint8_t* scales, int M, int K, void* out, bool fp32, int64_t ldo, cudaStream_t st) {
    const bool wide = aligned32(out, ldo * (fp32 ? 4 : 2));
    if (fp32)
        return wide ? dequantize<float, true>(codes, scales, M, K, out, ldo, st) : dequantize<float, false>(codes, scales, M, K, out, ldo, st);
    return wide ? dequantize<__nv_bfloat16, true>(codes, scales, M, K, out, ldo, st)
                : dequantize<__nv_bfloat16, false>(codes, scales, M, K, out, ldo, st);
}

} // namespace w8a8
