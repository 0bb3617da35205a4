// Host-side encoding of tensor maps for TMA.
#pragma once

#include <cstdint>
#include <cuda.h>
#include <cuda_runtime.h>

namespace w8a8 {

using EncodeTiledFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                   const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

inline EncodeTiledFn encode_tiled_fn() {
    static EncodeTiledFn fn = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess) p = nullptr;
        return reinterpret_cast<EncodeTiledFn>(p);
    }();
    return fn;
}

// 2-D row-major tensor [rows, cols], row stride ld_bytes, box [box_rows, box_cols].
inline bool encode_map_2d(CUtensorMap* tm, CUtensorMapDataType dt, const void* ptr, uint64_t rows, uint64_t cols, uint64_t ld_bytes,
                          uint32_t box_rows, uint32_t box_cols, CUtensorMapSwizzle swizzle) {
    EncodeTiledFn enc = encode_tiled_fn();
    if (enc == nullptr) return false;
    cuuint64_t dims[2] = {cols, rows};
    cuuint64_t strides[1] = {ld_bytes};
    cuuint32_t box[2] = {box_cols, box_rows};
    cuuint32_t estr[2] = {1, 1};
    return enc(tm, dt, 2, const_cast<void*>(ptr), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle,
               CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// MXFP4 codes [rows, K/2] in boxes of box_rows x 128 bytes (256 elements), 128-byte swizzle.
inline bool encode_mx_codes(CUtensorMap* tm, const uint8_t* p, int rows, int K, int64_t ld_bytes, int box_rows) {
    return encode_map_2d(tm, CU_TENSOR_MAP_DATA_TYPE_UINT8, p, rows, K / 2, ld_bytes, box_rows, 128, CU_TENSOR_MAP_SWIZZLE_128B);
}

// MXFP4 scale tiles (128 rows x 4 blocks, 512 bytes) as rows of 128 words: a box of two is what 128 matrix rows need for 256
// elements along K. The second row of the last box of an odd number of tiles belongs to the next 128 rows (or is past the
// end, and reads as zeros): it is not used.
inline bool encode_mx_scales(CUtensorMap* tm, const uint8_t* s, int rows, int K) {
    const uint64_t tiles = static_cast<uint64_t>((rows + 127) / 128) * ((K + 127) / 128);
    return encode_map_2d(tm, CU_TENSOR_MAP_DATA_TYPE_UINT32, s, tiles, 128, 512, 2, 128, CU_TENSOR_MAP_SWIZZLE_NONE);
}

} // namespace w8a8
