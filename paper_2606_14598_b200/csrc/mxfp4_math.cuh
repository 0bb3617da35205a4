// Arithmetic of the MXFP4 format (OCP Microscaling: E2M1 elements, one E8M0 scale for 32 of them), shared by the
// quantizer, the linear's activation path and the cache. Device code only.
//
//   amax = max |x| of the block             e = max(floor(log2(amax)) - 2, -127)      scale byte = e + 127
//   code = rne_e2m1(x * 2^-e), saturated at +-6 (amax in (6, 8) * 2^e is the only case that saturates)
//   value = e2m1(code) * 2^e                a block holding Inf or NaN: scale byte 255 (NaN), codes 0
//
// Everything but the rounding to E2M1 is exact in binary32: multiplying by 2^-e only moves the exponent (results
// below 2^-126 are far under the smallest rounding boundary 0.25, so what subnormal rounding does to them cannot
// show), and value * 2^e fits bf16 for every code and every byte that the quantizer writes (0 to 252: the smallest, 2^-128, is a
// bf16 subnormal). Under the bytes 253 and 254 the largest codes stand for more than fp32 holds: they read as infinities.
#pragma once

#include <cstdint>
#include <cuda_bf16.h>

namespace w8a8 {

constexpr int kMxBlock = 32;                 // elements that share a scale
constexpr int kScaleTileRows = 128;          // rows of a scale tile
constexpr int kScaleTileBlocks = 4;          // blocks (of 32 along K) of a scale tile
constexpr int kScaleTileBytes = 512;

// Byte offset, inside its tile, of the scale of row r, block c: the order in which tcgen05.cp.32x128b.warpx4 spreads
// 32 rows of 16 bytes over the lanes of tensor memory, so that a tile goes from global memory to the MMA untouched.
__host__ __device__ __forceinline__ int scale_in_tile(int r, int c) { return 16 * (r & 31) + 4 * (r >> 5) + c; }

// Scale byte of a block from the bit pattern of its largest magnitude as binary32. For a normal number the exponent
// field minus 2 is floor(log2) - 2 + 127; zero and subnormals clamp to byte 0. Inf and NaN (patterns order above all
// finite magnitudes) give 255.
__device__ __forceinline__ uint32_t mx_scale_byte(uint32_t amax_bits) {
    const int f = static_cast<int>(amax_bits >> 23);
    return f == 255 ? 255u : static_cast<uint32_t>(max(f - 2, 0));
}
// 2^-e as binary32 for scale bytes 0..252 (a block with byte 255 is written as zeros: factor 0 and finite stand-ins)
__device__ __forceinline__ float mx_inverse_scale(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }
// 2^e as bf16 bits (byte 0 is the subnormal 2^-127, byte 255 NaN)
__device__ __forceinline__ uint32_t mx_scale_bf16(uint32_t byte) { return byte == 0u ? 0x0040u : byte == 255u ? 0x7fc0u : byte << 7; }

// Eight binary32 values, already multiplied by 2^-e, to eight E2M1 codes: element 0 in the lowest nibble.
__device__ __forceinline__ uint32_t e2m1x8(const float (&y)[8]) {
    uint32_t r;
    asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b2, %6, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b3, %8, %7;\n\t"
        "mov.b32 %0, {b0, b1, b2, b3};\n\t}"
        : "=r"(r) : "f"(y[0]), "f"(y[1]), "f"(y[2]), "f"(y[3]), "f"(y[4]), "f"(y[5]), "f"(y[6]), "f"(y[7]));
    return r;
}

// Two bf16 products, each rounded once
__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
    const __nv_bfloat162 r = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
    return *reinterpret_cast<const uint32_t*>(&r);
}
// Eight codes times 2^e as eight bf16 values. The magnitudes' upper and lower bytes come from two eight-entry byte tables (a byte
// permute takes three index bits a nibble), the signs from a table of two; the product with a power of two is exact.
__device__ __forceinline__ uint4 mx_values8(uint32_t codes, uint32_t byte) {
    const uint32_t s1 = mx_scale_bf16(byte), s = s1 | (s1 << 16);
    const uint32_t idx = codes & 0x77777777u, sign = (codes >> 3) & 0x11111111u;
    uint32_t v[4];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t c = idx >> (16 * i);
        const uint32_t hi = __byte_perm(0x3f3f3f00u, 0x40404040u, c) | __byte_perm(0x00008000u, 0u, sign >> (16 * i));     // 0 .5 1 1.5 2 3 4 6
        const uint32_t lo = __byte_perm(0xc0800000u, 0xc0804000u, c);
        v[2 * i] = mul_bf16x2(__byte_perm(lo, hi, 0x5140), s);
        v[2 * i + 1] = mul_bf16x2(__byte_perm(lo, hi, 0x7362), s);
    }
    return make_uint4(v[0], v[1], v[2], v[3]);
}

// Largest |bf16| bit pattern of eight packed values, as an integer: patterns of magnitudes order like the magnitudes,
// with Inf and then NaN on top, so a non-finite element cannot hide behind a maximum that skips NaN.
__device__ __forceinline__ uint32_t absmax_bits8(const uint4& v) {
    uint32_t m = __vmaxu2(v.x & 0x7fff7fffu, v.y & 0x7fff7fffu);
    m = __vmaxu2(m, __vmaxu2(v.z & 0x7fff7fffu, v.w & 0x7fff7fffu));
    return max(m >> 16, m & 0xffffu) << 16;
}
__device__ __forceinline__ void unpack_bf16x8(const uint4& v, float (&f)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(w[i] << 16);
        f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
// Codes of eight bf16 values whose block has this scale byte. The scaling is done in bf16: exact, but for values that land
// below 2^-126, which round to code 0 all the same.
__device__ __forceinline__ uint32_t mx_codes8(const uint4& x, uint32_t byte) {
    if (byte == 255u) return 0u;
    const uint32_t i1 = (254u - byte) << 7, inv = i1 | (i1 << 16);
    float y[8];
    unpack_bf16x8(make_uint4(mul_bf16x2(x.x, inv), mul_bf16x2(x.y, inv), mul_bf16x2(x.z, inv), mul_bf16x2(x.w, inv)), y);
    return e2m1x8(y);
}

} // namespace w8a8
