// Arithmetic of the per-row int8 quantizer (paper, "The quantization recipe (reused)": symmetric per-token /
// per-channel int8 with scale = absmax / 127, round half to even), shared by the quantizer kernels and by the
// one-kernel path for small problems. Device code only.
#pragma once

#include "ptx.cuh"

#include <cuda_bf16.h>

namespace w8a8 {

// q = clamp(rne(x / s)) with the IEEE quotient, the definition.
__device__ __forceinline__ int quant_exact(float x, float s) {
    return max(-127, min(127, __float2int_rn(__fdiv_rn(x, s))));
}

// The IEEE quotient without a division instruction. With inv = RN(1 / s) (correctly rounded, once
// per row), q0 = RN(x * inv) is within 1.5 ulp of x / s; one fma pair (remainder r0 = x - s * q0,
// exact; q1 = RN(q0 + r0 * inv)) makes it faithful, and by Markstein's theorem a second pair then
// yields exactly RN(x / s): if the reciprocal is correctly rounded and q is faithful, RN(q + r * inv)
// with the exact remainder r is the correctly rounded quotient (no over/underflow; scales outside
// [1e-30, 1e30] take the division instead). Adding 1.5 * 2^23 rounds the quotient to the nearest
// integer, ties to even, and leaves the code in the low byte of the sum; |x / s| <= 127 * (1 + 2^-23)
// so the clamp to [-127, 127] cannot bind.
struct RowScale {
    float s, inv;
    bool fast;      // false for degenerate scales: every element takes the division
};
__device__ __forceinline__ RowScale make_row_scale(float amax) {
    RowScale r;
    r.s = amax > 0.f ? __fdiv_rn(amax, 127.0f) : 1.0f;
    r.inv = __frcp_rn(r.s);
    r.fast = r.s >= 1e-30f && r.s <= 1e30f;
    return r;
}
constexpr float MAGIC = 12582912.0f;               // 1.5 * 2^23

// the code of x in the low byte of the result (upper bytes are don't-care)
__device__ __forceinline__ uint32_t quant1(float x, const RowScale& rs) {
    const float q0 = __fmul_rn(x, rs.inv);
    const float r0 = __fmaf_rn(-rs.s, q0, x);
    const float q1 = __fmaf_rn(r0, rs.inv, q0);
    const float r1 = __fmaf_rn(-rs.s, q1, x);
    const float q2 = __fmaf_rn(r1, rs.inv, q1);
    return __float_as_uint(__fadd_rn(q2, MAGIC));
}
__device__ __forceinline__ uint32_t quant4(float a, float b, float c, float d, const RowScale& rs) {
    if (rs.fast) {
        const uint32_t lo = __byte_perm(quant1(a, rs), quant1(b, rs), 0x0040);
        const uint32_t hi = __byte_perm(quant1(c, rs), quant1(d, rs), 0x0040);
        return __byte_perm(lo, hi, 0x5410);
    }
    return (uint32_t(quant_exact(a, rs.s)) & 0xffu) | ((uint32_t(quant_exact(b, rs.s)) & 0xffu) << 8) |
           ((uint32_t(quant_exact(c, rs.s)) & 0xffu) << 16) | (uint32_t(quant_exact(d, rs.s)) << 24);
}

// |x| maximum of 8 packed bf16 values, kept packed (two running maxima)
__device__ __forceinline__ __nv_bfloat162 absmax8(const uint4& v, __nv_bfloat162 m) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) m = __hmax2(m, __habs2(*reinterpret_cast<const __nv_bfloat162*>(&w[i])));
    return m;
}
__device__ __forceinline__ float unpack_max(__nv_bfloat162 m) {
    const uint32_t mb = *reinterpret_cast<const uint32_t*>(&m);
    return fmaxf(__uint_as_float(mb << 16), __uint_as_float(mb & 0xffff0000u));
}
// Two quotients at a time with the packed fp32x2 instructions (each half rounds exactly like the scalar
// instruction): the same sequence as quant1 on a pair of values held in one 64-bit register.
struct RowScale2 {          // RowScale with its constants replicated into both halves
    uint64_t neg_s, inv, magic;
    uint64_t inv_hi, inv_lo;        // the reciprocal in two pieces, for bf16 inputs (see quant2)
};
__device__ __forceinline__ RowScale2 make_row_scale2(const RowScale& rs) {
    // inv_hi: the reciprocal cut to 16 significant bits; inv_lo: what is missing to 1 / s, to ~2^-39 of it
    const float inv_hi = __uint_as_float(__float_as_uint(rs.inv) & 0xffffff00u);
    const float inv_lo = rs.fast ? __fdiv_rn(__fmaf_rn(-rs.s, inv_hi, 1.0f), rs.s) : 0.f;
    return RowScale2{pack2(-rs.s, -rs.s), pack2(rs.inv, rs.inv), pack2(MAGIC, MAGIC), pack2(inv_hi, inv_hi), pack2(inv_lo, inv_lo)};
}
// Codes of the two bf16 values of `w` in byte 0 and byte 4 of the result. A bf16 value has 8 significant bits, so its
// product with the 16-bit inv_hi is exact; one fma adds x * inv_lo and rounds once: a faithful quotient (within an ulp
// of x / s) in two operations instead of three. The remainder pair then makes it the correctly rounded one as above.
__device__ __forceinline__ uint64_t quant2(uint32_t w, const RowScale2& r2) {
    const uint64_t x = pack2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
    const uint64_t p = mul2(x, r2.inv_hi);
    const uint64_t q1 = fma2(x, r2.inv_lo, p);
    const uint64_t r1 = fma2(r2.neg_s, q1, x);
    const uint64_t q2 = fma2(r1, r2.inv, q1);
    return add2(q2, r2.magic);
}
// Codes of two fp32 values in byte 0 and byte 4: the sequence of quant1 on a pair.
__device__ __forceinline__ uint64_t quant2f(uint64_t x, const RowScale2& r2) {
    const uint64_t q0 = mul2(x, r2.inv);
    const uint64_t q1 = fma2(fma2(r2.neg_s, q0, x), r2.inv, q0);
    const uint64_t q2 = fma2(fma2(r2.neg_s, q1, x), r2.inv, q1);
    return add2(q2, r2.magic);
}
__device__ __forceinline__ uint32_t gather4(uint64_t a, uint64_t b) {   // bytes 0 and 4 of a, then of b
    const uint32_t lo = __byte_perm(static_cast<uint32_t>(a), static_cast<uint32_t>(a >> 32), 0x0040);
    const uint32_t hi = __byte_perm(static_cast<uint32_t>(b), static_cast<uint32_t>(b >> 32), 0x0040);
    return __byte_perm(lo, hi, 0x5410);
}
// Four fp32 values -> four codes
__device__ __forceinline__ uint32_t quant4f(float a, float b, float c, float d, const RowScale& rs, const RowScale2& r2) {
    if (rs.fast) return gather4(quant2f(pack2(a, b), r2), quant2f(pack2(c, d), r2));
    return quant4(a, b, c, d, rs);
}
// amax / 127 and its reciprocal without a division (Markstein's theorem, as above): 1 / 127 correctly rounded, a faithful quotient and its exact
// remainder give the correctly rounded quotient. Scales near the ends of the range, where a remainder could underflow, take the division.
__device__ __forceinline__ RowScale head_scale(float amax) {
    if (amax < 1e-25f || amax > 1e25f) return make_row_scale(amax);
    const float inv127 = 1.0f / 127.0f;
    const float q = __fmul_rn(amax, inv127);
    const float s = __fmaf_rn(__fmaf_rn(-127.0f, q, amax), inv127, q);
    return RowScale{s, __frcp_rn(s), true};
}
// What quant8 needs of a scale; the low part of the reciprocal to 2^-40 of it (by a multiplication: its own error is 2^-24 of 2^-16)
__device__ __forceinline__ RowScale2 head_scale2(const RowScale& rs) {
    const float inv_hi = __uint_as_float(__float_as_uint(rs.inv) & 0xffffff00u);
    const float inv_lo = rs.fast ? __fmul_rn(__fmaf_rn(-rs.s, inv_hi, 1.0f), rs.inv) : 0.f;
    return RowScale2{pack2(-rs.s, -rs.s), pack2(rs.inv, rs.inv), pack2(MAGIC, MAGIC), pack2(inv_hi, inv_hi), pack2(inv_lo, inv_lo)};
}
// 8 packed bf16 -> 8 int8 codes (bf16 -> fp32 is exact: the 16 bits become the high half of the word)
__device__ __forceinline__ uint2 quant8(const uint4& v, const RowScale& rs, const RowScale2& r2) {
    if (rs.fast)
        return make_uint2(gather4(quant2(v.x, r2), quant2(v.y, r2)), gather4(quant2(v.z, r2), quant2(v.w, r2)));
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    float f[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(w[i] << 16);
        f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
    return make_uint2(quant4(f[0], f[1], f[2], f[3], rs), quant4(f[4], f[5], f[6], f[7], rs));
}

} // namespace w8a8
