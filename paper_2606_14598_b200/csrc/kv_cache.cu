// Paged cache of keys and values in few bits: quantized as it is written, read back as bf16.
//
//   int8   per (token, head): s = amax > 0 ? amax / 127 : 1, q = clamp(rne(x / s), +-127)    value = q * s
//   MXFP4  per block of 32 along the head (a head's last block may be shorter): see mxfp4_math.cuh
//
// Both directions move bytes: a write reads 2 and stores 1 (or 0.53) bytes an element, a read loads 1 (0.53) and stores
// 2. A lane takes 8 elements of a read, 16 of a write where sizes, strides and addresses allow it, else 8. All offsets into the
// cache are 64-bit.
//
// What bounds them, keys and values of 8 x 128 a token: HBM, at 6.5 TB/s of copy bandwidth. Reads: 120000 int8 tokens 120 us =
// 6.2 TB/s, 230000 MXFP4 tokens 200 us = 5.9 TB/s (16 elements a lane and 32-byte stores: no faster, not kept); small ones
// the chain sequence - page - codes (512 tokens of 36 x 128 5.5 us). Writes: 230000 MXFP4 tokens 183 us = 6.5 TB/s; int8 the
// instructions of the exact quotient, 120000 tokens 137 us = 5.4 TB/s (189 us with 8 elements a lane). Writes of heads that do not
// fill their lanes (int8: the next power of two; MXFP4: whole blocks of 32) pay for the idle ones: 8220 tokens of 16 x 72 take
// 35.0 us in int8 and 15.6 in MXFP4, for 9 and 7 us worth of bytes.
#include "../../include/kv_cache.h"
#include "internal.h"
#include "mxfp4_math.cuh"
#include "ptx.cuh"
#include "quant_math.cuh"

namespace w8a8 {
namespace {

constexpr int kThreads = 256;

struct Side {                      // keys or values
    const __nv_bfloat16* x;        // new tokens (write)
    int64_t st, sh;                // their strides in elements: token, head
    uint8_t* codes;
    void* scales;
    __nv_bfloat16* out;            // tokens read back (read)
    int64_t ot, oh;                // its strides
};

// How a CTA covers tokens: its threads stand for `width` lanes' worth of a token (slice blockIdx.y of it), `subs` tokens side by
// side, and go down the CTA's tokens with what they do within a token fixed: no index arithmetic per element.
struct Cover {
    int width, subs, slices, threads;
};
Cover make_cover(int lanes) {
    Cover c{};
    c.slices = (lanes + kThreads - 1) / kThreads;
    c.width = ((lanes + c.slices - 1) / c.slices + 31) / 32 * 32;
    if (c.slices == 1) c.width = lanes;
    c.subs = kThreads / c.width;
    c.threads = (c.subs * c.width + 31) / 32 * 32;
    return c;
}

// amax / 127 and its reciprocal without a division (Markstein's theorem, as in quant_math.cuh): 1 / 127 correctly rounded, a
// faithful quotient and its exact remainder give the correctly rounded quotient. Scales near the ends of the range, where a
// remainder could underflow, take the division.
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

// A unit is what shares a scale: a head of a token (int8) or a block of 32 of it (MXFP4); 2^lane_shift lanes, E elements each. 16
// elements a lane, loaded as 32 bytes, where sizes, strides and addresses allow it: what a unit costs beside its elements (its
// maximum, scale and places) is then shared by twice as many; else 8. Keys and values of UNROLL tokens are in flight at once.
template <int FMT, bool VALUES, int E>
__global__ void __launch_bounds__(kThreads, FMT == KV_CACHE_INT8 ? 3 : 4)
kv_write_kernel(const Side k, const Side v, const int64_t* slots, int64_t num_slots, int64_t tokens, int heads, int dim, int lane_shift, int tile,
                const Cover cover) {
    constexpr int UNROLL = E == 16 ? 2 : 4, SIDES = VALUES ? 2 : 1, WORDS = E / 2;
    grid_dep_wait();
    const int sub = static_cast<int>(threadIdx.x) / cover.width;
    const int lane = blockIdx.y * cover.width + static_cast<int>(threadIdx.x) - sub * cover.width;
    const int unit = lane >> lane_shift, gl = lane & ((1 << lane_shift) - 1);
    const int blocks = FMT == KV_CACHE_INT8 ? 1 : (dim + kMxBlock - 1) / kMxBlock;       // units of a head
    const int head = unit / blocks, d = (unit - head * blocks) * kMxBlock + gl * E;
    const bool mine = sub < cover.subs && head < heads && d < dim;
    const int64_t k_off = head * k.sh + d, v_off = VALUES ? head * v.sh + d : 0;
    const int code_off = FMT == KV_CACHE_INT8 ? head * dim + d : (head * dim + d) / 2;
    const int64_t token_codes = static_cast<int64_t>(heads) * dim / (FMT == KV_CACHE_INT8 ? 1 : 2), token_scales = static_cast<int64_t>(heads) * blocks;
    auto load = [](const __nv_bfloat16* p, uint32_t (&r)[WORDS]) {
        if (E == 16) {
            ldcg_32(p, r);
        } else {
            const uint4 q = __ldcg(reinterpret_cast<const uint4*>(p));
            r[0] = q.x; r[1] = q.y; r[2] = q.z; r[3] = q.w;
        }
    };
    for (int64_t t0 = static_cast<int64_t>(blockIdx.x) * tile; t0 < tokens; t0 += static_cast<int64_t>(gridDim.x) * tile) {
        const int count = static_cast<int>(tokens - t0 < tile ? tokens - t0 : tile);
        for (int base = 0; base < count; base += UNROLL * cover.subs) {          // (uniform: every lane takes part in the shuffles)
            uint32_t x[UNROLL][SIDES][WORDS];
            int64_t slot[UNROLL];
#pragma unroll
            for (int j = 0; j < UNROLL; ++j) {
                const int tt = base + j * cover.subs + sub;
                slot[j] = -1;
                if (mine && tt < count) {
                    const int64_t t = t0 + tt;
                    slot[j] = __ldcg(slots + t);
                    load(k.x + t * k.st + k_off, x[j][0]);
                    if (VALUES) load(v.x + t * v.st + v_off, x[j][SIDES - 1]);
                } else {
#pragma unroll
                    for (int q = 0; q < SIDES; ++q)
#pragma unroll
                        for (int i = 0; i < WORDS; ++i) x[j][q][i] = 0;
                }
            }
#pragma unroll
            for (int j = 0; j < UNROLL; ++j) {
                if (base + j * cover.subs >= count) break;                       // uniform
                const bool store = slot[j] >= 0 && slot[j] < num_slots;
#pragma unroll
                for (int q = 0; q < SIDES; ++q) {
                    const Side& s = q == 0 ? k : v;
                    uint4 part[E / 8];
                    uint32_t m = 0;
#pragma unroll
                    for (int i = 0; i < E / 8; ++i) {
                        part[i] = make_uint4(x[j][q][4 * i], x[j][q][4 * i + 1], x[j][q][4 * i + 2], x[j][q][4 * i + 3]);
                        m = max(m, absmax_bits8(part[i]));
                    }
                    if (FMT == KV_CACHE_INT8) {
                        for (int o = 1; o < 1 << lane_shift; o <<= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
                        // (every lane of a head works the scale out: sharing the scales of several tokens out over the lanes and passing
                        // them on by shuffles was slower, 206 against 198 us on 120000 tokens of 8 x 128 and 3.8 against 2.2 us on 48)
                        const bool finite = m < 0x7f800000u;
                        const RowScale rs = head_scale(finite ? __uint_as_float(m) : 0.f);
                        const RowScale2 r2 = head_scale2(rs);
                        uint2 c[E / 8];
#pragma unroll
                        for (int i = 0; i < E / 8; ++i) c[i] = finite ? quant8(part[i], rs, r2) : make_uint2(0, 0);
                        if (store) {
                            uint8_t* p = s.codes + slot[j] * token_codes + code_off;
                            if (E == 16) *reinterpret_cast<uint4*>(p) = make_uint4(c[0].x, c[0].y, c[E / 8 - 1].x, c[E / 8 - 1].y);
                            else *reinterpret_cast<uint2*>(p) = c[0];
                            if (gl == 0) static_cast<float*>(s.scales)[slot[j] * token_scales + unit] = finite ? rs.s : __uint_as_float(0x7fc00000u);
                        }
                    } else {
                        for (int o = 1; o < kMxBlock / E; o <<= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
                        const uint32_t byte = mx_scale_byte(m);
                        if (store) {
                            uint8_t* p = s.codes + slot[j] * token_codes + code_off;
                            if (E == 16) *reinterpret_cast<uint2*>(p) = make_uint2(mx_codes8(part[0], byte), mx_codes8(part[E / 8 - 1], byte));
                            else *reinterpret_cast<uint32_t*>(p) = mx_codes8(part[0], byte);
                            if (gl == 0) static_cast<uint8_t*>(s.scales)[slot[j] * token_scales + unit] = static_cast<uint8_t>(byte);
                        }
                    }
                }
            }
        }
    }
}

template <int FMT, bool VALUES>
auto write_kernel(bool wide) { return wide ? kv_write_kernel<FMT, VALUES, 16> : kv_write_kernel<FMT, VALUES, 8>; }

constexpr int kMaxTile = 32;       // tokens whose places a CTA looks up at a time, at most

// Eight int8 codes times a scale as bf16: a code plus 128, put in the low byte of 2^23, is exact in binary32
__device__ __forceinline__ uint4 int8_values8(uint2 c, float s) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t two = (i < 2 ? c.x : c.y) ^ 0x80808080u;
        const float a = __uint_as_float(__byte_perm(two, 0x4b000000u, (i & 1) ? 0x7442 : 0x7440)) - 8388736.f;
        const float b = __uint_as_float(__byte_perm(two, 0x4b000000u, (i & 1) ? 0x7443 : 0x7441)) - 8388736.f;
        const __nv_bfloat162 p = __floats2bfloat162_rn(a * s, b * s);
        w[i] = *reinterpret_cast<const uint32_t*>(&p);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// A CTA takes tiles of consecutive output tokens: first their cache rows (one thread a token: its sequence, its page), then
// their elements, 8 a lane, keys and values of UNROLL tokens in flight at once.
template <int FMT, bool VALUES>
__global__ void __launch_bounds__(kThreads, 4)
kv_read_kernel(const Side k, const Side v, const int32_t* table, int64_t table_stride, int max_pages, const int32_t* cu, const int32_t* starts, int seqs,
               int64_t total, int64_t num_pages, int page, int heads, int dim, int zero_rest, int tile, const Cover cover) {
    constexpr int UNROLL = 4, SIDES = VALUES ? 2 : 1;
    grid_dep_wait();
    __shared__ int64_t slots[kMaxTile];                           // cache row of each token of the tile, -1: reads as zeros, -2: left alone
    __shared__ int first;
    __shared__ int32_t first_begin, first_end;
    const int sub = static_cast<int>(threadIdx.x) / cover.width;
    const int lane = blockIdx.y * cover.width + static_cast<int>(threadIdx.x) - sub * cover.width;
    const int per_head = dim / 8, blocks = (dim + kMxBlock - 1) / kMxBlock;
    const int head = lane / per_head, d = (lane - head * per_head) * 8;
    const bool mine = sub < cover.subs && head < heads;
    const int code_off = FMT == KV_CACHE_INT8 ? head * dim + d : (head * dim + d) / 2;
    const int scale_off = FMT == KV_CACHE_INT8 ? head : head * blocks + d / kMxBlock;
    const int64_t token_codes = static_cast<int64_t>(heads) * dim / (FMT == KV_CACHE_INT8 ? 1 : 2);
    const int64_t token_scales = static_cast<int64_t>(heads) * (FMT == KV_CACHE_INT8 ? 1 : blocks);
    const int64_t k_off = head * k.oh + d, v_off = VALUES ? head * v.oh + d : 0;
    for (int64_t t0 = static_cast<int64_t>(blockIdx.x) * tile; t0 < total; t0 += static_cast<int64_t>(gridDim.x) * tile) {
        const int count = static_cast<int>(total - t0 < tile ? total - t0 : tile);
        // the sequence of the tile's first token, found by all threads at once: the first one that ends after it
        if (threadIdx.x == 0) first = seqs;
        __syncthreads();
        for (int b0 = 0; b0 < seqs; b0 += blockDim.x) {
            const int b = b0 + static_cast<int>(threadIdx.x);
            const int32_t end = b < seqs ? __ldcg(cu + b + 1) : 0;
            const int32_t before = b < seqs ? __ldcg(cu + b) : 0;
            const bool here = b < seqs && end > t0 && (b == 0 || before <= t0);
            if (here) { first = b; first_begin = before; first_end = end; }
            if (__syncthreads_or(here)) break;
        }
        for (int i = threadIdx.x; i < count; i += blockDim.x) {
            const int64_t t = t0 + i;
            int b = first;
            int32_t begin = b < seqs ? first_begin : 0, end = b < seqs ? first_end : 0;
            while (b < seqs && end <= t) {
                begin = end;
                if (++b < seqs) end = __ldcg(cu + b + 1);
            }
            int64_t row = zero_rest ? -1 : -2;                    // of no sequence
            if (b < seqs) {
                if (t >= begin) {
                    const int64_t at = t - begin + (starts != nullptr ? __ldcg(starts + b) : 0);
                    row = -1;
                    if (at >= 0 && at < INT32_MAX) {
                        const uint32_t p = static_cast<uint32_t>(at) / static_cast<uint32_t>(page);
                        if (p < static_cast<uint32_t>(max_pages)) {
                            const int64_t id = __ldcg(table + b * table_stride + p);
                            if (id >= 0 && id < num_pages) row = id * page + (at - static_cast<int64_t>(p) * page);
                        }
                    }
                }
            }
            slots[i] = row;
        }
        __syncthreads();
        if (mine) {
            for (int tt0 = sub; tt0 < count; tt0 += UNROLL * cover.subs) {
                uint2 c[UNROLL][SIDES];
                uint32_t scale[UNROLL][SIDES];
                bool store[UNROLL];
#pragma unroll
                for (int j = 0; j < UNROLL; ++j) {
                    const int tt = tt0 + j * cover.subs;
                    const int64_t slot = tt < count ? slots[tt] : -2;
                    store[j] = slot != -2;
#pragma unroll
                    for (int q = 0; q < SIDES; ++q) {
                        c[j][q] = make_uint2(0, 0);
                        scale[j][q] = 0;
                        if (slot >= 0) {
                            const Side& s = q == 0 ? k : v;
                            const uint8_t* codes = s.codes + slot * token_codes + code_off;
                            if (FMT == KV_CACHE_INT8) {
                                c[j][q] = __ldcg(reinterpret_cast<const uint2*>(codes));
                                scale[j][q] = __ldcg(static_cast<const uint32_t*>(s.scales) + slot * token_scales + scale_off);
                            } else {
                                c[j][q].x = __ldcg(reinterpret_cast<const uint32_t*>(codes));
                                scale[j][q] = __ldcg(static_cast<const uint8_t*>(s.scales) + slot * token_scales + scale_off);
                            }
                        }
                    }
                }
#pragma unroll
                for (int j = 0; j < UNROLL; ++j) {
                    if (!store[j]) continue;
                    const int64_t t = t0 + tt0 + j * cover.subs;
#pragma unroll
                    for (int q = 0; q < SIDES; ++q) {
                        const uint4 o = FMT == KV_CACHE_INT8 ? int8_values8(c[j][q], __uint_as_float(scale[j][q])) : mx_values8(c[j][q].x, scale[j][q]);
                        __nv_bfloat16* p = q == 0 ? k.out + t * k.ot + k_off : v.out + t * v.ot + v_off;
                        *reinterpret_cast<uint4*>(p) = o;
                    }
                }
            }
        }
        __syncthreads();                                          // slots[] is rewritten for the next tile
    }
}

// Tokens of a tile: the CTAs that an SM holds at once (four) take all tokens in one go where that makes tiles of at most kMaxTile.
// (4096 tokens of 8 x 80: tiles of 3 in 2.3 rounds 10.2 us to read.)
int tile_for(int64_t tokens, int slices) {
    const int64_t ctas = static_cast<int64_t>(sm_count()) * 4, tile = (tokens * slices + ctas - 1) / ctas;
    return static_cast<int>(tile < 1 ? 1 : tile > kMaxTile ? kMaxTile : tile);
}

dim3 grid_for(int64_t tokens, int tile, const Cover& c) {
    const int64_t ctas = (tokens + tile - 1) / tile, most = (static_cast<int64_t>(sm_count()) * 16 + c.slices - 1) / c.slices;
    return dim3(static_cast<unsigned>(ctas < most ? ctas : most), c.slices);
}

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

int check_shape(int fmt, int64_t heads, int64_t dim) {
    if ((fmt != KV_CACHE_INT8 && fmt != KV_CACHE_MXFP4) || heads <= 0 || dim <= 0 || dim > KV_CACHE_MAX_DIM || heads > KV_CACHE_MAX_WIDTH ||
        heads * dim > KV_CACHE_MAX_WIDTH)
        return W8A8_ERR_INVALID_ARG;
    return dim % 8 == 0 ? W8A8_OK : W8A8_ERR_ALIGNMENT;
}

int check_store(int fmt, const void* codes, const void* scales, int64_t places) {
    if (places > 0 && (codes == nullptr || scales == nullptr)) return W8A8_ERR_INVALID_ARG;
    if (!aligned(codes, 16) || !aligned(scales, fmt == KV_CACHE_INT8 ? 4 : 1)) return W8A8_ERR_ALIGNMENT;
    return W8A8_OK;
}

} // namespace
} // namespace w8a8

extern "C" {

using namespace w8a8;

int kv_cache_write(int fmt, const void* k, int64_t k_token_stride, int64_t k_head_stride, const void* v, int64_t v_token_stride,
                   int64_t v_head_stride, const int64_t* slots, int64_t tokens, int64_t heads, int64_t dim, void* k_codes, void* k_scales,
                   void* v_codes, void* v_scales, int64_t num_slots, void* stream) {
    if (int e = check_shape(fmt, heads, dim)) return e;
    if (tokens < 0 || num_slots < 0 || (tokens > 0 && (k == nullptr || slots == nullptr))) return W8A8_ERR_INVALID_ARG;
    if (int e = check_store(fmt, k_codes, k_scales, num_slots)) return e;
    if (!aligned(k, 16) || k_token_stride % 8 != 0 || k_head_stride % 8 != 0 || !aligned(slots, 8)) return W8A8_ERR_ALIGNMENT;
    if (v != nullptr) {
        if (int e = check_store(fmt, v_codes, v_scales, num_slots)) return e;
        if (!aligned(v, 16) || v_token_stride % 8 != 0 || v_head_stride % 8 != 0) return W8A8_ERR_ALIGNMENT;
    }
    if (int e = check_arch()) return e;
    if (tokens == 0 || num_slots == 0) return W8A8_OK;
    auto wide_side = [](const void* p, int64_t token_stride, int64_t head_stride) { return aligned(p, 32) && token_stride % 16 == 0 && head_stride % 16 == 0; };
    const bool wide = dim % 16 == 0 && wide_side(k, k_token_stride, k_head_stride) && (v == nullptr || wide_side(v, v_token_stride, v_head_stride));
    const int each = wide ? 16 : 8;                                // elements a lane
    int lane_shift = 0;
    while ((each << lane_shift) < (fmt == KV_CACHE_INT8 ? dim : kMxBlock)) ++lane_shift;
    const int blocks = fmt == KV_CACHE_INT8 ? 1 : static_cast<int>((dim + kMxBlock - 1) / kMxBlock);
    Side ks{}, vs{};
    ks.x = static_cast<const __nv_bfloat16*>(k);
    ks.st = k_token_stride;
    ks.sh = k_head_stride;
    ks.codes = static_cast<uint8_t*>(k_codes);
    ks.scales = k_scales;
    vs.x = static_cast<const __nv_bfloat16*>(v);
    vs.st = v_token_stride;
    vs.sh = v_head_stride;
    vs.codes = static_cast<uint8_t*>(v_codes);
    vs.scales = v_scales;
    const Cover cover = make_cover(static_cast<int>(heads) * blocks << lane_shift);
    const int tile = tile_for(tokens, cover.slices);
    const auto kern = fmt == KV_CACHE_INT8 ? (v != nullptr ? write_kernel<KV_CACHE_INT8, true>(wide) : write_kernel<KV_CACHE_INT8, false>(wide))
                                           : (v != nullptr ? write_kernel<KV_CACHE_MXFP4, true>(wide) : write_kernel<KV_CACHE_MXFP4, false>(wide));
    const cudaError_t e = launch_pdl(kern, grid_for(tokens, tile, cover), cover.threads, static_cast<cudaStream_t>(stream), ks, vs, slots, num_slots, tokens,
                                     static_cast<int>(heads), static_cast<int>(dim), lane_shift, tile, cover);
    return e == cudaSuccess ? W8A8_OK : W8A8_ERR_CUDA;
}

int kv_cache_read(int fmt, const void* k_codes, const void* k_scales, const void* v_codes, const void* v_scales, int64_t num_pages, int64_t page_size,
                  int64_t heads, int64_t dim, const int32_t* table, int64_t table_stride, int64_t max_pages, const int32_t* cu_seqlens,
                  const int32_t* starts, int64_t seqs, int64_t total, void* k_out, int64_t k_token_stride, int64_t k_head_stride, void* v_out,
                  int64_t v_token_stride, int64_t v_head_stride, void* stream) {
    const bool zero_rest = (fmt & KV_CACHE_ZERO_REST) != 0;
    fmt &= ~KV_CACHE_ZERO_REST;
    if (int e = check_shape(fmt, heads, dim)) return e;
    if (num_pages < 0 || page_size <= 0 || page_size > INT32_MAX || max_pages < 0 || max_pages > INT32_MAX || table_stride < max_pages || seqs < 0 ||
        seqs > INT32_MAX - 1 || total < 0 || total > INT32_MAX || (total > 0 && k_out == nullptr) || (seqs > 0 && cu_seqlens == nullptr) ||
        (seqs > 0 && max_pages > 0 && table == nullptr))
        return W8A8_ERR_INVALID_ARG;
    if (int e = check_store(fmt, k_codes, k_scales, num_pages)) return e;
    if (!aligned(k_out, 16) || k_token_stride % 8 != 0 || k_head_stride % 8 != 0 || !aligned(table, 4) || !aligned(cu_seqlens, 4) || !aligned(starts, 4))
        return W8A8_ERR_ALIGNMENT;
    if (v_out != nullptr) {
        if (int e = check_store(fmt, v_codes, v_scales, num_pages)) return e;
        if (!aligned(v_out, 16) || v_token_stride % 8 != 0 || v_head_stride % 8 != 0) return W8A8_ERR_ALIGNMENT;
    }
    if (int e = check_arch()) return e;
    if (total == 0 || (seqs == 0 && !zero_rest)) return W8A8_OK;
    Side ks{}, vs{};
    ks.codes = static_cast<uint8_t*>(const_cast<void*>(k_codes));
    ks.scales = const_cast<void*>(k_scales);
    ks.out = static_cast<__nv_bfloat16*>(k_out);
    ks.ot = k_token_stride;
    ks.oh = k_head_stride;
    vs.codes = static_cast<uint8_t*>(const_cast<void*>(v_codes));
    vs.scales = const_cast<void*>(v_scales);
    vs.out = static_cast<__nv_bfloat16*>(v_out);
    vs.ot = v_token_stride;
    vs.oh = v_head_stride;
    const Cover cover = make_cover(static_cast<int>(heads * (dim / 8)));
    const int tile = tile_for(total, cover.slices);
    const auto kern = fmt == KV_CACHE_INT8 ? (v_out != nullptr ? kv_read_kernel<KV_CACHE_INT8, true> : kv_read_kernel<KV_CACHE_INT8, false>)
                                           : (v_out != nullptr ? kv_read_kernel<KV_CACHE_MXFP4, true> : kv_read_kernel<KV_CACHE_MXFP4, false>);
    const cudaError_t e = launch_pdl(kern, grid_for(total, tile, cover), cover.threads, static_cast<cudaStream_t>(stream), ks, vs, table, table_stride,
                                     static_cast<int>(max_pages), cu_seqlens, starts, static_cast<int>(seqs), total, num_pages, static_cast<int>(page_size),
                                     static_cast<int>(heads), static_cast<int>(dim), zero_rest ? 1 : 0, tile, cover);
    return e == cudaSuccess ? W8A8_OK : W8A8_ERR_CUDA;
}

} // extern "C"
