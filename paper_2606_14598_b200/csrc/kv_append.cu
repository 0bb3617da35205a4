// New tokens on their way into the quantized cache: queries and keys rotated by position, keys and values quantized into their slots.
//
//   a' = a c - b s,  b' = b c + a s     (c, s) of a pair from the table row of the token's position on the pair's axis
//
// Products and sums are fp32 and rounded once each (no fused multiply-add), so that codes are specified to the bit. Keys go from fp32 to
// codes: rounding them to bf16 in between, as a rotation in a pass of its own would, loses a bit for nothing.
#include "../../include/kv_cache.h"
#include "internal.h"
#include "mxfp4_math.cuh"
#include "ptx.cuh"
#include "quant_math.cuh"

#include <cmath>

namespace w8a8 {
namespace {

constexpr int kThreads = 256;
enum { ROPE_NONE = 0, ROPE_HALVES = 1, ROPE_PAIRS = 2 };

struct Vectors {                   // bf16 [tokens, heads, dim]
    const __nv_bfloat16* x;
    int64_t st, sh;
};
struct Store {
    uint8_t* codes;
    void* scales;
};
struct AppendArgs {
    Vectors q, k, v;
    __nv_bfloat16* q_out;
    int64_t q_out_st, q_out_sh;
    Store ks, vs;
    const float* table;
    const int64_t *positions, *slots;
    const uint8_t* axis_of;
    int64_t position_stride, num_positions, num_slots, tokens;
    int q_heads, heads, dim, rot, axes;
    int lanes, subs, lane_shift;   // lanes of a head, heads side by side in a CTA, log2 of the lanes that share an int8 scale
};

// cos and sin of the eight elements that a lane holds, two groups of four that turn, each by the angles of its own pairs: four (pairs side by side:
// elements 2i and 2i + 1 share them) or eight. Kept while the lane walks the heads of its token.
template <int ROPE>
struct Turn {
    static constexpr int N = ROPE == ROPE_PAIRS ? 4 : 8;
    float c[N], s[N];
    bool on[2];                    // whether the group turns at all
    int64_t other[2];              // distance of a group's partners (halves)
};

template <int ROPE>
__device__ __forceinline__ void four_pairs(const AppendArgs& a, int64_t t, int pair, float* c, float* s) {
    int axis[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) axis[i] = a.axis_of != nullptr ? a.axis_of[pair + i] : 0;
    if (axis[0] == axis[1] && axis[0] == axis[2] && axis[0] == axis[3]) {
        const int64_t p = axis[0] < a.axes ? a.positions[axis[0] * a.position_stride + t] : -1;
        if (p >= 0 && p < a.num_positions) {
            const float* row = a.table + p * a.rot + pair;
            const float4 u = *reinterpret_cast<const float4*>(row), w = *reinterpret_cast<const float4*>(row + a.rot / 2);
            c[0] = u.x; c[1] = u.y; c[2] = u.z; c[3] = u.w;
            s[0] = w.x; s[1] = w.y; s[2] = w.z; s[3] = w.w;
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) c[i] = s[i] = __uint_as_float(0x7fc00000u);
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t p = axis[i] < a.axes ? a.positions[axis[i] * a.position_stride + t] : -1;
        const bool in = p >= 0 && p < a.num_positions;
        c[i] = in ? a.table[p * a.rot + pair + i] : __uint_as_float(0x7fc00000u);
        s[i] = in ? a.table[p * a.rot + a.rot / 2 + pair + i] : __uint_as_float(0x7fc00000u);
    }
}

template <int ROPE>
__device__ __forceinline__ void load_turn(const AppendArgs& a, int64_t t, int d, Turn<ROPE>& r) {
    const int half = a.rot / 2;
    if (ROPE == ROPE_PAIRS) {
        r.on[0] = r.on[1] = d < a.rot;
        if (d < a.rot) four_pairs<ROPE>(a, t, d / 2, r.c, r.s);
    } else if (ROPE == ROPE_HALVES) {
#pragma unroll
        for (int g = 0; g < 2; ++g) {                     // (a group of four is in one half: half is a multiple of four)
            const int e = d + 4 * g;
            const bool low = e < half;
            r.on[g] = e < a.rot;
            r.other[g] = low ? half : -half;
            if (!r.on[g]) continue;
            four_pairs<ROPE>(a, t, low ? e : e - half, r.c + 4 * g, r.s + 4 * g);
            if (low) {
#pragma unroll
                for (int i = 0; i < 4; ++i) r.s[4 * g + i] = -r.s[4 * g + i];
            }
        }
    }
}

// Partners of a lane's elements: nothing more to load where pairs lie side by side
template <int ROPE>
__device__ __forceinline__ void load_other(const __nv_bfloat16* p, const Turn<ROPE>& r, uint2 (&o)[2]) {
    if (ROPE == ROPE_HALVES) {
#pragma unroll
        for (int g = 0; g < 2; ++g)
            if (r.on[g]) o[g] = *reinterpret_cast<const uint2*>(p + 4 * g + r.other[g]);
    }
}

template <int ROPE>
__device__ __forceinline__ void rotate8(const uint4& x, const uint2 (&o)[2], const Turn<ROPE>& r, float (&f)[8]) {
    unpack_bf16x8(x, f);
    if (ROPE == ROPE_PAIRS) {
        if (r.on[0]) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float a = f[2 * i], b = f[2 * i + 1];
                f[2 * i] = __fsub_rn(__fmul_rn(a, r.c[i]), __fmul_rn(b, r.s[i]));
                f[2 * i + 1] = __fadd_rn(__fmul_rn(b, r.c[i]), __fmul_rn(a, r.s[i]));
            }
        }
    } else if (ROPE == ROPE_HALVES) {
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            if (!r.on[g]) continue;
            const float p[4] = {__uint_as_float(o[g].x << 16), __uint_as_float(o[g].x & 0xffff0000u), __uint_as_float(o[g].y << 16), __uint_as_float(o[g].y & 0xffff0000u)};
#pragma unroll
            for (int i = 0; i < 4; ++i) f[4 * g + i] = __fadd_rn(__fmul_rn(f[4 * g + i], r.c[4 * g + i]), __fmul_rn(p[i], r.s[4 * g + i]));
        }
    }
}

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&p);
}

// A CTA takes a token (and a part of its heads, blockIdx.y): its threads stand for `subs` heads side by side, eight elements a lane, and walk
// the queries', the keys' and the values' heads with their angles in registers.
template <int FMT, int ROPE>
__global__ void __launch_bounds__(kThreads) kv_append_kernel(const AppendArgs a) {
    constexpr int UNROLL = 2;
    grid_dep_wait();
    const int sub = static_cast<int>(threadIdx.x) / a.lanes, lane = static_cast<int>(threadIdx.x) - sub * a.lanes, d = lane * 8;
    const bool mine = sub < a.subs && d < a.dim;
    const int all = a.q_heads + a.heads * (a.v.x != nullptr ? 2 : 1), step = a.subs * static_cast<int>(gridDim.y);
    const int blocks = (a.dim + kMxBlock - 1) / kMxBlock;
    const int64_t token_codes = static_cast<int64_t>(a.heads) * a.dim / (FMT == KV_CACHE_INT8 ? 1 : 2);
    const int64_t token_scales = static_cast<int64_t>(a.heads) * (FMT == KV_CACHE_INT8 ? 1 : blocks);
    for (int64_t t = blockIdx.x; t < a.tokens; t += gridDim.x) {
        const int64_t slot = a.slots[t];
        const bool keep = slot >= 0 && slot < a.num_slots;
        Turn<ROPE> turn;
        if (mine) load_turn<ROPE>(a, t, d, turn);
        for (int base = static_cast<int>(blockIdx.y) * a.subs; base < all; base += UNROLL * step) {        // (uniform: every lane takes part in the shuffles)
            uint4 x[UNROLL];
            uint2 other[UNROLL][2];
#pragma unroll
            for (int j = 0; j < UNROLL; ++j) {
                const int h = base + j * step + sub;
                x[j] = make_uint4(0, 0, 0, 0);
                if (!mine || h >= all) continue;
                const bool is_q = h < a.q_heads, is_v = h >= a.q_heads + a.heads;
                const Vectors& from = is_q ? a.q : is_v ? a.v : a.k;
                const int local = is_q ? h : is_v ? h - a.q_heads - a.heads : h - a.q_heads;
                const __nv_bfloat16* p = from.x + t * from.st + local * from.sh + d;
                x[j] = *reinterpret_cast<const uint4*>(p);
                if (!is_v) load_other<ROPE>(p, turn, other[j]);
            }
            if (ROPE == ROPE_HALVES) __syncthreads();        // q_out may be q: a lane's partners are read before they are written over
#pragma unroll
            for (int j = 0; j < UNROLL; ++j) {
                const int h = base + j * step + sub;
                if (base + j * step >= all) break;           // uniform
                const bool live = mine && h < all, is_q = h < a.q_heads, is_v = h >= a.q_heads + a.heads;
                float f[8];
                if (is_v || !mine) unpack_bf16x8(x[j], f);
                else rotate8<ROPE>(x[j], other[j], turn, f);
                if (live && is_q)
                    *reinterpret_cast<uint4*>(a.q_out + t * a.q_out_st + h * a.q_out_sh + d) =
                        make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
                uint32_t top = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(f[i]) & 0x7fffffffu);
                if (!live) top = 0;
                const int shift = FMT == KV_CACHE_INT8 ? a.lane_shift : 2;
                for (int o = 1; o < 1 << shift; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
                if (!live || is_q || !keep) continue;
                const Store& to = is_v ? a.vs : a.ks;
                const int local = is_v ? h - a.q_heads - a.heads : h - a.q_heads;
                if (FMT == KV_CACHE_INT8) {
                    const bool fine = top < 0x7f800000u;
                    const RowScale rs = make_row_scale(fine ? __uint_as_float(top) : 0.f);
                    *reinterpret_cast<uint2*>(to.codes + slot * token_codes + local * a.dim + d) =
                        fine ? make_uint2(quant4(f[0], f[1], f[2], f[3], rs), quant4(f[4], f[5], f[6], f[7], rs)) : make_uint2(0, 0);
                    if (lane == 0) static_cast<float*>(to.scales)[slot * token_scales + local] = fine ? rs.s : __uint_as_float(0x7fc00000u);
                } else {
                    const uint32_t byte = mx_scale_byte(top);
                    const float inv = byte == 255u ? 0.f : mx_inverse_scale(byte);
                    float y[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) y[i] = byte == 255u ? 0.f : f[i] * inv;
                    *reinterpret_cast<uint32_t*>(to.codes + slot * token_codes + (local * a.dim + d) / 2) = e2m1x8(y);
                    if ((lane & 3) == 0) static_cast<uint8_t*>(to.scales)[slot * token_scales + local * blocks + lane / 4] = static_cast<uint8_t>(byte);
                }
            }
        }
    }
}

__global__ void __launch_bounds__(kThreads) rope_table_kernel(const double* inv_freq, int pairs, int64_t first, int64_t positions, double scale, float* cos_sin) {
    grid_dep_wait();
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; i < positions * pairs; i += static_cast<int64_t>(gridDim.x) * kThreads) {
        const int64_t p = i / pairs;
        const int pair = static_cast<int>(i - p * pairs);
        double s, c;
        sincos(static_cast<double>(first + p) * inv_freq[pair], &s, &c);
        cos_sin[p * 2 * pairs + pair] = static_cast<float>(c * scale);
        cos_sin[p * 2 * pairs + pairs + pair] = static_cast<float>(s * scale);
    }
}

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
bool vectors_aligned(const void* p, int64_t st, int64_t sh) { return aligned(p, 16) && st % 8 == 0 && sh % 8 == 0; }

template <int FMT>
auto append_kernel(int rope) {
    return rope == ROPE_NONE ? kv_append_kernel<FMT, ROPE_NONE> : rope == ROPE_HALVES ? kv_append_kernel<FMT, ROPE_HALVES> : kv_append_kernel<FMT, ROPE_PAIRS>;
}

} // namespace
} // namespace w8a8

extern "C" {

using namespace w8a8;

int kv_cache_append(int fmt, const void* q, int64_t q_token_stride, int64_t q_head_stride, int64_t q_heads, void* q_out, int64_t q_out_token_stride,
                    int64_t q_out_head_stride, const void* k, int64_t k_token_stride, int64_t k_head_stride, const void* v, int64_t v_token_stride,
                    int64_t v_head_stride, const float* cos_sin, int64_t num_positions, int64_t rot, int interleaved, const int64_t* positions,
                    int64_t position_stride, int64_t axes, const uint8_t* axis_of, const int64_t* slots, int64_t tokens, int64_t heads, int64_t dim,
                    void* k_codes, void* k_scales, void* v_codes, void* v_scales, int64_t num_slots, void* stream) {
    if ((fmt != KV_CACHE_INT8 && fmt != KV_CACHE_MXFP4) || heads <= 0 || dim <= 0 || dim > KV_CACHE_MAX_DIM || heads > KV_CACHE_MAX_WIDTH ||
        heads * dim > KV_CACHE_MAX_WIDTH || tokens < 0 || num_slots < 0 || (tokens > 0 && (k == nullptr || slots == nullptr)))
        return W8A8_ERR_INVALID_ARG;
    if (q_heads < 0 || q_heads > KV_CACHE_MAX_WIDTH || q_heads * dim > KV_CACHE_MAX_WIDTH || (tokens > 0 && q_heads > 0 && (q == nullptr || q_out == nullptr)))
        return W8A8_ERR_INVALID_ARG;
    if (num_slots > 0 && (k_codes == nullptr || k_scales == nullptr || (v != nullptr && (v_codes == nullptr || v_scales == nullptr)))) return W8A8_ERR_INVALID_ARG;
    if (cos_sin != nullptr && (rot <= 0 || rot > dim || num_positions < 0 || num_positions > INT32_MAX || axes <= 0 || axes > KV_CACHE_MAX_AXES || (axes > 1 && axis_of == nullptr) ||
                               (tokens > 0 && positions == nullptr) || (axes > 1 && position_stride < tokens)))
        return W8A8_ERR_INVALID_ARG;
    if (dim % 8 != 0 || !vectors_aligned(k, k_token_stride, k_head_stride) || !aligned(slots, 8) || !aligned(k_codes, 16) || !aligned(k_scales, fmt == KV_CACHE_INT8 ? 4 : 1))
        return W8A8_ERR_ALIGNMENT;
    if (v != nullptr && (!vectors_aligned(v, v_token_stride, v_head_stride) || !aligned(v_codes, 16) || !aligned(v_scales, fmt == KV_CACHE_INT8 ? 4 : 1)))
        return W8A8_ERR_ALIGNMENT;
    if (q_heads > 0 && (!vectors_aligned(q, q_token_stride, q_head_stride) || !vectors_aligned(q_out, q_out_token_stride, q_out_head_stride))) return W8A8_ERR_ALIGNMENT;
    if (cos_sin != nullptr && (rot % 8 != 0 || !aligned(cos_sin, 16) || !aligned(positions, 8))) return W8A8_ERR_ALIGNMENT;
    if (int e = check_arch()) return e;
    if (tokens == 0 || (num_slots == 0 && q_heads == 0)) return W8A8_OK;
    AppendArgs a{};
    a.q = {static_cast<const __nv_bfloat16*>(q), q_token_stride, q_head_stride};
    a.k = {static_cast<const __nv_bfloat16*>(k), k_token_stride, k_head_stride};
    a.v = {static_cast<const __nv_bfloat16*>(v), v_token_stride, v_head_stride};
    a.q_out = static_cast<__nv_bfloat16*>(q_out);
    a.q_out_st = q_out_token_stride;
    a.q_out_sh = q_out_head_stride;
    a.ks = {static_cast<uint8_t*>(k_codes), k_scales};
    a.vs = {static_cast<uint8_t*>(v_codes), v_scales};
    a.table = cos_sin;
    a.positions = positions;
    a.slots = slots;
    a.axis_of = axis_of;
    a.position_stride = position_stride;
    a.num_positions = num_positions;
    a.num_slots = num_slots;
    a.tokens = tokens;
    a.q_heads = static_cast<int>(q_heads);
    a.heads = static_cast<int>(heads);
    a.dim = static_cast<int>(dim);
    a.rot = static_cast<int>(rot);
    a.axes = static_cast<int>(axes);
    while ((8 << a.lane_shift) < dim) ++a.lane_shift;
    a.lanes = fmt == KV_CACHE_INT8 ? 1 << a.lane_shift : static_cast<int>((dim + kMxBlock - 1) / kMxBlock) * (kMxBlock / 8);
    a.subs = kThreads / a.lanes;
    const int all = static_cast<int>(q_heads + heads * (v != nullptr ? 2 : 1));
    // few tokens: their heads are shared out over more CTAs
    const int parts = (all + a.subs - 1) / a.subs;
    int64_t slices = tokens >= 4 * sm_count() ? 1 : (4 * sm_count() + tokens - 1) / tokens;
    if (slices > parts) slices = parts;
    const int64_t most = static_cast<int64_t>(sm_count()) * 32;
    const int rope = cos_sin == nullptr ? ROPE_NONE : interleaved != 0 ? ROPE_PAIRS : ROPE_HALVES;
    const cudaError_t e = launch_pdl(fmt == KV_CACHE_INT8 ? append_kernel<KV_CACHE_INT8>(rope) : append_kernel<KV_CACHE_MXFP4>(rope),
                                     dim3(static_cast<unsigned>(tokens < most ? tokens : most), static_cast<unsigned>(slices)), kThreads, static_cast<cudaStream_t>(stream), a);
    return e == cudaSuccess ? W8A8_OK : W8A8_ERR_CUDA;
}

int kv_cache_rope_table(const double* inv_freq, int64_t pairs, int64_t first, int64_t num_positions, double scale, float* cos_sin, void* stream) {
    if (pairs <= 0 || pairs > KV_CACHE_MAX_DIM || num_positions < 0 || num_positions > INT32_MAX || first < -(int64_t{1} << 52) || first > (int64_t{1} << 52) ||
        !std::isfinite(scale) || inv_freq == nullptr || (num_positions > 0 && cos_sin == nullptr))
        return W8A8_ERR_INVALID_ARG;
    if (!aligned(inv_freq, 8) || !aligned(cos_sin, 4)) return W8A8_ERR_ALIGNMENT;
    if (int e = check_arch()) return e;
    if (num_positions == 0) return W8A8_OK;
    const int64_t ctas = (num_positions * pairs + kThreads - 1) / kThreads, most = static_cast<int64_t>(sm_count()) * 32;
    const cudaError_t e = launch_pdl(rope_table_kernel, dim3(static_cast<unsigned>(ctas < most ? ctas : most)), kThreads, static_cast<cudaStream_t>(stream), inv_freq,
                                     static_cast<int>(pairs), first, num_positions, scale, cos_sin);
    return e == cudaSuccess ? W8A8_OK : W8A8_ERR_CUDA;
}

} // extern "C"
