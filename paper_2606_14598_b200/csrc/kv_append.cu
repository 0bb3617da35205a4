// New tokens on their way into the quantized cache: queries and keys rotated by position, keys and values quantized into their slots.
//
//   a' = a c - b s,  b' = b c + a s     (c, s) of a pair from the table row of the token's position on the pair's axis
//
// Products and sums are fp32 and rounded once each (no fused multiply-add), so that codes are specified to the bit. Keys go from fp32 to
// codes: rounding them to bf16 in between, as a rotation in a pass of its own would, loses a bit for nothing.
//
// A lane has eight elements of a head, of up to four heads at once, from the load to the codes in registers. 16000 tokens of 32 + 8 + 8 heads of 128 with a rotation, int8: 74 us, 56 at
// the copy's rate; 8220 tokens of 3 x 16 x 72, three axes, 4 bits: 32 us (13), where positions, axes and blocks that end inside a lane cost instructions; 48 tokens: 2.8 us, a launch.
// (SM clock 1935 MHz in the first of them, 1965 MHz in the others.)
#include "../../include/kv_cache.h"
#include "internal.h"
#include "mxfp4_math.cuh"
#include "ptx.cuh"
#include "quant_math.cuh"

#include <cmath>

namespace w8a8 {
namespace {

constexpr int kThreads = 256;
enum { ROPE_NONE = 0, ROPE_HALVES = 1, ROPE_PAIRS = 2, ROPE_HALVES_ANY = 3 };

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
    int lanes, lane_shift;         // lanes of a head, log2 of the lanes that share an int8 scale
};

// A lane holds eight elements of a head as two groups of four. Where it can, its groups are each other's partners:
//   ROPE_PAIRS       groups side by side, pairs side by side in them
//   ROPE_HALVES      lane i: elements 4i of the first half and 4i of the second; behind the rotated part, groups side by side. 4-bit: only where halves are
//                    whole blocks, which then lie in eight lanes' first or second groups
//   ROPE_HALVES_ANY  groups side by side, the partners of each loaded beside it (halves that end inside a block of the 4-bit format)
template <int ROPE>
struct Places {
    static constexpr int TURNS = ROPE == ROPE_HALVES_ANY ? 2 : 1;      // runs of four pairs whose angles the lane needs
    int at[2];                     // elements that the groups begin at
    bool on[TURNS];                // whether they turn
    int pair[TURNS];               // their first pairs
    uint32_t axis[TURNS];          // a byte a pair
    bool low[TURNS];               // HALVES_ANY: whether the group is in the first half
    __device__ __forceinline__ void init(const AppendArgs& a, int lane) {
        const int half = a.rot / 2;
        at[0] = 8 * lane;
        at[1] = 8 * lane + 4;
        if (ROPE == ROPE_NONE) return;
        if (ROPE == ROPE_HALVES && 4 * lane < half) {
            at[0] = 4 * lane;
            at[1] = 4 * lane + half;
        }
#pragma unroll
        for (int g = 0; g < TURNS; ++g) {
            low[g] = at[g] < half;
            on[g] = at[g] < a.rot;
            pair[g] = ROPE == ROPE_PAIRS ? at[0] / 2 : ROPE == ROPE_HALVES ? at[0] : low[g] ? at[g] : at[g] - half;
            if (ROPE == ROPE_HALVES) on[g] = at[0] < half;
            axis[g] = 0;
            if (on[g] && a.axis_of != nullptr) {
#pragma unroll
                for (int i = 0; i < 4; ++i) axis[g] |= static_cast<uint32_t>(a.axis_of[pair[g] + i]) << (8 * i);
            }
        }
    }
};
struct Angles {
    float c[4], s[4];
};
// Rows of the table that four pairs of token t go by (-1: outside), a token ahead of their use; all alike if the pairs have one axis
__device__ __forceinline__ void load_rows(const AppendArgs& a, int64_t t, uint32_t axis, int (&row)[4]) {
    const bool one = axis == (axis & 0xffu) * 0x01010101u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (i == 0 || !one) {
            const int its = static_cast<int>(axis >> (8 * i) & 0xffu);
            const int64_t p = its < a.axes ? a.positions[its * a.position_stride + t] : -1;
            row[i] = p >= 0 && p < a.num_positions ? static_cast<int>(p) : -1;
        } else {
            row[i] = row[0];
        }
    }
}
// The angles of four pairs; a position outside the table gives NaN
__device__ __forceinline__ void load_angles(const AppendArgs& a, const int (&row)[4], int pair, Angles& r) {
    const float nan = __uint_as_float(0x7fc00000u);
    if (row[0] == row[1] && row[0] == row[2] && row[0] == row[3] && row[0] >= 0) {
        const float* at = a.table + static_cast<int64_t>(row[0]) * a.rot + pair;
        const float4 u = *reinterpret_cast<const float4*>(at), w = *reinterpret_cast<const float4*>(at + a.rot / 2);
        r.c[0] = u.x; r.c[1] = u.y; r.c[2] = u.z; r.c[3] = u.w;
        r.s[0] = w.x; r.s[1] = w.y; r.s[2] = w.z; r.s[3] = w.w;
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float* at = a.table + static_cast<int64_t>(max(row[i], 0)) * a.rot + pair + i;
        r.c[i] = row[i] >= 0 ? at[0] : nan;
        r.s[i] = row[i] >= 0 ? at[a.rot / 2] : nan;
    }
}

__device__ __forceinline__ void unpack4(const uint2& x, float* f) {
    f[0] = __uint_as_float(x.x << 16);
    f[1] = __uint_as_float(x.x & 0xffff0000u);
    f[2] = __uint_as_float(x.y << 16);
    f[3] = __uint_as_float(x.y & 0xffff0000u);
}
// f: the lane's eight elements; o: (HALVES_ANY) the partners of both groups. (Scalar instructions: a product and a sum of the packed ones are made one by the
// assembler, in spite of their roundings.)
template <int ROPE>
__device__ __forceinline__ void rotate8(float (&f)[8], const uint2 (&o)[2], const Places<ROPE>& where, const Angles (&r)[Places<ROPE>::TURNS]) {
    if (ROPE == ROPE_PAIRS || ROPE == ROPE_HALVES) {
        if (!where.on[0]) return;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float& x = f[ROPE == ROPE_PAIRS ? 2 * i : i];
            float& y = f[ROPE == ROPE_PAIRS ? 2 * i + 1 : 4 + i];
            const float a = x, b = y;
            x = __fsub_rn(__fmul_rn(a, r[0].c[i]), __fmul_rn(b, r[0].s[i]));
            y = __fadd_rn(__fmul_rn(b, r[0].c[i]), __fmul_rn(a, r[0].s[i]));
        }
    } else if (ROPE == ROPE_HALVES_ANY) {
        constexpr int LAST = Places<ROPE>::TURNS - 1;
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            const int turn = g < LAST ? g : LAST;
            if (!where.on[turn]) continue;
            float p[4];
            unpack4(o[g], p);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float mine = __fmul_rn(f[4 * g + i], r[turn].c[i]), its = __fmul_rn(p[i], r[turn].s[i]);
                f[4 * g + i] = where.low[turn] ? __fsub_rn(mine, its) : __fadd_rn(mine, its);
            }
        }
    }
}

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&p);
}
__device__ __forceinline__ uint32_t top4(const float* f) {             // the largest pattern of a magnitude among four
    return max(max(__float_as_uint(f[0]) & 0x7fffffffu, __float_as_uint(f[1]) & 0x7fffffffu), max(__float_as_uint(f[2]) & 0x7fffffffu, __float_as_uint(f[3]) & 0x7fffffffu));
}

// How CTAs cover the vectors of one kind (queries, keys or values): a CTA's threads stand for `across` heads side by side of `down` tokens, and each goes on to UNROLL heads
// `across` apart; `parts` CTAs side by side take all heads. From there a CTA goes from token to token.
struct Cover {
    int across, down, parts, each;      // each: heads of a thread, UNROLL at most
};
// Four heads of a thread on their way at once: 74 and 32 us for the cases above, two: 81 and 42. (Partners of their own take as many registers again.)
constexpr __host__ __device__ int unroll_of(int rope) { return rope == ROPE_HALVES_ANY ? 2 : 4; }
enum { QUERIES = 0, KEYS = 1, VALUES = 2 };

template <int FMT, int ROPE, int KIND>
__device__ __forceinline__ void append_kind(const AppendArgs& a, const Cover& cover, const Vectors& v, const Store& store, int heads, int part, int row_of_ctas, int rows_of_ctas) {
    constexpr int TURNS = Places<ROPE>::TURNS, UNROLL = unroll_of(ROPE);
    constexpr bool APART = ROPE == ROPE_HALVES && KIND != VALUES;      // groups may lie apart
    const int sub = static_cast<int>(threadIdx.x) / a.lanes, lane = static_cast<int>(threadIdx.x) - sub * a.lanes;
    const int off = sub / cover.across, h0 = part * cover.across * cover.each + sub - off * cover.across;
    Places<ROPE> where;
    if (KIND == VALUES) {
        where.at[0] = 8 * lane;
        where.at[1] = 8 * lane + 4;
    } else {
        where.init(a, lane);
    }
    const bool mine = off < cover.down && 8 * lane < a.dim;
    const bool in_pairs = APART && where.on[0];
    const int apart = where.at[1] - where.at[0];                       // from the first group to the second
    const int blocks = (a.dim + kMxBlock - 1) / kMxBlock;
    const int64_t token_codes = static_cast<int64_t>(a.heads) * a.dim / (FMT == KV_CACHE_INT8 ? 1 : 2);
    const int64_t token_scales = static_cast<int64_t>(a.heads) * (FMT == KV_CACHE_INT8 ? 1 : blocks);
    // this thread's elements of its first token, and from head to head and token to token
    const int64_t first = static_cast<int64_t>(row_of_ctas) * cover.down + off, on = static_cast<int64_t>(rows_of_ctas) * cover.down;
    const __nv_bfloat16* from = v.x + first * v.st + h0 * v.sh + where.at[0];
    const int64_t next_head = cover.across * v.sh, next_token = on * v.st;
    __nv_bfloat16* out = KIND == QUERIES ? a.q_out + first * a.q_out_st + h0 * a.q_out_sh + where.at[0] : nullptr;
    const int64_t out_head = cover.across * a.q_out_sh, out_token = on * a.q_out_st;
    uint8_t* const codes = KIND == QUERIES ? nullptr : store.codes + (h0 * a.dim + where.at[0]) / (FMT == KV_CACHE_INT8 ? 1 : 2);
    const int codes_head = cover.across * a.dim / (FMT == KV_CACHE_INT8 ? 1 : 2);
    int row[TURNS][4];
    int64_t slot = -1;
    auto ahead = [&](int64_t t) {                                      // what a token needs first
        if (t >= a.tokens || !mine) return;
        if (KIND != QUERIES) slot = a.slots[t];
        if constexpr (ROPE != ROPE_NONE && KIND != VALUES) {
#pragma unroll
            for (int g = 0; g < TURNS; ++g)
                if (where.on[g]) load_rows(a, t, where.axis[g], row[g]);
        }
    };
    ahead(first);
    for (int64_t t = first; t - off < a.tokens; t += on, from += next_token, out += KIND == QUERIES ? out_token : 0) {     // (uniform: every lane takes part in the shuffles)
        const bool here = mine && t < a.tokens;
        const int64_t its_slot = slot;
        uint2 x[UNROLL][2], other[UNROLL][2];
#pragma unroll
        for (int j = 0; j < UNROLL; ++j) {
            x[j][0] = x[j][1] = make_uint2(0, 0);
            if (!here || j >= cover.each || h0 + j * cover.across >= heads) continue;
            const __nv_bfloat16* p = from + j * next_head;
            if (APART) {
                x[j][0] = *reinterpret_cast<const uint2*>(p);
                x[j][1] = *reinterpret_cast<const uint2*>(p + apart);
            } else {
                const uint4 w = *reinterpret_cast<const uint4*>(p);
                x[j][0] = make_uint2(w.x, w.y);
                x[j][1] = make_uint2(w.z, w.w);
            }
            if constexpr (ROPE == ROPE_HALVES_ANY && KIND != VALUES) {
                constexpr int LAST = TURNS - 1;
#pragma unroll
                for (int g = 0; g < 2; ++g)
                    if (where.on[g < LAST ? g : LAST]) other[j][g] = *reinterpret_cast<const uint2*>(p + 4 * g + (where.low[g < LAST ? g : LAST] ? a.rot / 2 : -(a.rot / 2)));
            }
        }
        Angles turn[TURNS];
        if constexpr (ROPE != ROPE_NONE && KIND != VALUES) {
#pragma unroll
            for (int g = 0; g < TURNS; ++g)
                if (here && where.on[g]) load_angles(a, row[g], where.pair[g], turn[g]);
        }
        ahead(t + on);
        if (ROPE == ROPE_HALVES_ANY && KIND == QUERIES) __syncthreads();         // q_out may be q: a lane's partners are read before they are written over
#pragma unroll
        for (int j = 0; j < UNROLL; ++j) {
            if (j >= cover.each || (part * cover.each + j) * cover.across >= heads) break;         // uniform
            const bool live = here && h0 + j * cover.across < heads;
            float f[8];
            unpack4(x[j][0], f);
            unpack4(x[j][1], f + 4);
            if constexpr (ROPE != ROPE_NONE && KIND != VALUES)
                if (here) rotate8<ROPE>(f, other[j], where, turn);
            if (KIND == QUERIES) {
                if (!live) continue;
                __nv_bfloat16* p = out + j * out_head;
                const uint2 lo = make_uint2(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3])), hi = make_uint2(pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
                if (APART) {
                    *reinterpret_cast<uint2*>(p) = lo;
                    *reinterpret_cast<uint2*>(p + apart) = hi;
                } else {
                    *reinterpret_cast<uint4*>(p) = make_uint4(lo.x, lo.y, hi.x, hi.y);
                }
                continue;
            }
            const bool keep = live && its_slot >= 0 && its_slot < a.num_slots;
            const uint4 packed = make_uint4(x[j][0].x, x[j][0].y, x[j][1].x, x[j][1].y);
            uint32_t top[2] = {0u, 0u};
            if (live) {
                if (KIND == VALUES) top[0] = top[1] = absmax_bits8(packed);
                else { top[0] = top4(f); top[1] = top4(f + 4); }
            }
            uint8_t* const p = codes + its_slot * token_codes + j * codes_head;
            if (FMT == KV_CACHE_INT8) {
                uint32_t m = max(top[0], top[1]);
                for (int o = 1; o < 1 << a.lane_shift; o <<= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
                if (!keep) continue;
                const bool fine = m < 0x7f800000u;
                const RowScale rs = head_scale(fine ? __uint_as_float(m) : 0.f);
                const RowScale2 r2 = head_scale2(rs);
                const uint2 c = !fine ? make_uint2(0, 0) : KIND == VALUES ? quant8(packed, rs, r2) : make_uint2(quant4f(f[0], f[1], f[2], f[3], rs, r2), quant4f(f[4], f[5], f[6], f[7], rs, r2));
                if (APART) {
                    *reinterpret_cast<uint32_t*>(p) = c.x;
                    *reinterpret_cast<uint32_t*>(p + apart) = c.y;
                } else {
                    *reinterpret_cast<uint2*>(p) = c;
                }
                if (lane == 0) static_cast<float*>(store.scales)[its_slot * token_scales + h0 + j * cover.across] = fine ? rs.s : __uint_as_float(0x7fc00000u);
            } else {
                // a block: four lanes, or the first or second groups of eight
                if (!in_pairs) top[0] = top[1] = max(top[0], top[1]);
#pragma unroll
                for (int g = 0; g < (APART ? 2 : 1); ++g) {
                    top[g] = max(top[g], __shfl_xor_sync(0xffffffffu, top[g], 1));
                    top[g] = max(top[g], __shfl_xor_sync(0xffffffffu, top[g], 2));
                    if (APART) {
                        const uint32_t its = __shfl_xor_sync(0xffffffffu, top[g], 4);
                        if (in_pairs) top[g] = max(top[g], its);
                    }
                }
                if (!keep) continue;
                const uint32_t byte[2] = {mx_scale_byte(top[0]), mx_scale_byte(top[APART ? 1 : 0])};
                uint32_t c;
                if (KIND == VALUES) {
                    c = mx_codes8(packed, byte[0]);
                } else {
                    float y[8];
#pragma unroll
                    for (int g = 0; g < 2; ++g) {
                        const float inv = byte[g] == 255u ? 0.f : mx_inverse_scale(byte[g]);
                        const uint64_t both = pack2(inv, inv);
                        unpack2(mul2(pack2(f[4 * g], f[4 * g + 1]), both), y[4 * g], y[4 * g + 1]);
                        unpack2(mul2(pack2(f[4 * g + 2], f[4 * g + 3]), both), y[4 * g + 2], y[4 * g + 3]);
                        if (byte[g] == 255u) y[4 * g] = y[4 * g + 1] = y[4 * g + 2] = y[4 * g + 3] = 0.f;
                    }
                    c = e2m1x8(y);
                }
                if (APART) {
                    *reinterpret_cast<uint16_t*>(p) = static_cast<uint16_t>(c);
                    *reinterpret_cast<uint16_t*>(p + apart / 2) = static_cast<uint16_t>(c >> 16);
                } else {
                    *reinterpret_cast<uint32_t*>(p) = c;
                }
                if (where.at[0] % kMxBlock == 0) {
                    uint8_t* s = static_cast<uint8_t*>(store.scales) + its_slot * token_scales + (h0 + j * cover.across) * blocks;
                    s[where.at[0] / kMxBlock] = static_cast<uint8_t>(byte[0]);
                    if (in_pairs) s[where.at[1] / kMxBlock] = static_cast<uint8_t>(byte[1]);
                }
            }
        }
    }
}

// blockIdx.y: a part of the queries' heads, of the keys' or of the values'. The three cost differently much a vector, so that their CTAs end at different times, and
// others take their places.
template <int FMT, int ROPE>
__global__ void __launch_bounds__(kThreads, 4) kv_append_kernel(const AppendArgs a, const Cover q, const Cover kv) {
    grid_dep_wait();
    grid_dep_launch_dependents();
    const int part = blockIdx.y;
    if (part < q.parts) append_kind<FMT, ROPE, QUERIES>(a, q, a.q, a.ks, a.q_heads, part, blockIdx.x, gridDim.x);
    else if (part < q.parts + kv.parts) append_kind<FMT, ROPE, KEYS>(a, kv, a.k, a.ks, a.heads, part - q.parts, blockIdx.x, gridDim.x);
    else append_kind<FMT, ROPE, VALUES>(a, kv, a.v, a.vs, a.heads, part - q.parts - kv.parts, blockIdx.x, gridDim.x);
}

// few: so few tokens that a head a thread, on more CTAs, is over sooner; else as many loads of a thread as can be are on their way (48 tokens: 2.9 us as few, 4.8 else; 300,
// two an SM, 6.1 either way; 450: 7.5 and 6.3)
Cover make_cover(int heads, int subs, int unroll, bool few) {
    Cover c{};
    if (heads == 0) return c;
    c.across = few ? heads : (heads + unroll - 1) / unroll;
    if (c.across > subs) c.across = subs;
    c.down = few ? 1 : subs / c.across;
    const int each = few ? 1 : unroll;
    c.parts = (heads + c.across * each - 1) / (c.across * each);
    c.each = each;
    return c;
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
    return rope == ROPE_NONE     ? kv_append_kernel<FMT, ROPE_NONE>
           : rope == ROPE_HALVES ? kv_append_kernel<FMT, ROPE_HALVES>
           : rope == ROPE_PAIRS  ? kv_append_kernel<FMT, ROPE_PAIRS>
                                 : kv_append_kernel<FMT, ROPE_HALVES_ANY>;
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
    const int rope = cos_sin == nullptr ? ROPE_NONE : interleaved != 0 ? ROPE_PAIRS : fmt == KV_CACHE_INT8 || rot % (2 * kMxBlock) == 0 ? ROPE_HALVES : ROPE_HALVES_ANY;
    a.lanes = fmt == KV_CACHE_INT8 ? 1 << a.lane_shift : static_cast<int>((dim + kMxBlock - 1) / kMxBlock) * (kMxBlock / 8);
    if (fmt != KV_CACHE_INT8 && rope == ROPE_HALVES) a.lanes = (a.lanes + 7) / 8 * 8;         // (blocks of eight lanes)
    const int subs = kThreads / a.lanes, unroll = unroll_of(rope);
    const bool few = tokens <= 2 * sm_count();
    const Cover q_cover = make_cover(a.q_heads, subs, unroll, few), kv_cover = make_cover(num_slots > 0 ? a.heads : 0, subs, unroll, few);
    const int parts = q_cover.parts + kv_cover.parts * (v != nullptr ? 2 : 1);
    // CTAs of a part: as many as an SM holds of them together, twice over (the kinds end at different times), and no more than there are tokens
    const int64_t fit = (static_cast<int64_t>(sm_count()) * 8 + parts - 1) / parts;
    const cudaError_t e = launch_pdl(fmt == KV_CACHE_INT8 ? append_kernel<KV_CACHE_INT8>(rope) : append_kernel<KV_CACHE_MXFP4>(rope),
                                     dim3(static_cast<unsigned>(tokens < fit ? tokens : fit), static_cast<unsigned>(parts)), kThreads, static_cast<cudaStream_t>(stream), a, q_cover, kv_cover);
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
