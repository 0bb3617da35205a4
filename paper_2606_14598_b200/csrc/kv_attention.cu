// Attention of new tokens over the quantized paged cache, on the codes.
//
//   o = sum_p softmax_p(scale * q . k_p) v_p,   k_p = code * s_k(p),  v_p = code * s_v(p)      (MXFP4: a scale for 32 elements)
//
// A token's scale factors out of both products: scores are (q . code) * s_k, and the values' scale multiplies the probability, so what the
// matrix instructions take are the codes themselves, converted in registers and exact: keys as fp16 beside queries that a power of two of their
// row brings into fp16's range, values as bf16 beside probabilities rounded to bf16 (their range is that of s_v).
//
// One pass over the cache with a running maximum and sum. The work is cut into units of a few dozen tokens of one head of one sequence, in one
// long list that the CTAs share out evenly whatever the sequences' lengths: a CTA's range holds ends of at most two items that others share,
// whose parts meet in the workspace and are added up, in the order of the tokens, by the CTA that arrives last.
#include "../../include/kv_cache.h"
#include "internal.h"
#include "mxfp4_math.cuh"
#include "ptx.cuh"

#include <cmath>
#include <cuda_fp16.h>

namespace w8a8 {
namespace {

constexpr int kWarps = 4, kThreads = 32 * kWarps;
constexpr int kStep = 16;                       // tokens that a warp takes at a time
constexpr int kTile = kStep * kWarps;           // tokens of a unit
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct AttentionArgs {
    const uint8_t *k_codes, *v_codes;
    const void *k_scales, *v_scales;
    const int32_t *table, *lens, *starts, *cu_q;
    const int64_t* tree;
    const __nv_bfloat16* q;
    __nv_bfloat16* out;
    float* lse;
    uint32_t* counters;
    float* parts;
    int64_t q_st, q_sh, o_st, o_sh, table_stride, tree_words;
    int num_pages, page, max_pages, heads, group, dim, seqs, total_q;
    int copy;                                   // bytes of an asynchronous copy: 16, 8 or 4, by the alignment of the heads in the cache
    float scale;
    int zero_rest;
};

// ------------------------------------------------------------------------------------------------ the list of work

struct Sequence {
    int begin, n;                               // its rows of q
    int before;                                 // tokens ahead of the new ones (negative if the cache holds fewer than n)
    int start, stop;                            // tokens that may be seen
    int tiles, row_tiles;
};
__device__ __forceinline__ Sequence read_sequence(const AttentionArgs& a, int b, int rows_of_tile) {
    Sequence s;
    const int begin = a.cu_q[b], end = a.cu_q[b + 1], len = a.lens[b];
    const int64_t most = static_cast<int64_t>(a.max_pages) * a.page;
    s.begin = max(0, min(begin, a.total_q));
    s.n = max(s.begin, min(end, a.total_q)) - s.begin;
    s.before = max(len, 0) - s.n;
    s.stop = static_cast<int>(min(static_cast<int64_t>(max(len, 0)), most));
    s.start = a.starts != nullptr ? max(0, min(a.starts[b], s.stop)) : 0;
    s.tiles = max(1, (s.stop - s.start + kTile - 1) / kTile);
    s.row_tiles = static_cast<int>((static_cast<int64_t>(s.n) * a.group + rows_of_tile - 1) / rows_of_tile);
    return s;
}
__device__ __forceinline__ int64_t units_of(const AttentionArgs& a, const Sequence& s) { return static_cast<int64_t>(a.heads) * s.row_tiles * s.tiles; }

struct Share {
    int64_t total, first_of_b;                  // units of all sequences; of those before b
    int64_t ctas;                               // CTAs that work: none without a unit
    int64_t begin, end;                         // this CTA's units
    int b;
};
// The sequence that unit `u` (of this CTA's range) belongs to, found by all threads at once; u < 0: only the total
__device__ __forceinline__ int64_t warp_scan(int64_t v) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t w = __shfl_up_sync(0xffffffffu, v, o);
        if ((threadIdx.x & 31) >= o) v += w;
    }
    return v;
}
template <int THREADS>
__device__ __forceinline__ Share share_out(const AttentionArgs& a, int rows_of_tile) {
    __shared__ int64_t of_warp[THREADS / 32];
    __shared__ int64_t first_unit;
    __shared__ int found;
    const int per = (a.seqs + THREADS - 1) / THREADS, b0 = min(a.seqs, static_cast<int>(threadIdx.x) * per), b1 = min(a.seqs, b0 + per);
    int64_t mine = 0;
    for (int b = b0; b < b1; ++b) mine += units_of(a, read_sequence(a, b, rows_of_tile));
    const int64_t scan = warp_scan(mine);
    if ((threadIdx.x & 31) == 31) of_warp[threadIdx.x >> 5] = scan;
    if (threadIdx.x == 0) found = a.seqs;
    __syncthreads();
    int64_t before = scan - mine, total = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) {
        if (w < static_cast<int>(threadIdx.x >> 5)) before += of_warp[w];
        total += of_warp[w];
    }
    const int64_t ctas = min(total, static_cast<int64_t>(gridDim.x)), u = blockIdx.x < ctas ? total * blockIdx.x / ctas : total;
    if (u >= before && u < before + mine) {
        for (int b = b0; b < b1; ++b) {
            const int64_t units = units_of(a, read_sequence(a, b, rows_of_tile));
            if (u < before + units) {
                found = b;
                first_unit = before;
                break;
            }
            before += units;
        }
    }
    __syncthreads();
    return Share{total, found < a.seqs ? first_unit : 0, ctas, u, blockIdx.x < ctas ? total * (blockIdx.x + 1) / ctas : u, found};
}

// The CTA whose range holds unit u (CTA c takes units total * c / ctas up to total * (c + 1) / ctas)
__device__ __forceinline__ int owner(int64_t u, const Share& s) { return static_cast<int>(((u + 1) * s.ctas - 1) / s.total); }

// ------------------------------------------------------------------------------------------------ small pieces

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&p);
}
__device__ __forceinline__ uint32_t sub_bf16x2(uint32_t a, uint32_t b) {
    const __nv_bfloat162 r = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
    return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ uint32_t sub_f16x2(uint32_t a, uint32_t b) {
    const __half2 r = __hsub2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
    return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ uint32_t mul_f16x2(uint32_t a, uint32_t b) {
    const __half2 r = __hmul2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
    return *reinterpret_cast<const uint32_t*>(&r);
}
// D += A * B, 16 x 8 x 16: rows g and g + 8 of A and D (g = lane / 4), column g of B, column pairs 2c, 2c + 1 of D (c = lane % 4)
__device__ __forceinline__ void mma_f16(float (&d)[4], const uint4& a, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_bf16(float (&d)[4], const uint4& a, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b0), "r"(b1));
}
template <int BYTES>
__device__ __forceinline__ void cp_async(uint32_t dst, const void* src, uint32_t valid) {      // valid: BYTES, or 0 for zeros
    if (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(valid) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(dst), "l"(src), "n"(BYTES), "r"(valid) : "memory");
}
// BYTES of a head's codes, of which those past `valid` are zeros, in pieces that the head's alignment allows
template <int BYTES>
__device__ __forceinline__ void copy_codes(uint32_t dst, const uint8_t* src, int valid, int piece) {
    if (BYTES == 16 && piece == 16) {
        cp_async<16>(dst, src, valid > 0 ? 16 : 0);
    } else if (BYTES >= 8 && piece >= 8) {
#pragma unroll
        for (int i = 0; i < BYTES; i += 8) cp_async<8>(dst + i, src + (valid > i ? i : 0), valid > i ? 8 : 0);
    } else {
#pragma unroll
        for (int i = 0; i < BYTES; i += 4) cp_async<4>(dst + i, src + (valid > i ? i : 0), valid > i ? 4 : 0);
    }
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// ------------------------------------------------------------------------------------------------ codes to matrix operands

// Four int8 codes as fp16: code + 128 in the low byte of 1024, minus 1152
__device__ __forceinline__ void int8_to_f16(uint32_t w, uint32_t (&r)[2]) {
    const uint32_t t = w ^ 0x80808080u;
    r[0] = sub_f16x2(__byte_perm(t, 0x64646464u, 0x4140), 0x64806480u);
    r[1] = sub_f16x2(__byte_perm(t, 0x64646464u, 0x4342), 0x64806480u);
}
// Codes in bytes 0 and 2 of x as bf16: the low seven bits in the fraction of 128, minus 128 or (sign bit) 256
__device__ __forceinline__ uint32_t int8_to_bf16(uint32_t x) { return sub_bf16x2((x & 0x007f007fu) | 0x43004300u, (x & 0x00800080u) | 0x43004300u); }
// Eight E2M1 codes as fp16 times 2^-14 (sign, two bits of exponent and one of fraction in their places): elements 0 2 | 1 3 | 4 6 | 5 7
__device__ __forceinline__ void e2m1_to_f16(uint32_t w, uint32_t mul, uint32_t (&r)[4]) {
    const uint32_t odd = (w & 0x80808080u) | ((w >> 3) & 0x0e0e0e0eu), even = ((w << 4) & 0x80808080u) | ((w << 1) & 0x0e0e0e0eu);
    r[0] = mul_f16x2(__byte_perm(even, 0u, 0x1404), mul);
    r[1] = mul_f16x2(__byte_perm(odd, 0u, 0x1404), mul);
    r[2] = mul_f16x2(__byte_perm(even, 0u, 0x3424), mul);
    r[3] = mul_f16x2(__byte_perm(odd, 0u, 0x3424), mul);
}
// E2M1 code i (0 to 3) of both halves of t as bf16 times 2^-126, times mul
template <int I>
__device__ __forceinline__ uint32_t e2m1_to_bf16(uint32_t t, uint32_t mul) {
    const uint32_t sign = (I < 3 ? t << (12 - 4 * I) : t) & 0x80008000u;
    const uint32_t mag = (I < 2 ? t << (6 - 4 * I) : t >> (4 * I - 6)) & 0x01c001c0u;
    return mul_bf16x2(sign | mag, mul);
}

template <int FMT, int DP> struct Layout {
    static constexpr int PER_BYTE = FMT == KV_CACHE_INT8 ? 1 : 2;
    static constexpr int ROW = DP / PER_BYTE;                                   // bytes of a head, padded
    static constexpr int KB = ROW / 4 < 16 ? ROW / 4 : 16, KCH = ROW / 4 / KB;  // keys: chunk j of lane c at byte (j * 4 + c) * KB
    static constexpr int VB = ROW / 8 < 16 ? ROW / 8 : 16, VCH = ROW / 8 / VB;  // values: chunk j of lane g at byte (j * 8 + g) * VB
    static constexpr int KC = KB * PER_BYTE, VC = VB * PER_BYTE;                // codes of a chunk
    static constexpr int KS = DP / 16;                                          // products of 16 along a head
    static constexpr int K_BYTES = kStep * ROW, SCALES = 2 * K_BYTES, FACTORS = SCALES + (FMT == KV_CACHE_INT8 ? 0 : 512), STAGE = FACTORS + 128 + 16;
    static constexpr int STAGES = ROW <= 128 ? 3 : 2;                           // steps in a warp's ring
    // element of q behind operand pair p, half e, of product s in lane c
    __device__ static __forceinline__ int element(int s, int c, int p, int e) {
        if (FMT == KV_CACHE_INT8) return (s / 4 * 4 + c) * KC + s % 4 * 4 + 2 * p + e;
        const int word = s / 2, words = KB / 4;
        return (word / words * 4 + c) * KC + word % words * 8 + s % 2 * 4 + p + 2 * e;
    }
};

// ------------------------------------------------------------------------------------------------ the kernel

template <int FMT, int DP, int MT>
struct Shared {
    using L = Layout<FMT, DP>;
    static constexpr int ROWS = 16 * MT;
    static constexpr int RING = kWarps * L::STAGES * L::STAGE, MERGE = kWarps * ROWS * (DP + 4) * 4;      // the ring, and over it the warps' results
    static constexpr int FRAGS = (RING > MERGE ? RING : MERGE), HALVES = FRAGS + MT * L::KS * 512, ROW_FACTOR = HALVES + ROWS * DP * 2;
    static constexpr int STATE = ROW_FACTOR + ROWS * 4, BYTES = STATE + 2 * kWarps * ROWS * 4;
};

template <int FMT, int DP, int MT>
__global__ void __launch_bounds__(kThreads, DP * MT <= 64 ? 4 : DP * MT <= 128 ? 3 : 2) kv_attention_kernel(const AttentionArgs a) {
    using L = Layout<FMT, DP>;
    using S = Shared<FMT, DP, MT>;
    constexpr int ROWS = S::ROWS;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ int last_one;
    grid_dep_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
    const Share share = share_out<kThreads>(a, ROWS);
    int64_t u = share.begin;
    const int64_t u_begin = u, u_end = share.end;
    int b = share.b;
    int64_t first_of_b = share.first_of_b;
    const int row_bytes = a.dim / L::PER_BYTE, blocks = (a.dim + kMxBlock - 1) / kMxBlock;
    const int64_t token_bytes = static_cast<int64_t>(a.heads) * row_bytes;
    uint8_t* const ring = smem + warp * L::STAGES * L::STAGE;
    const uint32_t ring_u32 = smem_u32(ring);

    while (u < u_end) {
        Sequence s = read_sequence(a, b, ROWS);
        while (b + 1 < a.seqs && u - first_of_b >= units_of(a, s)) {                  // (sequences without new tokens have no units)
            first_of_b += units_of(a, s);
            s = read_sequence(a, ++b, ROWS);
        }
        const int64_t of_b = u - first_of_b;
        const int item = static_cast<int>(of_b / s.tiles), tile0 = static_cast<int>(of_b - static_cast<int64_t>(item) * s.tiles);
        const int head = item / s.row_tiles, row0 = (item - head * s.row_tiles) * ROWS, rows = min(ROWS, s.n * a.group - row0);
        const int steps = static_cast<int>(min(static_cast<int64_t>(s.tiles - tile0), u_end - u));
        const int64_t item_begin = u - tile0, item_end = item_begin + s.tiles;
        const int first_token = s.start + tile0 * kTile + warp * kStep;

        // ---- the cache: a step's 16 tokens into a stage of the warp's ring, codes straight to the lane that will use them
        auto find = [&](int step) {                                 // slot of token lane % 16 of a step, -1: not seen
            const int t = first_token + step * kTile + (lane & 15);
            if (step >= steps || t >= s.stop) return -1;
            const uint32_t p = static_cast<uint32_t>(t) / static_cast<uint32_t>(a.page);
            const int id = a.table[b * a.table_stride + p];
            return id >= 0 && id < a.num_pages ? id * a.page + (t - static_cast<int>(p) * a.page) : -1;
        };
        auto issue = [&](int step, int slot) {
            if (step < steps) {
                const uint32_t st = ring_u32 + step % L::STAGES * L::STAGE;
                const uint32_t seen = __ballot_sync(0xffffffffu, slot >= 0) & 0xffffu;
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int at = __shfl_sync(0xffffffffu, slot, i * 8 + g);
                    const uint8_t* src = a.k_codes + max(at, 0) * token_bytes + head * row_bytes;
#pragma unroll
                    for (int j = 0; j < L::KCH; ++j) {
                        const int off = (j * 4 + c) * L::KB, valid = at >= 0 ? row_bytes - off : 0;
                        copy_codes<L::KB>(st + ((i * L::KCH + j) * 32 + lane) * L::KB, src + (valid > 0 ? off : 0), valid, a.copy);
                    }
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int at = __shfl_sync(0xffffffffu, slot, (i >> 1) * 8 + 2 * c + (i & 1));
                    const uint8_t* src = a.v_codes + max(at, 0) * token_bytes + head * row_bytes;
#pragma unroll
                    for (int j = 0; j < L::VCH; ++j) {
                        const int off = (j * 8 + g) * L::VB, valid = at >= 0 ? row_bytes - off : 0;
                        copy_codes<L::VB>(st + L::K_BYTES + ((i * L::VCH + j) * 32 + lane) * L::VB, src + (valid > 0 ? off : 0), valid, a.copy);
                    }
                }
                // scales: lanes 0 to 15 the keys', 16 to 31 the values'
                const int at = __shfl_sync(0xffffffffu, slot, lane & 15);
                const void* scales = lane < 16 ? a.k_scales : a.v_scales;
                const int64_t entry = static_cast<int64_t>(max(at, 0)) * a.heads + head;
                if (FMT == KV_CACHE_INT8) {
                    cp_async<4>(st + L::FACTORS + lane * 4, static_cast<const float*>(scales) + entry, at >= 0 ? 4 : 0);
                } else {                                            // the aligned words that hold the head's bytes, two at most
                    const uint8_t* p = static_cast<const uint8_t*>(scales) + entry * blocks;
                    const int shift = static_cast<int>(reinterpret_cast<uintptr_t>(p) & 3);
                    cp_async<4>(st + L::SCALES + lane * 16, p - shift, at >= 0 ? 4 : 0);
                    const bool two = shift + blocks > 4;
                    cp_async<4>(st + L::SCALES + lane * 16 + 4, p - shift + (two ? 4 : 0), at >= 0 && two ? 4 : 0);
                    *reinterpret_cast<int*>(ring + step % L::STAGES * L::STAGE + L::SCALES + lane * 16 + 8) = shift;
                }
                if (lane == 0) *reinterpret_cast<uint32_t*>(ring + step % L::STAGES * L::STAGE + L::FACTORS + 128) = seen;
            }
            cp_async_commit();
        };
        int slot;
        {
            int slots[L::STAGES];
#pragma unroll
            for (int i = 0; i < L::STAGES; ++i) slots[i] = find(i);
#pragma unroll
            for (int i = 0; i < L::STAGES - 1; ++i) issue(i, slots[i]);
            slot = slots[L::STAGES - 1];
        }

        // ---- queries: rows of fp16 times a power of two, then as operands of the products
        __half* const halves = reinterpret_cast<__half*>(smem + S::HALVES);
        float* const row_factor = reinterpret_cast<float*>(smem + S::ROW_FACTOR);
        for (int r = warp; r < ROWS; r += kWarps) {
            uint4 x = make_uint4(0, 0, 0, 0);
            if (r < rows && lane * 8 < a.dim) {
                const int node = (row0 + r) / a.group, h = head * a.group + (row0 + r) - node * a.group;
                x = *reinterpret_cast<const uint4*>(a.q + static_cast<int64_t>(s.begin + node) * a.q_st + h * a.q_sh + lane * 8);
            }
            uint32_t top = absmax_bits8(x);
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
            const int field = static_cast<int>(top >> 23);
            // the largest magnitude goes to [2^14, 2^15): elements down to 2^-28 of it stay exact
            const int up = field == 255 ? 0 : min(126, max(-126, 141 - max(field, 1)));
            const float mul = __uint_as_float((127 + up) << 23);
            float f[8];
            unpack_bf16x8(x, f);
            if (lane * 8 < DP) {
                __half2 h[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) h[i] = __floats2half2_rn(f[2 * i] * mul, f[2 * i + 1] * mul);
                *reinterpret_cast<uint4*>(halves + r * DP + lane * 8) = *reinterpret_cast<const uint4*>(h);
            }
            if (lane == 0) row_factor[r] = a.scale * kLog2e * __uint_as_float((127 - up) << 23);
        }
        __syncthreads();
        uint4* const frags = reinterpret_cast<uint4*>(smem + S::FRAGS);
        for (int e = threadIdx.x; e < MT * L::KS * 32; e += kThreads) {
            const int ln = e & 31, ks = e / 32 % L::KS, r = e / 32 / L::KS * 16 + (ln >> 2);
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const __half* from = halves + (r + (i & 1) * 8) * DP;
                const __half2 p = __halves2half2(from[L::element(ks, ln & 3, i >> 1, 0)], from[L::element(ks, ln & 3, i >> 1, 1)]);
                w[i] = *reinterpret_cast<const uint32_t*>(&p);
            }
            frags[e] = make_uint4(w[0], w[1], w[2], w[3]);
        }
        __syncthreads();

        // ---- the steps
        float o[MT][DP / 8][4], m[MT][2], l[MT][2], factor[MT][2];
#pragma unroll
        for (int i = 0; i < MT; ++i) {
#pragma unroll
            for (int j = 0; j < DP / 8; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[i][j][e] = 0.f;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                m[i][e] = -INFINITY;
                l[i][e] = 0.f;
                factor[i][e] = row_factor[i * 16 + e * 8 + g];
            }
        }
        for (int step = 0; step < steps; ++step) {
            cp_async_wait<L::STAGES - 2>();
            __syncwarp();
            issue(step + L::STAGES - 1, slot);
            slot = find(step + L::STAGES);
            uint8_t* const st = ring + step % L::STAGES * L::STAGE;
            const uint32_t seen16 = *reinterpret_cast<const uint32_t*>(st + L::FACTORS + 128);
            float* const factors = reinterpret_cast<float*>(st + L::FACTORS);
            uint32_t k_mul[2][L::KCH], v_mul[2][L::VCH];
            bool poison = false;
            if (FMT == KV_CACHE_MXFP4) {
                // a token's bytes and the largest of them, 2^(it - 127) being the token's factor: lane by lane, then for all to read
                const uint4 raw = *reinterpret_cast<const uint4*>(st + L::SCALES + lane * 16);
                uint64_t bytes = (static_cast<uint64_t>(raw.x) | static_cast<uint64_t>(raw.y) << 32) >> (8 * raw.z);
                if (blocks < 8) bytes &= (uint64_t{1} << (8 * blocks)) - 1;
                const uint32_t lo = static_cast<uint32_t>(bytes), hi = static_cast<uint32_t>(bytes >> 32);
                const bool nan = (__vcmpeq4(lo, 0xffffffffu) | __vcmpeq4(hi, 0xffffffffu)) != 0;
                // (values: a block that is NaN is so by itself, the token's other blocks are not)
                uint32_t top = __vmaxu4(lo & ~__vcmpeq4(lo, 0xffffffffu), hi & ~__vcmpeq4(hi, 0xffffffffu));
                top = __vmaxu4(top, top >> 16);
                top = max(top & 0xffu, (top >> 8) & 0xffu);
                poison = __any_sync(0xffffffffu, nan && lane >= 16);
                *reinterpret_cast<uint2*>(st + L::SCALES + lane * 16) = make_uint2(lo, hi);
                *reinterpret_cast<uint32_t*>(st + L::SCALES + lane * 16 + 8) = top;
                factors[lane] = nan && lane < 16 ? __uint_as_float(0x7fc00000u) : __uint_as_float(top == 0 ? 0x00400000u : top << 23);
                __syncwarp();
                const uint8_t* const sb = st + L::SCALES;
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int largest = sb[(i * 8 + g) * 16 + 8];
#pragma unroll
                    for (int j = 0; j < L::KCH; ++j) {
                        const int e = 29 + sb[(i * 8 + g) * 16 + (j * 4 + c) * L::KC / kMxBlock] - largest;        // 2^14 * 2^(byte - largest)
                        k_mul[i][j] = e > 0 ? static_cast<uint32_t>(e) * 0x04000400u : 0u;
                    }
#pragma unroll
                    for (int j = 0; j < L::VCH; ++j) {
                        uint32_t two = 0;
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const uint8_t* p = sb + (16 + i * 8 + 2 * c + h) * 16;
                            const int byte = p[(j * 8 + g) * L::VC / kMxBlock], e = 253 + byte - p[8];              // 2^126 * 2^(byte - largest)
                            two |= (byte == 255 ? 0x7fc0u : e > 0 ? static_cast<uint32_t>(e) << 7 : 0u) << (16 * h);
                        }
                        v_mul[i][j] = two;
                    }
                }
            }
            // scores
            float sc[MT][2][4];
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) sc[i][j][e] = 0.f;
#pragma unroll
            for (int j = 0; j < L::KCH; ++j) {
                uint32_t w[2][L::KB / 4];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const uint8_t* p = st + ((i * L::KCH + j) * 32 + lane) * L::KB;
                    if (L::KB == 16) *reinterpret_cast<uint4*>(w[i]) = *reinterpret_cast<const uint4*>(p);
                    else *reinterpret_cast<uint2*>(w[i]) = *reinterpret_cast<const uint2*>(p);
                }
#pragma unroll
                for (int x = 0; x < L::KB / 4; ++x) {
                    constexpr int PER = FMT == KV_CACHE_INT8 ? 1 : 2;           // products that a word feeds
                    uint32_t r[2][2 * PER];
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        if constexpr (FMT == KV_CACHE_INT8) int8_to_f16(w[i][x], r[i]);
                        else e2m1_to_f16(w[i][x], k_mul[i][j], r[i]);
                    }
#pragma unroll
                    for (int y = 0; y < PER; ++y) {
                        const int ks = (j * (L::KB / 4) + x) * PER + y;
#pragma unroll
                        for (int i = 0; i < MT; ++i) {
                            const uint4 q = frags[(i * L::KS + ks) * 32 + lane];
                            mma_f16(sc[i][0], q, r[0][2 * y], r[0][2 * y + 1]);
                            mma_f16(sc[i][1], q, r[1][2 * y], r[1][2 * y + 1]);
                        }
                    }
                }
            }
            // softmax: this lane's tokens are 2c, 2c + 1, 8 + 2c and 9 + 2c of the step
            const int t0 = first_token + step * kTile;
            const bool masked = seen16 != 0xffffu || t0 + kStep > s.before;
            float kf[4], vf[4];
            *reinterpret_cast<float2*>(kf) = *reinterpret_cast<const float2*>(factors + 2 * c);
            *reinterpret_cast<float2*>(kf + 2) = *reinterpret_cast<const float2*>(factors + 8 + 2 * c);
            *reinterpret_cast<float2*>(vf) = *reinterpret_cast<const float2*>(factors + 16 + 2 * c);
            *reinterpret_cast<float2*>(vf + 2) = *reinterpret_cast<const float2*>(factors + 24 + 2 * c);
            uint4 p[MT];
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                uint32_t sees[2] = {15u, 15u};
                if (masked) {
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int node = min(row0 + i * 16 + e * 8 + g, s.n * a.group - 1) / a.group;
                        sees[e] = 0;
#pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            const int at = (x >> 1) * 8 + 2 * c + (x & 1), j = t0 + at - s.before;
                            bool see = (seen16 >> at & 1u) != 0;
                            if (see && j >= 0) {
                                if (a.tree == nullptr) see = j <= node;
                                else see = (j >> 6) < a.tree_words && (a.tree[static_cast<int64_t>(s.begin + node) * a.tree_words + (j >> 6)] >> (j & 63) & 1) != 0;
                            }
                            sees[e] |= static_cast<uint32_t>(see) << x;
                        }
                    }
                    if (FMT == KV_CACHE_MXFP4 && poison) {
                        // NaN blocks of values, for the rows that see them only: taken out of the product, put into the sums
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            uint32_t bad = 0;
                            for (int x = 0; x < 4; ++x) {
                                if (!(sees[e] >> x & 1u)) continue;
                                const uint8_t* bytes = st + L::SCALES + (16 + (x >> 1) * 8 + 2 * c + (x & 1)) * 16;
                                for (int k = 0; k < blocks; ++k) bad |= static_cast<uint32_t>(bytes[k] == 255) << k;
                            }
                            bad |= __shfl_xor_sync(0xffffffffu, bad, 1);
                            bad |= __shfl_xor_sync(0xffffffffu, bad, 2);
#pragma unroll
                            for (int j = 0; j < L::VCH; ++j)
#pragma unroll
                                for (int h = 0; h < 2; ++h)
                                    if (bad >> ((j * 8 + 2 * c + h) * L::VC / kMxBlock) & 1u)
#pragma unroll
                                        for (int x = 0; x < L::VC; ++x) o[i][j * L::VC + x][2 * e + h] = __uint_as_float(0x7fc00000u);
                        }
                    }
                }
                float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float v = sc[i][j][e] * kf[2 * j + (e & 1)] * factor[i][e >> 1];
                        if (masked && !(sees[e >> 1] >> (2 * j + (e & 1)) & 1u)) v = -INFINITY;
                        sc[i][j][e] = v;
                        top[e >> 1] = fmaxf(top[e >> 1], v);
                    }
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    top[e] = fmaxf(top[e], __shfl_xor_sync(0xffffffffu, top[e], 1));
                    top[e] = fmaxf(top[e], __shfl_xor_sync(0xffffffffu, top[e], 2));
                }
                // the running maximum may lag by 2^8: nothing is rescaled for less
                if (__any_sync(0xffffffffu, top[0] > m[i][0] + 8.f || top[1] > m[i][1] + 8.f)) {
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const float now = fmaxf(m[i][e], top[e]), scale = now == -INFINITY ? 1.f : ex2(m[i][e] - now);
                        m[i][e] = now;
                        l[i][e] *= scale;
#pragma unroll
                        for (int j = 0; j < DP / 8; ++j) {
                            o[i][j][2 * e] *= scale;
                            o[i][j][2 * e + 1] *= scale;
                        }
                    }
                }
                const float base[2] = {m[i][0] == -INFINITY ? 0.f : m[i][0], m[i][1] == -INFINITY ? 0.f : m[i][1]};
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float x = ex2(sc[i][j][e] - base[e >> 1]);
                        l[i][e >> 1] += x;
                        sc[i][j][e] = masked && !(sees[e >> 1] >> (2 * j + (e & 1)) & 1u) ? 0.f : x * vf[2 * j + (e & 1)];
                    }
                p[i] = make_uint4(pack_bf16(sc[i][0][0], sc[i][0][1]), pack_bf16(sc[i][0][2], sc[i][0][3]), pack_bf16(sc[i][1][0], sc[i][1][1]),
                                  pack_bf16(sc[i][1][2], sc[i][1][3]));
            }
            if (FMT == KV_CACHE_MXFP4 && masked && poison) {
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < L::VCH; ++j) {
                        if ((v_mul[i][j] & 0xffffu) == 0x7fc0u) v_mul[i][j] &= 0xffff0000u;
                        if (v_mul[i][j] >> 16 == 0x7fc0u) v_mul[i][j] &= 0xffffu;
                    }
            }
            // values
#pragma unroll
            for (int j = 0; j < L::VCH; ++j) {
                uint32_t w[4][L::VB / 4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint8_t* from = st + L::K_BYTES + ((i * L::VCH + j) * 32 + lane) * L::VB;
                    if constexpr (L::VB == 16) *reinterpret_cast<uint4*>(w[i]) = *reinterpret_cast<const uint4*>(from);
                    else if constexpr (L::VB == 8) *reinterpret_cast<uint2*>(w[i]) = *reinterpret_cast<const uint2*>(from);
                    else w[i][0] = *reinterpret_cast<const uint32_t*>(from);
                }
#pragma unroll
                for (int x = 0; x < L::VB / 4; ++x) {
#pragma unroll
                    for (int half = 0; half < 2; ++half) {                      // two bytes of each token's word, tokens side by side
                        const uint32_t t0w = __byte_perm(w[0][x], w[1][x], half ? 0x7632 : 0x5410), t1w = __byte_perm(w[2][x], w[3][x], half ? 0x7632 : 0x5410);
                        if constexpr (FMT == KV_CACHE_INT8) {
#pragma unroll
                            for (int y = 0; y < 2; ++y) {
                                const uint32_t b0 = int8_to_bf16(y ? t0w >> 8 : t0w), b1 = int8_to_bf16(y ? t1w >> 8 : t1w);
#pragma unroll
                                for (int i = 0; i < MT; ++i) mma_bf16(o[i][j * L::VC + x * 4 + half * 2 + y], p[i], b0, b1);
                            }
                        } else {
                            const uint32_t b0[4] = {e2m1_to_bf16<0>(t0w, v_mul[0][j]), e2m1_to_bf16<1>(t0w, v_mul[0][j]), e2m1_to_bf16<2>(t0w, v_mul[0][j]),
                                                    e2m1_to_bf16<3>(t0w, v_mul[0][j])};
                            const uint32_t b1[4] = {e2m1_to_bf16<0>(t1w, v_mul[1][j]), e2m1_to_bf16<1>(t1w, v_mul[1][j]), e2m1_to_bf16<2>(t1w, v_mul[1][j]),
                                                    e2m1_to_bf16<3>(t1w, v_mul[1][j])};
#pragma unroll
                            for (int y = 0; y < 4; ++y)
#pragma unroll
                                for (int i = 0; i < MT; ++i) mma_bf16(o[i][j * L::VC + x * 8 + half * 4 + y], p[i], b0[y], b1[y]);
                        }
                    }
                }
            }
        }
        cp_async_wait<0>();

        // ---- the warps' results meet in shared memory
        __syncthreads();
        float* const merge = reinterpret_cast<float*>(smem);
        float* const state = reinterpret_cast<float*>(smem + S::STATE);                       // [warp][row] maxima, then sums
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int r = i * 16 + e * 8 + g;
                float sum = l[i][e];
                sum += __shfl_xor_sync(0xffffffffu, sum, 1);
                sum += __shfl_xor_sync(0xffffffffu, sum, 2);
                if (c == 0) {
                    state[warp * ROWS + r] = m[i][e];
                    state[(kWarps + warp) * ROWS + r] = sum;
                }
                float* to = merge + (warp * ROWS + r) * (DP + 4);
#pragma unroll
                for (int j = 0; j < L::VCH; ++j)
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int x = 0; x < L::VC; x += 4)
                            *reinterpret_cast<float4*>(to + (j * 8 + 2 * c + h) * L::VC + x) =
                                make_float4(o[i][j * L::VC + x][2 * e + h], o[i][j * L::VC + x + 1][2 * e + h], o[i][j * L::VC + x + 2][2 * e + h], o[i][j * L::VC + x + 3][2 * e + h]);
            }
        __syncthreads();
        const bool whole = tile0 == 0 && steps == s.tiles;
        constexpr int PART = ROWS * (DP + 2);
        float* const part = a.parts + (2 * static_cast<int64_t>(blockIdx.x) + (u_begin > item_begin ? 0 : 1)) * PART;
        auto finish = [&](int r, int d, const float (&v)[4], float top, float sum) {          // four elements of a row
            const int node = (row0 + r) / a.group, h = head * a.group + (row0 + r) - node * a.group;
            const float inv = sum == 0.f ? 0.f : 1.f / sum;
            const uint2 two = sum == 0.f ? make_uint2(0, 0) : make_uint2(pack_bf16(v[0] * inv, v[1] * inv), pack_bf16(v[2] * inv, v[3] * inv));
            *reinterpret_cast<uint2*>(a.out + static_cast<int64_t>(s.begin + node) * a.o_st + h * a.o_sh + d) = two;
            if (d == 0 && a.lse != nullptr)
                a.lse[static_cast<int64_t>(s.begin + node) * a.heads * a.group + h] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * kLn2;
        };
        const int quads = a.dim / 4;
        for (int e = threadIdx.x; e < rows * quads; e += kThreads) {
            const int r = e / quads, d = (e - r * quads) * 4;
            float top = -INFINITY;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) top = fmaxf(top, state[w * ROWS + r]);
            float v[4] = {0.f, 0.f, 0.f, 0.f}, sum = 0.f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                const float weight = top == -INFINITY ? 1.f : ex2(state[w * ROWS + r] - top);
                const float4 x = *reinterpret_cast<const float4*>(merge + (w * ROWS + r) * (DP + 4) + d);
                sum += weight * state[(kWarps + w) * ROWS + r];
                v[0] += weight * x.x; v[1] += weight * x.y; v[2] += weight * x.z; v[3] += weight * x.w;
            }
            if (whole) {
                finish(r, d, v, top, sum);
            } else {
                *reinterpret_cast<float4*>(part + r * DP + d) = make_float4(v[0], v[1], v[2], v[3]);
                if (d == 0) {
                    part[ROWS * DP + r] = top;
                    part[ROWS * DP + ROWS + r] = sum;
                }
            }
        }
        if (!whole) {
            const int first = owner(item_begin, share), last = owner(item_end - 1, share);
            // (place of the item's counter: sequences' row tiles one after another, a place more for each that ends in the middle of one)
            uint32_t* const counter = a.counters + (static_cast<int64_t>(b) + static_cast<int64_t>(s.begin) * a.group / ROWS + row0 / ROWS) * a.heads + head;
            __threadfence();
            __syncthreads();
            if (threadIdx.x == 0) last_one = atomicAdd(counter, 1u) == static_cast<uint32_t>(last - first);
            __syncthreads();
            if (last_one) {
                if (threadIdx.x == 0) *counter = 0;
                __threadfence();
                for (int e = threadIdx.x; e < rows * quads; e += kThreads) {
                    const int r = e / quads, d = (e - r * quads) * 4;
                    float v[4] = {0.f, 0.f, 0.f, 0.f}, sum = 0.f, top = -INFINITY;
                    for (int x = first; x <= last; ++x) {
                        const float* from = a.parts + (2 * static_cast<int64_t>(x) + (x == first ? 1 : 0)) * PART;
                        const float4 y = __ldcg(reinterpret_cast<const float4*>(from + r * DP + d));
                        const float its_top = __ldcg(from + ROWS * DP + r), its_sum = __ldcg(from + ROWS * DP + ROWS + r);
                        const float now = fmaxf(top, its_top);
                        const float mine = now == -INFINITY ? 1.f : ex2(top - now), its = now == -INFINITY ? 1.f : ex2(its_top - now);
                        top = now;
                        sum = sum * mine + its_sum * its;
                        v[0] = v[0] * mine + y.x * its; v[1] = v[1] * mine + y.y * its; v[2] = v[2] * mine + y.z * its; v[3] = v[3] * mine + y.w * its;
                    }
                    finish(r, d, v, top, sum);
                }
            }
        }
        __syncthreads();                                            // shared memory is the next item's
        u += steps;
    }
    if (a.zero_rest != 0) {                                         // rows of no sequence
        const int lo = a.seqs > 0 ? max(0, min(a.cu_q[0], a.total_q)) : a.total_q, hi = a.seqs > 0 ? max(lo, min(a.cu_q[a.seqs], a.total_q)) : a.total_q;
        const int q_heads = a.heads * a.group, eights = a.dim / 8;
        const int64_t rest = lo + (a.total_q - hi), each = static_cast<int64_t>(q_heads) * eights;
        for (int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; i < rest * each; i += static_cast<int64_t>(gridDim.x) * kThreads) {
            int64_t t = i / each;
            const int e = static_cast<int>(i - t * each), h = e / eights, d = (e - h * eights) * 8;
            t = t < lo ? t : hi + (t - lo);
            *reinterpret_cast<uint4*>(a.out + t * a.o_st + h * a.o_sh + d) = make_uint4(0, 0, 0, 0);
            if (d == 0 && a.lse != nullptr) a.lse[t * q_heads + h] = -INFINITY;
        }
    }
}

// ------------------------------------------------------------------------------------------------ host

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

constexpr int kSmallestRows = 16;                   // rows of the smallest item: the most items, so the most counters
constexpr int kMostCtas = 4;                        // CTAs on an SM
constexpr size_t kAlign = 256;

size_t counters_bytes(int64_t seqs, int64_t total_q, int64_t q_heads, int64_t heads) {
    const int64_t group = q_heads / heads;
    return (static_cast<size_t>(seqs + total_q * group / kSmallestRows + 1) * heads * sizeof(uint32_t) + kAlign - 1) / kAlign * kAlign;
}
int padded(int64_t dim) { return dim <= 64 ? 64 : dim <= 128 ? 128 : 256; }
size_t parts_bytes(int64_t dim) { return static_cast<size_t>(sm_count()) * kMostCtas * 2 * 32 * (padded(dim) + 2) * sizeof(float); }
bool sizes_fine(int64_t seqs, int64_t total_q, int64_t q_heads, int64_t heads, int64_t dim) {
    return seqs >= 0 && seqs < INT32_MAX && total_q >= 0 && total_q <= INT32_MAX && heads > 0 && q_heads > 0 && q_heads <= KV_CACHE_MAX_WIDTH && q_heads % heads == 0 && dim > 0 &&
           dim <= KV_CACHE_MAX_DIM && q_heads * dim <= KV_CACHE_MAX_WIDTH && heads * dim <= KV_CACHE_MAX_WIDTH && total_q * q_heads <= INT32_MAX;
}

template <int FMT, int DP, int MT>
cudaError_t launch(const AttentionArgs& a, cudaStream_t st) {
    static PerDeviceOnce once;
    static int per_sm = 1;                          // (the same on every device that the library runs on)
    constexpr int bytes = Shared<FMT, DP, MT>::BYTES;
    const auto kern = kv_attention_kernel<FMT, DP, MT>;
    cudaError_t e = once.run([&] {
        const cudaError_t set = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
        if (set != cudaSuccess) return set;
        int n = 0;
        const cudaError_t asked = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kern, kThreads, bytes);
        per_sm = n < 1 ? 1 : n > kMostCtas ? kMostCtas : n;
        return asked;
    });
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(sm_count() * per_sm));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = bytes;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kern, a);
}
template <int FMT>
cudaError_t launch_for(const AttentionArgs& a, int64_t most_rows, cudaStream_t st) {
    const int dp = padded(a.dim);
    const bool two = most_rows > 16;
    if (dp == 64) return two ? launch<FMT, 64, 2>(a, st) : launch<FMT, 64, 1>(a, st);
    if (dp == 128) return two ? launch<FMT, 128, 2>(a, st) : launch<FMT, 128, 1>(a, st);
    return launch<FMT, 256, 1>(a, st);
}

} // namespace
} // namespace w8a8

extern "C" {

using namespace w8a8;

size_t kv_cache_attention_zeroed_bytes(int64_t seqs, int64_t total_q, int64_t q_heads, int64_t heads, int64_t dim) {
    return sizes_fine(seqs, total_q, q_heads, heads, dim) ? counters_bytes(seqs, total_q, q_heads, heads) : 0;
}
size_t kv_cache_attention_workspace_bytes(int64_t seqs, int64_t total_q, int64_t q_heads, int64_t heads, int64_t dim) {
    return sizes_fine(seqs, total_q, q_heads, heads, dim) ? counters_bytes(seqs, total_q, q_heads, heads) + parts_bytes(dim) : 0;
}

int kv_cache_attention(int fmt, const void* k_codes, const void* k_scales, const void* v_codes, const void* v_scales, int64_t num_pages, int64_t page_size,
                       int64_t heads, int64_t dim, const int32_t* table, int64_t table_stride, int64_t max_pages, const int32_t* lens, const int32_t* starts,
                       const int32_t* cu_q, int64_t seqs, const void* q, int64_t q_token_stride, int64_t q_head_stride, int64_t q_heads, int64_t total_q,
                       const int64_t* tree, int64_t tree_words, float scale, void* out, int64_t out_token_stride, int64_t out_head_stride, float* lse,
                       void* workspace, size_t workspace_bytes, void* stream) {
    const bool zero_rest = (fmt & KV_CACHE_ZERO_REST) != 0;
    fmt &= ~KV_CACHE_ZERO_REST;
    if ((fmt != KV_CACHE_INT8 && fmt != KV_CACHE_MXFP4) || !sizes_fine(seqs, total_q, q_heads, heads, dim)) return W8A8_ERR_INVALID_ARG;
    if (num_pages < 0 || page_size <= 0 || page_size > INT32_MAX || num_pages > INT32_MAX / page_size || max_pages < 0 || max_pages > INT32_MAX || table_stride < max_pages ||
        (seqs > 0 && (lens == nullptr || cu_q == nullptr)) || (seqs > 0 && max_pages > 0 && table == nullptr) || (total_q > 0 && (q == nullptr || out == nullptr)) ||
        (tree != nullptr && (tree_words <= 0 || tree_words > INT32_MAX)) || !std::isfinite(scale))
        return W8A8_ERR_INVALID_ARG;
    if (num_pages > 0 && (k_codes == nullptr || k_scales == nullptr || v_codes == nullptr || v_scales == nullptr)) return W8A8_ERR_INVALID_ARG;
    if (dim % 8 != 0 || !aligned(k_codes, 16) || !aligned(v_codes, 16) || !aligned(k_scales, 4) || !aligned(v_scales, 4) || !aligned(table, 4) || !aligned(lens, 4) ||
        !aligned(starts, 4) || !aligned(cu_q, 4) || !aligned(tree, 8) || !aligned(lse, 4) || !aligned(q, 16) || q_token_stride % 8 != 0 || q_head_stride % 8 != 0 ||
        !aligned(out, 16) || out_token_stride % 8 != 0 || out_head_stride % 8 != 0)
        return W8A8_ERR_ALIGNMENT;
    if (workspace == nullptr || !aligned(workspace, kAlign) || workspace_bytes < kv_cache_attention_workspace_bytes(seqs, total_q, q_heads, heads, dim)) return W8A8_ERR_WORKSPACE;
    if (int e = check_arch()) return e;
    if (total_q == 0 || (seqs == 0 && !zero_rest)) return W8A8_OK;
    AttentionArgs a{};
    a.k_codes = static_cast<const uint8_t*>(k_codes);
    a.v_codes = static_cast<const uint8_t*>(v_codes);
    a.k_scales = k_scales;
    a.v_scales = v_scales;
    a.table = table;
    a.lens = lens;
    a.starts = starts;
    a.cu_q = cu_q;
    a.tree = tree;
    a.q = static_cast<const __nv_bfloat16*>(q);
    a.out = static_cast<__nv_bfloat16*>(out);
    a.lse = lse;
    a.counters = static_cast<uint32_t*>(workspace);
    a.parts = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + counters_bytes(seqs, total_q, q_heads, heads));
    a.q_st = q_token_stride;
    a.q_sh = q_head_stride;
    a.o_st = out_token_stride;
    a.o_sh = out_head_stride;
    a.table_stride = table_stride;
    a.tree_words = tree_words;
    a.num_pages = static_cast<int>(num_pages);
    a.page = static_cast<int>(page_size);
    a.max_pages = static_cast<int>(max_pages);
    a.heads = static_cast<int>(heads);
    a.group = static_cast<int>(q_heads / heads);
    a.dim = static_cast<int>(dim);
    a.seqs = static_cast<int>(seqs);
    a.total_q = static_cast<int>(total_q);
    const int64_t row_bytes = fmt == KV_CACHE_INT8 ? dim : dim / 2;
    a.copy = row_bytes % 16 == 0 ? 16 : row_bytes % 8 == 0 ? 8 : 4;
    a.scale = scale;
    a.zero_rest = zero_rest ? 1 : 0;
    const int64_t most_rows = total_q * a.group / (seqs > 0 ? seqs : 1);
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    const cudaError_t e = fmt == KV_CACHE_INT8 ? launch_for<KV_CACHE_INT8>(a, most_rows, st) : launch_for<KV_CACHE_MXFP4>(a, most_rows, st);
    return e == cudaSuccess ? W8A8_OK : W8A8_ERR_CUDA;
}

} // extern "C"
