// What the kernels of the attention over the cache share: the list of work, conversions of codes, results and their merging. Device code only.
#pragma once

#include "../../include/kv_cache.h"
#include "mxfp4_math.cuh"
#include "ptx.cuh"
#include "scale_words.h"

#include <cuda.h>
#include <cuda_fp16.h>

namespace w8a8 {
namespace attention {

constexpr int kMostBox = 64;                    // tokens of a box of codes, at most
constexpr float kNone = -3e38f;                 // reference of a row that has seen nothing (finite, so that differences are numbers)
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
    int page_shift;                             // log2 of the page, or -1
    int box, box_step;                          // tokens of a box of codes, elements from a box to the one beside it; 0: no boxes
    float scale;
    int zero_rest;
    int *status, *sticky;
    uint64_t limit_ns;
    int starve;                                 // test hook: the first load of every CTA never arrives
};

// ------------------------------------------------------------------------------------------------ the list of work

struct Sequence {
    int begin, n;                               // its rows of q
    int before;                                 // tokens ahead of the new ones (negative if the cache holds fewer than n)
    int start, stop;                            // tokens that may be seen
    int base;                                   // where the units begin: start, rounded down to whole boxes
    int tiles, row_tiles;
};
template <int TILE>                             // tokens of a unit
__device__ __forceinline__ Sequence read_sequence(const AttentionArgs& a, int b, int rows_of_tile) {
    Sequence s;
    const int begin = a.cu_q[b], end = a.cu_q[b + 1], len = a.lens[b];
    const int64_t most = static_cast<int64_t>(a.max_pages) * a.page;
    s.begin = max(0, min(begin, a.total_q));
    s.n = max(s.begin, min(end, a.total_q)) - s.begin;
    s.before = max(len, 0) - s.n;
    s.stop = static_cast<int>(min(static_cast<int64_t>(max(len, 0)), most));
    s.start = a.starts != nullptr ? max(0, min(a.starts[b], s.stop)) : 0;
    s.base = s.start & ~(kMostBox - 1);
    s.tiles = max(1, (s.stop - s.base + TILE - 1) / TILE);
    s.row_tiles = static_cast<int>((static_cast<int64_t>(s.n) * a.group + rows_of_tile - 1) / rows_of_tile);
    return s;
}
__device__ __forceinline__ int64_t units_of(const AttentionArgs& a, const Sequence& s) { return static_cast<int64_t>(a.heads) * s.row_tiles * s.tiles; }

// a / b of what is not negative: in 32 bits where it fits (a division of 64 bits takes several times as long, and a CTA begins with a few)
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) {
    return ((a | b) >> 32) == 0 ? static_cast<int64_t>(static_cast<uint32_t>(a) / static_cast<uint32_t>(b)) : a / b;
}

struct Share {
    int64_t total, first_of_b;                  // units of all sequences; of those before b
    int64_t ctas;                               // CTAs that work: none without a unit
    int64_t begin, end;                         // this CTA's units
    int b;
};
__device__ __forceinline__ int64_t warp_scan(int64_t v) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t w = __shfl_up_sync(0xffffffffu, v, o);
        if ((threadIdx.x & 31) >= o) v += w;
    }
    return v;
}
// This CTA's units, and the sequence that the first of them belongs to: found by all threads at once
template <int THREADS, int TILE>
__device__ __forceinline__ Share share_out(const AttentionArgs& a, int rows_of_tile) {
    __shared__ int64_t of_warp[THREADS / 32];
    __shared__ int64_t first_unit;
    __shared__ int found;
    const int per = (a.seqs + THREADS - 1) / THREADS, b0 = min(a.seqs, static_cast<int>(threadIdx.x) * per), b1 = min(a.seqs, b0 + per);
    int64_t mine = 0;
    for (int b = b0; b < b1; ++b) mine += units_of(a, read_sequence<TILE>(a, b, rows_of_tile));
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
    // up to four units a CTA: no more CTAs than it takes for the one with the most units to have no fewer. 5 sequences of 7 nodes and 1500 tokens, 940 units, are over after 2
    // units a CTA on 470 CTAs as on 592, which share more items and SMs: 21.5 us against 24.2. (Longer ranges gain nothing, and that they end at different times spreads the
    // joining of parts: 104 against 107 us for 12 sequences of up to 30000 tokens.)
    const int64_t most = max(quotient(total + gridDim.x - 1, gridDim.x), int64_t{1}), ctas = most <= 4 ? quotient(total + most - 1, most) : static_cast<int64_t>(gridDim.x);
    const int64_t u = blockIdx.x < ctas ? quotient(total * blockIdx.x, ctas) : total;
    if (u >= before && u < before + mine) {
        for (int b = b0; b < b1; ++b) {
            const int64_t units = units_of(a, read_sequence<TILE>(a, b, rows_of_tile));
            if (u < before + units) {
                found = b;
                first_unit = before;
                break;
            }
            before += units;
        }
    }
    __syncthreads();
    return Share{total, found < a.seqs ? first_unit : 0, ctas, u, blockIdx.x < ctas ? quotient(total * (blockIdx.x + 1), ctas) : u, found};
}

// The CTA whose range holds unit u (CTA c takes units total * c / ctas up to total * (c + 1) / ctas)
__device__ __forceinline__ int owner(int64_t u, const Share& s) { return static_cast<int>(quotient((u + 1) * s.ctas - 1, s.total)); }

// ------------------------------------------------------------------------------------------------ small pieces

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float y;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
    return y;
}
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&p);
}
__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
    const __half2 p = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&p);
}
__device__ __forceinline__ float lg2(float x) {
    float y;
    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
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
__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// 8 x 8 halves, lane (g, c) holding row g, columns 2c and 2c + 1: the transpose in the same places
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
template <int BYTES>
__device__ __forceinline__ void cp_async(uint32_t dst, const void* src, uint32_t valid) {      // valid: BYTES, or 0 for zeros
    if (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(valid) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(dst), "l"(src), "n"(BYTES), "r"(valid) : "memory");
}
// one arrival on `bar` (not counted as pending by it) once the copies that this thread has asked for are there
__device__ __forceinline__ void cp_async_mbar_arrive(uint32_t bar) { asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
// a box of a head's codes (16-byte chunks swizzled), rows one token apart
__device__ __forceinline__ void tma_load_3d(uint32_t smem_dst, const void* tmap, uint32_t bar, int x, int y, int z) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                 ::"r"(smem_dst), "l"(reinterpret_cast<uint64_t>(tmap)), "r"(bar), "r"(x), "r"(y), "r"(z) : "memory");
}

// ------------------------------------------------------------------------------------------------ codes to matrix operands

// Four int8 codes, bytes 0 and 1 and bytes 2 and 3, as fp16: code + 128 in the low byte of 1024, minus 1152
__device__ __forceinline__ void int8_to_f16(uint32_t w, uint32_t& r0, uint32_t& r1) {
    const uint32_t t = w ^ 0x80808080u;
    r0 = sub_f16x2(__byte_perm(t, 0x64646464u, 0x4140), 0x64806480u);
    r1 = sub_f16x2(__byte_perm(t, 0x64646464u, 0x4342), 0x64806480u);
}
// Eight E2M1 codes as fp16, in pairs
__device__ __forceinline__ void e2m1_to_f16(uint32_t w, uint32_t (&r)[4]) {
    asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t"
        "mov.b32 {b0, b1, b2, b3}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, b0;\n\t"
        "cvt.rn.f16x2.e2m1x2 %1, b1;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, b2;\n\t"
        "cvt.rn.f16x2.e2m1x2 %3, b3;\n\t}"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(w));
}

// ------------------------------------------------------------------------------------------------ results

// Four elements of a row, on their way from parts to the output: o stands for o * 2^(m_l + m_o), l for l * 2^m_l. (m_o is of the size of the values' scales; with m_l in it, which
// may be any fp32 number, it would be rounded to that one's spacing, and the result with it.)
struct Row {
    float o[4] = {0.f, 0.f, 0.f, 0.f}, m_o = kNone, m_l = kNone, l = 0.f;
    __device__ __forceinline__ void add(const float4& x, float its_m_o, float its_m_l, float its_l) {
        const float now_l = fmaxf(m_l, its_m_l), down = m_l - now_l, its_down = its_m_l - now_l;
        const float now_o = fmaxf(m_o + down, its_m_o + its_down), mine_o = ex2(m_o + down - now_o), its_o = ex2(its_m_o + its_down - now_o);
        l = l * ex2(down) + its_l * ex2(its_down);
        o[0] = o[0] * mine_o + x.x * its_o;
        o[1] = o[1] * mine_o + x.y * its_o;
        o[2] = o[2] * mine_o + x.z * its_o;
        o[3] = o[3] * mine_o + x.w * its_o;
        m_o = now_o;
        m_l = now_l;
    }
    // r: row of the sequence's new tokens and the group's heads. The result is o * 2^m_o / l, 4-bit: / 2^12. The power
    // may be more than fp32 spans while the result is not: it is applied in two halves.
    template <int FMT>
    __device__ __forceinline__ float2 scale() const {           // o times x, times y, times y is the result (l == 0: it is 0)
        return make_float2(1.f / l, ex2(fminf(fmaxf(0.5f * (m_o - (FMT == KV_CACHE_INT8 ? 0.f : 12.f)), -126.f), 126.f)));
    }
    __device__ __forceinline__ void write_lse(const AttentionArgs& a, const Sequence& s, int node, int h) const {
        if (a.lse != nullptr) a.lse[static_cast<int64_t>(s.begin + node) * a.heads * a.group + h] = l == 0.f ? -INFINITY : (m_l + log2f(l)) * kLn2;
    }
    template <int FMT>
    __device__ __forceinline__ void finish(const AttentionArgs& a, const Sequence& s, int head, int r, int d) const {
        const int node = r / a.group, h = head * a.group + r - node * a.group;
        float v[4];
        const float2 by = scale<FMT>();
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = l == 0.f ? 0.f : o[i] * by.x * by.y * by.y;
        *reinterpret_cast<uint2*>(a.out + static_cast<int64_t>(s.begin + node) * a.o_st + h * a.o_sh + d) = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
        if (d == 0) write_lse(a, s, node, h);
    }
};
constexpr __host__ __device__ int part_floats(int rows, int dp) { return rows * (dp + 4); }

// Rows of no sequence
template <int THREADS>
__device__ __forceinline__ void zero_rest(const AttentionArgs& a) {
    if (a.zero_rest == 0) return;
    const int lo = a.seqs > 0 ? max(0, min(a.cu_q[0], a.total_q)) : a.total_q, hi = a.seqs > 0 ? max(lo, min(a.cu_q[a.seqs], a.total_q)) : a.total_q;
    const int q_heads = a.heads * a.group, eights = a.dim / 8;
    const int64_t rest = lo + (a.total_q - hi), each = static_cast<int64_t>(q_heads) * eights;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * THREADS + threadIdx.x; i < rest * each; i += static_cast<int64_t>(gridDim.x) * THREADS) {
        int64_t t = i / each;
        const int e = static_cast<int>(i - t * each), h = e / eights, d = (e - h * eights) * 8;
        t = t < lo ? t : hi + (t - lo);
        *reinterpret_cast<uint4*>(a.out + t * a.o_st + h * a.o_sh + d) = make_uint4(0, 0, 0, 0);
        if (d == 0 && a.lse != nullptr) a.lse[t * q_heads + h] = -INFINITY;
    }
}

// Whether this segment of an item is the last to arrive, of those that CTAs `first` to `last` work on: its threads (which `sync` brings together, `me` of
// them) find all parts written.
template <int ROWS, typename Sync>
__device__ __forceinline__ bool last_to_arrive(const AttentionArgs& a, const Sequence& s, int b, int head, int row0, int first, int last, int me, int* last_one, Sync sync) {
    // (place of the item's counter: sequences' row tiles one after another, a place more for each that ends in the middle of one)
    uint32_t* const counter = a.counters + (static_cast<int64_t>(b) + static_cast<int64_t>(s.begin) * a.group / ROWS + row0 / ROWS) * a.heads + head;
    __threadfence();
    sync();
    if (me == 0) *last_one = atomicAdd(counter, 1u) == static_cast<uint32_t>(last - first);
    sync();
    if (!*last_one) return false;
    if (me == 0) *counter = 0;
    __threadfence();
    return true;
}

// ---- kv_attention_tc.cu : the attention for many rows of queries a head (the maps: codes of keys and of values in boxes of a.box tokens of a head)
bool many_rows_fits(int dim);                                              // what the kernel can run
size_t many_rows_part_bytes();                                             // scratch for the parts of any call
cudaError_t launch_many_rows(int fmt, const CUtensorMap& k_map, const CUtensorMap& v_map, const AttentionArgs& a, int64_t rows, cudaStream_t st);

} // namespace attention
} // namespace w8a8
