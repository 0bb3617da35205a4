// Attention over the quantized cache for many rows of queries a head: trees of drafted tokens with grouped heads, chains, prompts.
//
// Both products run on the tensor memory's matrix unit, 128 rows of queries at a time: S = Q K^T with Q and K in shared memory, O += P V with P in
// tensor memory, where it lies over the scores it came from. Eight warps turn the cache's codes into fp16 tiles of 128 tokens (keys: the codes, whose scale goes
// to the scores; values: codes times scale, relative to the largest scale so far), a thread a row does the softmax, one warp issues the products.
//
// Two softmax warpgroups, each with scores and an O of its own: of the same 128 rows and every other tile of tokens, or (PAIR) of 128 rows each and all
// tiles, which then are converted once for 256 rows. What bounds it: the exponentials (128 x 128 a tile at 16 a cycle: 1024 cycles, the two products' time) and the
// issue slots of softmax and conversion.
#include "internal.h"
#include "kv_attention.cuh"

#include <cmath>

namespace w8a8 {
namespace attention {
namespace {

constexpr int kTok = 128;                       // tokens of a tile
constexpr int kRows = 128;                      // rows of a product
constexpr int kConvertWarp = 8, kMmaWarp = 16, kThreads = 32 * 17, kConverters = 256, kSoftmax = 256;
constexpr int kWaitMany = 41;                   // which wait gave up, for the status word: this and the 8 after it
constexpr int kSlots = 4;                       // tiles whose factors are kept

template <int FMT, int DP, bool PAIR>
struct Plan {
    static constexpr int ROWS = PAIR ? 2 * kRows : kRows;
    static constexpr int PER_BYTE = FMT == KV_CACHE_INT8 ? 1 : 2;
    static constexpr int TILE = kTok * DP * 2, PANEL = kTok * 128;             // an fp16 tile of tokens or queries: panels of 64 elements (128 bytes) a row
    static constexpr int K = 0, V = K + 2 * TILE, Q = V + 2 * TILE, FACTORS = Q + (PAIR ? 2 : 1) * TILE;
    static constexpr int NANS = FACTORS + kSlots * kTok * 4;                   // NaN blocks of a token's values, a byte each
    static constexpr int SIGMA = NANS + kSlots * kTok, ANY_NAN = SIGMA + kSlots * 4, OF_WARP = ANY_NAN + kSlots * 4, STATE = OF_WARP + 2 * 8 * 4;
    static constexpr int BARS = STATE + 2 * kRows * 16, BYTES = BARS + 16 * 8 + 16 + 1024;
    static constexpr int O = 2 * kTok;                                         // tensor memory: scores (and weights) of the two, then their O
    static_assert(O + 2 * DP <= 512 && BYTES <= 227 * 1024, "");
    // codes: a thread takes a chunk of 16 bytes of every PASS-th token
    static constexpr int CHUNKS = DP / PER_BYTE / 16, PASS = kConverters / CHUNKS, EACH = kTok / PASS, CODES = 16 * PER_BYTE;
};
enum Bar { K_FULL = 0, V_FULL = 2, K_EMPTY = 4, V_EMPTY = 6, S_FULL = 8, P_FULL = 10, O_DONE = 12, Q_FULL = 14, DRAINED = 15 };

// A CTA's segments, one after another: (sequence, head, rows) and a run of its tiles. Every role walks them by itself.
template <int ROWS>
struct Segments {
    const AttentionArgs& a;
    const Share share;
    int64_t u, first_of_b;
    int b;
    Sequence s;
    int head, row0, rows, tile0, tiles;
    int64_t item_begin, item_end;
    __device__ __forceinline__ Segments(const AttentionArgs& args, const Share& sh) : a(args), share(sh), u(sh.begin), first_of_b(sh.first_of_b), b(sh.b), tiles(0) {}
    __device__ __forceinline__ bool next() {
        u += tiles;
        if (u >= share.end) return false;
        s = read_sequence<kTok>(a, b, ROWS);
        while (b + 1 < a.seqs && u - first_of_b >= units_of(a, s)) {
            first_of_b += units_of(a, s);
            s = read_sequence<kTok>(a, ++b, ROWS);
        }
        const int64_t of_b = u - first_of_b;
        const int item = static_cast<int>(of_b / s.tiles);
        tile0 = static_cast<int>(of_b - static_cast<int64_t>(item) * s.tiles);
        head = item / s.row_tiles;
        row0 = (item - head * s.row_tiles) * ROWS;
        rows = min(ROWS, s.n * a.group - row0);
        tiles = static_cast<int>(min(static_cast<int64_t>(s.tiles - tile0), share.end - u));
        item_begin = u - tile0;
        item_end = item_begin + s.tiles;
        return true;
    }
    __device__ __forceinline__ int token(int tile) const { return s.base + (tile0 + tile) * kTok; }        // first of a tile
    __device__ __forceinline__ bool whole() const { return tile0 == 0 && tiles == s.tiles; }
};

__device__ __forceinline__ void named_sync(int id, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }

// 16 bytes of codes, `valid` of them there (a multiple of 4; the rest zeros), in loads that the head's alignment allows
__device__ __forceinline__ uint4 load_codes(const uint8_t* p, int valid, int align) {
    uint4 x = make_uint4(0, 0, 0, 0);
    if (valid <= 0) return x;
    if (align == 16) return __ldcg(reinterpret_cast<const uint4*>(p));
    if (align == 8) {
        const uint2 lo = __ldcg(reinterpret_cast<const uint2*>(p)), hi = valid > 8 ? __ldcg(reinterpret_cast<const uint2*>(p) + 1) : make_uint2(0, 0);
        return make_uint4(lo.x, lo.y, hi.x, hi.y);
    }
    const uint32_t* q = reinterpret_cast<const uint32_t*>(p);
    x.x = __ldcg(q);
    if (valid > 4) x.y = __ldcg(q + 1);
    if (valid > 8) x.z = __ldcg(q + 2);
    if (valid > 12) x.w = __ldcg(q + 3);
    return x;
}

// Elements first to first + 7 of row r of a tile: where their 16 bytes are
__device__ __forceinline__ uint32_t place(int r, int first) { return (first >> 6) * (kTok * 128) + r * 128 + ((((first >> 3) & 7) ^ (r & 7)) << 4); }

__device__ __forceinline__ void store_16(uint32_t addr, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}

// New tokens j0 to j0 + 31 of a sequence (below 0: what comes before them) that a node sees, as bits
__device__ __forceinline__ uint32_t sees32(const AttentionArgs& a, int64_t row_of_tree, int node, int j0) {
    if (j0 + 31 < 0) return ~0u;
    if (a.tree == nullptr) return j0 + 31 <= node ? ~0u : j0 > node ? 0u : ~0u >> (31 - (node - j0));
    uint32_t bits = j0 < 0 ? (1u << -j0) - 1 : 0u;              // (-31 .. -1: that many tokens of before; 0 and more: none)
    const int64_t* words = a.tree + row_of_tree * a.tree_words;
    const int from = max(j0, 0), w = from >> 6, at = from & 63;
    uint64_t x = w < a.tree_words ? static_cast<uint64_t>(words[w]) >> at : 0u;
    if (at > 32 && w + 1 < a.tree_words) x |= static_cast<uint64_t>(words[w + 1]) << (64 - at);
    return bits | static_cast<uint32_t>(x) << (from - j0);
}

template <int FMT, int DP, bool PAIR>
__global__ void __launch_bounds__(kThreads, 1) many_rows_kernel(const AttentionArgs a) {
    using L = Plan<FMT, DP, PAIR>;
    constexpr int ROWS = L::ROWS;
    extern __shared__ uint8_t raw_smem[];
    uint8_t* const smem = raw_smem + (1024 - (smem_u32(raw_smem) & 1023)) % 1024;
    const uint32_t base = smem_u32(smem);
    __shared__ int abort_flag, last_one;
    __shared__ uint32_t tmem_slot;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t bars = base + L::BARS;
    auto bar = [&](int which, int i) { return bars + 8 * (which + i); };
    if (threadIdx.x == 0) {
        abort_flag = 0;
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar(K_FULL, i), 8);
            mbar_init(bar(V_FULL, i), 8);
            mbar_init(bar(K_EMPTY, i), 1);
            mbar_init(bar(V_EMPTY, i), 1);
            mbar_init(bar(S_FULL, i), 1);
            mbar_init(bar(P_FULL, i), 4);
            mbar_init(bar(O_DONE, i), 1);
        }
        mbar_init(bar(Q_FULL, 0), 8);
        mbar_init(bar(DRAINED, 0), 1);
        fence_mbar_init();
    }
    const WaitCtl ctl{&abort_flag, a.status, a.sticky, a.limit_ns};
    grid_dep_wait();
    const Share share = share_out<kThreads, kTok>(a, ROWS);
    // tensor memory is taken behind the wait for the kernel ahead (whose CTAs may still want theirs), and dependents are released behind that
    if (warp == kMmaWarp) {
        tmem_alloc(smem_u32(&tmem_slot), 512);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    grid_dep_launch_dependents();
    const uint32_t tmem = tmem_slot;
    float* const factors = reinterpret_cast<float*>(smem + L::FACTORS);          // [slot][token]: of the keys; -1: not seen by anybody
    volatile int* const sigmas = reinterpret_cast<volatile int*>(smem + L::SIGMA);        // [slot]: values are relative to 2^this
    volatile int* const any_nan = reinterpret_cast<volatile int*>(smem + L::ANY_NAN);     // [slot]: whether values of the tile are NaN
    uint8_t* const nans = smem + L::NANS;
    Segments<ROWS> seg(a, share);

    if (warp == kMmaWarp) {
        // ---- products. A job is a tile of tokens for one of the two softmax warpgroups: every other tile, or (PAIR) each tile for both.
        uint32_t tile_base = 0, jobs_of[2] = {0, 0}, segments = 0;
        constexpr uint32_t kQk = make_f16_idesc(kRows, kTok, false), kPv = make_f16_idesc(kRows, DP, true);
        while (seg.next()) {
            const int jobs = PAIR ? 2 * seg.tiles : seg.tiles;
            mbar_wait(bar(Q_FULL, 0), segments & 1, ctl, kWaitMany, kStatusTimeout);
            auto scores = [&](int n) {
                const uint32_t t = tile_base + (PAIR ? n >> 1 : n), buf = t & 1, w = n & 1;
                if (!PAIR || w == 0) mbar_wait(bar(K_FULL, buf), t >> 1 & 1, ctl, kWaitMany + 1, kStatusTimeout);
                tc_fence_after();
                if (lane == 0) {
                    const uint32_t q = base + L::Q + (PAIR ? w * L::TILE : 0), k = base + L::K + buf * L::TILE;
#pragma unroll
                    for (int i = 0; i < DP / 16; ++i) {
                        const uint32_t off = (i / 4) * L::PANEL + (i % 4) * 32;
                        mma_f16_ss(tmem + w * kTok, make_kmajor_sw128_desc(q + off), make_kmajor_sw128_desc(k + off), kQk, i > 0);
                    }
                    tc_commit(bar(S_FULL, w));
                    if (!PAIR || w == 1) tc_commit(bar(K_EMPTY, buf));
                }
                __syncwarp();
            };
            for (int n = 0; n < min(2, jobs); ++n) scores(n);
            for (int n = 0; n < jobs; ++n) {
                const uint32_t t = tile_base + (PAIR ? n >> 1 : n), buf = t & 1, w = n & 1;
                if (!PAIR || w == 0) mbar_wait(bar(V_FULL, buf), t >> 1 & 1, ctl, kWaitMany + 2, kStatusTimeout);
                mbar_wait(bar(P_FULL, w), jobs_of[w] & 1, ctl, kWaitMany + 3, kStatusTimeout);
                ++jobs_of[w];
                tc_fence_after();
                if (lane == 0) {
                    const uint32_t v = base + L::V + buf * L::TILE;
                    const bool first = n < 2;
#pragma unroll
                    for (int i = 0; i < kTok / 16; ++i)
                        mma_f16_ts(tmem + L::O + w * DP, tmem + w * kTok + 8 * i, make_mnmajor_sw128_desc(v + i * 16 * 128, L::PANEL), kPv, !first || i > 0);
                    tc_commit(bar(O_DONE, w));
                    if (!PAIR || w == 1) tc_commit(bar(V_EMPTY, buf));
                }
                __syncwarp();
                if (n + 2 < jobs) scores(n + 2);
            }
            tile_base += seg.tiles;
            ++segments;
        }
        if (lane == 0) tc_commit(bar(DRAINED, 0));                               // (whatever became of the waits, no product is left when the CTA goes)
        mbar_drain(bar(DRAINED, 0), 0, a.limit_ns);
    } else if (warp >= kConvertWarp) {
        // ---- codes to fp16 tiles. The codes of the next tile are on their way while this one is converted.
        constexpr int EACH = L::EACH;
        const int me = threadIdx.x - 32 * kConvertWarp, chunk = me % L::CHUNKS, tok = me / L::CHUNKS;
        const int row_bytes = a.dim / L::PER_BYTE, blocks = (a.dim + kMxBlock - 1) / kMxBlock, off = chunk * 16;
        const int align = row_bytes % 16 == 0 ? 16 : row_bytes % 8 == 0 ? 8 : 4;
        const int64_t token_bytes = static_cast<int64_t>(a.heads) * row_bytes;
        int* const of_warp = reinterpret_cast<int*>(smem + L::OF_WARP);
        bool more = seg.next();
        int tile = 0;                           // of the segment: the next to look up
        int slots[EACH];
        bool seen[EACH];
        int head = 0;
        auto look_up = [&] {                    // where the tokens of that tile are; then on to the next one
            const int t0 = seg.token(tile) + tok;
            head = seg.head;
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                const int t = t0 + i * L::PASS;
                slots[i] = -1;
                seen[i] = false;
                if (more && t >= seg.s.start && t < seg.s.stop) {
                    const int p = a.page_shift >= 0 ? t >> a.page_shift : t / a.page, id = a.table[seg.b * a.table_stride + p];
                    if (id >= 0 && id < a.num_pages) slots[i] = id * a.page + (t - p * a.page);
                }
                seen[i] = slots[i] >= 0;
            }
            if (more && ++tile == seg.tiles) {
                more = seg.next();
                tile = 0;
            }
        };
        uint4 kx[EACH], vx[EACH];               // codes
        uint32_t ksc[EACH], vsc[EACH], next_vsc[EACH];     // int8: the scale; 4-bit: the byte of this chunk's block
        int now[EACH], now_head = 0, sigma = -126;
        bool now_seen[EACH];
        auto fetch_codes = [&](const uint8_t* codes, uint4 (&x)[EACH], const int (&where)[EACH], int h) {
#pragma unroll
            for (int i = 0; i < EACH; ++i)
                x[i] = where[i] >= 0 ? load_codes(codes + where[i] * token_bytes + h * row_bytes + off, row_bytes - off, align) : make_uint4(0, 0, 0, 0);
        };
        auto fetch_scales = [&](const void* scales, uint32_t (&sc)[EACH]) {
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                const int64_t entry = static_cast<int64_t>(max(slots[i], 0)) * a.heads + head;
                sc[i] = 0;
                if (slots[i] >= 0) {
                    if (FMT == KV_CACHE_INT8) sc[i] = __ldcg(static_cast<const uint32_t*>(scales) + entry);
                    else if (chunk < blocks) sc[i] = __ldcg(static_cast<const uint8_t*>(scales) + entry * blocks + chunk);
                }
            }
        };
        auto take_over = [&] {
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                now[i] = slots[i];
                now_seen[i] = seen[i];
                vsc[i] = next_vsc[i];
            }
            now_head = head;
            fetch_codes(a.v_codes, vx, now, now_head);
        };
        static_assert(FMT == KV_CACHE_INT8 || L::CODES == kMxBlock, "a chunk is a block");
        look_up();
        fetch_codes(a.k_codes, kx, slots, head);
        fetch_scales(a.k_scales, ksc);
        fetch_scales(a.v_scales, next_vsc);
        take_over();
        const int64_t tiles_in_all = share.end - share.begin;
        int64_t left_of_item = 0;               // tiles of the current segment still to come: the values' reference starts anew with each
        Segments<ROWS> at(a, share);
        for (int64_t t = 0; t < tiles_in_all; ++t) {
            if (left_of_item == 0) {
                at.next();
                left_of_item = at.tiles;
                sigma = -126;
            }
            --left_of_item;
            const uint32_t buf = t & 1, slot = t & (kSlots - 1), phase = (static_cast<uint32_t>(t) >> 1 & 1) ^ 1;
            look_up();                          // of the tile after this one
            // keys
            mbar_wait(bar(K_EMPTY, buf), phase, ctl, kWaitMany + 4, kStatusTimeout);
            const uint32_t k_tile = base + L::K + buf * L::TILE, v_tile = base + L::V + buf * L::TILE;
            int top_sigma = -126, nan_any = 0;
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                const int r = tok + i * L::PASS;
                const uint32_t w[4] = {kx[i].x, kx[i].y, kx[i].z, kx[i].w};
                if (FMT == KV_CACHE_INT8) {
                    uint32_t f[8];
#pragma unroll
                    for (int j = 0; j < 4; ++j) int8_to_f16(w[j], f[2 * j], f[2 * j + 1]);
                    if (!now_seen[i])
#pragma unroll
                        for (int j = 0; j < 8; ++j) f[j] = 0;
                    store_16(k_tile + place(r, chunk * 16), f[0], f[1], f[2], f[3]);
                    store_16(k_tile + place(r, chunk * 16 + 8), f[4], f[5], f[6], f[7]);
                    if (chunk == 0) {
                        factors[slot * kTok + r] = now_seen[i] ? __uint_as_float(ksc[i]) : -1.f;
                        nans[slot * kTok + r] = 0;
                    }
                    const uint32_t bits = vsc[i];
                    if (now_seen[i] && (bits & 0x7f800000u) == 0x7f800000u) {
                        nan_any = 1;
                        if (chunk == 0) nans[slot * kTok + r] = 0xff;
                    } else if (now_seen[i]) {
                        top_sigma = max(top_sigma, static_cast<int>(bits >> 23) - 126);         // s < 2^this
                    }
                } else {
                    // the token's largest byte: of the lanes that hold its chunks
                    const bool nan = chunk < blocks && ksc[i] == 255u;
                    uint32_t top = nan ? 0u : ksc[i], bad = nan ? 1u : 0u, vbad = chunk < blocks && vsc[i] == 255u && now_seen[i] ? 1u << chunk : 0u;
#pragma unroll
                    for (int o = 1; o < L::CHUNKS; o <<= 1) {
                        top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
                        bad |= __shfl_xor_sync(0xffffffffu, bad, o);
                        vbad |= __shfl_xor_sync(0xffffffffu, vbad, o);
                    }
                    const int e = 27 + static_cast<int>(ksc[i]) - static_cast<int>(top);
                    const uint32_t mul = nan || e <= 0 ? 0u : static_cast<uint32_t>(e) * 0x04000400u;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        uint32_t f[4];
                        e2m1_to_f16(w[j], f);
                        store_16(k_tile + place(r, chunk * 32 + 8 * j), mul_f16x2(f[0], mul), mul_f16x2(f[1], mul), mul_f16x2(f[2], mul), mul_f16x2(f[3], mul));
                    }
                    if (chunk == 0) {
                        factors[slot * kTok + r] = !now_seen[i] ? -1.f : bad != 0 ? __uint_as_float(0x7fc00000u) : __uint_as_float(top == 0 ? 0x00400000u : top << 23);
                        nans[slot * kTok + r] = static_cast<uint8_t>(vbad);
                    }
                    nan_any |= vbad != 0;
                    if (now_seen[i] && chunk < blocks && vsc[i] != 255u) top_sigma = max(top_sigma, static_cast<int>(vsc[i]) - 127);
                }
            }
            // the largest scale of values so far (fp32 exponents: all of them fit a byte)
            const int warp_top = __reduce_max_sync(0xffffffffu, top_sigma), warp_nan = __any_sync(0xffffffffu, nan_any);
            if (lane == 0) of_warp[buf * 8 + warp - kConvertWarp] = warp_top * 2 + (warp_nan ? 1 : 0);
            named_sync(1, kConverters);
            int nan_of_all = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int its = of_warp[buf * 8 + i];
                sigma = max(sigma, its >> 1);
                nan_of_all |= its & 1;
            }
            if (me == 0) {
                sigmas[slot] = sigma;
                any_nan[slot] = nan_of_all;
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(K_FULL, buf));
            const bool another = t + 1 < tiles_in_all;
            if (another) {
                fetch_codes(a.k_codes, kx, slots, head);
                fetch_scales(a.k_scales, ksc);
                fetch_scales(a.v_scales, next_vsc);
            }
            // values: times their scale over 2^sigma, brought to 2^15 at most
            mbar_wait(bar(V_EMPTY, buf), phase, ctl, kWaitMany + 5, kStatusTimeout);
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                const int r = tok + i * L::PASS;
                const uint32_t w[4] = {vx[i].x, vx[i].y, vx[i].z, vx[i].w};
                if (FMT == KV_CACHE_INT8) {
                    const float s = __uint_as_float(vsc[i]);
                    const bool fine = now_seen[i] && (vsc[i] & 0x7f800000u) != 0x7f800000u;
                    // (two factors: 2^(8 - sigma) alone may be more than fp32 holds)
                    const float by = fine ? s * __uint_as_float(static_cast<uint32_t>(127 - sigma / 2) << 23) * __uint_as_float(static_cast<uint32_t>(127 + 8 - (sigma - sigma / 2)) << 23) : 0.f;
                    const uint32_t mul = pack_f16(by, by);
                    uint32_t f[8];
#pragma unroll
                    for (int j = 0; j < 4; ++j) int8_to_f16(w[j], f[2 * j], f[2 * j + 1]);
#pragma unroll
                    for (int j = 0; j < 8; ++j) f[j] = fine ? mul_f16x2(f[j], mul) : 0u;
                    store_16(v_tile + place(r, chunk * 16), f[0], f[1], f[2], f[3]);
                    store_16(v_tile + place(r, chunk * 16 + 8), f[4], f[5], f[6], f[7]);
                } else {
                    const int e = 27 + static_cast<int>(vsc[i]) - 127 - sigma;       // (2^12 * 2^(byte - 127 - sigma), subnormal from 0 down)
                    const uint32_t bits = e > 0 ? static_cast<uint32_t>(e) << 10 : 512u >> min(-e, 31), mul = !now_seen[i] || vsc[i] == 255u ? 0u : bits * 0x00010001u;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        uint32_t f[4];
                        e2m1_to_f16(w[j], f);
                        store_16(v_tile + place(r, chunk * 32 + 8 * j), mul_f16x2(f[0], mul), mul_f16x2(f[1], mul), mul_f16x2(f[2], mul), mul_f16x2(f[3], mul));
                    }
                }
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(V_FULL, buf));
            if (another) take_over();
        }
    } else {
        // ---- softmax: a thread a row
        const int w = warp >> 2, row = threadIdx.x & (kRows - 1);
        const uint32_t lanes = static_cast<uint32_t>(32 * (warp & 3)) << 16, s_tmem = tmem + lanes + w * kTok, o_tmem = tmem + lanes + L::O + w * DP;
        float* const state = reinterpret_cast<float*>(smem + L::STATE);          // [warpgroup][row]: references of o and of the sum, the sum, NaN blocks
        uint32_t tile_base = 0, jobs = 0;                                        // jobs of this warpgroup so far
        while (seg.next()) {
            const int r = (PAIR ? w * kRows : 0) + row;                          // of the item's rows
            const bool live = r < seg.rows, warp_live = (PAIR ? w * kRows : 0) + 32 * (warp & 3) < seg.rows;
            const int node = (seg.row0 + min(r, seg.rows - 1)) / a.group, h = seg.head * a.group + (seg.row0 + min(r, seg.rows - 1)) - node * a.group;
            // queries: a power of two brings the row's largest magnitude to [2^14, 2^15)
            float factor;
            {
                const __nv_bfloat16* from = a.q + static_cast<int64_t>(seg.s.begin + node) * a.q_st + h * a.q_sh;
                uint32_t top = 0;
                for (int d = 0; d < a.dim; d += 8) top = max(top, absmax_bits8(*reinterpret_cast<const uint4*>(from + d)));
                const int field = static_cast<int>(top >> 23), up = field == 255 ? 0 : min(126, max(-126, 141 - max(field, 1)));
                const float mul = a.scale < 0.f ? -__uint_as_float((127 + up) << 23) : __uint_as_float((127 + up) << 23);
                factor = fabsf(a.scale) * kLog2e * __uint_as_float((127 - up) << 23) * (FMT == KV_CACHE_INT8 ? 1.f : 0x1p-12f);
                const uint32_t to = base + L::Q + (PAIR ? w * L::TILE : 0);
                // (one tile of queries: each warpgroup writes every other eight elements)
                for (int d = PAIR ? 0 : 8 * w; d < DP; d += PAIR ? 8 : 16) {
                    float f[8];
                    unpack_bf16x8(live && d < a.dim ? *reinterpret_cast<const uint4*>(from + d) : make_uint4(0, 0, 0, 0), f);
                    store_16(to + place(row, d), pack_f16(f[0] * mul, f[1] * mul), pack_f16(f[2] * mul, f[3] * mul), pack_f16(f[4] * mul, f[5] * mul), pack_f16(f[6] * mul, f[7] * mul));
                }
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(Q_FULL, 0));
            float m = kNone;
            uint64_t l2 = 0;
            int sigma = -126;
            uint32_t poison = 0;                                                 // blocks of this row's output that are NaN
            const uint64_t f2 = pack2(factor, factor);
            bool first = true;
            for (int t = PAIR ? 0 : w; t < seg.tiles; t += PAIR ? 1 : 2, ++jobs) {
                const uint32_t slot = (tile_base + t) & (kSlots - 1);
                mbar_wait(bar(S_FULL, w), jobs & 1, ctl, kWaitMany + 6, kStatusTimeout);
                tc_fence_after();
                if (warp_live) {
                    const float* const kf = factors + slot * kTok;
                    const int j0 = seg.token(t) - seg.s.before;
                    uint32_t sees[4];
#pragma unroll
                    for (int ch = 0; ch < 4; ++ch) {
                        sees[ch] = __ballot_sync(0xffffffffu, kf[32 * ch + lane] != -1.f);
                        if (j0 + 32 * ch + 31 >= 0) sees[ch] &= sees32(a, seg.s.begin + node, node, j0 + 32 * ch);
                    }
                    if (any_nan[slot] != 0) {
                        for (int x = 0; x < kTok; ++x)
                            if (sees[x >> 5] >> (x & 31) & 1u) poison |= nans[slot * kTok + x];
                    }
                    // the row's largest score
                    float top = -INFINITY;
#pragma unroll
                    for (int ch = 0; ch < 4; ++ch) {
                        uint32_t v[32];
                        tmem_ld_32x32b_x32(s_tmem + 32 * ch, v);
                        tmem_wait_ld();
                        const bool all = sees[ch] == ~0u;
#pragma unroll
                        for (int x = 0; x < 32; x += 4) {
                            const float4 k = *reinterpret_cast<const float4*>(kf + 32 * ch + x);
                            float p, q, y, z;
                            unpack2(mul2(pack2(__uint_as_float(v[x]), __uint_as_float(v[x + 1])), pack2(k.x, k.y)), p, q);
                            unpack2(mul2(pack2(__uint_as_float(v[x + 2]), __uint_as_float(v[x + 3])), pack2(k.z, k.w)), y, z);
                            if (!all) {
                                if (!(sees[ch] >> x & 1u)) p = -INFINITY;
                                if (!(sees[ch] >> x & 2u)) q = -INFINITY;
                                if (!(sees[ch] >> x & 4u)) y = -INFINITY;
                                if (!(sees[ch] >> x & 8u)) z = -INFINITY;
                            }
                            top = fmaxf(top, fmaxf(fmaxf(p, q), fmaxf(y, z)));
                        }
                    }
                    top = top == -INFINITY ? kNone : top * factor;
                    // references move when a weight would pass 2^15, to put it at 2^7, or when the values' does
                    const int its_sigma = sigmas[slot];
                    if (__any_sync(0xffffffffu, top > m + 15.f || its_sigma != sigma)) {
                        const float now = top > m + 15.f ? top - 7.f : m, by_l = ex2(m - now);
                        l2 = mul2(l2, pack2(by_l, by_l));
                        if (!first) {
                            const float by = by_l * ex2(static_cast<float>(max(sigma - its_sigma, -252)) * 0.5f) * ex2(static_cast<float>(max(sigma - its_sigma, -252)) * 0.5f);
                            mbar_wait(bar(O_DONE, w), (jobs - 1) & 1, ctl, kWaitMany + 7, kStatusTimeout);
                            tc_fence_after();
#pragma unroll
                            for (int ch = 0; ch < DP / 16; ++ch) {
                                uint32_t v[16];
                                tmem_ld_32x32b_x16(o_tmem + 16 * ch, v);
                                tmem_wait_ld();
#pragma unroll
                                for (int x = 0; x < 16; ++x) v[x] = __float_as_uint(__uint_as_float(v[x]) * by);
                                tmem_st_32x32b_x16(o_tmem + 16 * ch, v);
                            }
                        }
                        m = now;
                        sigma = its_sigma;
                    }
                    first = false;
                    // weights, over the scores that they came from
                    const uint64_t m2 = pack2(-m, -m);
#pragma unroll
                    for (int ch = 0; ch < 4; ++ch) {
                        uint32_t v[32], p[16];
                        tmem_ld_32x32b_x32(s_tmem + 32 * ch, v);
                        tmem_wait_ld();
                        const bool all = sees[ch] == ~0u;
#pragma unroll
                        for (int x = 0; x < 32; x += 2) {
                            const uint64_t k = *reinterpret_cast<const uint64_t*>(kf + 32 * ch + x);
                            float y, z;
                            unpack2(fma2(mul2(pack2(__uint_as_float(v[x]), __uint_as_float(v[x + 1])), k), f2, m2), y, z);
                            if (!all) {
                                if (!(sees[ch] >> x & 1u)) y = -INFINITY;
                                if (!(sees[ch] >> x & 2u)) z = -INFINITY;
                            }
                            y = ex2(y);
                            z = ex2(z);
                            l2 = add2(l2, pack2(y, z));
                            p[x / 2] = pack_f16(y, z);
                        }
                        tmem_st_32x32b_x16(s_tmem + 16 * ch, p);
                    }
                    tmem_wait_st();
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(P_FULL, w));
            }
            // ---- results: o of this warpgroup, or of both, over the sums
            float l, other;
            unpack2(l2, l, other);
            l += other;
            // (reference of o with the values' in it: int8 tiles are 2^8 too large, 4-bit ones 2^12, which the results take account of)
            float m_o = m + static_cast<float>(sigma - (FMT == KV_CACHE_INT8 ? 8 : 0));
            const bool had = PAIR || w < seg.tiles;
            if (had) mbar_wait(bar(O_DONE, w), (jobs - 1) & 1, ctl, kWaitMany + 8, kStatusTimeout);
            if (!PAIR) {
                *reinterpret_cast<float4*>(state + (w * kRows + row) * 4) = make_float4(m_o, m, l, __uint_as_float(poison));
            }
            named_sync(2, kSoftmax);
            tc_fence_after();
            const bool whole = seg.whole();
            constexpr int PART = part_floats(ROWS, DP);
            float* const part = a.parts + (2 * static_cast<int64_t>(blockIdx.x) + (share.begin > seg.item_begin ? 0 : 1)) * PART;
            if (warp_live) {
                const float nan = __uint_as_float(0x7fc00000u);
                float by[2] = {1.f, 0.f}, m_l = m;
                const bool two = !PAIR && seg.tiles > 1;
                if (!PAIR) {
                    const float4 s0 = *reinterpret_cast<const float4*>(state + row * 4), s1 = *reinterpret_cast<const float4*>(state + (kRows + row) * 4);
                    m_o = two ? fmaxf(s0.x, s1.x) : s0.x;
                    m_l = two ? fmaxf(s0.y, s1.y) : s0.y;
                    l = s0.z;
                    poison = __float_as_uint(s0.w);
                    if (two) {
                        by[0] = ex2(s0.x - m_o);
                        by[1] = ex2(s1.x - m_o);
                        l = s0.z * ex2(s0.y - m_l) + s1.z * ex2(s1.y - m_l);
                        poison |= __float_as_uint(s1.w);
                    }
                }
                // (one item's rows: each warpgroup takes half of the elements)
                constexpr int WIDTH = PAIR ? DP : DP / 2;
                const int d0 = PAIR ? 0 : w * WIDTH;
#pragma unroll
                for (int ch = 0; ch < WIDTH / 16; ++ch) {
                    uint32_t v[16];
                    float o[16];
                    tmem_ld_32x32b_x16(tmem + lanes + L::O + (PAIR ? w * DP : 0) + d0 + 16 * ch, v);
                    tmem_wait_ld();
#pragma unroll
                    for (int x = 0; x < 16; ++x) o[x] = __uint_as_float(v[x]) * by[0];
                    if (two) {
                        tmem_ld_32x32b_x16(tmem + lanes + L::O + DP + d0 + 16 * ch, v);
                        tmem_wait_ld();
#pragma unroll
                        for (int x = 0; x < 16; ++x) o[x] += __uint_as_float(v[x]) * by[1];
                    }
                    const int d = d0 + 16 * ch;
                    const uint32_t bad = FMT == KV_CACHE_INT8 ? poison : poison >> (d / kMxBlock) & 1u;
                    if (live) {
#pragma unroll
                        for (int x = 0; x < 16; x += 4) {
                            if (d + x >= a.dim) break;
                            Row out;
                            out.m_o = m_o;
                            out.m_l = m_l;
                            out.l = l;
#pragma unroll
                            for (int e = 0; e < 4; ++e) out.o[e] = bad != 0 ? nan : o[x + e];
                            if (whole) out.finish<FMT>(a, seg.s, seg.head, seg.row0 + r, d + x);
                            else *reinterpret_cast<float4*>(part + r * DP + d + x) = make_float4(out.o[0], out.o[1], out.o[2], out.o[3]);
                        }
                        if (!whole && d == 0) *reinterpret_cast<float4*>(part + ROWS * DP + 4 * r) = make_float4(m_o, m_l, l, 0.f);
                    }
                }
            }
            tc_fence_before();
            named_sync(2, kSoftmax);                                             // o and the states may be written over
            if (!whole)
                merge_parts<FMT, ROWS, DP, kSoftmax>(a, seg.s, seg.b, seg.head, seg.row0, seg.rows, owner(seg.item_begin, share), owner(seg.item_end - 1, share),
                                                     threadIdx.x, &last_one, [] { named_sync(2, kSoftmax); });
            tile_base += seg.tiles;
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == kMmaWarp) tmem_dealloc(tmem, 512);
    zero_rest<kThreads>(a);
}

template <int FMT, int DP, bool PAIR>
cudaError_t launch(const AttentionArgs& a, cudaStream_t st) {
    static PerDeviceOnce once;
    constexpr int bytes = Plan<FMT, DP, PAIR>::BYTES;
    const auto kern = many_rows_kernel<FMT, DP, PAIR>;
    cudaError_t e = once.run([&] { return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes); });
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(sm_count()));
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
cudaError_t launch_for(const AttentionArgs& a, int64_t rows, cudaStream_t st) {
    if (a.dim <= 64) return rows > kRows ? launch<FMT, 64, true>(a, st) : launch<FMT, 64, false>(a, st);
    return rows > kRows ? launch<FMT, 128, true>(a, st) : launch<FMT, 128, false>(a, st);
}

} // namespace

bool many_rows_fits(int dim) { return dim <= 128; }
size_t many_rows_part_bytes(int64_t most_rows, int64_t dim) {
    if (dim > 128) return 0;
    return static_cast<size_t>(sm_count()) * 2 * part_floats(most_rows > kRows ? 2 * kRows : kRows, dim <= 64 ? 64 : 128) * sizeof(float);
}
cudaError_t launch_many_rows(int fmt, const AttentionArgs& a, int64_t rows, cudaStream_t st) {
    return fmt == KV_CACHE_INT8 ? launch_for<KV_CACHE_INT8>(a, rows, st) : launch_for<KV_CACHE_MXFP4>(a, rows, st);
}

} // namespace attention
} // namespace w8a8
