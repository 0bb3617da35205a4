// Attention over the quantized cache for many rows of queries a head: trees of drafted tokens with grouped heads, chains, prompts.
//
// Both products run on the tensor memory's matrix unit, 128 rows of queries at a time: S = Q K^T with Q and K in shared memory, O += P V with P in
// tensor memory, where it lies over the scores it came from. Two warps bring the cache's codes into shared memory, keys and values; four and four turn them into fp16 tiles
// of 128 tokens; a thread a row does the softmax; one thread issues the products. Tiles and codes of either side go round in rings of their own.
//
// Keys in int8 are the codes, exact, and a token's scale goes to its scores. Keys in 4 bits are codes times their block's scale relative to the tile's largest (powers of
// two: exact down to 2^-36 of it), so that one factor stands for all scores of a tile. Values are codes times scale, relative to the largest scale so far.
//
// Two softmax warpgroups, each with scores and an O of its own: of the same 128 rows and every other tile of tokens, or (PAIR) of 128 rows each and all
// tiles, which then are converted once for 256 rows (61 nodes, 8 queries a head, int8: 3 sequences of 20000 tokens 167 us against 184 without, one of 60000 210 against 237).
//
// What bounds it: no one thing. A tile of 128 tokens and 128 rows in int8 takes some 3700 cycles, of which HBM's share is 1060, the products' 1024, the exponentials' 1024 and
// the issue slots' (softmax, conversion) 1500: they meet in a chain (scores, softmax, products) two of which are under way, all that tensor memory has room for. 12 x 32
// nodes behind 6000 tokens: 76 us (16 at the copy's rate), of which some 25 are beginnings and ends: queries, a first tile, parts. 4 bits, 3 x 61 nodes, 256 rows a tile, behind
// 20000 tokens: 152 us (53, bound by the products, at cuBLAS's rate).
#include "internal.h"
#include "kv_attention.cuh"

#include <cmath>
#include <type_traits>

namespace w8a8 {
namespace attention {
namespace {

constexpr int kTok = 128;                       // tokens of a tile
constexpr int kRows = 128;                      // rows of a product
constexpr int kSoftmax = 256, kConverters = 128;            // threads that do the softmax; that turn keys, or values, to fp16
constexpr int kKeyWarp = 8, kValueWarp = 12, kMmaWarp = 16, kLoadWarp = 17, kThreads = 32 * 19;
constexpr int kWaitMany = 41;                   // which wait gave up, for the status word: this and the 11 after it
constexpr int kSlots = 4;                       // tiles whose factors are kept

template <int FMT, int DP, bool PAIR>
struct Plan {
    static constexpr int ROWS = PAIR ? 2 * kRows : kRows;
    static constexpr int PER_BYTE = FMT == KV_CACHE_INT8 ? 1 : 2, ROW = DP / PER_BYTE;     // bytes of a head, padded
    static constexpr int TILE = kTok * DP * 2, PANEL = kTok * 128;             // an fp16 tile of tokens or queries: panels of 64 elements (128 bytes) a row
    // a ring of fp16 tiles of keys, one of values, and rings of their codes on their way
    static constexpr int KEYS = 2, VALUES = DP == 128 ? 1 : 2, RAW_KEYS = FMT == KV_CACHE_INT8 ? 2 : 3, RAW_VALUES = RAW_KEYS - (PAIR && DP == 128 ? 1 : 0);
    static constexpr int V_TILES = KEYS * TILE, Q = V_TILES + VALUES * TILE, RAW = Q + (PAIR ? 2 : 1) * TILE, RAW_V = RAW + RAW_KEYS * kTok * ROW;
    static constexpr int MORE = RAW_V + RAW_VALUES * kTok * ROW;
    // with the codes of keys come the scales of keys and values (4-bit: the two words that hold a head's bytes) and a byte a token: 0x80 where it
    // may be seen, and (4-bit) where in the words its bytes begin
    static constexpr int WORDS = FMT == KV_CACHE_INT8 ? 1 : 2, V_SCALES = kTok * 4 * WORDS, FLAGS = 2 * V_SCALES, MORE_BYTES = FLAGS + kTok;
    static constexpr int FACTORS = MORE + RAW_KEYS * MORE_BYTES;
    static constexpr int ONES = FACTORS + kSlots * kTok * 4;                   // factors of scores that have theirs already
    static constexpr int NANS = ONES + kTok * 4;                               // NaN blocks of a token's values, a byte each
    static constexpr int SIGMA = NANS + kSlots * kTok, SPECIAL = SIGMA + kSlots * 4, OF_WARP = SPECIAL + kSlots * 4, OF_V = OF_WARP + 2 * 8 * 4, OF_K = OF_V + kSlots * kTok * 4, OF_TILE = OF_K + (FMT == KV_CACHE_INT8 ? 0 : 2 * kTok * 4);
    static constexpr int FACTOR = OF_TILE + kSlots * 4;         // of the scores; the queries' maxima and odd rows of the warps
    static constexpr int POWERS = FACTOR + 24 * 4, STATE = POWERS + 2 * kRows * 4, BARS = STATE + 4 * kSoftmax * 8, BYTES = BARS + 33 * 8 + 1024;
    static constexpr int O = 2 * kTok;                                         // tensor memory: scores (and weights) of the two, then their O
    static_assert(O + 2 * DP <= 512 && BYTES <= 226 * 1024, "");
    // codes: a thread converts a chunk of 16 bytes of every PASS-th token
    static constexpr int CHUNKS = ROW / 16, PASS = kConverters / CHUNKS, CODES = 16 * PER_BYTE;
    // byte `off` of row r of a tile of codes, as boxes arrive: chunks of 16 bytes change places by the row
    __device__ static __forceinline__ int raw_place(int r, int off) {
        const int turn = ROW == 128 ? r & 7 : ROW == 64 ? (r >> 1) & 3 : (r >> 2) & 1;
        return r * ROW + (off ^ (turn << 4));
    }
};
enum Bar {
    K_FULL = 0, K_EMPTY = 2, V_FULL = 4, V_EMPTY = 6, RAW_K_FULL = 8, RAW_K_EMPTY = 11, RAW_V_FULL = 14, RAW_V_EMPTY = 17,
    S_FULL = 20, P_FULL = 22, O_DONE = 24, SCALES_FULL = 26, Q_FULL = 30, FACTOR_FULL = 31, DRAINED = 32
};

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
        const int item = static_cast<int>(quotient(of_b, s.tiles));
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

// mbar_wait for roles that walk on to their end when a wait of the CTA has given up: those after it do not wait
static __device__ __noinline__ bool wait_slow(uint32_t bar, uint32_t parity, const WaitCtl& ctl, int where, int status_code) {
    return *static_cast<volatile int*>(ctl.abort_flag) == 0 && mbar_wait_slow(bar, parity, ctl, where, status_code);
}
__device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity, const WaitCtl& ctl, int where, int status_code) {
    if (mbar_try_wait(bar, parity)) return true;
    return wait_slow(bar, parity, ctl, where, status_code);
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

// A position in a ring of N: which slot, and how often it came round
template <int N>
struct Turn {
    uint32_t slot = 0, phase = 0;
    __device__ __forceinline__ void next() {
        if (++slot == N) {
            slot = 0;
            phase ^= 1;
        }
    }
};

template <int FMT, int DP, bool PAIR>
__global__ void __launch_bounds__(kThreads, 1) many_rows_kernel(const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map, const AttentionArgs a) {
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
    if (threadIdx.x < kTok) reinterpret_cast<float*>(smem + L::ONES)[threadIdx.x] = 1.f;
    if (threadIdx.x == 0) {
        abort_flag = 0;
        for (int i = 0; i < 3; ++i) {
            mbar_init(bar(RAW_K_FULL, i), 64);
            mbar_init(bar(RAW_K_EMPTY, i), 4);
            mbar_init(bar(RAW_V_FULL, i), 64);
            mbar_init(bar(RAW_V_EMPTY, i), 4);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar(K_FULL, i), 4);
            mbar_init(bar(K_EMPTY, i), 1);
            mbar_init(bar(V_FULL, i), 4);
            mbar_init(bar(V_EMPTY, i), 1);
            mbar_init(bar(S_FULL, i), 1);
            mbar_init(bar(P_FULL, i), 4);
            mbar_init(bar(O_DONE, i), 1);
        }
        for (int i = 0; i < kSlots; ++i) mbar_init(bar(SCALES_FULL, i), 4);
        mbar_init(bar(Q_FULL, 0), 8);
        mbar_init(bar(FACTOR_FULL, 0), 8);
        mbar_init(bar(DRAINED, 0), 1);
        fence_mbar_init();
    }
    const WaitCtl ctl{&abort_flag, a.status, a.sticky, a.limit_ns};
    grid_dep_wait();
    // tensor memory is taken behind the wait for the kernel ahead (whose CTAs may still want theirs), and dependents are released behind that
    if (warp == kMmaWarp) {
        tmem_alloc(smem_u32(&tmem_slot), 512);
        tmem_relinquish();
    }
    const Share share = share_out<kThreads, kTok>(a, ROWS);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    grid_dep_launch_dependents();
    const uint32_t tmem = tmem_slot;
    float* const factors = reinterpret_cast<float*>(smem + L::FACTORS);          // [slot][token]: of the scores; -1: not seen by anybody
    volatile int* const sigmas = reinterpret_cast<volatile int*>(smem + L::SIGMA);        // [slot]: values are relative to 2^this
    volatile float* const tile_factors = reinterpret_cast<volatile float*>(smem + L::OF_TILE);      // 4-bit: [slot]: of all scores of a tile
    volatile int* const special = reinterpret_cast<volatile int*>(smem + L::SPECIAL);     // [slot]: whether values of the tile are NaN (1), tokens not to be seen (2), scores large (4), rows odd (8)
    uint8_t* const nans = smem + L::NANS;
    const int row_bytes = a.dim / L::PER_BYTE, blocks = (a.dim + kMxBlock - 1) / kMxBlock;
    Segments<ROWS> seg(a, share);

    if (warp == kMmaWarp) {
        // ---- products. A job is a tile of tokens for one of the two softmax warpgroups: every other tile, or (PAIR) each tile for both. One thread, and as few
        // instructions between products as can be: the queue in front of the matrix unit is short, so that it stands still meanwhile.
        if (lane == 0) {
            constexpr uint32_t kQk = make_f16_idesc(kRows, kTok, false), kPv = make_f16_idesc(kRows, DP, true);
            const uint64_t k_desc = make_kmajor_sw128_desc(base), v_desc = make_mnmajor_sw128_desc(base + L::V_TILES, L::PANEL);
            const uint32_t k_lo = static_cast<uint32_t>(k_desc), k_hi = static_cast<uint32_t>(k_desc >> 32), v_lo = static_cast<uint32_t>(v_desc), v_hi = static_cast<uint32_t>(v_desc >> 32);
            uint32_t segments = 0, p_phase[2] = {0, 0};
            Turn<L::KEYS> k_at;
            Turn<L::VALUES> v_at;
            // (addresses in units of 16 bytes; the tiles end well below what the field holds)
            auto scores = [&](auto which) {
                constexpr uint32_t w = decltype(which)::value;
                if (!PAIR || w == 0) {
                    wait(bar(K_FULL, k_at.slot), k_at.phase, ctl, kWaitMany + 1, kStatusTimeout);
                    tc_fence_after();
                }
                const uint32_t q = k_lo + (L::Q + (PAIR ? w * L::TILE : 0)) / 16, k = k_lo + k_at.slot * (L::TILE / 16);
#pragma unroll
                for (int i = 0; i < DP / 16; ++i) {
                    const uint32_t off = ((i / 4) * L::PANEL + (i % 4) * 32) / 16;
                    mma_f16_ss(tmem + w * kTok, q + off, k_hi, k + off, k_hi, kQk, i > 0);
                }
                tc_commit(bar(S_FULL, w));
                if (!PAIR || w == 1) {
                    tc_commit(bar(K_EMPTY, k_at.slot));
                    k_at.next();
                }
            };
            auto values = [&](auto which, bool first) {
                constexpr uint32_t w = decltype(which)::value;
                if (!PAIR || w == 0) wait(bar(V_FULL, v_at.slot), v_at.phase, ctl, kWaitMany + 2, kStatusTimeout);
                wait(bar(P_FULL, w), p_phase[w], ctl, kWaitMany + 3, kStatusTimeout);
                p_phase[w] ^= 1;
                tc_fence_after();
                const uint32_t v = v_lo + v_at.slot * (L::TILE / 16);
#pragma unroll
                for (int i = 0; i < kTok / 16; ++i) mma_f16_ts(tmem + L::O + w * DP, tmem + w * kTok + 8 * i, v + i * 16 * 128 / 16, v_hi, kPv, !first || i > 0);
                tc_commit(bar(O_DONE, w));
                if (!PAIR || w == 1) {
                    tc_commit(bar(V_EMPTY, v_at.slot));
                    v_at.next();
                }
            };
            const std::integral_constant<uint32_t, 0> zero{};
            const std::integral_constant<uint32_t, 1> one{};
            while (seg.next()) {
                const int jobs = PAIR ? 2 * seg.tiles : seg.tiles;
                wait(bar(Q_FULL, 0), segments & 1, ctl, kWaitMany, kStatusTimeout);
                ++segments;
                scores(zero);
                if (jobs > 1) scores(one);
#pragma unroll 1
                for (int n = 0; n < jobs; n += 2) {
                    values(zero, n == 0);
                    if (n + 2 < jobs) scores(zero);
                    if (n + 1 == jobs) break;
                    values(one, n == 0);
                    if (n + 3 < jobs) scores(one);
                }
            }
        }
        __syncwarp();
        if (lane == 0) tc_commit(bar(DRAINED, 0));                               // (whatever became of the waits, no product is left when the CTA goes)
        mbar_drain(bar(DRAINED, 0), 0, a.limit_ns);
    } else if (warp >= kLoadWarp) {
        // ---- codes and scales into shared memory: a warp for keys (and all scales), one for values. A lane has four tokens of a tile; codes come as boxes of tokens
        // that lie side by side in any page, or (heads that are not whole 16-byte pieces) piece by piece. (Loops are not unrolled: what bounds a warp that comes
        // round once a tile, beside others that run other code, is the fetching of its instructions.)
        const int64_t token_bytes = static_cast<int64_t>(a.heads) * row_bytes;
        const bool runs = a.page % 4 == 0;                                       // a lane's tokens lie side by side
        const int side = warp - kLoadWarp;
        const uint32_t raws = side == 0 ? L::RAW_KEYS : L::RAW_VALUES;
        const uint32_t fulls = bar(side == 0 ? RAW_K_FULL : RAW_V_FULL, 0), empties = bar(side == 0 ? RAW_K_EMPTY : RAW_V_EMPTY, 0), raw_at = base + (side == 0 ? L::RAW : L::RAW_V);
        const void* const map = side == 0 ? &k_map : &v_map;
        int64_t table_of = 0;
        auto look_up = [&](int t, int stop) { return t < stop ? a.table[table_of + (a.page_shift >= 0 ? t >> a.page_shift : t / a.page)] : -1; };
        auto slot_of = [&](int id, int t) { return id >= 0 && id < a.num_pages ? id * a.page + (a.page_shift >= 0 ? t & (a.page - 1) : t % a.page) : -1; };
        uint32_t slot = 0, phase = 1, unit = 0;
        bool going = true;
        while (going && seg.next()) {
            table_of = seg.b * a.table_stride;
            const int stop = seg.s.stop, head = seg.head;
            int t0 = seg.token(0) + 4 * lane, id = look_up(t0, stop);            // (of the first of a lane's tokens, a tile ahead)
#pragma unroll 1
            for (int left = seg.tiles; left > 0; --left) {
                const int t = t0, first = slot_of(id, t);
                t0 += kTok;
                if (left > 1) id = look_up(t0, stop);
                // (once a wait of the CTA has given up, slots are called empty that are not)
                going = __all_sync(0xffffffffu, wait(empties + 8 * slot, phase, ctl, kWaitMany + 4, kStatusTimeout) && *static_cast<volatile int*>(&abort_flag) == 0);
                if (!going) break;
                const uint32_t full = fulls + 8 * slot, to = raw_at + slot * kTok * L::ROW, rest = base + L::MORE + slot * L::MORE_BYTES;
                const uint32_t its_slot = slot;
                if (++slot == raws) {
                    slot = 0;
                    phase ^= 1;
                }
                if (unit++ == 0 && a.starve != 0 && side == 0) {
                    going = false;
                    break;
                }
                if (a.box >= 4) {                                                // boxes that begin with the first token of a lane
#pragma unroll 1
                    for (int l = 0; l < 32; l += a.box / 4) {
                        const int from = __shfl_sync(0xffffffffu, first, l);
                        if (lane == 0 && from >= 0) {
                            mbar_expect_tx(full, a.box * L::ROW);
                            tma_load_3d(to + 4 * l * L::ROW, map, full, 0, head, from);
                        }
                    }
                }
#pragma unroll 1
                for (int i = 0; i < 4; ++i) {
                    if (side == 1 && a.box >= 4) break;                          // (nothing else for values)
                    const int from = i == 0 ? first : t + i >= stop ? -1 : !runs ? slot_of(look_up(t + i, stop), t + i) : first >= 0 ? first + i : -1;
                    if (a.box > 0) {
                        if (a.box < 4 && from >= 0 && i % a.box == 0) {          // smaller boxes
                            mbar_expect_tx(full, a.box * L::ROW);
                            tma_load_3d(to + (4 * lane + i) * L::ROW, map, full, 0, head, from);
                        }
                    } else {
                        const uint8_t* const codes = side == 0 ? a.k_codes : a.v_codes;
                        constexpr int kPieces = L::ROW / 8;
#pragma unroll 1
                        for (int e = lane; e < 32 * kPieces; e += 32) {
                            const int its_lane = e / kPieces, r = 4 * its_lane + i, off = (e - its_lane * kPieces) * 8, its = __shfl_sync(0xffffffffu, from, its_lane);
                            const int64_t where = max(its, 0) * token_bytes + head * row_bytes + off;
                            const int valid = its >= 0 ? row_bytes - off : 0;
                            if (row_bytes % 8 == 0) {
                                cp_async<8>(to + L::raw_place(r, off), codes + (valid > 0 ? where : 0), valid > 0 ? 8 : 0);
                            } else {
#pragma unroll
                                for (int x = 0; x < 8; x += 4) cp_async<4>(to + L::raw_place(r, off) + x, codes + (valid > x ? where + x : 0), valid > x ? 4 : 0);
                            }
                        }
                    }
                    if (side == 0) {                                             // with the keys, all scales
                        const int64_t entry = static_cast<int64_t>(max(from, 0)) * a.heads + head;
                        const uint32_t at = rest + (4 * lane + i) * 4 * L::WORDS, there = from >= 0 ? 4 : 0;
                        uint32_t flag = from >= 0 && t + i >= seg.s.start ? 0x80u : 0u;
                        if (FMT == KV_CACHE_INT8) {
                            cp_async<4>(at, static_cast<const float*>(a.k_scales) + entry, there);
                            cp_async<4>(at + L::V_SCALES, static_cast<const float*>(a.v_scales) + entry, there);
                        } else {
                            const ScaleWords its = scale_words(entry, blocks);
                            const uint8_t *const k_words = static_cast<const uint8_t*>(a.k_scales) + its.from, *const v_words = static_cast<const uint8_t*>(a.v_scales) + its.from;
                            if (flag != 0) flag |= static_cast<uint32_t>(its.shift);
                            const int one = from >= 0 ? its.bytes(0) : 0;
                            cp_async<4>(at, k_words, one);
                            cp_async<4>(at + L::V_SCALES, v_words, one);
                            if (blocks != 4 && blocks != 2) {                    // (bytes of a token may lie across two words)
                                const int two = from >= 0 ? its.bytes(1) : 0;
                                cp_async<4>(at + 4, k_words + (two > 0 ? 4 : 0), two);
                                cp_async<4>(at + L::V_SCALES + 4, v_words + (two > 0 ? 4 : 0), two);
                            }
                        }
                        smem[L::MORE + its_slot * L::MORE_BYTES + L::FLAGS + 4 * lane + i] = static_cast<uint8_t>(flag);
                    }
                }
                mbar_arrive(full);
                cp_async_mbar_arrive(full);                                      // once this lane's own copies are there
            }
        }
        // nothing is on its way when the CTA goes: what was asked for has been waited for by those who convert it, unless a wait gave up
        if (!going || abort_flag != 0) {
            asm volatile("cp.async.wait_all;" ::: "memory");
            for (uint32_t last = unit > raws ? unit - raws : 0; last < unit; ++last) mbar_drain(fulls + 8 * (last % raws), last / raws & 1, a.limit_ns);
        }
    } else if (warp >= kKeyWarp) {
        // ---- codes to fp16 tiles, keys by four warps and values by four: a thread has a chunk of 16 bytes of every PASS-th token (PASS is a multiple of 8, so that its
        // chunks are swizzled alike). The keys' warps work out the scales of both.
        const bool keys = warp < kValueWarp;
        const int me = threadIdx.x & (kConverters - 1), chunk = me % L::CHUNKS, tok = me / L::CHUNKS;
        static_assert(FMT == KV_CACHE_INT8 || L::CODES == kMxBlock, "a chunk is a block");
        static_assert(L::PASS % 8 == 0 && kConverters == kTok, "");
        uint8_t* const v_scales = smem + L::OF_V;                                // [slot][token]: int8: the values' scales, 4-bit: their four bytes
        const uint32_t raw_from = base + L::raw_place(tok, chunk * 16);
        uint32_t to[L::CODES / 8];
#pragma unroll
        for (int j = 0; j < L::CODES / 8; ++j) to[j] = base + place(tok, chunk * L::CODES + 8 * j);
        auto convert = [&](uint32_t raw, uint32_t tile, auto multiplier) {       // of a token: two equal halves
            const uint32_t from = raw_from + raw;
#pragma unroll 2
            for (int i = 0; i < kTok / L::PASS; ++i) {
                uint32_t w[4];
                asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(from + i * L::PASS * L::ROW) : "memory");
                const uint32_t mul = multiplier(tok + i * L::PASS), at = tile + i * L::PASS * 128;
                if (FMT == KV_CACHE_INT8) {
                    uint32_t f[8];
#pragma unroll
                    for (int j = 0; j < 4; ++j) int8_to_f16(w[j], f[2 * j], f[2 * j + 1]);
                    if (mul != 0x3c003c00u) {
#pragma unroll
                        for (int j = 0; j < 8; ++j) f[j] = mul_f16x2(f[j], mul);
                        if (static_cast<int>(mul) < 0)
#pragma unroll
                            for (int j = 0; j < 8; ++j) f[j] = mul_f16x2(f[j], 0x84008400u);
                    }
                    store_16(to[0] + at, f[0], f[1], f[2], f[3]);
                    store_16(to[1] + at, f[4], f[5], f[6], f[7]);
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        uint32_t f[4];
                        e2m1_to_f16(w[j], f);
                        store_16(to[j] + at, mul_f16x2(f[0], mul), mul_f16x2(f[1], mul), mul_f16x2(f[2], mul), mul_f16x2(f[3], mul));
                    }
                }
            }
        };
        uint32_t t = 0;                                                          // tiles so far
        if (keys) {
            int* const of_warp = reinterpret_cast<int*>(smem + L::OF_WARP);
            uint8_t* const k_scales = smem + L::OF_K;                            // 4-bit: [tile % 2][token]: their four bytes
            Turn<L::RAW_KEYS> raw;
            Turn<L::KEYS> ring;
            uint32_t segments = 0;
            while (seg.next()) {
                int sigma = -126;                                                // the values' reference starts anew with each segment
                wait(bar(FACTOR_FULL, 0), segments & 1, ctl, kWaitMany + 10, kStatusTimeout);
                ++segments;
                const volatile float* const of_segment = reinterpret_cast<const volatile float*>(smem + L::FACTOR);
                const float factor = of_segment[0];
                const int odd = __any_sync(0xffffffffu, of_segment[16 + (lane & 7)] != 0.f) ? 8 : 0;
                for (int left = seg.tiles; left > 0; --left, ++t) {
                    const uint32_t slot = t & (kSlots - 1);
                    wait(bar(RAW_K_FULL, raw.slot), raw.phase, ctl, kWaitMany + 5, kStatusTimeout);
                    // (the products of two tiles back are done, so those of four back with their values: nobody reads this slot of the factors)
                    wait(bar(K_EMPTY, ring.slot), ring.phase ^ 1, ctl, kWaitMany + 6, kStatusTimeout);
                    // scales: a thread a token
                    int word;                                                    // this warp's: the largest exponent of a value's scale, and what is special
                    const uint8_t* const rest = smem + L::MORE + raw.slot * L::MORE_BYTES;
                    const uint32_t flag = rest[L::FLAGS + me];
                    const bool in = flag != 0;
                    int top_sigma = -126;
                    bool nan = false;
                    float k_factor = 0.f;
                    uint32_t top_of_k = 0;
                    if (FMT == KV_CACHE_INT8) {
                        const uint32_t vs = reinterpret_cast<const uint32_t*>(rest + L::V_SCALES)[me];
                        k_factor = reinterpret_cast<const float*>(rest)[me];
                        nan = in && (vs & 0x7f800000u) == 0x7f800000u;
                        if (in && !nan) top_sigma = static_cast<int>(vs >> 23) - 126;               // s < 2^this
                        nans[slot * kTok + me] = nan ? 0xff : 0;
                        reinterpret_cast<uint32_t*>(v_scales)[slot * kTok + me] = in && !nan ? vs : 0u;     // (finite is what matters)
                    } else {
                        const uint32_t* const its = reinterpret_cast<const uint32_t*>(rest) + 2 * me;
                        const uint32_t shift = 8 * (flag & 3), there = blocks == 4 ? ~0u : (1u << (8 * blocks)) - 1;
                        const uint32_t kb = __funnelshift_r(its[0], its[1], shift) & there, vb = __funnelshift_r(its[kTok * 2], its[kTok * 2 + 1], shift) & there;
                        const uint32_t k_nan = __vcmpeq4(kb, ~0u), v_nan = __vcmpeq4(vb, ~0u);
                        uint32_t k_top = kb & ~k_nan, v_top = vb & ~v_nan;
                        k_top = __vmaxu4(k_top, k_top >> 16);
                        if (in) top_of_k = max(k_top & 0xffu, k_top >> 8 & 0xffu);
                        v_top = __vmaxu4(v_top, v_top >> 16);
                        nan = in && v_nan != 0;
                        if (in) top_sigma = max(-126, static_cast<int>(max(v_top & 0xffu, v_top >> 8 & 0xffu)) - 127);
                        reinterpret_cast<uint32_t*>(k_scales)[(t & 1) * kTok + me] = in ? kb : 0u;
                        nans[slot * kTok + me] = static_cast<uint8_t>((v_nan & 1u) | (v_nan >> 7 & 2u) | (v_nan >> 14 & 4u) | (v_nan >> 21 & 8u));
                        reinterpret_cast<uint32_t*>(v_scales)[slot * kTok + me] = in ? vb & ~v_nan : 0u;        // (those not seen may be above what is seen: finite is what matters)
                    }
                    k_factor *= factor;
                    factors[slot * kTok + me] = in ? k_factor : -1.f;
                    word = __reduce_max_sync(0xffffffffu, top_sigma) * 8 + (__any_sync(0xffffffffu, nan) ? 1 : 0) + (__any_sync(0xffffffffu, !in) ? 2 : 0) +
                           (FMT == KV_CACHE_INT8 && __any_sync(0xffffffffu, in && k_factor > 0x1p-9f) ? 4 : 0);
                    if (FMT == KV_CACHE_MXFP4) top_of_k = __reduce_max_sync(0xffffffffu, top_of_k);
                    if (lane == 0) {
                        of_warp[(t & 1) * 8 + warp - kKeyWarp] = word;
                        of_warp[(t & 1) * 8 + 4 + warp - kKeyWarp] = static_cast<int>(top_of_k);
                    }
                    named_sync(1, kConverters);
                    int all = 0;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int its = of_warp[(t & 1) * 8 + i];
                        if (FMT == KV_CACHE_MXFP4) top_of_k = max(top_of_k, static_cast<uint32_t>(of_warp[(t & 1) * 8 + 4 + i]));
                        sigma = max(sigma, its >> 3);                            // the largest scale of values so far (an exponent of fp32)
                        all |= its & 7;
                    }
                    if (me == 0) {
                        sigmas[slot] = sigma;
                        all |= odd;
                        if (FMT == KV_CACHE_MXFP4) {                             // (0 and infinity are no factors of -infinity and 0)
                            const float of_tile = fminf(fmaxf(factor * __uint_as_float(top_of_k == 0 ? 0x00400000u : top_of_k << 23) * 0x1p-12f, 1.2e-38f), 3e38f);
                            tile_factors[slot] = of_tile;
                            if (of_tile > 0x1p-17f) all |= 4;
                        }
                        special[slot] = all;
                    }
                    if (lane == 0) mbar_arrive(bar(SCALES_FULL, slot));
                    const uint32_t from = L::RAW + raw.slot * kTok * L::ROW, tile = ring.slot * L::TILE;
                    if constexpr (FMT == KV_CACHE_INT8) convert(from, tile, [](int) { return 0x3c003c00u; });
                    else convert(from, tile, [&](int r) {                        // 2^12 * 2^(byte - top), subnormal from e = 0 down (2^-39 of the tile's largest keys)
                        const int its = k_scales[((t & 1) * kTok + r) * 4 + chunk], e = 27 + its - static_cast<int>(top_of_k);
                        return (its == 255 ? 0x7e00u : e > 0 ? static_cast<uint32_t>(e) << 10 : 512u >> min(-e, 31)) * 0x00010001u;
                    });
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) {
                        mbar_arrive(bar(K_FULL, ring.slot));
                        mbar_arrive(bar(RAW_K_EMPTY, raw.slot));
                    }
                    raw.next();
                    ring.next();
                }
            }
        } else {
            Turn<L::RAW_VALUES> raw;
            Turn<L::VALUES> ring;
            for (const uint32_t units = static_cast<uint32_t>(share.end - share.begin); t < units; ++t) {
                // values: times their scale over 2^sigma, brought to 2^15 at most
                const uint32_t slot = t & (kSlots - 1);
                wait(bar(SCALES_FULL, slot), t / kSlots & 1, ctl, kWaitMany + 11, kStatusTimeout);
                const int sigma = sigmas[slot];
                wait(bar(RAW_V_FULL, raw.slot), raw.phase, ctl, kWaitMany + 5, kStatusTimeout);
                wait(bar(V_EMPTY, ring.slot), ring.phase ^ 1, ctl, kWaitMany + 6, kStatusTimeout);
                const uint32_t from = L::RAW_V + raw.slot * kTok * L::ROW, tile = L::V_TILES + ring.slot * L::TILE;
                if constexpr (FMT == KV_CACHE_INT8) {
                    // (two factors, as 2^(8 - sigma) alone may be more than fp32 holds)
                    const float by0 = __uint_as_float(static_cast<uint32_t>(127 - sigma / 2) << 23), by1 = __uint_as_float(static_cast<uint32_t>(127 + 8 - (sigma - sigma / 2)) << 23);
                    convert(from, tile, [&](int r) {
                        const float by = reinterpret_cast<const float*>(v_scales)[slot * kTok + r] * by0 * by1;
                        // (where fp16 holds only part of it, in two steps: 2^14 times as much, negative, then times -2^-14)
                        return by >= 0x1p-14f ? pack_f16(by, by) : pack_f16(by * -0x1p14f, by * -0x1p14f);
                    });
                } else {
                    convert(from, tile, [&](int r) {                             // 2^12 * 2^(byte - 127 - sigma), subnormal from e = 0 down
                        const int e = 27 + static_cast<int>(v_scales[(slot * kTok + r) * 4 + chunk]) - 127 - sigma;
                        return (e > 0 ? static_cast<uint32_t>(e) << 10 : 512u >> min(-e, 31)) * 0x00010001u;
                    });
                }
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(bar(V_FULL, ring.slot));
                    mbar_arrive(bar(RAW_V_EMPTY, raw.slot));
                }
                raw.next();
                ring.next();
            }
        }
    } else {
        // ---- softmax: a thread a row. Scores times their tokens' factors are powers of two.
        const int w = warp >> 2, row = threadIdx.x & (kRows - 1);
        const uint32_t lanes = static_cast<uint32_t>(32 * (warp & 3)) << 16, s_tmem = tmem + lanes + w * kTok, o_tmem = tmem + lanes + L::O + w * DP;
        float* const state = reinterpret_cast<float*>(smem + L::STATE);          // [warpgroup][row]: references of o (beside the sum's) and of the sum, the sum, NaN blocks
        volatile float* const of_segment = reinterpret_cast<volatile float*>(smem + L::FACTOR);         // the scores' factor, [8 + warp]: the queries' maxima, [16 + warp]: 1 with odd rows
        volatile uint32_t* const powers = reinterpret_cast<volatile uint32_t*>(smem + L::POWERS);       // [row]: what its queries are multiplied by
        uint32_t tile_base = 0, jobs = 0;                                        // jobs of this warpgroup so far
        while (seg.next()) {
            const int r = (PAIR ? w * kRows : 0) + row;                          // of the item's rows
            const bool live = r < seg.rows, warp_live = (PAIR ? w * kRows : 0) + 32 * (warp & 3) < seg.rows;
            const int node = (seg.row0 + min(r, seg.rows - 1)) / a.group;
            // queries: a power of two, which the tokens' factors take account of, brings the largest magnitude of all rows to [2^14, 2^15) (a larger one counts as 2^15: factors stay
            // within fp32). It serves the rows whose own largest is 2^-8 of that or more, so 2^6 after it. Others are odd, and have their own: no row's result depends on how large its
            // neighbours are. Their scores are brought to the common power in tensor memory (exact), which costs the segment a trip for each tile.
            // DP / 8 lanes a row; all rows are on their way at once, those of one tile of
            // rows in registers, those of two by way of the places that they go to (twice through registers costs 10 us).
            int common_up;
            {
                constexpr int LANES = DP / 8, AT_ONCE = 32 / LANES, STEPS = ROWS / 8 / AT_ONCE;
                const int d = lane % LANES * 8;
                uint4 x[PAIR ? 1 : STEPS] = {};
                auto row_of = [&](int i) { return (warp * STEPS + i) * AT_ONCE + lane / LANES; };
                auto place_of = [&](int i) { return base + L::Q + (row_of(i) / kRows) * L::TILE + place(row_of(i) % kRows, d); };
                auto from = [&](int i, bool& valid) {
                    const int q_row = row_of(i), its = (seg.row0 + q_row) / a.group, its_head = seg.head * a.group + (seg.row0 + q_row) - its * a.group;
                    valid = q_row < seg.rows && d < a.dim;
                    return a.q + (valid ? static_cast<int64_t>(seg.s.begin + its) * a.q_st + its_head * a.q_sh + d : 0);
                };
                auto read = [&](int i) {
                    if (!PAIR) return x[PAIR ? 0 : i];
                    uint4 v;
                    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(place_of(i)) : "memory");
                    return v;
                };
                bool valid;
                if (PAIR) {
#pragma unroll 1
                    for (int i = 0; i < STEPS; ++i) {
                        const __nv_bfloat16* const p = from(i, valid);
                        cp_async<16>(place_of(i), p, valid ? 16 : 0);
                    }
                    asm volatile("cp.async.wait_all;" ::: "memory");
                } else {
#pragma unroll
                    for (int i = 0; i < (PAIR ? 1 : STEPS); ++i) {
                        const __nv_bfloat16* const p = from(i, valid);
                        x[i] = valid ? *reinterpret_cast<const uint4*>(p) : make_uint4(0, 0, 0, 0);
                    }
                }
                // largest magnitudes, of N steps' rows at a time: lanes swap halves of what they hold, until each has one row's (what is Inf or NaN sets no power)
                constexpr int N = PAIR ? 4 : STEPS;
                uint32_t top = 0;
                int my_row = 0;
#pragma unroll 1
                for (int i = 0; i < STEPS; i += N) {
                    uint32_t its[N];
#pragma unroll
                    for (int j = 0; j < N; ++j) {
                        its[j] = absmax_bits8(read(i + j));
                        if (its[j] >= 0x7f800000u) its[j] = 0;
                    }
#pragma unroll
                    for (int o = LANES / 2, n = N; o > 0; o /= 2, n = n > 1 ? n / 2 : 1) {
                        if (n == 1) its[0] = max(its[0], __shfl_xor_sync(0xffffffffu, its[0], o));
#pragma unroll
                        for (int j = 0; j < n / 2; ++j) {
                            const bool upper = (lane & o) != 0;
                            its[j] = max(upper ? its[j + n / 2] : its[j], __shfl_xor_sync(0xffffffffu, upper ? its[j] : its[j + n / 2], o));
                        }
                    }
                    top = its[0];
                    my_row = row_of(i + lane % LANES / (LANES / N));
                    if (PAIR) powers[my_row] = top;
                }
                if (PAIR) {                                                      // (32 rows a warp)
                    __syncwarp();
                    my_row = warp * 32 + lane;
                    top = powers[my_row];
                }
                uint32_t largest = __reduce_max_sync(0xffffffffu, top);
                if (lane == 0) of_segment[8 + warp] = __uint_as_float(largest);
                named_sync(2, kSoftmax);
#pragma unroll
                for (int i = 0; i < 8; ++i) largest = max(largest, __float_as_uint(of_segment[8 + i]));
                const int field = static_cast<int>(top >> 23), common = min(static_cast<int>(largest >> 23), 141);
                common_up = min(126, 141 - max(common, 1));
                const bool odd = top != 0 && (field > common || field + 8 < common);
                const bool any_odd = __any_sync(0xffffffffu, odd);
                if (lane == 0) of_segment[16 + warp] = any_odd ? 1.f : 0.f;
                if (threadIdx.x == 0) of_segment[0] = fabsf(a.scale) * kLog2e * __uint_as_float((127 - common_up) << 23);
                if (lane == 0) mbar_arrive(bar(FACTOR_FULL, 0));
                const uint32_t my_power = static_cast<uint32_t>(127 + (odd ? min(126, 141 - max(field, 1)) : common_up)) << 23;
                powers[my_row] = my_power;
                if (PAIR) __syncwarp();
#pragma unroll(PAIR ? 4 : STEPS)
                for (int i = 0; i < STEPS; ++i) {
                    const float power = __uint_as_float(PAIR ? powers[row_of(i)] : __shfl_sync(0xffffffffu, my_power, (lane & ~(LANES - 1)) + i * (LANES / N)));
                    const float mul = a.scale < 0.f ? -power : power;
                    float f[8];
                    unpack_bf16x8(read(i), f);
                    store_16(place_of(i), pack_f16(f[0] * mul, f[1] * mul), pack_f16(f[2] * mul, f[3] * mul), pack_f16(f[4] * mul, f[5] * mul), pack_f16(f[6] * mul, f[7] * mul));
                }
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(Q_FULL, 0));
            float m = kNone;
            uint64_t l2 = 0;
            int sigma = -126;
            uint32_t poison = 0;                                                 // blocks of this row's output that are NaN
            bool first = true;
#pragma unroll 1
            for (int t = PAIR ? 0 : w; t < seg.tiles; t += PAIR ? 1 : 2, ++jobs) {
                const uint32_t slot = (tile_base + t) & (kSlots - 1);
                wait(bar(S_FULL, w), jobs & 1, ctl, kWaitMany + 7, kStatusTimeout);
                tc_fence_after();
                if (warp_live) {
                    const float* kf = factors + slot * kTok;
                    const int j0 = seg.token(t) - seg.s.before;
                    // which of 32 tokens this row sees: those that anybody does, and of the new ones its own
                    auto sees32_of = [&](int ch) {
                        uint32_t sees = __ballot_sync(0xffffffffu, kf[32 * ch + lane] != -1.f);
                        if (j0 + 32 * ch + 31 >= 0) sees &= sees32(a, seg.s.begin + node, node, j0 + 32 * ch);
                        return sees;
                    };
                    const int its_special = special[slot];
                    if ((its_special & 1) != 0) {
#pragma unroll 1
                        for (int ch = 0; ch < 4; ++ch) {
                            const uint32_t sees = sees32_of(ch);
#pragma unroll 1
                            for (int x = 0; x < 32; ++x)
                                if (sees >> x & 1u) poison |= nans[slot * kTok + x + 32 * ch];
                        }
                    }
                    float tile_factor = FMT == KV_CACHE_MXFP4 ? tile_factors[slot] : 1.f;
                    // Tiles with tokens that not all rows see (a sequence's last ones): scores with their factors, or -inf, put back in their places. So are those of rows with powers
                    // of their own, and scores that may be beyond 2^20 (before their factors they are below 2^29 or 2^37): of a product that is not rounded before its reference is
                    // taken off, which was, more than 2^15 might be left.
                    if (j0 + kTok > 0 || its_special > 1) {
                        if ((its_special & 8) != 0) tile_factor = fminf(tile_factor * __uint_as_float(((254u + common_up) << 23) - powers[r]), 3e38f);
#pragma unroll 1
                        for (int ch = 0; ch < 16; ++ch) {
                            uint32_t v[8];
                            tmem_ld_32x32b_x8(s_tmem + 8 * ch, v);
                            const uint32_t sees = sees32_of(ch / 4) >> (8 * (ch & 3));
                            tmem_wait_ld();
#pragma unroll
                            for (int i = 0; i < 8; ++i) v[i] = sees >> i & 1u ? __float_as_uint(__uint_as_float(v[i]) * (FMT == KV_CACHE_INT8 ? kf[8 * ch + i] * tile_factor : tile_factor)) : 0xff800000u;
                            tmem_st_32x32b_x8(s_tmem + 8 * ch, v);
                        }
                        tmem_wait_st();
                        kf = reinterpret_cast<const float*>(smem + L::ONES);
                        tile_factor = 1.f;
                    }
                    // the row's largest score: 16 columns at a time, the next ones on their way
                    float top = -INFINITY;
                    {
                        uint32_t v[2][16];
                        tmem_ld_32x32b_x16(s_tmem, v[0]);
#pragma unroll 1
                        for (int ch = 0; ch < 8; ch += 2) {
#pragma unroll
                            for (int half = 0; half < 2; ++half) {
                                tmem_wait_ld();
                                tmem_ld_32x32b_x16(s_tmem + 16 * ((ch + half + 1) & 7), v[half ^ 1]);
                                const uint32_t (&x)[16] = v[half];
#pragma unroll
                                for (int i = 0; i < 16; i += 4) {
                                    if (FMT == KV_CACHE_MXFP4) {
                                        top = max3(max3(top, __uint_as_float(x[i]), __uint_as_float(x[i + 1])), __uint_as_float(x[i + 2]), __uint_as_float(x[i + 3]));
                                        continue;
                                    }
                                    const float4 k = *reinterpret_cast<const float4*>(kf + 16 * (ch + half) + i);
                                    float p, q, y, z;
                                    unpack2(mul2(pack2(__uint_as_float(x[i]), __uint_as_float(x[i + 1])), pack2(k.x, k.y)), p, q);
                                    unpack2(mul2(pack2(__uint_as_float(x[i + 2]), __uint_as_float(x[i + 3])), pack2(k.z, k.w)), y, z);
                                    top = max3(max3(top, p, q), y, z);
                                }
                            }
                        }
                        tmem_wait_ld();
                    }
                    top = fmaxf(FMT == KV_CACHE_MXFP4 ? top * tile_factor : top, kNone);
                    // references move when a weight would pass 2^15, to put it at 2^7, or when the values' does
                    const int its_sigma = sigmas[slot];
                    if (__any_sync(0xffffffffu, top - m > 15.f || its_sigma != sigma)) {
                        const float now = top - m > 15.f ? top - 7.f : m, by_l = ex2(m - now);
                        l2 = mul2(l2, pack2(by_l, by_l));
                        if (!first) {
                            const float half = ex2(static_cast<float>(max(sigma - its_sigma, -252)) * 0.5f), by = by_l * half * half;
                            wait(bar(O_DONE, w), (jobs - 1) & 1, ctl, kWaitMany + 8, kStatusTimeout);
                            tc_fence_after();
#pragma unroll 1
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
                    {
                        uint32_t v[2][16];
                        uint64_t sum[2] = {0, 0};
                        tmem_ld_32x32b_x16(s_tmem, v[0]);
#pragma unroll 1
                        for (int ch = 0; ch < 8; ch += 2) {
#pragma unroll
                            for (int half = 0; half < 2; ++half) {
                                tmem_wait_ld();
                                if (half == 0 || ch < 6) tmem_ld_32x32b_x16(s_tmem + 16 * (ch + half + 1), v[half ^ 1]);
                                const uint32_t (&x)[16] = v[half];
                                uint32_t p[8];
#pragma unroll
                                for (int i = 0; i < 16; i += 4) {
                                    const float4 k = FMT == KV_CACHE_MXFP4 ? make_float4(tile_factor, tile_factor, tile_factor, tile_factor) : *reinterpret_cast<const float4*>(kf + 16 * (ch + half) + i);
                                    float y, z;
                                    unpack2(fma2(pack2(__uint_as_float(x[i]), __uint_as_float(x[i + 1])), pack2(k.x, k.y), m2), y, z);
                                    y = ex2(y);
                                    z = ex2(z);
                                    sum[0] = add2(sum[0], pack2(y, z));
                                    p[i / 2] = pack_f16(y, z);
                                    unpack2(fma2(pack2(__uint_as_float(x[i + 2]), __uint_as_float(x[i + 3])), pack2(k.z, k.w), m2), y, z);
                                    y = ex2(y);
                                    z = ex2(z);
                                    sum[1] = add2(sum[1], pack2(y, z));
                                    p[i / 2 + 1] = pack_f16(y, z);
                                }
                                tmem_st_32x32b_x8(s_tmem + 8 * (ch + half), p);
                            }
                        }
                        l2 = add2(l2, add2(sum[0], sum[1]));
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
            // (reference of o beside the sum's: the values'; int8 tiles are 2^8 too large, 4-bit ones 2^12, which the results take account of)
            float m_o = static_cast<float>(sigma - (FMT == KV_CACHE_INT8 ? 8 : 0)), m_l = m;
            if (PAIR || w < seg.tiles) wait(bar(O_DONE, w), (jobs - 1) & 1, ctl, kWaitMany + 9, kStatusTimeout);
            if (!PAIR) *reinterpret_cast<float4*>(state + (w * kRows + row) * 4) = make_float4(m_o, m, l, __uint_as_float(poison));
            named_sync(2, kSoftmax);
            tc_fence_after();
            const bool whole = seg.whole();
            // a part: elements 4q to 4q + 3 of row r at float4 q * ROWS + r (so that the threads of a warp, a row each, write and read side by side), then the states
            constexpr int PART = part_floats(ROWS, DP);
            float4* const part = reinterpret_cast<float4*>(a.parts + (2 * static_cast<int64_t>(blockIdx.x) + (share.begin > seg.item_begin ? 0 : 1)) * PART);
            // (one tile of rows: each warpgroup takes half of the elements)
            constexpr int WIDTH = PAIR ? DP : DP / 2;
            const int d0 = PAIR ? 0 : w * WIDTH, h = seg.head * a.group + seg.row0 + r - node * a.group;
            __nv_bfloat16* const to = a.out + static_cast<int64_t>(seg.s.begin + node) * a.o_st + h * a.o_sh;
            auto write8 = [&](const Row& state_of, float2 scale, const float* o, int d) {        // eight elements of this thread's row
                uint32_t packed[4];
                const float both = scale.x * scale.y;
#pragma unroll
                for (int e = 0; e < 4; ++e) packed[e] = state_of.l == 0.f ? 0u : pack_bf16(o[2 * e] * both * scale.y, o[2 * e + 1] * both * scale.y);
                *reinterpret_cast<uint4*>(to + d) = make_uint4(packed[0], packed[1], packed[2], packed[3]);
            };
            if (warp_live) {
                float by[2] = {1.f, 0.f};
                const bool two = !PAIR && seg.tiles > 1;
                if (!PAIR) {
                    const float4 s0 = *reinterpret_cast<const float4*>(state + row * 4), s1 = *reinterpret_cast<const float4*>(state + (kRows + row) * 4);
                    m_o = s0.x;
                    m_l = s0.y;
                    l = s0.z;
                    poison = __float_as_uint(s0.w);
                    if (two) {
                        m_l = fmaxf(s0.y, s1.y);
                        const float down0 = s0.y - m_l, down1 = s1.y - m_l;
                        m_o = fmaxf(s0.x + down0, s1.x + down1);
                        by[0] = ex2(s0.x + down0 - m_o);
                        by[1] = ex2(s1.x + down1 - m_o);
                        l = s0.z * ex2(down0) + s1.z * ex2(down1);
                        poison |= __float_as_uint(s1.w);
                    }
                }
                Row out;
                out.m_o = m_o;
                out.m_l = m_l;
                out.l = l;
                const float2 scale = out.scale<FMT>();
#pragma unroll 1
                for (int d = d0; d < d0 + WIDTH; d += 16) {
                    uint32_t v[16], u[16];
                    tmem_ld_32x32b_x16(tmem + lanes + L::O + (PAIR ? w * DP : 0) + d, v);
                    if (two) tmem_ld_32x32b_x16(tmem + lanes + L::O + DP + d, u);
                    tmem_wait_ld();
                    float o[16];
#pragma unroll
                    for (int x = 0; x < 16; ++x) o[x] = two ? __uint_as_float(v[x]) * by[0] + __uint_as_float(u[x]) * by[1] : __uint_as_float(v[x]);
                    if ((FMT == KV_CACHE_INT8 ? poison : poison >> (d / kMxBlock) & 1u) != 0)
#pragma unroll
                        for (int x = 0; x < 16; ++x) o[x] = __uint_as_float(0x7fc00000u);
                    if (!live) continue;
                    if (whole) {
#pragma unroll
                        for (int x = 0; x < 16; x += 8)
                            if (d + x < a.dim) write8(out, scale, o + x, d + x);
                    } else {
#pragma unroll
                        for (int x = 0; x < 16; x += 4) part[(d + x) / 4 * ROWS + r] = make_float4(o[x], o[x + 1], o[x + 2], o[x + 3]);
                    }
                }
                if (live && d0 == 0) {
                    if (whole) out.write_lse(a, seg.s, node, h);
                    else part[DP / 4 * ROWS + r] = make_float4(m_o, m_l, l, 0.f);
                }
            }
            tc_fence_before();
            named_sync(2, kSoftmax);                                             // o and the states may be written over
            if (!whole) {
                const int from = owner(seg.item_begin, share), until = owner(seg.item_end - 1, share);
                if (last_to_arrive<ROWS>(a, seg.s, seg.b, seg.head, seg.row0, from, until, threadIdx.x, &last_one, [] { named_sync(2, kSoftmax); })) {
                    if (live) {
                    // the parts of this thread's row and elements, in the order of the tokens: their states, then 32 elements at a time, several parts' loads on their way
                    auto part_of = [&](int x) { return reinterpret_cast<const float4*>(a.parts + (2 * static_cast<int64_t>(x) + (x == from ? 1 : 0)) * PART); };
                    Row sum;
#pragma unroll 2
                    for (int x = from; x <= until; ++x) {
                        const float4 its = __ldcg(part_of(x) + DP / 4 * ROWS + r);
                        const float now_l = fmaxf(sum.m_l, its.y), down = sum.m_l - now_l, its_down = its.y - now_l;
                        sum.l = sum.l * ex2(down) + its.z * ex2(its_down);
                        sum.m_l = now_l;
                        sum.m_o = fmaxf(sum.m_o + down, its.x + its_down);
                    }
                    const float2 scale = sum.scale<FMT>();
                    // by way of the queries' place or, where nothing follows in this CTA, of the tiles' too, so that several parts are on their way (46.6 to 44.3 us for 12 x 32
                    // nodes behind 1500 tokens, against 8 elements at a time by way of the queries' place)
                    constexpr int Q_BYTES = (PAIR ? 2 : 1) * L::TILE, EACH = DP == 128 ? 8 : 4, GROUP = EACH * 16 * kSoftmax, MOST = (L::Q + Q_BYTES) / GROUP;
                    static_assert(Q_BYTES >= GROUP && WIDTH % (4 * EACH) == 0 && MOST >= 4, "");
                    const bool at_end = seg.u + seg.tiles == share.end;
                    const int groups = at_end ? 4 : Q_BYTES / GROUP >= 2 ? 2 : 1;
                    const uint32_t stage = base + (at_end ? 0 : L::Q) + threadIdx.x * 16, m_stage = base + L::STATE + threadIdx.x * 8;
                    const int chunks = (max(0, min(WIDTH, a.dim - d0)) + 4 * EACH - 1) / (4 * EACH);
                    int in_chunk = 0, in_part = from, in_slot = 0;
                    auto ask = [&] {
                        if (in_chunk < chunks) {
                            const float4* const p = part_of(in_part);
#pragma unroll
                            for (int q = 0; q < EACH; ++q) cp_async<16>(stage + (in_slot * EACH + q) * kSoftmax * 16, p + (d0 / 4 + in_chunk * EACH + q) * ROWS + r, 16);
                            cp_async<8>(m_stage + in_slot * kSoftmax * 8, p + DP / 4 * ROWS + r, 8);
                            if (++in_part > until) {
                                in_part = from;
                                ++in_chunk;
                            }
                        }
                        cp_async_commit();
                        in_slot = in_slot + 1 == groups ? 0 : in_slot + 1;
                    };
#pragma unroll 1
                    for (int i = 0; i < groups; ++i) ask();
                    int slot = 0;
#pragma unroll 1
                    for (int c = 0; c < chunks; ++c) {
                        float o[4 * EACH];
#pragma unroll
                        for (int i = 0; i < 4 * EACH; ++i) o[i] = 0.f;
#pragma unroll 1
                        for (int x = from; x <= until; ++x) {
                            if (groups == 4) cp_async_wait<3>();
                            else if (groups == 2) cp_async_wait<1>();
                            else cp_async_wait<0>();
                            float its_m, its_l;
                            asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(its_m), "=f"(its_l) : "r"(m_stage + slot * kSoftmax * 8) : "memory");
                            float4 v[EACH];
#pragma unroll
                            for (int q = 0; q < EACH; ++q)
                                asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v[q].x), "=f"(v[q].y), "=f"(v[q].z), "=f"(v[q].w) : "r"(stage + (slot * EACH + q) * kSoftmax * 16) : "memory");
                            const float by = ex2(its_m + (its_l - sum.m_l) - sum.m_o);
#pragma unroll
                            for (int q = 0; q < EACH; ++q) {
                                o[4 * q] += v[q].x * by;
                                o[4 * q + 1] += v[q].y * by;
                                o[4 * q + 2] += v[q].z * by;
                                o[4 * q + 3] += v[q].w * by;
                            }
                            ask();                                               // (into the place just read)
                            slot = slot + 1 == groups ? 0 : slot + 1;
                        }
#pragma unroll
                        for (int x = 0; x < 4 * EACH; x += 8)
                            if (d0 + c * 4 * EACH + x < a.dim) write8(sum, scale, o + x, d0 + c * 4 * EACH + x);
                    }
                    if (d0 == 0) sum.write_lse(a, seg.s, node, h);
                    }
                    named_sync(2, kSoftmax);                                     // (the queries' place is free again)
                }
            }
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
cudaError_t launch(const CUtensorMap& k_map, const CUtensorMap& v_map, const AttentionArgs& a, cudaStream_t st) {
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
    return cudaLaunchKernelEx(&cfg, kern, k_map, v_map, a);
}
template <int FMT>
cudaError_t launch_for(const CUtensorMap& k, const CUtensorMap& v, const AttentionArgs& a, int64_t rows, cudaStream_t st) {
    if (a.dim <= 64) return rows > kRows ? launch<FMT, 64, true>(k, v, a, st) : launch<FMT, 64, false>(k, v, a, st);
    return rows > kRows ? launch<FMT, 128, true>(k, v, a, st) : launch<FMT, 128, false>(k, v, a, st);
}

} // namespace

bool many_rows_fits(int dim) { return dim <= 128; }
size_t many_rows_part_bytes() { return static_cast<size_t>(sm_count()) * 2 * part_floats(2 * kRows, 128) * sizeof(float); }
cudaError_t launch_many_rows(int fmt, const CUtensorMap& k_map, const CUtensorMap& v_map, const AttentionArgs& a, int64_t rows, cudaStream_t st) {
    return fmt == KV_CACHE_INT8 ? launch_for<KV_CACHE_INT8>(k_map, v_map, a, rows, st) : launch_for<KV_CACHE_MXFP4>(k_map, v_map, a, rows, st);
}

} // namespace attention
} // namespace w8a8
