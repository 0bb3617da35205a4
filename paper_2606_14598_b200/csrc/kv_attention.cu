// Attention of new tokens over the quantized paged cache, on the codes.
//
//   o = sum_p softmax_p(scale * q . k_p) v_p,   k_p = code * s_k(p),  v_p = code * s_v(p)      (MXFP4: a scale for 32 elements)
//
// A token's scale factors out of both products: scores are (q . code) * s_k, and the values' scale multiplies the probability, so what the
// matrix instructions take are the codes themselves, converted in registers and exact: keys as fp16 beside queries that a power of two of their
// row brings into fp16's range, values as fp16 beside weights (probability times s_v) relative to the row's own size.
//
// One pass over the cache with a running maximum and sum. The work is cut into units of a few dozen tokens of one head of one sequence, in one
// long list that the CTAs share out evenly whatever the sequences' lengths: a CTA's range holds ends of at most two items that others share,
// whose parts meet in the workspace and are added up, in the order of the tokens, by the CTA that arrives last.
//
// What bounds it: int8, HBM and the latency of loads (48 sequences of up to 4000 tokens, 8 heads of 128, 4 queries a head: 62 us, 39 at the copy's rate; loads alone, without
// the products, 55). 4 bits: issue slots, some 1100 instructions for 32 tokens of a head, most of them conversions (12 sequences of up to 30000, 8 heads, 8 queries: 106 us, 39;
// its 128 registers, for four CTAs an SM, spill 128 bytes).
// One sequence of 777 tokens: 9.5 us, launch, list, one step and the parts' meeting after one another. (SM clock 1965 MHz in all.)
#include "internal.h"
#include "kv_attention.cuh"
#include "tensor_map.h"

#include <cmath>

namespace w8a8 {

using namespace attention;

namespace {

constexpr int kWarps = 4, kThreads = 32 * kWarps;
constexpr int kWaitAttention = 40;              // which wait gave up, for the status word
// Where things are. The codes are the first operand of both products: keys as 16 tokens by 16 elements, values as 16 elements by 16 tokens, so that eight
// rows of queries are enough to fill the second. Lane (g, c) feeds the keys of tokens g and g + 8 (the elements of chunks that its c gives) and its own
// elements (by g) of the values of tokens 2c, 2c + 1, 2c + 8 and 2c + 9; which elements those are is free as long as queries and outputs follow.
template <int FMT, int DP, int TT> struct Layout {
    static constexpr int TOK = 16 * TT;                                         // tokens of a step
    static constexpr int PER_BYTE = FMT == KV_CACHE_INT8 ? 1 : 2;
    static constexpr int ROW = DP / PER_BYTE;                                   // bytes of a head, padded
    static constexpr int BOX = ROW < 128 ? ROW : 128, BOXES = ROW / BOX;        // bytes of a row of a box, boxes side by side: a box is swizzled
    static constexpr int KB = ROW / 4 < 16 ? ROW / 4 : 16, KCH = ROW / 4 / KB;  // keys: bytes of a chunk, chunks of a lane
    static constexpr int VB = ROW / 8 < 16 ? ROW / 8 : 16, VCH = ROW / 8 / VB;  // values
    static constexpr int VC = VB * PER_BYTE;                                    // codes of a chunk of values
    static constexpr int KS = DP / 16;                                          // products of 16 along a head
    static constexpr int BLOCKS = DP / kMxBlock;
    static constexpr int K_BYTES = TOK * ROW, CODES = 2 * K_BYTES;              // codes of a stage: a multiple of the swizzle's 1024 bytes
    // and what goes with them: scales (4-bit: the words that hold a head's bytes), the shifts of these words, a bit for each token that may be seen
    static constexpr int WORDS = FMT == KV_CACHE_INT8 ? 1 : BLOCKS > 4 ? 4 : 2;
    static constexpr int META = 2 * TOK * 4 * WORDS, SEEN = META + (FMT == KV_CACHE_INT8 ? 0 : 4 * TOK), REST = SEEN + 16;
    // per warp, not per stage: (4-bit) multipliers [side][block][token] fp16; factors of the keys (4-bit) and logarithms of the values' scales, fp32 [token]
    static constexpr int MULS = FMT == KV_CACHE_INT8 ? 0 : 2 * BLOCKS * TOK * 2, PREP = MULS + 2 * TOK * 4;

    __device__ static __forceinline__ int k_offset(int j, int c) {              // first byte of chunk j of lane c in a row
        return KB == 16 && KCH > 1 ? (j / 2) * 128 + (2 * c + (j & 1)) * 16 : c * KB;
    }
    __device__ static __forceinline__ int v_offset(int j, int g) { return j * 128 + g * VB; }
    // byte `off` of row r of one side of a stage: chunks of 16 bytes change places by the row
    __device__ static __forceinline__ int place(int r, int off) {
        const int box = off / BOX, in = off % BOX;
        const int turn = BOX == 128 ? r & 7 : BOX == 64 ? (r >> 1) & 3 : (r >> 2) & 1;
        return box * TOK * BOX + r * BOX + (in ^ (turn << 4));
    }
    // element of q behind operand pair p, half e, of product s in lane c
    __device__ static __forceinline__ int element(int s, int c, int p, int e) {
        constexpr int words = KB / 4, per_word = FMT == KV_CACHE_INT8 ? 1 : 2;
        const int word = s / per_word;
        return k_offset(word / words, c) * PER_BYTE + word % words * 4 * PER_BYTE + s % per_word * 4 + 2 * p + e;
    }
};

// ------------------------------------------------------------------------------------------------ the kernel

// CTAs that are to share an SM: what the registers of the sums allow, and 50 KB of codes in flight on it do with
template <int FMT, int DP, int NR> constexpr int resident() { return DP * NR <= 64 ? 4 : DP * NR <= 128 ? (FMT == KV_CACHE_INT8 ? 3 : 4) : DP * NR <= 256 ? 3 : 2; }

template <int FMT, int DP, int NR, int TT>
struct Shared {
    using L = Layout<FMT, DP, TT>;
    static constexpr int ROWS = 8 * NR;
    static constexpr int FRAGS_BYTES = NR * L::KS * 256, STATE_BYTES = 3 * kWarps * ROWS * 4 + ROWS * 4, MERGE = kWarps * ROWS * (DP + 4) * 4;
    // as many steps in a warp's ring as let the CTAs meant to share an SM do so (227 KB, less what each is charged and wants besides)
    static constexpr int EACH = 227 * 1024 / resident<FMT, DP, NR>() - 2 * 1024 - 512 - FRAGS_BYTES - STATE_BYTES - kWarps * L::PREP;
    static constexpr int FIT = EACH / (kWarps * (L::CODES + L::REST + 8)), STAGES = FIT > 4 ? 4 : FIT;
    static constexpr int RING = kWarps * STAGES * L::CODES;
    // the ring (and over it, at the end, the warps' results); operands of the queries; the rest
    static constexpr int FRAGS = (RING > MERGE ? RING : MERGE), REST = FRAGS + FRAGS_BYTES, PREP = REST + kWarps * STAGES * L::REST;
    static constexpr int ROW_FACTOR = PREP + kWarps * L::PREP, STATE = ROW_FACTOR + ROWS * 4, BARS = STATE + 3 * kWarps * ROWS * 4;
    static constexpr int BYTES = BARS + kWarps * STAGES * 8 + 1024;
    static_assert(STAGES >= 2 && L::CODES % 1024 == 0 && BARS % 8 == 0, "");
};

template <int FMT, int DP, int NR, int TT>
__global__ void __launch_bounds__(kThreads, resident<FMT, DP, NR>()) kv_attention_kernel(const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map,
                                                                                  const AttentionArgs a) {
    using L = Layout<FMT, DP, TT>;
    using S = Shared<FMT, DP, NR, TT>;
    constexpr int ROWS = S::ROWS, TOK = L::TOK, STAGES = S::STAGES;
    constexpr uint32_t kAllSeen = TOK == 32 ? 0xffffffffu : (1u << (TOK & 31)) - 1;
    extern __shared__ uint8_t raw_smem[];
    uint8_t* const smem = raw_smem + (1024 - (smem_u32(raw_smem) & 1023)) % 1024;
    __shared__ int last_one;
    __shared__ volatile int abort_flag;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
    const uint32_t bars = smem_u32(smem + S::BARS) + warp * STAGES * 8;
    if (threadIdx.x == 0) abort_flag = 0;
    if (lane == 0) {
#pragma unroll
        for (int i = 0; i < STAGES; ++i) mbar_init(bars + 8 * i, 1);
        fence_mbar_init();
    }
    const WaitCtl ctl{&abort_flag, a.status, a.sticky, a.limit_ns};
    grid_dep_wait();
    const Share share = share_out<kThreads, kWarps * TOK>(a, ROWS);             // (its barriers make the mbarriers known, too)
    int64_t u = share.begin;
    const int64_t u_begin = u, u_end = share.end;
    int b = share.b;
    int64_t first_of_b = share.first_of_b;
    const int row_bytes = a.dim / L::PER_BYTE, blocks = (a.dim + kMxBlock - 1) / kMxBlock;
    uint8_t* const ring = smem + warp * STAGES * L::CODES;
    uint8_t* const rest = smem + S::REST + warp * STAGES * L::REST;
    const uint32_t ring_u32 = smem_u32(ring), rest_u32 = smem_u32(rest);
    uint8_t* const prep = smem + S::PREP + warp * L::PREP;
    uint32_t loads = 0;                                             // of this warp: stage and parity of a step go by it

    // this lane's places in a stage
    const int k_at = L::place(g, L::k_offset(0, c));
    const int v_at[2] = {L::place(2 * c, L::v_offset(0, g)), L::place(2 * c + 1, L::v_offset(0, g))};

    bool gave_up = false;                                           // one of this warp's waits did
    while (u < u_end) {
        Sequence s = read_sequence<kWarps * TOK>(a, b, ROWS);
        while (b + 1 < a.seqs && u - first_of_b >= units_of(a, s)) {            // (sequences without new tokens have no units)
            first_of_b += units_of(a, s);
            s = read_sequence<kWarps * TOK>(a, ++b, ROWS);
        }
        const int64_t of_b = u - first_of_b;
        const int item = static_cast<int>(of_b / s.tiles), tile0 = static_cast<int>(of_b - static_cast<int64_t>(item) * s.tiles);
        const int head = item / s.row_tiles, row0 = (item - head * s.row_tiles) * ROWS, rows = min(ROWS, s.n * a.group - row0);
        const int steps = static_cast<int>(min(static_cast<int64_t>(s.tiles - tile0), u_end - u));
        const int64_t item_begin = u - tile0, item_end = item_begin + s.tiles;
        const int first_token = s.base + (tile0 * kWarps + warp) * TOK;

        // ---- the cache: a step's tokens into a stage of the warp's ring. A lane looks up the token of its number and copies its scales; codes come as
        // boxes of as many tokens as lie side by side in any page, or (heads that are not whole 16-byte pieces) piece by piece.
        auto find = [&](int step) {                                 // slot of a token, -1: no such page or behind the end
            const int t = first_token + step * (kWarps * TOK) + (lane & (TOK - 1));
            if (step >= steps || t >= s.stop) return -1;
            const int p = a.page_shift >= 0 ? t >> a.page_shift : t / a.page;
            const int id = a.table[b * a.table_stride + p];
            return id >= 0 && id < a.num_pages ? id * a.page + (t - p * a.page) : -1;
        };
        auto issue = [&](int step, int slot, uint32_t load) {
            if (step < steps && !gave_up && !(a.starve != 0 && warp == 0 && load == 0)) {
                const uint32_t stage = load % STAGES, st = ring_u32 + stage * L::CODES, more = rest_u32 + stage * L::REST, bar = bars + 8 * stage;
                const uint32_t seen = __ballot_sync(0xffffffffu, slot >= 0 && first_token + step * (kWarps * TOK) + (lane & (TOK - 1)) >= s.start) & kAllSeen;
                if (a.box > 0) {
                    const bool mine = slot >= 0 && lane < TOK && lane % a.box == 0;
                    const uint32_t boxes = __popc(__ballot_sync(0xffffffffu, mine));
                    if (lane == 0) mbar_arrive_expect_tx(bar, boxes * 2 * L::BOXES * a.box * L::BOX);
                    __syncwarp();
                    if (mine) {
#pragma unroll
                        for (int j = 0; j < L::BOXES; ++j) {
                            tma_load_3d(st + j * TOK * L::BOX + lane * L::BOX, &k_map, bar, j * a.box_step, head, slot);
                            tma_load_3d(st + L::K_BYTES + j * TOK * L::BOX + lane * L::BOX, &v_map, bar, j * a.box_step, head, slot);
                        }
                    }
                } else {
                    const int64_t token_bytes = static_cast<int64_t>(a.heads) * row_bytes;
                    constexpr int kPieces = L::ROW / 4;                         // four bytes each; two at a time where the head allows it
                    for (int e = lane; e < TOK * kPieces / 2; e += 32) {
                        const int r = e / (kPieces / 2), off = (e - r * (kPieces / 2)) * 8;
                        const int from = __shfl_sync(0xffffffffu, slot, r);
                        const int64_t where = max(from, 0) * token_bytes + head * row_bytes + off;
                        const uint32_t to = st + L::place(r, off);
                        const int valid = from >= 0 ? row_bytes - off : 0;
                        if (row_bytes % 8 == 0) {
                            cp_async<8>(to, a.k_codes + (valid > 0 ? where : 0), valid > 0 ? 8 : 0);
                            cp_async<8>(to + L::K_BYTES, a.v_codes + (valid > 0 ? where : 0), valid > 0 ? 8 : 0);
                        } else {
#pragma unroll
                            for (int i = 0; i < 8; i += 4) {
                                cp_async<4>(to + i, a.k_codes + (valid > i ? where + i : 0), valid > i ? 4 : 0);
                                cp_async<4>(to + i + L::K_BYTES, a.v_codes + (valid > i ? where + i : 0), valid > i ? 4 : 0);
                            }
                        }
                    }
                }
                if (lane < TOK) {
                    const int64_t entry = static_cast<int64_t>(max(slot, 0)) * a.heads + head;
                    if (FMT == KV_CACHE_INT8) {
                        cp_async<4>(more + lane * 4, static_cast<const float*>(a.k_scales) + entry, slot >= 0 ? 4 : 0);
                        cp_async<4>(more + TOK * 4 + lane * 4, static_cast<const float*>(a.v_scales) + entry, slot >= 0 ? 4 : 0);
                    } else {                                        // the words that hold the head's bytes
                        const ScaleWords its = scale_words(entry, blocks);
#pragma unroll
                        for (int side = 0; side < 2; ++side) {
                            const uint8_t* p = static_cast<const uint8_t*>(side == 0 ? a.k_scales : a.v_scales) + its.from;
#pragma unroll
                            for (int i = 0; i < (L::WORDS == 2 ? 2 : 3); ++i) {
                                const int there = slot >= 0 ? its.bytes(i) : 0;
                                cp_async<4>(more + ((side * TOK + lane) * L::WORDS + i) * 4, p + (there > 0 ? 4 * i : 0), there);
                            }
                        }
                        *reinterpret_cast<int*>(rest + stage * L::REST + L::META + lane * 4) = its.shift;
                    }
                }
                if (lane == 0) *reinterpret_cast<uint32_t*>(rest + stage * L::REST + L::SEEN) = seen;
            }
            cp_async_commit();
        };
        int slot;
        {
            int slots[STAGES + 1];
#pragma unroll
            for (int i = 0; i <= STAGES; ++i) slots[i] = find(i);
#pragma unroll
            for (int i = 0; i < STAGES; ++i) issue(i, slots[i], loads + i);
            slot = slots[STAGES];
        }

        // ---- queries: rows of fp16 times a power of two, then as operands of the products
        float* const row_factor = reinterpret_cast<float*>(smem + S::ROW_FACTOR);
        __half* const halves = reinterpret_cast<__half*>(smem + S::FRAGS);
        for (int r = warp; r < ROWS; r += kWarps) {
            uint4 x = make_uint4(0, 0, 0, 0);
            if (r < rows && lane * 8 < a.dim) {
                const int node = (row0 + r) / a.group, h = head * a.group + (row0 + r) - node * a.group;
                x = *reinterpret_cast<const uint4*>(a.q + static_cast<int64_t>(s.begin + node) * a.q_st + h * a.q_sh + lane * 8);
            }
            uint32_t top = absmax_bits8(x);
            top = __reduce_max_sync(0xffffffffu, top);
            const int field = static_cast<int>(top >> 23);
            // the largest magnitude goes to [2^14, 2^15): elements down to 2^-28 of it stay exact
            const int up = field == 255 ? 0 : min(126, max(-126, 141 - max(field, 1)));
            const float mul = __uint_as_float((127 + up) << 23);
            float f[8];
            unpack_bf16x8(x, f);
            if (lane * 8 < DP) {
                uint32_t h[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) h[i] = pack_f16(f[2 * i] * mul, f[2 * i + 1] * mul);
                *reinterpret_cast<uint4*>(halves + r * DP + lane * 8) = make_uint4(h[0], h[1], h[2], h[3]);
            }
            if (lane == 0) row_factor[r] = a.scale * kLog2e * __uint_as_float((127 - up) << 23) * (FMT == KV_CACHE_INT8 ? 1.f : 0x1p-12f);
        }
        __syncthreads();
        uint2* const frags = reinterpret_cast<uint2*>(smem + S::FRAGS);
        constexpr int EACH = NR * L::KS * 32 / kThreads;            // (rearranged in place, by way of registers)
        uint2 moved[EACH];
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int e = threadIdx.x + i * kThreads, ln = e & 31, ks = e / 32 % L::KS, r = e / 32 / L::KS * 8 + (ln >> 2);
            const __half* from = halves + r * DP;                   // (elements of a pair lie side by side)
            moved[i] = make_uint2(*reinterpret_cast<const uint32_t*>(from + L::element(ks, ln & 3, 0, 0)), *reinterpret_cast<const uint32_t*>(from + L::element(ks, ln & 3, 1, 0)));
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < EACH; ++i) frags[threadIdx.x + i * kThreads] = moved[i];
        __syncthreads();

        // ---- the steps. Kept per row: o and its reference m_l + m_o, the sum l of the exponentials and its reference m_l. m_l is the scores'; m_l + m_o is that of score
        // + logarithm of the value's scale, so that the weights that are rounded to fp16 are of the row's own size whatever the scales. (A score meets m_l before anything else is
        // added: that difference is small and exact where the score is large.) This lane's rows: pairs
        // 2c and 2c + 1 of every eight; its elements of o: those of its g.
        float o[DP / 16][NR][4];
        uint64_t l2[NR], m_l[NR], m_o[NR], factor[NR];
#pragma unroll
        for (int i = 0; i < NR; ++i) {
#pragma unroll
            for (int j = 0; j < DP / 16; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[j][i][e] = 0.f;
            m_l[i] = m_o[i] = pack2(kNone, kNone);
            l2[i] = 0;
            factor[i] = *reinterpret_cast<const uint64_t*>(row_factor + i * 8 + 2 * c);
        }
        uint2 queries[NR == 1 ? L::KS : 1];
        if (NR == 1) {
#pragma unroll
            for (int k = 0; k < (NR == 1 ? L::KS : 1); ++k) queries[k] = frags[k * 32 + lane];
        }
        for (int step = 0; step < steps && !gave_up; ++step, ++loads) {
            const int stage = static_cast<int>(loads % STAGES);
            uint8_t* const st = ring + stage * L::CODES;
            const uint8_t* const more = rest + stage * L::REST;
            cp_async_wait<STAGES - 1>();
            if (a.box > 0 && !__all_sync(0xffffffffu, mbar_wait(bars + 8 * stage, loads / STAGES & 1, ctl, kWaitAttention, kStatusTimeout))) {
                // boxes on their way come first, then this warp is done with loads (what it leaves is undefined)
                for (int i = 0; i < min(STAGES, steps - step); ++i) mbar_drain(bars + 8 * ((loads + i) % STAGES), (loads + i) / STAGES & 1, a.limit_ns);
                gave_up = true;
                break;
            }
            __syncwarp();
            const int slot_now = slot;
            slot = find(step + STAGES + 1);
            const uint32_t seen = *reinterpret_cast<const uint32_t*>(more + L::SEEN);
            const int t0 = first_token + step * (kWarps * TOK);
            const bool masked = seen != kAllSeen || t0 + TOK > s.before;
            float* const logs = reinterpret_cast<float*>(prep + L::MULS) + TOK;                 // of the values' scales
            const float* const kf = FMT == KV_CACHE_INT8 ? reinterpret_cast<const float*>(more) : logs - TOK;
            if (FMT == KV_CACHE_INT8) {
                if (lane < TOK) logs[lane] = lg2(reinterpret_cast<const float*>(more)[TOK + lane]);
                __syncwarp();
            }
            bool poison = false;
            if (FMT == KV_CACHE_MXFP4) {
                // a token's bytes; the largest of them, t, makes 2^(t - 127) the token's factor and 2^12 * 2^(byte - t) its blocks' multipliers
                constexpr int SIDES = TOK == 32 ? 2 : 1;
#pragma unroll
                for (int i = 0; i < SIDES; ++i) {
                    const int side = TOK == 32 ? i : lane >> 4, tok = lane & (TOK - 1);
                    const uint32_t* const words = reinterpret_cast<const uint32_t*>(more) + (side * TOK + tok) * L::WORDS;
                    const int shift = 8 * *reinterpret_cast<const int*>(more + L::META + tok * 4);
                    uint32_t lo = __funnelshift_r(words[0], words[1], shift), hi = L::BLOCKS > 4 ? __funnelshift_r(words[1], words[L::WORDS / 2], shift) : 0u;
                    if (blocks < 4) lo &= (1u << (8 * blocks)) - 1;
                    if (L::BLOCKS > 4 && blocks < 8) hi &= (1u << (8 * max(blocks - 4, 0))) - 1;
                    const uint32_t nan_lo = __vcmpeq4(lo, 0xffffffffu), nan_hi = L::BLOCKS > 4 ? __vcmpeq4(hi, 0xffffffffu) : 0u;
                    uint32_t top = __vmaxu4(lo & ~nan_lo, hi & ~nan_hi);
                    top = __vmaxu4(top, top >> 16);
                    top = max(top & 0xffu, (top >> 8) & 0xffu);
                    const bool nan = (nan_lo | nan_hi) != 0;
                    poison = poison || (nan && side == 1);
                    __half* const muls = reinterpret_cast<__half*>(prep) + side * L::BLOCKS * TOK + tok;
#pragma unroll
                    for (int k = 0; k < L::BLOCKS; ++k) {
                        const int byte = ((k < 4 ? lo : hi) >> (8 * (k & 3))) & 0xff, e = 27 + byte - static_cast<int>(top);
                        const uint16_t bits = side == 1 && byte == 255 ? 0x7e00 : static_cast<uint16_t>(max(e, 0) << 10);
                        *reinterpret_cast<uint16_t*>(muls + k * TOK) = bits;
                    }
                    reinterpret_cast<float*>(prep + L::MULS)[side * TOK + tok] =
                        side == 1 ? static_cast<float>(static_cast<int>(top) - 127) : nan ? __uint_as_float(0x7fc00000u) : __uint_as_float(top == 0 ? 0x00400000u : top << 23);
                }
                poison = __any_sync(0xffffffffu, poison);
                __syncwarp();
            }
            // scores: tokens 16t + g ([0], [1]) and 16t + 8 + g ([2], [3]) for rows 2c and 2c + 1
            float sc[TT][NR][4];
#pragma unroll
            for (int t = 0; t < TT; ++t)
#pragma unroll
                for (int i = 0; i < NR; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) sc[t][i][e] = 0.f;
#pragma unroll
            for (int j = 0; j < L::KCH; ++j) {
                uint32_t w[2 * TT][L::KB / 4], mul[2 * TT];
#pragma unroll
                for (int n = 0; n < 2 * TT; ++n) {
                    const uint8_t* p = st + (j / 2) * TOK * 128 + n * 8 * L::BOX + (k_at ^ ((j & 1) << 4));
                    if constexpr (L::KB == 16) *reinterpret_cast<uint4*>(w[n]) = *reinterpret_cast<const uint4*>(p);
                    else *reinterpret_cast<uint2*>(w[n]) = *reinterpret_cast<const uint2*>(p);
                    if constexpr (FMT == KV_CACHE_MXFP4)
                        mul[n] = 0x00010001u * *reinterpret_cast<const uint16_t*>(reinterpret_cast<const __half*>(prep) + L::k_offset(j, c) * 2 / kMxBlock * TOK + n * 8 + g);
                }
#pragma unroll
                for (int x = 0; x < L::KB / 4; ++x) {
                    constexpr int PER = FMT == KV_CACHE_INT8 ? 1 : 2;           // products that a word feeds
                    uint32_t r[2 * TT][2 * PER];
#pragma unroll
                    for (int n = 0; n < 2 * TT; ++n) {
                        if constexpr (FMT == KV_CACHE_INT8) {
                            int8_to_f16(w[n][x], r[n][0], r[n][1]);
                        } else {
                            e2m1_to_f16(w[n][x], r[n]);
#pragma unroll
                            for (int y = 0; y < 4; ++y) r[n][y] = mul_f16x2(r[n][y], mul[n]);
                        }
                    }
#pragma unroll
                    for (int y = 0; y < PER; ++y) {
                        const int ks = (j * (L::KB / 4) + x) * PER + y;
#pragma unroll
                        for (int i = 0; i < NR; ++i) {
                            const uint2 q = NR == 1 ? queries[NR == 1 ? ks : 0] : frags[(i * L::KS + ks) * 32 + lane];
#pragma unroll
                            for (int t = 0; t < TT; ++t) mma_f16(sc[t][i], r[2 * t][2 * y], r[2 * t + 1][2 * y], r[2 * t][2 * y + 1], r[2 * t + 1][2 * y + 1], q.x, q.y);
                        }
                    }
                }
            }
            // softmax: this lane's tokens are 8n + g
            float kfs[2 * TT], lvs[2 * TT];
#pragma unroll
            for (int n = 0; n < 2 * TT; ++n) {
                kfs[n] = kf[8 * n + g];
                lvs[n] = logs[8 * n + g];
            }
            uint32_t p[NR][2 * TT];
            bool clean = false;                                     // NaN blocks of values are taken out of the products
#pragma unroll
            for (int i = 0; i < NR; ++i) {
                uint32_t sees[2] = {~0u, ~0u};                      // rows 2c and 2c + 1: a bit for each of the lane's tokens
                if (masked) {
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int node = min(row0 + i * 8 + 2 * c + e, s.n * a.group - 1) / a.group;
                        sees[e] = 0;
#pragma unroll
                        for (int n = 0; n < 2 * TT; ++n) {
                            const int at = 8 * n + g, j = t0 + at - s.before;
                            bool see = (seen >> at & 1u) != 0;
                            if (see && j >= 0) {
                                if (a.tree == nullptr) see = j <= node;
                                else see = (j >> 6) < a.tree_words && (a.tree[static_cast<int64_t>(s.begin + node) * a.tree_words + (j >> 6)] >> (j & 63) & 1) != 0;
                            }
                            sees[e] |= static_cast<uint32_t>(see) << n;
                        }
                    }
                    if (FMT == KV_CACHE_MXFP4 && poison) {
                        // NaN blocks of values, for the rows that see them only: put into the sums here, kept out of the product below
                        clean = true;
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            uint32_t bad = 0;
                            for (int n = 0; n < 2 * TT; ++n) {
                                if (!(sees[e] >> n & 1u)) continue;
                                const uint16_t* its = reinterpret_cast<const uint16_t*>(prep) + L::BLOCKS * TOK + 8 * n + g;
                                for (int k = 0; k < blocks; ++k) bad |= static_cast<uint32_t>(its[k * TOK] == 0x7e00) << k;
                            }
                            __syncwarp();
#pragma unroll
                            for (int x = 4; x < 32; x <<= 1) bad |= __shfl_xor_sync(0xffffffffu, bad, x);       // (the lanes that share its rows)
#pragma unroll
                            for (int j = 0; j < L::VCH; ++j)
                                if (bad >> (L::v_offset(j, g) * L::PER_BYTE / kMxBlock) & 1u)
#pragma unroll
                                    for (int x = 0; x < L::VC; ++x) o[(j * L::VC + x) / 2][i][(x & 1) * 2 + e] = __uint_as_float(0x7fc00000u);
                        }
                    }
                }
                // scores in powers of two; the largest of each row
                float top_l[2] = {kNone, kNone}, top_o[2] = {kNone, kNone};
                uint64_t score[2 * TT];
#pragma unroll
                for (int n = 0; n < 2 * TT; ++n) {
                    float x, y;
                    // (factors first: the key's alone may take a product past fp32 that the row's brings back)
                    unpack2(mul2(pack2(sc[n / 2][i][(n & 1) * 2], sc[n / 2][i][(n & 1) * 2 + 1]), mul2(pack2(kfs[n], kfs[n]), factor[i])), x, y);
                    if (masked) {
                        if (!(sees[0] >> n & 1u)) x = -INFINITY;
                        if (!(sees[1] >> n & 1u)) y = -INFINITY;
                    }
                    top_l[0] = fmaxf(top_l[0], x);
                    top_l[1] = fmaxf(top_l[1], y);
                    score[n] = pack2(x, y);
                }
                // Sums and weights may outgrow their references before these move: weights stay below 2^15 and are 2^7 at most where they moved last
                // (fp16 keeps all its bits down to 2^-21 of that)
                float ml[2], mo[2];
                unpack2(m_l[i], ml[0], ml[1]);
                unpack2(m_o[i], mo[0], mo[1]);
                if (__any_sync(0xffffffffu, top_l[0] - ml[0] > 16.f || top_l[1] - ml[1] > 16.f)) {
                    float by_l[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
#pragma unroll
                        for (int x = 4; x < 32; x <<= 1) top_l[e] = fmaxf(top_l[e], __shfl_xor_sync(0xffffffffu, top_l[e], x));
                        const float now_l = fmaxf(ml[e], top_l[e]);
                        by_l[e] = ex2(ml[e] - now_l);
                        mo[e] = fmaxf(mo[e] + (ml[e] - now_l), kNone);
                        ml[e] = now_l;
                    }
                    m_l[i] = pack2(ml[0], ml[1]);
                    m_o[i] = pack2(mo[0], mo[1]);
                    l2[i] = mul2(l2[i], pack2(by_l[0], by_l[1]));
                }
                // relative to m_l, without and with the values' scales
                const uint64_t minus_l = pack2(-ml[0], -ml[1]);
#pragma unroll
                for (int n = 0; n < 2 * TT; ++n) {
                    float x, y;
                    score[n] = add2(score[n], minus_l);
                    unpack2(score[n], x, y);
                    l2[i] = add2(l2[i], pack2(ex2(x), ex2(y)));
                    score[n] = add2(score[n], pack2(lvs[n], lvs[n]));
                    unpack2(score[n], x, y);
                    top_o[0] = fmaxf(top_o[0], x);
                    top_o[1] = fmaxf(top_o[1], y);
                }
                if (__any_sync(0xffffffffu, top_o[0] - mo[0] > 15.f || top_o[1] - mo[1] > 15.f)) {
                    float by_o[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
#pragma unroll
                        for (int x = 4; x < 32; x <<= 1) top_o[e] = fmaxf(top_o[e], __shfl_xor_sync(0xffffffffu, top_o[e], x));
                        const float now_o = fmaxf(mo[e], top_o[e] - 7.f);
                        by_o[e] = ex2(mo[e] - now_o);
                        mo[e] = now_o;
                    }
                    m_o[i] = pack2(mo[0], mo[1]);
#pragma unroll
                    for (int j = 0; j < DP / 16; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[j][i][e] *= by_o[e & 1];
                }
                const uint64_t minus_o = pack2(-mo[0], -mo[1]);
#pragma unroll
                for (int n = 0; n < 2 * TT; ++n) {
                    float x, y;
                    unpack2(add2(score[n], minus_o), x, y);
                    if (FMT == KV_CACHE_INT8 && masked) {           // (the scale of a token that is not seen may be NaN)
                        if (!(sees[0] >> n & 1u)) x = -INFINITY;
                        if (!(sees[1] >> n & 1u)) y = -INFINITY;
                    }
                    p[i][n] = transpose8(pack_f16(ex2(x), ex2(y)));
                }
            }
            // values, 16 tokens at a time
#pragma unroll
            for (int t = 0; t < TT; ++t)
#pragma unroll
                for (int j = 0; j < L::VCH; ++j) {
                    uint32_t w[4][L::VB / 4], mul[2];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint8_t* from = st + L::K_BYTES + j * TOK * 128 + (16 * t + (i >> 1) * 8) * L::BOX + v_at[i & 1];
                        if constexpr (L::VB == 16) *reinterpret_cast<uint4*>(w[i]) = *reinterpret_cast<const uint4*>(from);
                        else if constexpr (L::VB == 8) *reinterpret_cast<uint2*>(w[i]) = *reinterpret_cast<const uint2*>(from);
                        else w[i][0] = *reinterpret_cast<const uint32_t*>(from);
                    }
                    if constexpr (FMT == KV_CACHE_MXFP4) {
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            mul[i] = *reinterpret_cast<const uint32_t*>(reinterpret_cast<const __half*>(prep) + (L::BLOCKS + L::v_offset(j, g) * 2 / kMxBlock) * TOK + 16 * t + 8 * i + 2 * c);
                            if (clean) {
                                if ((mul[i] & 0xffffu) == 0x7e00u) mul[i] &= 0xffff0000u;
                                if (mul[i] >> 16 == 0x7e00u) mul[i] &= 0xffffu;
                            }
                        }
                    }
#pragma unroll
                    for (int x = 0; x < L::VB / 4; ++x) {
                        if constexpr (FMT == KV_CACHE_INT8) {
#pragma unroll
                            for (int half = 0; half < 2; ++half) {              // two elements of each token: tokens side by side
                                uint32_t a0, a1, a2, a3;
                                int8_to_f16(__byte_perm(w[0][x], w[1][x], half ? 0x7362 : 0x5140), a0, a1);
                                int8_to_f16(__byte_perm(w[2][x], w[3][x], half ? 0x7362 : 0x5140), a2, a3);
#pragma unroll
                                for (int i = 0; i < NR; ++i) mma_f16(o[(j * L::VC + x * 4) / 2 + half][i], a0, a1, a2, a3, p[i][2 * t], p[i][2 * t + 1]);
                            }
                        } else {
                            uint32_t f[4][4];
#pragma unroll
                            for (int i = 0; i < 4; ++i) e2m1_to_f16(w[i][x], f[i]);
#pragma unroll
                            for (int y = 0; y < 4; ++y) {
                                const uint32_t a0 = mul_f16x2(__byte_perm(f[0][y], f[1][y], 0x5410), mul[0]), a1 = mul_f16x2(__byte_perm(f[0][y], f[1][y], 0x7632), mul[0]);
                                const uint32_t a2 = mul_f16x2(__byte_perm(f[2][y], f[3][y], 0x5410), mul[1]), a3 = mul_f16x2(__byte_perm(f[2][y], f[3][y], 0x7632), mul[1]);
#pragma unroll
                                for (int i = 0; i < NR; ++i) mma_f16(o[(j * L::VC + x * 8) / 2 + y][i], a0, a1, a2, a3, p[i][2 * t], p[i][2 * t + 1]);
                            }
                        }
                    }
                }
            __syncwarp();                                           // every lane is done with the stage
            issue(step + STAGES, slot_now, loads + STAGES);
        }
        cp_async_wait<0>();

        // ---- the warps' results meet in shared memory
        __syncthreads();
        float* const merge = reinterpret_cast<float*>(smem);
        float* const state = reinterpret_cast<float*>(smem + S::STATE);                       // [warp][row]: references of o, of the sums, the sums
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            float sum[2], ml[2], mo[2];
            unpack2(l2[i], sum[0], sum[1]);
            unpack2(m_l[i], ml[0], ml[1]);
            unpack2(m_o[i], mo[0], mo[1]);
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int r = i * 8 + 2 * c + e;
#pragma unroll
                for (int x = 4; x < 32; x <<= 1) sum[e] += __shfl_xor_sync(0xffffffffu, sum[e], x);
                if (g == 0) {
                    state[warp * ROWS + r] = mo[e];
                    state[(kWarps + warp) * ROWS + r] = ml[e];
                    state[(2 * kWarps + warp) * ROWS + r] = sum[e];
                }
                float* to = merge + (warp * ROWS + r) * (DP + 4);
#pragma unroll
                for (int j = 0; j < L::VCH; ++j)
#pragma unroll
                    for (int x = 0; x < L::VC; x += 4) {
                        const int at = (j * L::VC + x) / 2;
                        *reinterpret_cast<float4*>(to + L::v_offset(j, g) * L::PER_BYTE + x) = make_float4(o[at][i][e], o[at][i][2 + e], o[at + 1][i][e], o[at + 1][i][2 + e]);
                    }
            }
        }
        __syncthreads();
        const bool whole = tile0 == 0 && steps == s.tiles;
        constexpr int PART = part_floats(ROWS, DP);
        float* const part = a.parts + (2 * static_cast<int64_t>(blockIdx.x) + (u_begin > item_begin ? 0 : 1)) * PART;
        const int quads = a.dim / 4;
        for (int e = threadIdx.x; e < rows * quads; e += kThreads) {
            const int r = e / quads, d = (e - r * quads) * 4;
            Row v;
#pragma unroll
            for (int w = 0; w < kWarps; ++w)
                v.add(*reinterpret_cast<const float4*>(merge + (w * ROWS + r) * (DP + 4) + d), state[w * ROWS + r], state[(kWarps + w) * ROWS + r], state[(2 * kWarps + w) * ROWS + r]);
            if (whole) {
                v.finish<FMT>(a, s, head, row0 + r, d);
            } else {
                *reinterpret_cast<float4*>(part + r * DP + d) = make_float4(v.o[0], v.o[1], v.o[2], v.o[3]);
                if (d == 0) *reinterpret_cast<float4*>(part + ROWS * DP + 4 * r) = make_float4(v.m_o, v.m_l, v.l, 0.f);
            }
        }
        const int from = owner(item_begin, share), until = owner(item_end - 1, share);
        if (!whole && last_to_arrive<ROWS>(a, s, b, head, row0, from, until, threadIdx.x, &last_one, [] { __syncthreads(); })) {
            for (int e = threadIdx.x; e < rows * quads; e += kThreads) {         // the parts, added up in the order of the tokens
                const int r = e / quads, d = (e - r * quads) * 4;
                Row v;
#pragma unroll 4
                for (int x = from; x <= until; ++x) {
                    const float* p = a.parts + (2 * static_cast<int64_t>(x) + (x == from ? 1 : 0)) * PART;
                    const float4 its = __ldcg(reinterpret_cast<const float4*>(p + ROWS * DP + 4 * r));
                    v.add(__ldcg(reinterpret_cast<const float4*>(p + r * DP + d)), its.x, its.y, its.z);
                }
                v.finish<FMT>(a, s, head, row0 + r, d);
            }
        }
        fence_proxy_async_smem();                                   // what threads have written here is overwritten by boxes
        __syncthreads();
        u += steps;
    }
    zero_rest<kThreads>(a);
}

// ------------------------------------------------------------------------------------------------ host

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

constexpr int kSmallestRows = 8;                    // rows of the smallest item: the most items, so the most counters
constexpr int kMostCtas = 4;                        // CTAs on an SM
// Rows of a sequence and head up to which the kernel of this file is chosen, which reads the cache once for 16 of them; the other's time does not depend on them. 16
// sequences of up to 6000 tokens, 8 heads of 128, trees, here and there: int8, 16 rows 55 and 86 us, 32 rows 82 and 87, 48 rows 113 and 88; 4 bits, 16 rows 58 and 79, 24 rows 80 and 79,
// 32 rows 92 and 80, 48 rows 129 and 82. (One border for both; in 4 bits it lies higher than it need.)
constexpr int kFewRows = 32;
constexpr size_t kAlign = 256;

size_t counters_bytes(int64_t seqs, int64_t total_q, int64_t q_heads, int64_t heads) {
    const int64_t group = q_heads / heads;
    return kAlign + (static_cast<size_t>(seqs + total_q * group / kSmallestRows + 1) * heads * sizeof(uint32_t) + kAlign - 1) / kAlign * kAlign;
}
int padded(int64_t dim) { return dim <= 64 ? 64 : dim <= 128 ? 128 : 256; }
// The same for every call, though most need less of it: what is left of a workspace is then what it has for counters, whatever calls it was made for, so that one with too few of
// them is refused and never finds old parts where zeros should be.
size_t parts_bytes() {
    const size_t few = static_cast<size_t>(sm_count()) * kMostCtas * 2 * part_floats(16, KV_CACHE_MAX_DIM) * sizeof(float), many = many_rows_part_bytes();
    return ((few > many ? few : many) + kAlign - 1) / kAlign * kAlign;
}
bool sizes_fine(int64_t seqs, int64_t total_q, int64_t q_heads, int64_t heads, int64_t dim) {
    return seqs >= 0 && seqs < INT32_MAX && total_q >= 0 && total_q <= INT32_MAX && heads > 0 && q_heads > 0 && q_heads <= KV_CACHE_MAX_WIDTH && q_heads % heads == 0 && dim > 0 &&
           dim <= KV_CACHE_MAX_DIM && q_heads * dim <= KV_CACHE_MAX_WIDTH && heads * dim <= KV_CACHE_MAX_WIDTH && total_q * q_heads <= INT32_MAX;
}

// Whether two sets of [tokens][heads][dim] elements share any, given where the second begins. Exact where strides are equal (slices of one buffer); where they are not,
// sets that reach into one another count as sharing.
bool overlap(int64_t tokens, int64_t heads, int64_t dim, int64_t st, int64_t sh, int64_t to, int64_t to_st, int64_t to_sh) {
    using Wide = __int128;
    if (tokens == 1) st = to_st = 0;
    if (heads == 1) sh = to_sh = 0;
    auto first = [&](int64_t t, int64_t h) { return (t < 0 ? static_cast<Wide>(tokens - 1) * t : 0) + (h < 0 ? static_cast<Wide>(heads - 1) * h : 0); };
    auto end = [&](int64_t t, int64_t h) { return (t > 0 ? static_cast<Wide>(tokens - 1) * t : 0) + (h > 0 ? static_cast<Wide>(heads - 1) * h : 0) + dim; };
    if (to + first(to_st, to_sh) >= end(st, sh) || first(st, sh) >= to + end(to_st, to_sh)) return false;
    if (st != to_st || sh != to_sh) return true;
    const Wide each = end(0, sh), apart = st > 0 ? (to % st + st) % st : 0;
    if (st > 0 && sh >= 0 && each <= apart && apart <= st - each) return false;           // tokens' heads lie side by side
    // a head of the second lies `to` + h * sh + t * st from one of the first, for some differences h and t of heads and tokens: those t count that bring it nearest
    for (int64_t h = 1 - heads; h < heads; ++h) {
        const Wide at = to + static_cast<Wide>(h) * sh;
        for (int more = -1; more <= 1; ++more) {
            Wide t = st != 0 ? -at / st + more : 0;
            t = t < 1 - tokens ? 1 - tokens : t > tokens - 1 ? tokens - 1 : t;
            const Wide gap = at + t * st;
            if (gap < dim && -gap < dim) return true;
        }
    }
    return false;
}

// Codes of a side as [slots][heads][bytes of a head], in boxes of `box` tokens of one head. Rows of a box are padded with zeros.
bool encode_codes(CUtensorMap* tm, const void* codes, int64_t slots, int64_t heads, int64_t row_bytes, int box, int box_bytes) {
    EncodeTiledFn enc = encode_tiled_fn();
    if (enc == nullptr) return false;
    const cuuint64_t dims[3] = {static_cast<cuuint64_t>(row_bytes), static_cast<cuuint64_t>(heads), static_cast<cuuint64_t>(slots)};
    const cuuint64_t strides[2] = {static_cast<cuuint64_t>(row_bytes), static_cast<cuuint64_t>(heads * row_bytes)};
    const cuuint32_t boxes[3] = {static_cast<cuuint32_t>(box_bytes), 1, static_cast<cuuint32_t>(box)}, steps[3] = {1, 1, 1};
    return enc(tm, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, const_cast<void*>(codes), dims, strides, boxes, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
               box_bytes == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : box_bytes == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_32B,
               box_bytes == 128 ? CU_TENSOR_MAP_L2_PROMOTION_L2_128B : CU_TENSOR_MAP_L2_PROMOTION_L2_64B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The maps of both sides, and a.box: tokens that lie side by side in any page, from any token that a box starts at; 0 where heads are not whole 16-byte pieces
bool encode_sides(CUtensorMap (&maps)[2], AttentionArgs& a, int fmt, int most) {
    const int per_byte = fmt == KV_CACHE_INT8 ? 1 : 2, row = padded(a.dim) / per_byte, row_bytes = a.dim / per_byte, box_bytes = row < 128 ? row : 128;
    a.box = 0;
    a.box_step = box_bytes;
    if (row_bytes % 16 != 0 || a.num_pages == 0) return true;
    a.box = most;
    while (a.page % a.box != 0) a.box /= 2;
    if (a.box * box_bytes % 128 != 0) a.box = 0;                // (a box goes to a 128-byte boundary)
    if (a.box == 0) return true;
    const int64_t slots = static_cast<int64_t>(a.num_pages) * a.page;
    return encode_codes(&maps[0], a.k_codes, slots, a.heads, row_bytes, a.box, box_bytes) && encode_codes(&maps[1], a.v_codes, slots, a.heads, row_bytes, a.box, box_bytes);
}

template <int FMT, int DP, int NR, int TT>
cudaError_t launch(const CUtensorMap (&maps)[2], const AttentionArgs& a, cudaStream_t st) {
    using S = Shared<FMT, DP, NR, TT>;
    static PerDeviceOnce once;
    static int per_sm = 1;                          // (the same on every device that the library runs on)
    constexpr int bytes = S::BYTES;
    const auto kern = kv_attention_kernel<FMT, DP, NR, TT>;
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
    return cudaLaunchKernelEx(&cfg, kern, maps[0], maps[1], a);
}
template <int FMT>
cudaError_t launch_for(const CUtensorMap (&maps)[2], const AttentionArgs& a, int64_t rows, cudaStream_t st) {
    const int dp = padded(a.dim);
    if (dp == 64) return rows <= 8 ? launch<FMT, 64, 1, 2>(maps, a, st) : launch<FMT, 64, 2, 2>(maps, a, st);
    if (dp == 128) return rows <= 8 ? launch<FMT, 128, 1, 2>(maps, a, st) : launch<FMT, 128, 2, 2>(maps, a, st);
    return rows <= 8 ? launch<FMT, 256, 1, 1>(maps, a, st) : launch<FMT, 256, 2, 1>(maps, a, st);
}

} // namespace
} // namespace w8a8

extern "C" {

using namespace w8a8;

size_t kv_cache_attention_zeroed_bytes(int64_t seqs, int64_t total_q, int64_t q_heads, int64_t heads, int64_t dim) {
    return sizes_fine(seqs, total_q, q_heads, heads, dim) ? counters_bytes(seqs, total_q, q_heads, heads) : 0;
}
size_t kv_cache_attention_workspace_bytes(int64_t seqs, int64_t total_q, int64_t q_heads, int64_t heads, int64_t dim) {
    return sizes_fine(seqs, total_q, q_heads, heads, dim) ? counters_bytes(seqs, total_q, q_heads, heads) + parts_bytes() : 0;
}

int kv_cache_attention(int fmt, const void* k_codes, const void* k_scales, const void* v_codes, const void* v_scales, int64_t num_pages, int64_t page_size,
                       int64_t heads, int64_t dim, const int32_t* table, int64_t table_stride, int64_t max_pages, const int32_t* lens, const int32_t* starts,
                       const int32_t* cu_q, int64_t seqs, const void* q, int64_t q_token_stride, int64_t q_head_stride, int64_t q_heads, int64_t total_q,
                       const int64_t* tree, int64_t tree_words, float scale, void* out, int64_t out_token_stride, int64_t out_head_stride, float* lse,
                       void* workspace, size_t workspace_bytes, void* stream) {
    const bool zero_rest = (fmt & KV_CACHE_ZERO_REST) != 0;
    fmt &= ~KV_CACHE_ZERO_REST;
    if ((fmt != KV_CACHE_INT8 && fmt != KV_CACHE_MXFP4) || !sizes_fine(seqs, total_q, q_heads, heads, dim)) return W8A8_ERR_INVALID_ARG;
    if (num_pages < 0 || page_size <= 0 || page_size > INT32_MAX || num_pages > INT32_MAX / page_size || max_pages < 0 || max_pages > (INT32_MAX - 4095) / page_size || table_stride < max_pages ||
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
    if (overlap(total_q, q_heads, dim, q_token_stride, q_head_stride, (reinterpret_cast<intptr_t>(out) - reinterpret_cast<intptr_t>(q)) / 2, out_token_stride, out_head_stride))
        return W8A8_ERR_INVALID_ARG;
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
    a.counters = reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(workspace) + kAlign);          // behind the status word
    // parts at the end of what is given, so that a call with fewer sequences leaves alone what must be zero for one with more
    a.parts = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + workspace_bytes / kAlign * kAlign - parts_bytes());
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
    a.page_shift = (page_size & (page_size - 1)) == 0 ? 0 : -1;
    while (a.page_shift >= 0 && (int64_t{1} << a.page_shift) < page_size) ++a.page_shift;
    a.scale = scale;
    a.status = static_cast<int*>(workspace);
    a.sticky = sticky_status_word();
    a.limit_ns = wait_limit_ns();
    a.zero_rest = zero_rest ? 1 : 0;
    a.starve = starve_mode() == kStarveGemm ? 1 : 0;
    const int64_t rows = (total_q * a.group + seqs - 1) / (seqs > 0 ? seqs : 1);       // of a sequence and head, on average
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    CUtensorMap maps[2] = {};
    const bool many = rows > kFewRows && many_rows_fits(a.dim);
    if (!encode_sides(maps, a, fmt, many ? kMostBox : padded(a.dim) == 256 ? 16 : 32)) return W8A8_ERR_CUDA;      // (few rows: a step's tokens)
    const cudaError_t e = many                     ? launch_many_rows(fmt, maps[0], maps[1], a, rows, st)
                          : fmt == KV_CACHE_INT8 ? launch_for<KV_CACHE_INT8>(maps, a, rows, st)
                                                 : launch_for<KV_CACHE_MXFP4>(maps, a, rows, st);
    return e == cudaSuccess ? W8A8_OK : W8A8_ERR_CUDA;
}

} // extern "C"
