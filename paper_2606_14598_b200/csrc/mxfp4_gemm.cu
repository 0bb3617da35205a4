// Tensor-core MXFP4 GEMM with bias, for sm_100a.
//
//   out[m,n] = bf16(sum_b 2^(ea + ew) * sum_{k in b} qa[m,k] * qw[n,k] + bias[n])
//              tcgen05.mma.kind::mxf4.block_scale (E2M1 x E2M1, one E8M0 scale for 32 elements along K), fp32 in TMEM
//
// One persistent CTA per SM; with CG = 2 the CTAs of a pair share a tile of 256 x BN (each loads its 128 rows of A and half
// of the W tile, the leader issues one MMA for both). Operand bytes per instruction and their layout are those of the int8
// GEMM (128 bytes of a row are 256 elements here), so a k-block takes the tensor pipe as long as an int8 one and carries
// twice the arithmetic; on top of it come the scales: 1 KB for 128 rows and 256 elements, copied from shared into tensor
// memory (tcgen05.cp) in front of the MMAs that read them.
//
// Tensor memory: 512 columns hold two accumulators of BN columns and the scales of four k-blocks (for each half of a k-block 4
// columns for A and 4 for every 128 columns of the tile). Two accumulators of 256 columns would leave no room for scales, so at
// BN = 256 they overlap by 128 columns ([0,256) and [128,384)): the epilogue takes the shared columns into registers first and
// hands them on, and the next tile's MMAs run under the rest of the epilogue.
//
// Warp roles: 0 TMA producer, 1 MMA issuer (and TMEM allocation), 2-5 epilogue (tcgen05.ld 32x32b, thread = row; bias; bf16;
// swizzled staging; TMA store of 32 x 32 boxes, which clips ragged edges), 6 copies scales into tensor memory, 7 loads them.
//
// What bounds it: the tensor queue and the way operands take to it, not HBM (the operands of a 4110 x 4608 -> 13824 product come
// out of L2). There 121-125 us = 4.2-4.3 PFLOP/s in a short run, 0.64-0.66 of four times the measured bf16 rate (8192 cubed 213-217 us,
// 5.1 PFLOP/s, 0.77); over seconds the power limit takes the SM clock to 1.65 GHz and it is 138 us. With parts left out: MMAs alone
// 86 us (162 cycles an MMA of 256 x 256 x 64 where 128 would be the pipe's), with scale copies 94 (a copy or commit holds the queue
// 35-45 cycles; in the MMA thread they made it 159), with operand loads 110, with the hand-over of the shared columns 120 (0.5 us
// a tile from the accumulator's completion to the peer's answer). Tried without gain: bands in the
// tile order, L2 hints, one commit for both CTAs, stages of one k-block (258 against 217 us on 8192 cubed), stores straight from registers.
//
// Every wait is bounded as in the int8 GEMM: on expiry the status word is set, all roles unwind, TMEM is freed.
#include "../../include/mxfp4_linear.h"
#include "internal.h"
#include "mxfp4_math.cuh"
#include "ptx.cuh"
#include "tensor_map.h"

namespace w8a8 {
namespace {

constexpr int BM = 128;             // rows of A per CTA (= TMEM lanes)
constexpr int BKB = 128;            // bytes of K per k-block: one 128-byte swizzle row
constexpr int BK = 2 * BKB;         // elements of K per k-block
constexpr int MMA_K = 64;           // elements of K per instruction
constexpr int EPI_THREADS = 128;
constexpr int SCALE_WARP = 6, SCALE_LOAD_WARP = 7;
constexpr int NUM_THREADS = 64 + EPI_THREADS + 64;
constexpr int SCALE_STAGES = 3;                        // stages of the scales' own ring, where they have one
constexpr int SMEM_MAX = 232448;
constexpr int SF_TILE_BYTES = 2 * kScaleTileBytes;     // 128 rows of scales for one k-block
constexpr int SF_BUFS = 4;                             // k-blocks whose scales tensor memory holds

enum Where { W_PRODUCER_EMPTY = 1, W_MMA_FULL = 2, W_MMA_TMEM_EMPTY = 3, W_EPI_TMEM_FULL = 4, W_SCALES = 5 };

template <int CG, int BN, int STAGES, int KBS>
struct Layout {
    static constexpr int A_BYTES = BM * BKB;
    static constexpr int B_ROWS = BN / CG;
    static constexpr int B_BYTES = B_ROWS * BKB;
    static constexpr int SFB_TILES = (BN + 127) / 128;
    static constexpr int SF_KB_BYTES = (1 + SFB_TILES) * SF_TILE_BYTES;       // scales of one k-block: A, then W
    // Scales in a ring of their own, fetched and copied ahead of the operands (see the scale warp), or in the operands' stages.
    static constexpr bool OWN_RING = BN < 256;
    static constexpr int KB_BYTES = A_BYTES + B_BYTES + (OWN_RING ? 0 : SF_KB_BYTES);       // one k-block of a stage
    static constexpr int STAGE_BYTES = KBS * KB_BYTES;
    static constexpr int SF_STAGE_BYTES = KBS * SF_KB_BYTES;
    static constexpr int OFF_SF = STAGES * STAGE_BYTES;
    static constexpr int BOX_BYTES = 32 * 64;                   // one 32-row x 32-column bf16 box
    static constexpr int BOXES = 2;                             // boxes that alternate per epilogue warp
    static constexpr int OFF_STAGING = OFF_SF + (OWN_RING ? SCALE_STAGES * SF_STAGE_BYTES : 0);
    static constexpr int OFF_BARS = OFF_STAGING + 4 * BOXES * BOX_BYTES;
    static constexpr int NUM_FULL = STAGES * KBS;               // a barrier per k-block
    static constexpr int NUM_SCALE_BARS = OWN_RING ? 2 * SCALE_STAGES : SF_BUFS;
    static constexpr int NUM_BARS = NUM_FULL + STAGES + 2 + 2 + NUM_SCALE_BARS;     // full, empty, tfull[2], tempty[2], scales
    static constexpr int OFF_TMEM = OFF_BARS + NUM_BARS * 8;
    static constexpr int OFF_ABORT = OFF_TMEM + 4;
    static constexpr int USED = OFF_ABORT + 4;
    static constexpr int DYN_BYTES = USED + 1024 <= SMEM_MAX ? USED + 1024 : SMEM_MAX;
    // tensor memory: two accumulators (overlapping by SHARED columns), then the scales: per half of a k-block 4 columns of A
    // and 4 for each 128 columns of W
    static constexpr int SF_HALF = 4 + 4 * SFB_TILES;
    static constexpr int SF_COLS = SF_BUFS * 2 * SF_HALF;
    static constexpr int SHARED = 2 * BN + SF_COLS <= 512 ? 0 : 128;
    static constexpr int SLOT1 = BN - SHARED;                   // first column of the second accumulator
    static constexpr int SF_COL = SLOT1 + BN;
    static constexpr int TMEM_COLS = SF_COL + SF_COLS <= 256 ? 256 : 512;
    static_assert(SF_COL + SF_COLS <= 512, "accumulators and scales fit tensor memory");
    static_assert(USED <= SMEM_MAX, "shared memory budget");
    static_assert(B_BYTES % 1024 == 0 && KB_BYTES % 1024 == 0, "operand tiles start on a swizzle-atom boundary");
};

struct RunCtl {
    int* status;
    int* sticky;
    uint64_t wait_limit_ns;
    int after_quantizer;
    int starve;
};

__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
    __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t*>(&v);
}

template <int CG, int BN, int STAGES, int KBS>
__global__ void __launch_bounds__(NUM_THREADS, 1)
mx_gemm_kernel(const __grid_constant__ CUtensorMap tm_a, const __grid_constant__ CUtensorMap tm_b, const __grid_constant__ CUtensorMap tm_sa,
               const __grid_constant__ CUtensorMap tm_sb, const __grid_constant__ CUtensorMap tm_out, const float* bias, int M, int N, int K,
               const RunCtl rc) {
    using L = Layout<CG, BN, STAGES, KBS>;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* base_ptr = smem_raw + (base - smem_u32(smem_raw));
    // (dynamic shared memory starts on a 1024-byte boundary when a kernel has no static one; the largest layout has no slack)
    if (base + L::USED > smem_u32(smem_raw) + L::DYN_BYTES) {
        grid_dep_wait();
        if (threadIdx.x == 0) atomicCAS(rc.status, 0, W8A8_ERR_CUDA);
        return;
    }
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = CG == 2 ? cluster_ctarank() : 0u;
    const bool leader = rank == 0;
    const uint32_t bars = base + L::OFF_BARS;
    auto full_bar = [&](int s, int sub) { return bars + 8u * (s * KBS + sub); };                        // used in the leader
    auto empty_bar = [&](int s) { return bars + 8u * (L::NUM_FULL + s); };                              // one per CTA
    auto tfull_bar = [&](int b) { return bars + 8u * (L::NUM_FULL + STAGES + b); };                     // one per CTA
    auto tempty_bar = [&](int b) { return bars + 8u * (L::NUM_FULL + STAGES + 2 + b); };                // used in the leader
    // scales in tensor memory: one barrier a buffer, used in the leader; with a ring of their own one a stage and CTA
    auto scale_bar = [&](int b) { return bars + 8u * (L::NUM_FULL + STAGES + 4 + b); };
    auto sfull_bar = [&](int s) { return bars + 8u * (L::NUM_FULL + STAGES + 4 + SCALE_STAGES + s); };  // (ring) scales landed: used in the leader
    volatile uint32_t* tmem_holder = reinterpret_cast<volatile uint32_t*>(base_ptr + L::OFF_TMEM);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(base_ptr + L::OFF_ABORT);
    const WaitCtl ctl{abort_flag, rc.status, rc.sticky, rc.wait_limit_ns};

    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) {
            for (int sub = 0; sub < KBS; ++sub) mbar_init(full_bar(s, sub), 1);
            mbar_init(empty_bar(s), 1);
        }
        for (int b = 0; b < L::NUM_SCALE_BARS; ++b) mbar_init(scale_bar(b), 1);
        for (int b = 0; b < 2; ++b) { mbar_init(tfull_bar(b), 1); mbar_init(tempty_bar(b), 4 * CG); }
        *abort_flag = 0;
        fence_mbar_init();
        prefetch_tensormap(&tm_a);
        prefetch_tensormap(&tm_b);
        prefetch_tensormap(&tm_sa);
        prefetch_tensormap(&tm_sb);
        prefetch_tensormap(&tm_out);
    }
    // Tensor memory of a pair. A barrier of the cluster before the allocation: it concerns both CTAs, and only the barrier says that the peer
    // has begun (without it a pair whose peer started late, beside CTAs of a kernel ahead, waited in its allocation for good). One after
    // it, before the permit, which is the pair's too, goes back.
    if (CG == 2) {
        __syncwarp();
        cluster_sync_all();
    }
    if (warp == 1) {
        if (CG == 2) tmem_alloc_pair(base + L::OFF_TMEM, L::TMEM_COLS);
        else tmem_alloc(base + L::OFF_TMEM, L::TMEM_COLS);
    }
    tc_fence_before();
    __syncthreads();
    if (CG == 2) cluster_sync_all();
    tc_fence_after();
    if (warp == 1) { if (CG == 2) tmem_relinquish_pair(); else tmem_relinquish(); }
    const uint32_t tmem_base = *tmem_holder;
    // Only now: a kernel behind this one that allocates tensor memory and then waits for this one must not get there first.
    grid_dep_launch_dependents();

    constexpr int TILE_M = BM * CG;
    const int num_nb = (N + BN - 1) / BN;
    const int num_tiles = (M + TILE_M - 1) / TILE_M * num_nb;
    const int num_kb = (K + BK - 1) / BK;
    const int num_ks = (num_kb + KBS - 1) / KBS;                // stages a tile takes
    const int ktiles = (K + kScaleTileBlocks * kMxBlock - 1) / (kScaleTileBlocks * kMxBlock);
    const int first_tile = blockIdx.x / CG, tile_step = gridDim.x / CG;

    if (warp == 0) {
        // ------------------------------------------------------------ TMA producer (both CTAs of a pair)
        if (lane == 0) {
            int stage = 0, issued = 0;
            uint32_t phase = 0;
            bool ok = true, withhold = rc.starve != 0;
            const uint64_t keep = l2_policy_evict_last();
            auto load = [&](const CUtensorMap* tm, uint32_t dst, uint32_t bar, int x, int y) {
                if (CG == 2) tma_load_2d_pair_hint(dst, tm, bar, x, y, keep);
                else tma_load_2d_hint(dst, tm, bar, x, y, keep);
            };
            // The loads of stage ks of a tile into ring slot st. A stage always receives all its k-blocks: what lies past the end
            // of K arrives as zeros and is not used.
            auto load_stage = [&](int t, int ks, int st) {
                const int m0 = (t / num_nb) * TILE_M + rank * BM, n0 = (t % num_nb) * BN;
#pragma unroll
                for (int sub = 0; sub < KBS; ++sub) {
                    const int kb = ks * KBS + sub;
                    const uint32_t s = base + st * L::STAGE_BYTES + sub * L::KB_BYTES;
                    const uint32_t bar = CG == 2 ? mapa_shared(full_bar(st, sub), 0) : full_bar(st, sub);
                    if (leader) mbar_arrive_expect_tx(full_bar(st, sub), CG * L::KB_BYTES);
                    load(&tm_b, s + L::A_BYTES, bar, kb * BKB, n0 + rank * L::B_ROWS);
                    load(&tm_a, s, bar, kb * BKB, m0);
                    if (!L::OWN_RING) {
#pragma unroll
                        for (int i = 0; i < L::SFB_TILES; ++i)
                            load(&tm_sb, s + L::A_BYTES + L::B_BYTES + (1 + i) * SF_TILE_BYTES, bar, 0, (n0 / kScaleTileRows + i) * ktiles + 2 * kb);
                        load(&tm_sa, s + L::A_BYTES + L::B_BYTES, bar, 0, m0 / kScaleTileRows * ktiles + 2 * kb);
                    }
                }
            };
            // The weights of the first ring of stages are on their way to L2 while the kernel ahead finishes. They are read after
            // it is complete, like everything else: it may be the one that writes them.
            if (first_tile < num_tiles) {
                const int n0 = (first_tile % num_nb) * BN;
                for (int kb = 0; kb < min(STAGES * KBS, num_kb); ++kb) {
                    tma_prefetch_2d_hint(&tm_b, kb * BKB, n0 + rank * L::B_ROWS, keep);
#pragma unroll
                    for (int i = 0; i < L::SFB_TILES; ++i) tma_prefetch_2d_hint(&tm_sb, 0, (n0 / kScaleTileRows + i) * ktiles + 2 * kb, keep);
                }
            }
            grid_dep_wait();
            if (!rc.after_quantizer && blockIdx.x == 0) *rc.status = 0;
            for (int t = first_tile; t < num_tiles && ok; t += tile_step) {
                for (int ks = 0; ks < num_ks; ++ks) {
                    if (!mbar_wait(empty_bar(stage), phase ^ 1u, ctl, W_PRODUCER_EMPTY, kStatusTimeout)) { ok = false; break; }
                    if (withhold) {
                        withhold = false;      // test hook: this stage never arrives; the bounded waits run out
                    } else {
                        load_stage(t, ks, stage);
                        ++issued;
                    }
                    if (++stage == STAGES) { stage = 0; phase ^= 1u; }
                }
            }
            if (!ok && leader) {
                // let copies that are still in flight land before the CTA goes away
                int s = stage;
                uint32_t ph = phase;
                for (int i = 0; i < STAGES && i < issued; ++i) {
                    if (s == 0) { s = STAGES; ph ^= 1u; }
                    --s;
                    for (int sub = 0; sub < KBS; ++sub) {
                        const uint64_t t0 = globaltimer_ns();
                        while (!mbar_try_wait(full_bar(s, sub), ph) && globaltimer_ns() - t0 < 10000000ull) {}
                    }
                }
            }
        }
        __syncwarp();
    } else if (warp == SCALE_LOAD_WARP) {
        // ------------------------------------------------------------ TMA producer of the scales (both CTAs of a pair)
        // A ring of its own: its stages come free as soon as they have been copied to tensor memory, so scales are fetched and
        // copied well ahead of the operands that they go with.
        if (L::OWN_RING && lane == 0) {
            const uint64_t keep = l2_policy_evict_last();
            grid_dep_wait();                                   // the activations' scales come from the kernel ahead
            int st = 0, issued = 0;
            uint32_t phase = 0;
            bool ok = true;
            for (int t = first_tile; t < num_tiles && ok; t += tile_step) {
                const int mt = ((t / num_nb) * TILE_M + static_cast<int>(rank) * BM) / kScaleTileRows, nt = (t % num_nb) * BN / kScaleTileRows;
                for (int ks = 0; ks < num_ks; ++ks) {
                    if (issued >= SCALE_STAGES && !mbar_wait(scale_bar(st), phase ^ 1u, ctl, W_PRODUCER_EMPTY, kStatusTimeout)) { ok = false; break; }
                    const uint32_t bar = CG == 2 ? mapa_shared(sfull_bar(st), 0) : sfull_bar(st);
                    if (leader) mbar_arrive_expect_tx(sfull_bar(st), CG * L::SF_STAGE_BYTES);
#pragma unroll
                    for (int sub = 0; sub < KBS; ++sub) {
                        const uint32_t dst = base + L::OFF_SF + st * L::SF_STAGE_BYTES + sub * L::SF_KB_BYTES;
                        const int x = 2 * (ks * KBS + sub);
#pragma unroll
                        for (int i = 0; i <= L::SFB_TILES; ++i) {
                            const CUtensorMap* tm = i == 0 ? &tm_sa : &tm_sb;
                            const int y = (i == 0 ? mt : nt + i - 1) * ktiles + x;
                            if (CG == 2) tma_load_2d_pair_hint(dst + i * SF_TILE_BYTES, tm, bar, 0, y, keep);
                            else tma_load_2d_hint(dst + i * SF_TILE_BYTES, tm, bar, 0, y, keep);
                        }
                    }
                    ++issued;
                    if (++st == SCALE_STAGES) { st = 0; phase ^= 1u; }
                }
            }
            if (!ok && leader) {
                for (int i = 0; i < SCALE_STAGES && i < issued; ++i) {      // let copies in flight land
                    if (st == 0) { st = SCALE_STAGES; phase ^= 1u; }
                    --st;
                    const uint64_t t0 = globaltimer_ns();
                    while (!mbar_try_wait(sfull_bar(st), phase) && globaltimer_ns() - t0 < 10000000ull) {}
                }
            }
        }
        __syncwarp();
    } else if (warp == SCALE_WARP) {
        // ------------------------------------------------------------ scales: shared -> tensor memory (leader CTA only)
        // A thread of its own: in front of the MMAs, in their thread, every copy would hold the tensor pipe up. Tensor memory
        // holds the scales of two stages. With a ring of their own the scales of a stage are copied before its operands have landed
        // (4110 x 4608 -> 13824 at 256 x 192 118 against 132 us, 512 x 12288 -> 4608 at 128 x 128 18.8 against 20.8 us); the
        // 256 x 256 tile, whose copies take a third longer, does better with copies and hand-over k-block by k-block (111 against
        // 124 us on 4110 x 12288 -> 4608).
        if (L::OWN_RING) {
            if (lane == 0 && leader) {
                int st = 0, n = 0;                                 // n: stages so far; buffers of stage n: n % BACK
                uint32_t phase = 0;
                bool ok = true;
                constexpr int BACK = SF_BUFS / KBS;                // stages whose scales tensor memory holds
                for (int t = first_tile; t < num_tiles && ok; t += tile_step) {
                    for (int ks = 0; ks < num_ks; ++ks, ++n) {
                        if (!mbar_wait(sfull_bar(st), phase, ctl, W_SCALES, kStatusTimeout)) { ok = false; break; }
                        // the MMAs that used these buffers are done
                        if (n >= BACK && !mbar_wait(empty_bar((n - BACK) % STAGES), ((n - BACK) / STAGES) & 1, ctl, W_SCALES, kStatusTimeout)) { ok = false; break; }
                        tc_fence_after();
#pragma unroll
                        for (int sub = 0; sub < KBS; ++sub) {
                            const uint32_t s = base + L::OFF_SF + st * L::SF_STAGE_BYTES + sub * L::SF_KB_BYTES;
                            const uint32_t sf = tmem_base + L::SF_COL + (n % BACK * KBS + sub) * 2 * L::SF_HALF;
#pragma unroll
                            for (int h = 0; h < 2; ++h)            // halves of 128 elements: one scale tile each
#pragma unroll
                                for (int q = 0; q <= L::SFB_TILES; ++q)
                                    tc_cp_scales<CG>(sf + h * L::SF_HALF + 4 * q, make_scale_desc(s + q * SF_TILE_BYTES + h * kScaleTileBytes));
                        }
                        if (CG == 2) { tc_commit_pair(scale_bar(st)); tc_commit_pair(mapa_shared(scale_bar(st), 1)); }
                        else tc_commit(scale_bar(st));
                        if (++st == SCALE_STAGES) { st = 0; phase ^= 1u; }
                    }
                }
            }
        } else if (lane == 0 && leader) {
            int stage = 0, i = 0;                              // i: k-blocks so far, buffer i % SF_BUFS
            uint32_t phase = 0;
            bool ok = true;
            constexpr int BACK = SF_BUFS / KBS;                // stages back whose MMAs must be done with the buffer
            int s_done = 0;                                    // stages whose completion has been waited for
            for (int t = first_tile; t < num_tiles && ok; t += tile_step) {
                for (int ks = 0; ks < num_ks && ok; ++ks) {
                    const int now = i / KBS;                   // running stage number
                    if (now >= BACK) {
                        s_done = now - BACK;
                        if (!mbar_wait(empty_bar(s_done % STAGES), (s_done / STAGES) & 1, ctl, W_SCALES, kStatusTimeout)) { ok = false; break; }
                    }
#pragma unroll
                    for (int sub = 0; sub < KBS; ++sub, ++i) {
                        if (!mbar_wait(full_bar(stage, sub), phase, ctl, W_SCALES, kStatusTimeout)) { ok = false; break; }
                        tc_fence_after();
                        const uint32_t s = base + stage * L::STAGE_BYTES + sub * L::KB_BYTES + L::A_BYTES + L::B_BYTES;
                        const uint32_t sf = tmem_base + L::SF_COL + (i % SF_BUFS) * 2 * L::SF_HALF;
#pragma unroll
                        for (int h = 0; h < 2; ++h) {          // halves of 128 elements: one scale tile each
                            tc_cp_scales<CG>(sf + h * L::SF_HALF, make_scale_desc(s + h * kScaleTileBytes));
#pragma unroll
                            for (int q = 0; q < L::SFB_TILES; ++q)
                                tc_cp_scales<CG>(sf + h * L::SF_HALF + 4 + 4 * q,
                                                 make_scale_desc(s + (1 + q) * SF_TILE_BYTES + h * kScaleTileBytes));
                        }
                        if (CG == 2) tc_commit_pair(scale_bar(i % SF_BUFS));
                        else tc_commit(scale_bar(i % SF_BUFS));
                    }
                    if (++stage == STAGES) { stage = 0; phase ^= 1u; }
                }
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        // ------------------------------------------------------------ MMA issuer (leader CTA only)
        if (lane == 0 && leader) {
            constexpr uint32_t idesc_lo = make_mxf4_idesc(TILE_M, BN, 0), idesc_hi = make_mxf4_idesc(TILE_M, BN, 2);
            int stage = 0, c = 0, n = 0;                      // n: stages so far
            uint32_t phase = 0;
            bool ok = true;
            for (int t = first_tile; t < num_tiles && ok; t += tile_step, ++c) {
                if (L::SHARED > 0) {
                    // the columns shared with the previous tile have been read (and with them all of the tile before that)
                    if (c > 0 && !mbar_wait(tempty_bar((c - 1) & 1), ((c - 1) >> 1) & 1, ctl, W_MMA_TMEM_EMPTY, kStatusTimeout)) break;
                } else {
                    if (c > 1 && !mbar_wait(tempty_bar(c & 1), ((c >> 1) & 1) ^ 1u, ctl, W_MMA_TMEM_EMPTY, kStatusTimeout)) break;
                }
                tc_fence_after();
                const uint32_t d = tmem_base + (c & 1) * L::SLOT1;
                // the tile's first column within its first scale tile, in tensor-memory columns of 32 rows
                const uint32_t sfb_shift = ((t % num_nb) * BN % kScaleTileRows) / 32;
                for (int ks = 0; ks < num_ks && ok; ++ks, ++n) {
                    if (L::OWN_RING && !mbar_wait(scale_bar(n % SCALE_STAGES), (n / SCALE_STAGES) & 1, ctl, W_MMA_FULL, kStatusTimeout)) { ok = false; break; }
#pragma unroll
                    for (int sub = 0; sub < KBS; ++sub) {
                        const int buf = n % (SF_BUFS / KBS) * KBS + sub;           // of the k-block's scales
                        if (!mbar_wait(full_bar(stage, sub), phase, ctl, W_MMA_FULL, kStatusTimeout) ||
                            (!L::OWN_RING && !mbar_wait(scale_bar(buf), (n / (SF_BUFS / KBS)) & 1, ctl, W_MMA_FULL, kStatusTimeout))) { ok = false; break; }
                        tc_fence_after();
                        const int kb = ks * KBS + sub;
                        const uint32_t s = base + stage * L::STAGE_BYTES + sub * L::KB_BYTES;
                        const uint64_t da = make_kmajor_sw128_desc(s), db = make_kmajor_sw128_desc(s + L::A_BYTES);
                        const uint32_t sf = tmem_base + L::SF_COL + buf * 2 * L::SF_HALF;
                        const int left = K - kb * BK;                      // elements of K this k-block holds (none past the end)
#pragma unroll
                        for (int k = 0; k < BK / MMA_K; ++k) {             // 64 elements = 32 bytes: +2 in 16-byte units
                            const uint32_t sfa = sf + (k >> 1) * L::SF_HALF;
                            if (k * MMA_K < left)
                                mma_mxf4_ss<CG>(d, da + 2 * k, db + 2 * k, (k & 1) ? idesc_hi : idesc_lo, sfa, sfa + 4 + sfb_shift, (kb | k) ? 1u : 0u);
                        }
                    }
                    if (!ok) break;
                    // the stage (and its scales' buffers) are free once these MMAs have read them
                    if (CG == 2) { tc_commit_pair(empty_bar(stage)); tc_commit_pair(mapa_shared(empty_bar(stage), 1)); }
                    else tc_commit(empty_bar(stage));
                    if (++stage == STAGES) { stage = 0; phase ^= 1u; }
                }
                if (!ok) break;
                if (CG == 2) { tc_commit_pair(tfull_bar(c & 1)); tc_commit_pair(mapa_shared(tfull_bar(c & 1), 1)); }
                else tc_commit(tfull_bar(c & 1));
            }
        }
        __syncwarp();
    } else {
        // ------------------------------------------------------------ epilogue
        const int lg = warp & 3;                       // TMEM lane group this warp may read
        const int stg_off = L::OFF_STAGING + (warp - 2) * L::BOXES * L::BOX_BYTES;
        const uint64_t stream_out = l2_policy_evict_first();
        constexpr int CHUNKS = BN / 32;                // 32 accumulator columns of this thread's row
        constexpr int GROUP = L::SHARED > 0 ? L::SHARED / 32 : 2;      // chunks loaded together
        static_assert(CHUNKS % GROUP == 0, "whole groups");
        grid_dep_wait();
        int c = 0;
        bool ok = true;
        for (int t = first_tile; t < num_tiles; t += tile_step, ++c) {
            const int slot = c & 1;
            const int m0 = (t / num_nb) * TILE_M + rank * BM, n0 = (t % num_nb) * BN;
            if (ok && !mbar_wait(tfull_bar(slot), (c >> 1) & 1, ctl, W_EPI_TMEM_FULL, kStatusTimeout)) ok = false;
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            tc_fence_after();
            const uint32_t t_row = tmem_base + (static_cast<uint32_t>(lg * 32) << 16) + slot * L::SLOT1;
            // the group that holds the columns shared with the next tile comes first
            const bool down = L::SHARED > 0 && slot == 0;
#pragma unroll 1
            for (int g = 0; g < CHUNKS / GROUP; ++g) {
                const int g0 = (down ? CHUNKS / GROUP - 1 - g : g) * GROUP;
                uint32_t v[GROUP][32];
#pragma unroll
                for (int j = 0; j < GROUP; ++j) tmem_ld_32x32b_x32(t_row + (g0 + j) * 32, v[j]);
                tmem_wait_ld();
                if (g == (L::SHARED > 0 ? 0 : CHUNKS / GROUP - 1)) {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) {
                        if (!leader) mbar_arrive_cluster(mapa_shared(tempty_bar(slot), 0));
                        else mbar_arrive(tempty_bar(slot));
                    }
                }
#pragma unroll
                for (int j = 0; j < GROUP; ++j) {
                    const int n = n0 + (g0 + j) * 32;
                    const int off = stg_off + (j & (L::BOXES - 1)) * L::BOX_BYTES;
                    if (lane == 0) bulk_wait_group_read<L::BOXES - 1>();       // the store that used this box has read it
                    __syncwarp();
#pragma unroll
                    for (int q = 0; q < 4; ++q) {                              // 8 columns = 16 bytes at a time
                        float f[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) f[e] = __uint_as_float(v[j][8 * q + e]);
                        if (bias != nullptr && n + 8 * q < N) {
                            const float4 b0 = __ldcg(reinterpret_cast<const float4*>(bias + n + 8 * q));
                            const float4 b1 = __ldcg(reinterpret_cast<const float4*>(bias + n + 8 * q) + 1);
                            f[0] += b0.x; f[1] += b0.y; f[2] += b0.z; f[3] += b0.w;
                            f[4] += b1.x; f[5] += b1.y; f[6] += b1.z; f[7] += b1.w;
                        }
                        *reinterpret_cast<uint4*>(base_ptr + off + lane * 64 + ((q ^ ((lane >> 1) & 3)) << 4)) =
                            make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
                    }
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) {
                        tma_store_2d_hint(&tm_out, base + off, n, m0 + lg * 32, stream_out);
                        bulk_commit_group();
                    }
                    __syncwarp();                              // (what follows may be a warp-wide load of tensor memory)
                }
            }
        }
        if (lane == 0) bulk_wait_group<0>();
    }

    tc_fence_before();
    __syncthreads();
    if (CG == 2) cluster_sync_all();            // nobody leaves while the peer may still signal its barriers
    tc_fence_after();
    if (warp == 1) {
        if (CG == 2) tmem_dealloc_pair(tmem_base, L::TMEM_COLS);
        else tmem_dealloc(tmem_base, L::TMEM_COLS);
    }
    if (CG == 2) {
        __syncwarp();
        cluster_sync_all();                     // neither is gone while the other frees its half
    }
}

// ---------------------------------------------------------------------------- host side

template <int CG, int BN, int STAGES, int KBS>
int launch_cfg(const MxLinearArgs& a, cudaStream_t st) {
    using L = Layout<CG, BN, STAGES, KBS>;
    auto kern = mx_gemm_kernel<CG, BN, STAGES, KBS>;
    static PerDeviceOnce smem_opt_in;
    if (smem_opt_in.run([&] { return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, L::DYN_BYTES); }) != cudaSuccess)
        return W8A8_ERR_CUDA;
    CUtensorMap tm_a, tm_b, tm_sa, tm_sb, tm_out;
    if (!encode_mx_codes(&tm_a, a.qa, a.M, a.K, a.ldqa, BM) || !encode_mx_codes(&tm_b, a.qw, a.N, a.K, a.K / 2, L::B_ROWS) ||
        !encode_mx_scales(&tm_sa, a.sa, a.M, a.K) || !encode_mx_scales(&tm_sb, a.sw, a.N, a.K) ||
        !encode_map_2d(&tm_out, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, a.out, a.M, a.N, a.ldo * 2, 32, 32, CU_TENSOR_MAP_SWIZZLE_64B))
        return W8A8_ERR_CUDA;
    const int64_t tiles = static_cast<int64_t>((a.M + BM * CG - 1) / (BM * CG)) * ((a.N + BN - 1) / BN);
    if (tiles > INT32_MAX / 2) return W8A8_ERR_INVALID_ARG;
    const int64_t most = sm_count() / CG;
    const int64_t waves = (tiles + most - 1) / most;
    // the fewest groups that need no more waves than all of them would: every group gets the same number of tiles
    const int groups = static_cast<int>(waves >= 3 ? (tiles + waves - 1) / waves : (tiles < most ? tiles : most));
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(CG * groups);
    cfg.blockDim = dim3(NUM_THREADS);
    cfg.dynamicSmemBytes = L::DYN_BYTES;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    int na = 0;
    if (CG == 2) {
        attr[na].id = cudaLaunchAttributeClusterDimension;
        attr[na].val.clusterDim.x = 2;
        attr[na].val.clusterDim.y = 1;
        attr[na].val.clusterDim.z = 1;
        ++na;
    }
    attr[na].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[na].val.programmaticStreamSerializationAllowed = 1;
    ++na;
    cfg.attrs = attr;
    cfg.numAttrs = na;
    RunCtl rc{};
    rc.status = a.status;
    rc.sticky = sticky_status_word();
    rc.wait_limit_ns = wait_limit_ns();
    rc.after_quantizer = a.after_quantizer ? 1 : 0;
    rc.starve = starve_mode() == kStarveGemm ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kern, tm_a, tm_b, tm_sa, tm_sb, tm_out, a.bias, a.M, a.N, a.K, rc) == cudaSuccess ? W8A8_OK : W8A8_ERR_CUDA;
}

} // namespace

// The configuration with the lowest estimated time. Fitted on 20 shapes from (128, 256, 256) to (8192, 8192, 8192): launch,
// fill and last epilogue, then for every wave of tiles its k-blocks and what the hand-over between tiles leaves exposed
// (microseconds). Measured on codes, 256 x 256 pairs / 256 x 192 pairs / 128 x 128: 8192 cubed 213 / 231 / 295 us, 4110 x 4608 -> 4608
// 52.9 / 49.9 / 61.9, 2048 x 4608 -> 12288 63.8 / 59.7 / 76.4, 1024 x 4608 -> 4608 17.5 / 20.9 / 17.9, 512 x 12288 -> 4608
// 29.5 / 25.8 / 21.8.
int choose_mx_config(int M, int N, int K) {
    struct { int cg, bn; double fixed, per_kb, per_tile; } const c[] = {{2, 256, 4.5, 0.455, 0.8}, {2, 192, 4.0, 0.39, 0.1}, {1, 128, 2.8, 0.345, 0.0}};
    int best = 0;
    double best_us = 0.0;
    for (int i = 0; i < 3; ++i) {
        const int64_t tiles = static_cast<int64_t>((M + BM * c[i].cg - 1) / (BM * c[i].cg)) * ((N + c[i].bn - 1) / c[i].bn);
        const int64_t groups = sm_count() / c[i].cg, waves = (tiles + groups - 1) / groups;
        const double us = c[i].fixed + waves * ((K + BK - 1) / BK * c[i].per_kb + c[i].per_tile);
        if (i == 0 || us < 0.97 * best_us) { best = i; best_us = us; }       // on near ties the earlier one
    }
    return best;
}

int launch_mx_gemm(const MxLinearArgs& a, int config, cudaStream_t st) {
    switch (config) {
        case 0: return launch_cfg<2, 256, 3, 2>(a, st);
        case 1: return launch_cfg<2, 192, 3, 2>(a, st);
        case 2: return launch_cfg<1, 128, 3, 2>(a, st);
        default: return W8A8_ERR_INVALID_ARG;
    }
}

} // namespace w8a8
