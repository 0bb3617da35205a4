// MXFP4 linear for few tokens (at most 64): the weights are streamed once, K is cut over clusters of CTAs. Up to 8 tokens in one
// launch, activations quantized where they are used; above that their codes come from a quantizer ahead.
//
// The work is reading the weights (N * K * 0.53 bytes); everything is laid out for that stream. The tensor cores take the weights
// as their first operand (128 output channels = the rows of tcgen05.mma, M = 128) and the tokens as the second (N = 16 to 64),
// so that a CTA streams 128 rows of W through a TMA ring whose first stages are prefetched into L2 before the kernel ahead has
// finished (and read after it, since it may have written them). K is cut over the CTAs of a cluster until the grid fills two CTAs an SM; the partial
// sums stay in the shared memory of their CTAs; each CTA reads the others' for its share of the tokens and adds them in the order of
// the ranks (the result does not depend on timing). While the weights are on their way the other warps quantize the tokens'
// k-blocks straight into the swizzled operand tile of the same ring stage. Accumulators are transposed (lane = output channel, column = token): they
// go through shared memory, so that a warp stores 256 contiguous bytes a token.
//
// What bounds it: HBM where there is enough to stream (2 x 4608 -> 27648, 67.9 MB: 13.8-14.5 us, 4.7-4.9 TB/s, 0.72-0.75 of the copy
// bandwidth), else the chain launch - first bytes - MMAs - cluster barrier - stores (1 x 4608 -> 4608, 11.3 MB: 6.5 us, of which a
// call on a 256 x 512 weight takes 3.9). The first tiles reach shared memory after the kernel ahead, out of L2: 0.3 us at one token,
// 1.0 us at 64 (10.4 us for 64 x 4608 -> 4608) more than loads ahead of it would take. Measured when those were loaded ahead: scale copies
// in the MMA thread and four accumulators instead of one, no difference (the stream sets the pace); tokens of all k-blocks quantized up
// front, 54 KB of shared memory less for the ring, 15.7 against 14.5 us; partial sums sent to one CTA, 8.2 against 6.2 us.
#include "../../include/mxfp4_linear.h"
#include "internal.h"
#include "mxfp4_math.cuh"
#include "ptx.cuh"
#include "tensor_map.h"

namespace w8a8 {
namespace {

constexpr int ROWS = 128;                 // output channels of a CTA
constexpr int BKB = 128;                  // bytes of K per k-block
constexpr int BK = 2 * BKB;               // elements of K per k-block
constexpr int MMA_K = 64;
constexpr int kMaxStages = 5;
constexpr int kMaxCluster = 8;
constexpr int kCrowdTokens = 4;           // up to here three CTAs fit an SM
constexpr int W_BYTES = ROWS * BKB;
constexpr int SF_BYTES = 2 * kScaleTileBytes;

// The kernel's variants. NT: tokens the MMA takes. WARPS that quantize bf16 tokens (0: the tokens come as codes, through TMA).
// CTAS an SM: shared memory of at least a CTA's share keeps further ones off it, so that all CTAs on an SM (of this kernel or of
// the one behind it) find tensor memory: no CTA of a cluster waits for columns that another cluster's CTA holds, and a
// quarter of it stays free.
template <int NT_, int QUANT_WARPS_, int CTAS_>
struct Variant {
    static constexpr int NT = NT_, QUANT_WARPS = QUANT_WARPS_, CTAS = CTAS_;
    static constexpr bool QUANT = QUANT_WARPS > 0;
    // warps: 0 TMA producer, 1 MMA issuer, 2 scale copies, 3 and up quantize; 4..7 epilogue (one for each quarter of tensor memory)
    static constexpr int THREADS = 32 * (3 + (QUANT_WARPS > 5 ? QUANT_WARPS : 5));
    static constexpr int TOKEN_BYTES = NT * BKB;                           // codes of the tokens, one k-block
    static constexpr int OFF_TOKENS = W_BYTES + SF_BYTES, OFF_TOKEN_SF = OFF_TOKENS + TOKEN_BYTES;       // scales in tile layout
    static constexpr int STAGE_BYTES = OFF_TOKEN_SF + SF_BYTES;
    static constexpr int SF_COL = NT < 32 ? 32 : NT;                       // accumulator, then per stage 8 columns of weight and 8 of token scales
    static constexpr int STAGES = NT <= 32 ? kMaxStages : 4;
    static constexpr int TMEM_COLS = 128;
    static constexpr int LEAST_SMEM = (CTAS == 3 ? 60 : 80) * 1024;
    static_assert(SF_COL + STAGES * 16 <= TMEM_COLS, "tensor memory");
};

enum Where { W_EMPTY = 1, W_FULL = 2, W_ACTS = 3, W_DONE = 4 };

struct Args {
    const void* A;                        // bf16 [M,K] (variants that quantize)
    int64_t lda;
    const float* bias;
    __nv_bfloat16* out;
    int64_t ldo;
    int M, N, K;
    int stages;
    int* status;
    int* sticky;
    uint64_t wait_limit_ns;
    int starve;
};

template <typename V>
__global__ void __launch_bounds__(V::THREADS, V::CTAS)
mx_skinny_kernel(const __grid_constant__ CUtensorMap tm_w, const __grid_constant__ CUtensorMap tm_sw, const __grid_constant__ CUtensorMap tm_a,
                 const __grid_constant__ CUtensorMap tm_sa, const Args a) {
    constexpr int NT = V::NT;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t bars[4 * kMaxStages + 1];
    __shared__ uint32_t tmem_holder;
    __shared__ int abort_word;
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* base_ptr = smem_raw + (base - smem_u32(smem_raw));
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint32_t rank, split;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(split));
    const uint32_t bar0 = smem_u32(bars);
    auto full_bar = [&](int s) { return bar0 + 8u * s; };
    auto empty_bar = [&](int s) { return bar0 + 8u * (kMaxStages + s); };
    auto scale_bar = [&](int s) { return bar0 + 8u * (2 * kMaxStages + s); };
    auto acts_bar = [&](int s) { return bar0 + 8u * (3 * kMaxStages + s); };
    const uint32_t done_bar = bar0 + 8u * (4 * kMaxStages);
    const WaitCtl ctl{&abort_word, a.status, a.sticky, a.wait_limit_ns};

    // this CTA's output channels and its k-blocks
    const int n0 = static_cast<int>(blockIdx.x / split) * ROWS;
    const int num_kb = (a.K + BK - 1) / BK;
    const int kb0 = static_cast<int>(static_cast<int64_t>(num_kb) * rank / split), kb1 = static_cast<int>(static_cast<int64_t>(num_kb) * (rank + 1) / split);
    const int ktiles = (a.K + kScaleTileBlocks * kMxBlock - 1) / (kScaleTileBlocks * kMxBlock);
    if (threadIdx.x == 0) {
        for (int s = 0; s < a.stages; ++s) {
            mbar_init(full_bar(s), 1);
            mbar_init(empty_bar(s), 1);
            mbar_init(scale_bar(s), 1);
            mbar_init(acts_bar(s), a.M);       // (variants that quantize) one arrival a token
        }
        mbar_init(done_bar, 1);
        abort_word = 0;
        fence_mbar_init();
        prefetch_tensormap(&tm_w);
        prefetch_tensormap(&tm_sw);
        if (!V::QUANT) { prefetch_tensormap(&tm_a); prefetch_tensormap(&tm_sa); }
    }
    if (warp == 1) { tmem_alloc(smem_u32(&tmem_holder), V::TMEM_COLS); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_holder;
    // Only now: a kernel behind this one that allocates tensor memory and then waits for this one must not get there first.
    grid_dep_launch_dependents();

    if (warp == 0) {
        if (lane == 0) {
            const uint64_t once = l2_policy_evict_first();
            constexpr int BYTES = W_BYTES + SF_BYTES + (V::QUANT ? 0 : V::TOKEN_BYTES + SF_BYTES);
            auto load = [&](int kb, int stage) {
                const uint32_t s = base + stage * V::STAGE_BYTES;
                mbar_arrive_expect_tx(full_bar(stage), BYTES);
                tma_load_2d_hint(s, &tm_w, full_bar(stage), kb * BKB, n0, once);
                tma_load_2d_hint(s + W_BYTES, &tm_sw, full_bar(stage), 0, n0 / kScaleTileRows * ktiles + 2 * kb, once);
                if (!V::QUANT) {
                    tma_load_2d(s + V::OFF_TOKENS, &tm_a, full_bar(stage), kb * BKB, 0);
                    tma_load_2d(s + V::OFF_TOKEN_SF, &tm_sa, full_bar(stage), 0, 2 * kb);
                }
            };
            int stage = 0, issued = 0;
            uint32_t phase = 0;
            bool withhold = a.starve != 0;
            // The weights of the first ring of stages are on their way to L2 while the kernel ahead finishes. They are read after
            // it is complete, like everything else: it may be the one that writes them.
            for (int kb = kb0; kb < min(kb1, kb0 + a.stages); ++kb) {
                tma_prefetch_2d_hint(&tm_w, kb * BKB, n0, once);
                tma_prefetch_2d_hint(&tm_sw, 0, n0 / kScaleTileRows * ktiles + 2 * kb, once);
            }
            grid_dep_wait();
            for (int kb = kb0; kb < kb1; ++kb) {
                if (issued >= a.stages && !mbar_wait(empty_bar(stage), phase ^ 1u, ctl, W_EMPTY, kStatusTimeout)) break;
                if (withhold) withhold = false;          // test hook: this stage never arrives; the bounded waits run out
                else load(kb, stage);
                if (++stage == a.stages) { stage = 0; phase ^= 1u; }
                ++issued;
            }
            // the last copies have landed before the CTA goes away (they have long been used, unless a wait ran out)
            for (int i = 0; i < a.stages && i < issued; ++i) {
                if (stage == 0) { stage = a.stages; phase ^= 1u; }
                --stage;
                const uint64_t t0 = globaltimer_ns();
                while (!mbar_try_wait(full_bar(stage), phase) && globaltimer_ns() - t0 < (*ctl.abort_flag ? 10000000ull : a.wait_limit_ns)) {}
            }
        }
        __syncwarp();
    } else if (warp == 2) {
        // ------------------------------------------------------------ scales: shared -> tensor memory
        // (in the MMA thread each copy, and the wait of the MMAs for it, would be on the path of every k-block)
        if (lane == 0) {
            bool ok = true;
            int stage = 0;
            uint32_t phase = 0;
            for (int kb = kb0; kb < kb1 && ok; ++kb) {
                // (the stage's columns are free: its bytes were requested after the MMAs that used them had completed)
                if (!mbar_wait(full_bar(stage), phase, ctl, W_FULL, kStatusTimeout) ||
                    (V::QUANT && !mbar_wait(acts_bar(stage), phase, ctl, W_ACTS, kStatusTimeout))) {
                    ok = false;
                    break;
                }
                tc_fence_after();
                const uint32_t s = base + stage * V::STAGE_BYTES, sf = tmem + V::SF_COL + stage * 16;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if (h * 2 * MMA_K < a.K - kb * BK) {
                        tc_cp_scales<1>(sf + 4 * h, make_scale_desc(s + W_BYTES + h * kScaleTileBytes));
                        tc_cp_scales<1>(sf + 8 + 4 * h, make_scale_desc(s + V::OFF_TOKEN_SF + h * kScaleTileBytes));
                    }
                }
                tc_commit(scale_bar(stage));
                if (++stage == a.stages) { stage = 0; phase ^= 1u; }
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        if (lane == 0) {
            constexpr uint32_t idesc_lo = make_mxf4_idesc(ROWS, NT, 0), idesc_hi = make_mxf4_idesc(ROWS, NT, 2);
            bool ok = true;
            int stage = 0;
            uint32_t phase = 0;
            for (int kb = kb0; kb < kb1 && ok; ++kb) {
                if (!mbar_wait(full_bar(stage), phase, ctl, W_FULL, kStatusTimeout) ||
                    (V::QUANT && !mbar_wait(acts_bar(stage), phase, ctl, W_ACTS, kStatusTimeout)) ||
                    !mbar_wait(scale_bar(stage), phase, ctl, W_FULL, kStatusTimeout)) {
                    ok = false;
                    break;
                }
                tc_fence_after();
                const uint32_t s = base + stage * V::STAGE_BYTES;
                const uint64_t dw = make_kmajor_sw128_desc(s), dt = make_kmajor_sw128_desc(s + V::OFF_TOKENS);
                const uint32_t sf = tmem + V::SF_COL + stage * 16;
                const int left = a.K - kb * BK;
#pragma unroll
                for (int k = 0; k < BK / MMA_K; ++k) {
                    if (k * MMA_K < left)
                        mma_mxf4_ss<1>(tmem, dw + 2 * k, dt + 2 * k, (k & 1) ? idesc_hi : idesc_lo, sf + 4 * (k >> 1), sf + 8 + 4 * (k >> 1),
                                       (kb > kb0 || k > 0) ? 1u : 0u);
                }
                tc_commit(empty_bar(stage));
                if (++stage == a.stages) { stage = 0; phase ^= 1u; }
            }
            if (ok) tc_commit(done_bar);
        }
        __syncwarp();
    } else {
        // every warp that may write global memory waits for the kernel ahead
        grid_dep_wait();
        if (blockIdx.x == 0 && warp == 3 && lane == 0) *a.status = 0;
        bool ok = true;
        if (V::QUANT && warp < 3 + V::QUANT_WARPS) {
            // Tokens: a warp takes 256 elements (one k-block) of one token at a time, a lane 8 of them. A warp serves one ring stage,
            // so that it waits for every use of the stage in turn (an mbarrier's parity cannot tell a use from the one after the
            // next), and some of the tokens.
            const int stage = (warp - 3) % a.stages, sub = (warp - 3) / a.stages;
            const int subs = (V::QUANT_WARPS - stage + a.stages - 1) / a.stages;    // warps of this stage
            const int mine = sub < a.M ? (a.M - sub + subs - 1) / subs : 0;         // tokens sub, sub + subs, ...
            const int blocks = (kb1 - kb0 - stage + a.stages - 1) / a.stages;       // k-blocks of this stage (stages <= k-blocks)
            const int units = mine * blocks, div = mine > 0 ? mine : 1;
            auto token_of = [&](int u) { return sub + u % div * subs; };
            constexpr int U = 4;                               // units whose loads are in flight together
            for (int u0 = 0; u0 < units && ok; u0 += U) {
                uint4 x[U];
#pragma unroll
                for (int j = 0; j < U; ++j) {
                    const int u = u0 + j, m = token_of(u), kb = kb0 + stage + u / div * a.stages, k = kb * BK + lane * 8;
                    x[j] = make_uint4(0, 0, 0, 0);
                    if (u < units && k < a.K) x[j] = __ldcg(reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(a.A) + m * a.lda + k));
                }
#pragma unroll
                for (int j = 0; j < U; ++j) {
                    const int u = u0 + j;
                    if (u >= units) break;                     // uniform over the warp
                    const int m = token_of(u), use = u / div;
                    uint32_t top = absmax_bits8(x[j]);
                    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
                    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
                    const uint32_t byte = mx_scale_byte(top);
                    const uint32_t codes = mx_codes8(x[j], byte);
                    uint32_t word = byte << (((lane >> 2) & 3) * 8);
                    word |= __shfl_xor_sync(0xffffffffu, word, 4);
                    word |= __shfl_xor_sync(0xffffffffu, word, 8);
                    // the stage's previous k-block has been multiplied
                    if (ok && use > 0 && !mbar_wait(empty_bar(stage), (use - 1) & 1, ctl, W_EMPTY, kStatusTimeout)) ok = false;
                    if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
                    uint8_t* st = base_ptr + stage * V::STAGE_BYTES;
                    // row m of the 128-byte-swizzled tile; scales of half of the k-block at row m of their tile
                    *reinterpret_cast<uint32_t*>(st + V::OFF_TOKENS + m * BKB + (((lane >> 2) ^ (m & 7)) << 4) + (lane & 3) * 4) = codes;
                    if ((lane & 15) == 0)
                        *reinterpret_cast<uint32_t*>(st + V::OFF_TOKEN_SF + (lane >> 4) * kScaleTileBytes + scale_in_tile(m, 0)) = word;
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(acts_bar(stage));
                }
            }
            __syncwarp();
        }
        // ------------------------------------------------------------ sums to shared memory (warps 4..7: all TMEM lanes)
        // The CTA's MMAs are done and its copies have landed and been used: the ring is free. [token][channel], fp32.
        if (warp >= 4 && warp < 8) {
            if (ok && !mbar_wait(done_bar, 0, ctl, W_DONE, kStatusTimeout)) ok = false;
            ok = __all_sync(0xffffffffu, ok) != 0;
            if (ok) {
                tc_fence_after();
                const uint32_t t_row = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16);
                float* mine = reinterpret_cast<float*>(base_ptr) + (warp & 3) * 32 + lane;
#pragma unroll 1
                for (int c = 0; c * 16 < a.M; ++c) {
                    uint32_t r[16];
                    tmem_ld_32x32b_x16(t_row + c * 16, r);
                    tmem_wait_ld();
#pragma unroll
                    for (int j = 0; j < 16; ++j) mine[(c * 16 + j) * ROWS] = __uint_as_float(r[j]);
                }
                tc_fence_before();
            }
        }
        __syncwarp();
    }
    if (split > 1) cluster_sync_all();
    else __syncthreads();
    // ---------------------------------------------------------------- the cluster's sums added up, bias, bf16
    // A CTA finishes its share of the tokens: four channels a thread, a token's 128 channels (256 bytes) a warp. (All threads may
    // write: the warps that have waited for the kernel ahead were at the barrier too.)
    {
        const int m_lo = a.M * static_cast<int>(rank) / static_cast<int>(split), m_hi = a.M * static_cast<int>(rank + 1) / static_cast<int>(split);
        for (int i = threadIdx.x; i < (m_hi - m_lo) * (ROWS / 4); i += V::THREADS) {
            const int m = m_lo + i / (ROWS / 4), ch = i % (ROWS / 4) * 4, n = n0 + ch;
            const uint32_t at = base + (m * ROWS + ch) * 4;
            float4 v[kMaxCluster];
#pragma unroll
            for (uint32_t q = 0; q < kMaxCluster; ++q)
                if (q < split) v[q] = ld_cluster_f32x4(mapa_shared(at, q));
            float4 s = v[0];
#pragma unroll
            for (uint32_t q = 1; q < kMaxCluster; ++q)
                if (q < split) { s.x += v[q].x; s.y += v[q].y; s.z += v[q].z; s.w += v[q].w; }
            if (n < a.N) {
                if (a.bias != nullptr) {
                    const float4 b = __ldcg(reinterpret_cast<const float4*>(a.bias + n));
                    s.x += b.x; s.y += b.y; s.z += b.z; s.w += b.w;
                }
                const __nv_bfloat162 lo = __floats2bfloat162_rn(s.x, s.y), hi = __floats2bfloat162_rn(s.z, s.w);
                *reinterpret_cast<uint2*>(a.out + static_cast<int64_t>(m) * a.ldo + n) =
                    make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
            }
        }
    }
    __syncwarp();
    if (split > 1) cluster_sync_all();          // nobody leaves while its sums may still be read
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 1) tmem_dealloc(tmem, V::TMEM_COLS);
}

// K is cut as long as the grid stays within two CTAs an SM and a part keeps two and a half k-blocks. Clusters of 4 and more that fill
// the GPU beyond one CTA an SM can only all be placed with three CTAs an SM (up to 4 tokens, a ring of three stages).
// (Measured with parts of 1 / 2 / 4 / 8: 1 x 4608 -> 13824, 108 tiles, 12.2 / 9.9 / 14.0 / 18.2 us; 1 x 12288 -> 4608, 36 tiles,
// 23.2 / 14.3 / 11.0 / 9.8 us; 50 x 4608 -> 9216, 72 tiles in 4 parts, two CTAs an SM, 15.9 us, the tiled GEMM 13.9.)
// It goes by the sizes alone, so that tokens that come as codes give the same bits.
struct Split {
    int parts;
    bool crowded;      // needs three CTAs an SM
};
Split split_for(int M, int N, int K) {
    const int64_t tiles = (static_cast<int64_t>(N) + ROWS - 1) / ROWS, num_kb = (K + BK - 1) / BK, sms = sm_count();
    Split s{1, false};
    while (s.parts < kMaxCluster && num_kb >= 5 * s.parts) {
        const int64_t ctas = tiles * s.parts * 2;
        const bool crowded = s.parts >= 2 && ctas > sms;
        if (ctas > 2 * sms || (crowded && M > kCrowdTokens)) break;
        s.parts *= 2;
        s.crowded = crowded;
    }
    return s;
}

template <typename V>
int launch_variant(const MxLinearArgs& g, const void* A, int64_t lda, cudaStream_t st) {
    const Split cut = split_for(g.M, g.N, g.K);
    const int split = cut.parts, kb_most = ((g.K + BK - 1) / BK + split - 1) / split;
    int stages = cut.crowded ? 3 : V::STAGES;
    static_assert(2 * (V::STAGES * V::STAGE_BYTES + 4096) <= 228 * 1024, "two CTAs an SM");
    if (stages > kb_most) stages = kb_most;
    int most = stages * V::STAGE_BYTES;                       // (the sums come into the ring when it is done)
    static_assert(V::NT * ROWS * 4 <= V::LEAST_SMEM, "the sums fit");
    if (most < V::LEAST_SMEM) most = V::LEAST_SMEM;
    const auto kern = mx_skinny_kernel<V>;
    static PerDeviceOnce opt_in;
    constexpr int MOST_SMEM = (V::STAGES * V::STAGE_BYTES > V::LEAST_SMEM ? V::STAGES * V::STAGE_BYTES : V::LEAST_SMEM) + 1024;
    if (opt_in.run([&] { return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, MOST_SMEM); }) != cudaSuccess) return W8A8_ERR_CUDA;
    CUtensorMap tm_w, tm_sw, tm_a, tm_sa;
    if (!encode_mx_codes(&tm_w, g.qw, g.N, g.K, g.K / 2, ROWS) || !encode_mx_scales(&tm_sw, g.sw, g.N, g.K)) return W8A8_ERR_CUDA;
    if (V::QUANT) {
        tm_a = tm_w;      // unused
        tm_sa = tm_sw;
    } else if (!encode_mx_codes(&tm_a, g.qa, g.M, g.K, g.ldqa, V::NT) || !encode_mx_scales(&tm_sa, g.sa, g.M, g.K)) {
        return W8A8_ERR_CUDA;
    }
    Args a{};
    a.A = A; a.lda = lda; a.bias = g.bias; a.out = static_cast<__nv_bfloat16*>(g.out); a.ldo = g.ldo;
    a.M = g.M; a.N = g.N; a.K = g.K; a.stages = stages;
    a.status = g.status; a.sticky = sticky_status_word(); a.wait_limit_ns = wait_limit_ns();
    a.starve = starve_mode() == kStarveGemm ? 1 : 0;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((g.N + ROWS - 1) / ROWS * split);
    cfg.blockDim = dim3(V::THREADS);
    cfg.dynamicSmemBytes = most + 1024;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = split;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kern, tm_w, tm_sw, tm_a, tm_sa, a) == cudaSuccess ? W8A8_OK : W8A8_ERR_CUDA;
}

} // namespace

bool mx_skinny_fits(int M) { return M <= kMxSkinnyMost; }
// (This kernel against the tiled GEMM, quantizer included: 17 x 4608 -> 4608 8.9 / 12.2 us, 32 x 4608 -> 13824 13.5 / 15.5, 64 x 12288 -> 4608
// 15.3 / 21.9, 64 x 4608 -> 4608 10.7 / 12.2, 64 x 768 -> 512 9.5 / 6.9. By M and K alone: about even on 48 x 1056 -> 2048, 8.4 / 8.0, and
// 64 x 4608 -> 27648, 22.3 / 21.6; beyond that the tiled kernel's reuse of the tokens wins, 64 x 2048 -> 60000 30.7 / 22.1.)
bool mx_skinny_preferred(int M, int K) { return M <= 16 || (M <= kMxSkinnyMost && K > 2 * BK); }

// Up to 4 tokens 5 warps quantize and three CTAs fit an SM; more tokens need 10 warps.
int launch_mx_skinny_bf16(const MxLinearArgs& g, const void* A, int64_t lda, cudaStream_t st) {
    return g.M <= kCrowdTokens ? launch_variant<Variant<16, 5, 3>>(g, A, lda, st) : launch_variant<Variant<16, 10, 2>>(g, A, lda, st);
}

int launch_mx_skinny_codes(const MxLinearArgs& g, cudaStream_t st) {
    if (g.M <= 16) return launch_variant<Variant<16, 0, 3>>(g, nullptr, 0, st);
    if (g.M <= 32) return launch_variant<Variant<32, 0, 2>>(g, nullptr, 0, st);
    if (g.M <= 48) return launch_variant<Variant<48, 0, 2>>(g, nullptr, 0, st);
    return launch_variant<Variant<64, 0, 2>>(g, nullptr, 0, st);
}

} // namespace w8a8
