// MXFP4 linear for a handful of tokens (at most 16), in one launch: activations are quantized where they are used, the
// weights are streamed once.
//
// The work is reading the weights (N * K * 0.53 bytes); everything is laid out for that stream. The tensor cores take the weights
// as their first operand (128 output channels = the rows of tcgen05.mma, M = 128) and the tokens as the second (N = 16),
// so that a CTA streams 128 rows of W through a TMA ring whose first stages are requested before the kernel ahead has
// finished (weights do not depend on it). K is cut over the CTAs of a cluster until the grid fills two CTAs an SM; the partial
// sums meet in the first CTA's shared memory and are added in the order of the ranks (the result does not depend on
// timing). While the weights are on their way the other warps quantize the tokens' k-blocks straight into the swizzled
// operand tile of the same ring stage. Accumulators are transposed (lane = output channel, column = token): a warp stores 64
// contiguous bytes a token.
#include "../../include/mxfp4_linear.h"
#include "internal.h"
#include "mxfp4_math.cuh"
#include "ptx.cuh"
#include "tensor_map.h"

namespace w8a8 {
namespace {

constexpr int NT = 16;                    // tokens
constexpr int ROWS = 128;                 // output channels of a CTA
constexpr int BKB = 128;                  // bytes of K per k-block
constexpr int BK = 2 * BKB;               // elements of K per k-block
constexpr int MMA_K = 64;
// Warps: 0 TMA producer, 1 MMA issuer, 2 scale copies, 3 and up quantize (4..7 epilogue). Up to 4 tokens 5 warps quantize, and
// three CTAs fit an SM; more tokens need 10 (8 x 4608 -> 4608: 9.4 against 10.0 us; 1 x 12288 -> 4608 in 8 parts: 15 against 9.8 us).
constexpr int kFewTokens = 4;
template <bool FEW> constexpr int QUANT_WARPS = FEW ? 5 : 10;
template <bool FEW> constexpr int THREADS = 32 * (3 + QUANT_WARPS<FEW>);
constexpr int kMaxStages = 5;             // 5 x 20 KB: two CTAs an SM
constexpr int kMaxCluster = 8;
constexpr int W_BYTES = ROWS * BKB;
constexpr int SF_BYTES = 2 * kScaleTileBytes;
constexpr int ACT_BYTES = NT * BKB;       // codes of 16 tokens, one k-block
constexpr int OFF_ACT = W_BYTES + SF_BYTES, OFF_ACT_SF = OFF_ACT + ACT_BYTES;      // the tokens' scales in tile layout (rows 0..15 are used)
constexpr int STAGE_BYTES = OFF_ACT_SF + SF_BYTES;
constexpr int TMEM_COLS = 128;            // the accumulator, then per stage 8 columns of weight and 8 of token scales
constexpr int SF_COL = 32;
// At least this much shared memory keeps a fourth CTA off the SM: three (of this kernel or of the one behind it) always find
// tensor memory, so no CTA of a cluster waits for columns that another cluster's CTA holds, and a quarter of it stays free.
constexpr int kLeastSmem = 60 * 1024;
static_assert(SF_COL + kMaxStages * 16 <= TMEM_COLS, "tensor memory");

enum Where { W_EMPTY = 1, W_FULL = 2, W_ACTS = 3, W_DONE = 4 };

struct Args {
    const void* A;                        // bf16 [M,K] (CODES = false) or codes
    int64_t lda;                          // elements / bytes
    const uint8_t* sa;                    // scale tiles of codes
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

template <bool CODES, bool FEW>
__global__ void __launch_bounds__(THREADS<FEW>, FEW ? 3 : 2)
mx_skinny_kernel(const __grid_constant__ CUtensorMap tm_w, const __grid_constant__ CUtensorMap tm_sw, const Args a) {
    constexpr int kQuantWarps = QUANT_WARPS<FEW>;
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
            mbar_init(acts_bar(s), a.M);       // one arrival a token
        }
        mbar_init(done_bar, 1);
        abort_word = 0;
        fence_mbar_init();
        prefetch_tensormap(&tm_w);
        prefetch_tensormap(&tm_sw);
    }
    if (warp == 1) { tmem_alloc(smem_u32(&tmem_holder), TMEM_COLS); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_holder;
    // Only now: a kernel behind this one that allocates tensor memory and then waits for this one must not get there first.
    grid_dep_launch_dependents();

    if (warp == 0) {
        if (lane == 0) {
            const uint64_t once = l2_policy_evict_first();
            int stage = 0, issued = 0;
            uint32_t phase = 0;
            bool withhold = a.starve != 0;
            for (int kb = kb0; kb < kb1; ++kb) {
                if (kb - kb0 >= a.stages && !mbar_wait(empty_bar(stage), phase ^ 1u, ctl, W_EMPTY, kStatusTimeout)) break;
                if (withhold) {
                    withhold = false;          // test hook: this stage never arrives; the bounded waits run out
                } else {
                    const uint32_t s = base + stage * STAGE_BYTES;
                    mbar_arrive_expect_tx(full_bar(stage), W_BYTES + SF_BYTES);
                    tma_load_2d_hint(s, &tm_w, full_bar(stage), kb * BKB, n0, once);
                    tma_load_2d_hint(s + W_BYTES, &tm_sw, full_bar(stage), 0, n0 / kScaleTileRows * ktiles + 2 * kb, once);
                }
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
                if (!mbar_wait(full_bar(stage), phase, ctl, W_FULL, kStatusTimeout) || !mbar_wait(acts_bar(stage), phase, ctl, W_ACTS, kStatusTimeout)) {
                    ok = false;
                    break;
                }
                tc_fence_after();
                const uint32_t s = base + stage * STAGE_BYTES + W_BYTES, act_sf = base + stage * STAGE_BYTES + OFF_ACT_SF;
                const uint32_t sf = tmem + SF_COL + stage * 16;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if (h * 2 * MMA_K < a.K - kb * BK) {
                        tc_cp_scales<1>(sf + 4 * h, make_scale_desc(s + h * kScaleTileBytes));
                        tc_cp_scales<1>(sf + 8 + 4 * h, make_scale_desc(act_sf + h * kScaleTileBytes));
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
                if (!mbar_wait(full_bar(stage), phase, ctl, W_FULL, kStatusTimeout) || !mbar_wait(acts_bar(stage), phase, ctl, W_ACTS, kStatusTimeout) ||
                    !mbar_wait(scale_bar(stage), phase, ctl, W_FULL, kStatusTimeout)) {
                    ok = false;
                    break;
                }
                tc_fence_after();
                const uint64_t dw = make_kmajor_sw128_desc(base + stage * STAGE_BYTES), dt = make_kmajor_sw128_desc(base + stage * STAGE_BYTES + OFF_ACT);
                const uint32_t sf = tmem + SF_COL + stage * 16;
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
        // Tokens: a warp takes 256 elements (one k-block) of one token at a time, a lane 8 of them. A warp serves one ring stage,
        // so that it waits for every use of the stage in turn (an mbarrier's parity cannot tell a use from the one after the
        // next), and some of the tokens.
        grid_dep_wait();
        if (blockIdx.x == 0 && warp == 3 && lane == 0) *a.status = 0;
        const int stage = (warp - 3) % a.stages, sub = (warp - 3) / a.stages;
        const int subs = (kQuantWarps - stage + a.stages - 1) / a.stages;       // warps of this stage
        const int mine = sub < a.M ? (a.M - sub + subs - 1) / subs : 0;         // tokens sub, sub + subs, ...
        const int blocks = (kb1 - kb0 - stage + a.stages - 1) / a.stages;       // k-blocks of this stage (stages <= k-blocks)
        const int units = mine * blocks, div = mine > 0 ? mine : 1;
        auto token_of = [&](int u) { return sub + u % div * subs; };
        bool ok = true;
        constexpr int U = 4;                               // units whose loads are in flight together
        for (int u0 = 0; u0 < units && ok; u0 += U) {
            uint4 x[U];
            uint32_t word[U];
#pragma unroll
            for (int j = 0; j < U; ++j) {
                const int u = u0 + j, m = token_of(u), kb = kb0 + stage + u / div * a.stages, k = kb * BK + lane * 8;
                x[j] = make_uint4(0, 0, 0, 0);
                word[j] = 0;
                if (u < units && k < a.K) {
                    if (CODES) {
                        const int t = kb * 2 + (lane >> 4);
                        x[j].x = __ldcg(reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(a.A) + m * a.lda + k / 2));
                        word[j] = __ldcg(reinterpret_cast<const uint32_t*>(a.sa + static_cast<int64_t>(t) * kScaleTileBytes + scale_in_tile(m, 0)));
                    } else {
                        x[j] = __ldcg(reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(a.A) + m * a.lda + k));
                    }
                }
            }
#pragma unroll
            for (int j = 0; j < U; ++j) {
                const int u = u0 + j;
                if (u >= units) break;                     // uniform over the warp
                const int m = token_of(u), use = u / div;
                uint32_t codes = x[j].x;
                if (!CODES) {
                    float f[8];
                    unpack_bf16x8(x[j], f);
                    uint32_t top = absmax_bits8(x[j]);
                    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
                    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
                    const uint32_t byte = mx_scale_byte(top);
                    codes = mx_codes8(f, byte);
                    word[j] = byte << (((lane >> 2) & 3) * 8);
                    word[j] |= __shfl_xor_sync(0xffffffffu, word[j], 4);
                    word[j] |= __shfl_xor_sync(0xffffffffu, word[j], 8);
                }
                // the stage's previous k-block has been multiplied
                if (ok && use > 0 && !mbar_wait(empty_bar(stage), (use - 1) & 1, ctl, W_EMPTY, kStatusTimeout)) ok = false;
                if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
                uint8_t* st = base_ptr + stage * STAGE_BYTES;
                // row m of the 128-byte-swizzled tile; scales of half of the k-block at row m of their tile
                *reinterpret_cast<uint32_t*>(st + OFF_ACT + m * BKB + (((lane >> 2) ^ (m & 7)) << 4) + (lane & 3) * 4) = codes;
                if ((lane & 15) == 0)
                    *reinterpret_cast<uint32_t*>(st + OFF_ACT_SF + (lane >> 4) * kScaleTileBytes + scale_in_tile(m, 0)) = word[j];
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(acts_bar(stage));
            }
        }
        // ------------------------------------------------------------ partial sums and epilogue (warps 4..7: all TMEM lanes)
        float v[NT];
        if (warp >= 4 && warp < 8) {
            if (ok && !mbar_wait(done_bar, 0, ctl, W_DONE, kStatusTimeout)) ok = false;
            ok = __all_sync(0xffffffffu, ok) != 0;
            if (ok) {
                tc_fence_after();
                const uint32_t t_row = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16);
                uint32_t r[NT];
                tmem_ld_32x32b_x16(t_row, r);
                tmem_wait_ld();
                tc_fence_before();
#pragma unroll
                for (int j = 0; j < NT; ++j) v[j] = __uint_as_float(r[j]);
            }
        }
        // Every CTA of the cluster has done its MMAs, and its copies have landed: the rings are free. The partial sums go into
        // the first CTA's, and are there after the second barrier.
        if (split > 1) {
            __syncwarp();
            cluster_sync_all();
            if (warp >= 4 && warp < 8 && ok) {
                if (rank != 0) {
                    // into the first CTA's slot for this rank: [token][channel]
                    const uint32_t dst = mapa_shared(base + (rank - 1) * a.M * ROWS * 4 + ((warp & 3) * 32 + lane) * 4, 0);
                    for (int j = 0; j < NT; ++j)
                        if (j < a.M) asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(dst + j * ROWS * 4), "f"(v[j]) : "memory");
                }
            }
            __syncwarp();
            cluster_sync_all();
        }
        if (warp >= 4 && warp < 8 && ok && rank == 0) {
            const int ch = (warp & 3) * 32 + lane, n = n0 + ch;
            const float* part = reinterpret_cast<const float*>(base_ptr) + ch;
            const float b = a.bias != nullptr && n < a.N ? __ldcg(a.bias + n) : 0.f;
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                if (j < a.M) {
                    float s = v[j];
                    for (uint32_t q = 1; q < split; ++q) s += part[((q - 1) * a.M + j) * ROWS];
                    if (n < a.N) a.out[static_cast<int64_t>(j) * a.ldo + n] = __float2bfloat16_rn(s + b);
                }
            }
        }
    }
    if (warp < 3 && split > 1) {
        cluster_sync_all();
        cluster_sync_all();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 1) tmem_dealloc(tmem, TMEM_COLS);
}

// K is cut as long as the grid stays within two CTAs an SM and a part keeps two and a half k-blocks. Clusters of 8 that fill the
// GPU can only all be placed with three CTAs an SM. (Measured with parts of 1 / 2 / 4 / 8: 1 x 4608 -> 13824, 108 tiles,
// 12.2 / 9.9 / 14.0 / 18.2 us; 1 x 12288 -> 4608, 36 tiles, 23.2 / 14.3 / 11.0 / 9.8 us.)
int split_for(int N, int K, bool few) {
    const int64_t tiles = (static_cast<int64_t>(N) + ROWS - 1) / ROWS, num_kb = (K + BK - 1) / BK;
    int split = 1;
    while (split < kMaxCluster && tiles * split * 2 <= (split * 2 == kMaxCluster && !few ? 1 : 2) * sm_count() && num_kb >= 5 * split) split *= 2;
    return split;
}

} // namespace

bool mx_skinny_fits(int M) { return M <= NT; }
// (16 x 4608 -> 13824: 17.4 us here, 16.0 us quantized by a kernel of its own in front of the tiled GEMM; 8 x 4608 -> 4608: 9.4 and 12.9 us)
bool mx_skinny_preferred(int M) { return M <= 12; }

int launch_mx_skinny(const MxLinearArgs& g, const void* A, bool codes, int64_t lda, const uint8_t* sa, cudaStream_t st) {
    const bool few = g.M <= kFewTokens;
    const int split = split_for(g.N, g.K, few), kb_most = ((g.K + BK - 1) / BK + split - 1) / split;
    const int ring_most = split == kMaxCluster ? 3 : kMaxStages;         // 60 KB: three CTAs an SM
    const int stages = kb_most < ring_most ? kb_most : ring_most;
    const int ring = stages * STAGE_BYTES, part = (split - 1) * g.M * ROWS * 4;      // (partial sums come into the ring when it is done)
    const int most = ring > part ? ring : part, smem = (most > kLeastSmem ? most : kLeastSmem) + 1024;
    const auto kern = few ? (codes ? mx_skinny_kernel<true, true> : mx_skinny_kernel<false, true>)
                          : (codes ? mx_skinny_kernel<true, false> : mx_skinny_kernel<false, false>);
    static PerDeviceOnce opt_in[2][2];
    constexpr int kMostSmem = kMaxStages * STAGE_BYTES + 1024;
    static_assert((kMaxCluster - 1) * NT * ROWS * 4 <= kMaxStages * STAGE_BYTES, "the partial sums fit in the largest ring");
    if (opt_in[few][codes].run([&] { return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostSmem); }) != cudaSuccess)
        return W8A8_ERR_CUDA;
    CUtensorMap tm_w, tm_sw;
    if (!encode_mx_codes(&tm_w, g.qw, g.N, g.K, g.K / 2, ROWS) || !encode_mx_scales(&tm_sw, g.sw, g.N, g.K)) return W8A8_ERR_CUDA;
    Args a{};
    a.A = A; a.lda = lda; a.sa = sa; a.bias = g.bias; a.out = static_cast<__nv_bfloat16*>(g.out); a.ldo = g.ldo;
    a.M = g.M; a.N = g.N; a.K = g.K; a.stages = stages;
    a.status = g.status; a.sticky = sticky_status_word(); a.wait_limit_ns = wait_limit_ns();
    a.starve = starve_mode() == kStarveGemm ? 1 : 0;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((g.N + ROWS - 1) / ROWS * split);
    cfg.blockDim = dim3(few ? THREADS<true> : THREADS<false>);
    cfg.dynamicSmemBytes = smem;
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
    return cudaLaunchKernelEx(&cfg, kern, tm_w, tm_sw, a) == cudaSuccess ? W8A8_OK : W8A8_ERR_CUDA;
}

} // namespace w8a8
