// MXFP4 linear for a handful of tokens (at most 16), in one launch: activations are quantized where they are used, the
// weights are streamed once.
//
// The work is reading the weights (N * K * 0.53 bytes); everything is laid out for that stream. The tensor cores take the weights
// as their first operand (128 output channels = the rows of tcgen05.mma, M = 128) and the tokens as the second (N = 16),
// so that a CTA streams 128 rows of W through a TMA ring whose first stages are requested before the kernel ahead has
// finished (weights do not depend on it). K is cut over the CTAs of a cluster until the grid covers the SMs; the partial
// sums meet in the first CTA's shared memory and are added in the order of the ranks (the result does not depend on
// timing). While the weights are on their way the other warps quantize the tokens' part of K straight into the swizzled
// operand tile. Accumulators are transposed (lane = output channel, column = token): a warp stores 64 contiguous bytes a token.
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
constexpr int kWarps = 8;                 // 0 TMA producer, 1 MMA issuer, 2..7 quantize; 4..7 epilogue
constexpr int kQuantWarps = 6;
constexpr int kMaxStages = 6;
constexpr int kMaxKb = 24;                // k-blocks of a CTA (their activations stay in shared memory)
constexpr int kMaxCluster = 8;
constexpr int W_BYTES = ROWS * BKB;
constexpr int SF_BYTES = 2 * kScaleTileBytes;
constexpr int STAGE_BYTES = W_BYTES + SF_BYTES;
constexpr int ACT_BYTES = NT * BKB;       // codes of 16 tokens, one k-block
constexpr int ACT_SF_BYTES = SF_BYTES;    // their scales in tile layout (rows 0..15 are used)
constexpr int TMEM_COLS = 128;            // 16 accumulator columns, then per stage 8 of weight and 8 of token scales
constexpr int SF_COL = 32;

enum Where { W_EMPTY = 1, W_FULL = 2, W_ACTS = 3, W_DONE = 4 };

struct Args {
    const void* A;                        // bf16 [M,K] (CODES = false) or codes
    int64_t lda;                          // elements / bytes
    const uint8_t* sa;                    // scale tiles of codes
    const float* bias;
    __nv_bfloat16* out;
    int64_t ldo;
    int M, N, K;
    int stages, kb_most;                  // ring stages; k-blocks the activation buffers hold
    int* status;
    int* sticky;
    uint64_t wait_limit_ns;
    int starve;
};

template <bool CODES>
__global__ void __launch_bounds__(kWarps * 32)
mx_skinny_kernel(const __grid_constant__ CUtensorMap tm_w, const __grid_constant__ CUtensorMap tm_sw, const Args a) {
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t bars[2 * kMaxStages + 2];
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
    const uint32_t acts_bar = bar0 + 8u * (2 * kMaxStages), done_bar = acts_bar + 8u;
    const WaitCtl ctl{&abort_word, a.status, a.sticky, a.wait_limit_ns};

    // this CTA's output channels and its k-blocks
    const int n0 = static_cast<int>(blockIdx.x / split) * ROWS;
    const int num_kb = (a.K + BK - 1) / BK;
    const int kb0 = static_cast<int>(static_cast<int64_t>(num_kb) * rank / split), kb1 = static_cast<int>(static_cast<int64_t>(num_kb) * (rank + 1) / split);
    const int ktiles = (a.K + kScaleTileBlocks * kMxBlock - 1) / (kScaleTileBlocks * kMxBlock);
    // shared memory: ring, token codes and scales of every k-block of this CTA, partial sums of the other ranks
    const int off_act = a.stages * STAGE_BYTES, off_act_sf = off_act + a.kb_most * ACT_BYTES, off_part = off_act_sf + a.kb_most * ACT_SF_BYTES;

    if (threadIdx.x == 0) {
        for (int s = 0; s < a.stages; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
        mbar_init(acts_bar, kQuantWarps);
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
    if (split > 1) cluster_arrive();           // (the others' shared memory is written to after the matching wait)

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
                    mbar_arrive_expect_tx(full_bar(stage), STAGE_BYTES);
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
    } else if (warp == 1) {
        if (lane == 0) {
            constexpr uint32_t idesc_lo = make_mxf4_idesc(ROWS, NT, 0), idesc_hi = make_mxf4_idesc(ROWS, NT, 2);
            bool ok = mbar_wait(acts_bar, 0, ctl, W_ACTS, kStatusTimeout);
            int stage = 0;
            uint32_t phase = 0;
            for (int kb = kb0; kb < kb1 && ok; ++kb) {
                // (the stage's scale columns are free too: its bytes were requested after the MMAs that used it had completed)
                if (!mbar_wait(full_bar(stage), phase, ctl, W_FULL, kStatusTimeout)) { ok = false; break; }
                tc_fence_after();
                const uint32_t s = base + stage * STAGE_BYTES, act = base + off_act + (kb - kb0) * ACT_BYTES, act_sf = base + off_act_sf + (kb - kb0) * ACT_SF_BYTES;
                const uint64_t dw = make_kmajor_sw128_desc(s), dt = make_kmajor_sw128_desc(act);
                const uint32_t sf = tmem + SF_COL + stage * 16;
                const int left = a.K - kb * BK;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if (h * 2 * MMA_K < left) {
                        tc_cp_scales<1>(sf + 4 * h, make_scale_desc(s + W_BYTES + h * kScaleTileBytes));
                        tc_cp_scales<1>(sf + 8 + 4 * h, make_scale_desc(act_sf + h * kScaleTileBytes));
                    }
                }
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
        // tokens: a warp takes 256 elements (one k-block) of one token at a time, a lane 8 of them
        grid_dep_wait();
        if (blockIdx.x == 0 && warp == 2 && lane == 0) *a.status = 0;
        const int units = a.M * (kb1 - kb0);
        constexpr int U = 4;                               // units whose loads are in flight together
        for (int u0 = warp - 2; u0 < units; u0 += kQuantWarps * U) {
            uint4 x[U];
            uint32_t word[U];
#pragma unroll
            for (int j = 0; j < U; ++j) {
                const int u = u0 + j * kQuantWarps, m = u % a.M, kb = kb0 + u / a.M, k = kb * BK + lane * 8;
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
                const int u = u0 + j * kQuantWarps;
                if (u >= units) break;                     // uniform over the warp
                const int m = u % a.M, i = u / a.M;
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
                // row m of the 128-byte-swizzled tile; scales of half of the k-block at row m of their tile
                *reinterpret_cast<uint32_t*>(base_ptr + off_act + i * ACT_BYTES + m * BKB + (((lane >> 2) ^ (m & 7)) << 4) + (lane & 3) * 4) = codes;
                if ((lane & 15) == 0)
                    *reinterpret_cast<uint32_t*>(base_ptr + off_act_sf + i * ACT_SF_BYTES + (lane >> 4) * kScaleTileBytes + scale_in_tile(m, 0)) = word[j];
            }
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(acts_bar);
        __syncwarp();
        // ------------------------------------------------------------ partial sums and epilogue (warps 4..7: all TMEM lanes)
        if (split > 1) cluster_wait();
        bool ok = true;
        float v[NT];
        if (warp >= 4) {
            if (!mbar_wait(done_bar, 0, ctl, W_DONE, kStatusTimeout)) ok = false;
            ok = __all_sync(0xffffffffu, ok) != 0;
            if (ok) {
                tc_fence_after();
                const uint32_t t_row = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16);
                uint32_t r[NT];
                asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                             : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
                               "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                             : "r"(t_row) : "memory");
                tmem_wait_ld();
                tc_fence_before();
#pragma unroll
                for (int j = 0; j < NT; ++j) v[j] = __uint_as_float(r[j]);
                if (rank != 0) {
                    // into the first CTA's slot for this rank: [token][channel]
                    const uint32_t dst = mapa_shared(base + off_part + (rank - 1) * a.M * ROWS * 4 + ((warp & 3) * 32 + lane) * 4, 0);
                    for (int j = 0; j < NT; ++j)
                        if (j < a.M) asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(dst + j * ROWS * 4), "f"(v[j]) : "memory");
                }
            }
        }
        if (split > 1) cluster_sync_all();
        if (warp >= 4 && ok && rank == 0) {
            const int ch = (warp & 3) * 32 + lane, n = n0 + ch;
            const float* part = reinterpret_cast<const float*>(base_ptr + off_part) + ch;
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
    if (warp < 2 && split > 1) {
        cluster_wait();
        cluster_sync_all();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 1) tmem_dealloc(tmem, TMEM_COLS);
}

struct Plan {
    int split, stages, kb_most, smem;
};

// K is cut until the grid covers the SMs, as long as a CTA keeps two k-blocks; further where the tokens of a longer part
// would not fit in shared memory.
Plan plan_for(int M, int N, int K) {
    const int tiles = (N + ROWS - 1) / ROWS, num_kb = (K + BK - 1) / BK;
    Plan p{};
    p.split = 1;
    while (p.split < kMaxCluster && ((tiles * p.split * 2 <= sm_count() && num_kb >= 4 * p.split) || (num_kb + p.split - 1) / p.split > kMaxKb)) p.split *= 2;
    p.kb_most = (num_kb + p.split - 1) / p.split;
    // two CTAs an SM where the ring and the tokens leave room for that
    p.stages = p.kb_most < kMaxStages ? p.kb_most : kMaxStages;
    auto bytes = [&] { return p.stages * STAGE_BYTES + p.kb_most * (ACT_BYTES + ACT_SF_BYTES) + (p.split - 1) * M * ROWS * 4 + 1024; };
    while (p.stages > 3 && bytes() > 112 * 1024) --p.stages;
    p.smem = bytes();
    return p;
}

} // namespace

bool mx_skinny_fits(int M, int N, int K) {
    return M <= NT && (K + BK - 1) / BK <= kMaxKb * kMaxCluster;
}

int launch_mx_skinny(const MxLinearArgs& g, const void* A, bool codes, int64_t lda, const uint8_t* sa, cudaStream_t st) {
    const Plan p = plan_for(g.M, g.N, g.K);
    const auto kern = codes ? mx_skinny_kernel<true> : mx_skinny_kernel<false>;
    static PerDeviceOnce opt_in[2];
    constexpr int kMostSmem = 200 * 1024;
    if (p.smem > kMostSmem || opt_in[codes].run([&] { return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostSmem); }) != cudaSuccess)
        return W8A8_ERR_CUDA;
    CUtensorMap tm_w, tm_sw;
    if (!encode_mx_codes(&tm_w, g.qw, g.N, g.K, g.K / 2, ROWS) || !encode_mx_scales(&tm_sw, g.sw, g.N, g.K)) return W8A8_ERR_CUDA;
    Args a{};
    a.A = A; a.lda = lda; a.sa = sa; a.bias = g.bias; a.out = static_cast<__nv_bfloat16*>(g.out); a.ldo = g.ldo;
    a.M = g.M; a.N = g.N; a.K = g.K; a.stages = p.stages; a.kb_most = p.kb_most;
    a.status = g.status; a.sticky = sticky_status_word(); a.wait_limit_ns = wait_limit_ns();
    a.starve = starve_mode() == kStarveGemm ? 1 : 0;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((g.N + ROWS - 1) / ROWS * p.split);
    cfg.blockDim = dim3(kWarps * 32);
    cfg.dynamicSmemBytes = p.smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = p.split;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kern, tm_w, tm_sw, a) == cudaSuccess ? W8A8_OK : W8A8_ERR_CUDA;
}

} // namespace w8a8
