// Paged cache of keys and values in few bits: quantized as it is written, read back as bf16.
//
//   int8   per (token, head): s = amax > 0 ? amax / 127 : 1, q = clamp(rne(x / s), +-127)    value = q * s
//   MXFP4  per block of 32 along the head (a head's last block may be shorter): see mxfp4_math.cuh
//
// Both directions move bytes: a write reads 2 and stores 1 (or 0.53) bytes an element, a read loads 1 (0.53) and stores
// 2. A lane handles 8 elements. All offsets into the cache are 64-bit.
#include "../../include/kv_cache.h"
#include "internal.h"
#include "mxfp4_math.cuh"
#include "ptx.cuh"
#include "quant_math.cuh"

namespace w8a8 {
namespace {

constexpr int kThreads = 256;

struct Side {                      // keys or values
    const __nv_bfloat16* x;        // new tokens (write)
    int64_t st, sh;                // their strides in elements: token, head
    uint8_t* codes;
    void* scales;
    __nv_bfloat16* out;            // tokens read back (read)
    int64_t ot, oh;                // its strides
};

// A group of LPG lanes (a power of two, at least dim / 8) quantizes one head of one token.
template <int FMT>
__global__ void __launch_bounds__(kThreads)
kv_write_kernel(const Side k, const Side v, const int64_t* __restrict__ slots, int64_t num_slots, int64_t groups, int heads, int dim, int lpg) {
    grid_dep_wait();
    const Side s = blockIdx.y == 0 ? k : v;
    const int lane = threadIdx.x & 31;
    const int gl = lane & (lpg - 1);                              // lane within its group
    const int per_warp = 32 / lpg;
    const int64_t warps = static_cast<int64_t>(gridDim.x) * (kThreads / 32);
    for (int64_t g0 = (static_cast<int64_t>(blockIdx.x) * (kThreads / 32) + (threadIdx.x >> 5)) * per_warp; g0 < groups; g0 += warps * per_warp) {
        const int64_t g = g0 + lane / lpg;
        const int64_t t = g / heads;
        const int h = static_cast<int>(g - t * heads);
        const bool mine = g < groups && gl * 8 < dim;
        uint4 x = make_uint4(0, 0, 0, 0);
        int64_t slot = -1;
        if (g < groups) slot = __ldcg(slots + t);
        if (mine) x = __ldcg(reinterpret_cast<const uint4*>(s.x + t * s.st + h * s.sh + gl * 8));
        const bool store = mine && slot >= 0 && slot < num_slots;
        const int64_t row = slot * heads + h;
        uint32_t m = absmax_bits8(x);
        if (FMT == KV_CACHE_INT8) {
            for (int o = 1; o < lpg; o <<= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
            const bool finite = m < 0x7f800000u;
            const RowScale rs = make_row_scale(finite ? __uint_as_float(m) : 0.f);
            const RowScale2 r2 = make_row_scale2(rs);
            uint2 q = make_uint2(0, 0);
            if (finite) q = quant8(x, rs, r2);
            if (store) {
                *reinterpret_cast<uint2*>(s.codes + row * dim + gl * 8) = q;
                if (gl == 0) static_cast<float*>(s.scales)[row] = finite ? rs.s : __uint_as_float(0x7fc00000u);
            }
        } else {
            m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
            m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
            const uint32_t byte = mx_scale_byte(m);
            float f[8];
            unpack_bf16x8(x, f);
            if (store) {
                *reinterpret_cast<uint32_t*>(s.codes + row * (dim / 2) + gl * 4) = mx_codes8(f, byte);
                if ((gl & 3) == 0) static_cast<uint8_t*>(s.scales)[row * ((dim + 31) / 32) + gl / 4] = static_cast<uint8_t>(byte);
            }
        }
    }
}

constexpr int kTile = 32;          // tokens a CTA reads at a time

// Eight int8 codes times a scale as bf16
__device__ __forceinline__ uint4 int8_values8(uint2 c, float s) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t two = i < 2 ? c.x : c.y;
        const float a = static_cast<float>(static_cast<int8_t>(two >> ((i & 1) * 16)));
        const float b = static_cast<float>(static_cast<int8_t>(two >> ((i & 1) * 16 + 8)));
        const __nv_bfloat162 p = __floats2bfloat162_rn(a * s, b * s);
        w[i] = *reinterpret_cast<const uint32_t*>(&p);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

template <int FMT>
__global__ void __launch_bounds__(kThreads)
kv_read_kernel(const Side k, const Side v, const int32_t* __restrict__ table, int64_t table_stride, int max_pages, const int32_t* __restrict__ cu,
               const int32_t* __restrict__ starts, int seqs, int64_t total, int64_t num_pages, int page, int heads, int dim) {
    grid_dep_wait();
    __shared__ int64_t rows[kTile];                               // cache row of each token of the tile, -1: none, -2: leave alone
    const Side s = blockIdx.y == 0 ? k : v;
    const int chunks = heads * (dim / 8);                         // pieces of 8 elements a token has
    for (int64_t t0 = static_cast<int64_t>(blockIdx.x) * kTile; t0 < total; t0 += static_cast<int64_t>(gridDim.x) * kTile) {
        __syncthreads();
        const int count = static_cast<int>(total - t0 < kTile ? total - t0 : kTile);
        if (static_cast<int>(threadIdx.x) < count) {
            const int64_t t = t0 + threadIdx.x;
            int lo = 0, hi = seqs;                                // the first sequence that ends after t
            while (lo < hi) {
                const int mid = (lo + hi) >> 1;
                if (__ldcg(cu + mid + 1) > t) hi = mid;
                else lo = mid + 1;
            }
            int64_t row = -2;
            if (lo < seqs && t >= __ldcg(cu + lo)) {
                const int64_t at = t - __ldcg(cu + lo) + (starts != nullptr ? __ldcg(starts + lo) : 0);
                const int64_t p = at / page;
                row = -1;
                if (at >= 0 && p < max_pages) {
                    const int64_t id = __ldcg(table + lo * table_stride + p);
                    if (id >= 0 && id < num_pages) row = id * page + at % page;
                }
            }
            rows[threadIdx.x] = row;
        }
        __syncthreads();
        for (int i = threadIdx.x; i < count * chunks; i += kThreads) {
            const int tt = i / chunks, c = i - tt * chunks;
            const int h = c / (dim / 8), d = (c - h * (dim / 8)) * 8;
            const int64_t slot = rows[tt];
            if (slot == -2) continue;
            uint4 o = make_uint4(0, 0, 0, 0);
            if (slot >= 0) {
                const int64_t row = slot * heads + h;
                if (FMT == KV_CACHE_INT8)
                    o = int8_values8(__ldcg(reinterpret_cast<const uint2*>(s.codes + row * dim + d)), __ldcg(static_cast<const float*>(s.scales) + row));
                else
                    o = mx_values8(__ldcg(reinterpret_cast<const uint32_t*>(s.codes + row * (dim / 2) + d / 2)),
                                   __ldcg(static_cast<const uint8_t*>(s.scales) + row * ((dim + 31) / 32) + d / 32));
            }
            *reinterpret_cast<uint4*>(s.out + (t0 + tt) * s.ot + h * s.oh + d) = o;
        }
    }
}

// Launched so that it may be set up while the kernel ahead of it is finishing (it waits before it touches memory).
template <typename... P, typename... A>
cudaError_t launch(void (*kern)(P...), dim3 grid, cudaStream_t st, A... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(kThreads);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kern, P(args)...);
}

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

int check_shape(int fmt, int64_t heads, int64_t dim) {
    if ((fmt != KV_CACHE_INT8 && fmt != KV_CACHE_MXFP4) || heads <= 0 || dim <= 0 || heads > 65536 || dim > KV_CACHE_MAX_DIM) return W8A8_ERR_INVALID_ARG;
    return dim % 8 == 0 ? W8A8_OK : W8A8_ERR_ALIGNMENT;
}

int check_store(int fmt, const void* codes, const void* scales) {
    if (codes == nullptr || scales == nullptr) return W8A8_ERR_INVALID_ARG;
    if (!aligned(codes, 16) || !aligned(scales, fmt == KV_CACHE_INT8 ? 4 : 1)) return W8A8_ERR_ALIGNMENT;
    return W8A8_OK;
}

} // namespace
} // namespace w8a8

extern "C" {

using namespace w8a8;

int kv_cache_write(int fmt, const void* k, int64_t k_token_stride, int64_t k_head_stride, const void* v, int64_t v_token_stride,
                   int64_t v_head_stride, const int64_t* slots, int64_t tokens, int64_t heads, int64_t dim, void* k_codes, void* k_scales,
                   void* v_codes, void* v_scales, int64_t num_slots, void* stream) {
    if (int e = check_shape(fmt, heads, dim)) return e;
    if (tokens < 0 || num_slots < 0 || k == nullptr || (tokens > 0 && slots == nullptr)) return W8A8_ERR_INVALID_ARG;
    if (int e = check_store(fmt, k_codes, k_scales)) return e;
    if (!aligned(k, 16) || k_token_stride % 8 != 0 || k_head_stride % 8 != 0 || !aligned(slots, 8)) return W8A8_ERR_ALIGNMENT;
    if (v != nullptr) {
        if (int e = check_store(fmt, v_codes, v_scales)) return e;
        if (!aligned(v, 16) || v_token_stride % 8 != 0 || v_head_stride % 8 != 0) return W8A8_ERR_ALIGNMENT;
    }
    if (int e = check_arch()) return e;
    if (tokens == 0 || num_slots == 0) return W8A8_OK;
    int lpg = 1;
    while (lpg * 8 < dim) lpg <<= 1;
    if (fmt == KV_CACHE_MXFP4 && lpg < 4) lpg = 4;               // a block's four lanes stay together
    Side ks{}, vs{};
    ks.x = static_cast<const __nv_bfloat16*>(k);
    ks.st = k_token_stride;
    ks.sh = k_head_stride;
    ks.codes = static_cast<uint8_t*>(k_codes);
    ks.scales = k_scales;
    vs.x = static_cast<const __nv_bfloat16*>(v);
    vs.st = v_token_stride;
    vs.sh = v_head_stride;
    vs.codes = static_cast<uint8_t*>(v_codes);
    vs.scales = v_scales;
    const int64_t groups = tokens * heads;
    const int64_t per_cta = (kThreads / 32) * (32 / lpg);
    const int64_t ctas = (groups + per_cta - 1) / per_cta, most = static_cast<int64_t>(sm_count()) * 8;
    const dim3 grid(static_cast<unsigned>(ctas < most ? ctas : most), v != nullptr ? 2 : 1);
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    const cudaError_t e = fmt == KV_CACHE_INT8
        ? launch(kv_write_kernel<KV_CACHE_INT8>, grid, st, ks, vs, slots, num_slots, groups, static_cast<int>(heads), static_cast<int>(dim), lpg)
        : launch(kv_write_kernel<KV_CACHE_MXFP4>, grid, st, ks, vs, slots, num_slots, groups, static_cast<int>(heads), static_cast<int>(dim), lpg);
    return e == cudaSuccess ? W8A8_OK : W8A8_ERR_CUDA;
}

int kv_cache_read(int fmt, const void* k_codes, const void* k_scales, const void* v_codes, const void* v_scales, int64_t num_pages, int64_t page_size,
                  int64_t heads, int64_t dim, const int32_t* table, int64_t table_stride, int64_t max_pages, const int32_t* cu_seqlens,
                  const int32_t* starts, int64_t seqs, int64_t total, void* k_out, int64_t k_token_stride, int64_t k_head_stride, void* v_out,
                  int64_t v_token_stride, int64_t v_head_stride, void* stream) {
    if (int e = check_shape(fmt, heads, dim)) return e;
    if (num_pages < 0 || page_size <= 0 || page_size > INT32_MAX || max_pages < 0 || max_pages > INT32_MAX || table_stride < max_pages || seqs < 0 ||
        seqs > INT32_MAX - 1 || total < 0 || total > INT32_MAX || k_out == nullptr || (seqs > 0 && cu_seqlens == nullptr) ||
        (seqs > 0 && max_pages > 0 && table == nullptr))
        return W8A8_ERR_INVALID_ARG;
    if (int e = check_store(fmt, k_codes, k_scales)) return e;
    if (!aligned(k_out, 16) || k_token_stride % 8 != 0 || k_head_stride % 8 != 0 || !aligned(table, 4) || !aligned(cu_seqlens, 4) || !aligned(starts, 4))
        return W8A8_ERR_ALIGNMENT;
    if (v_out != nullptr) {
        if (int e = check_store(fmt, v_codes, v_scales)) return e;
        if (!aligned(v_out, 16) || v_token_stride % 8 != 0 || v_head_stride % 8 != 0) return W8A8_ERR_ALIGNMENT;
    }
    if (int e = check_arch()) return e;
    if (total == 0 || seqs == 0) return W8A8_OK;
    Side ks{}, vs{};
    ks.codes = static_cast<uint8_t*>(const_cast<void*>(k_codes));
    ks.scales = const_cast<void*>(k_scales);
    ks.out = static_cast<__nv_bfloat16*>(k_out);
    ks.ot = k_token_stride;
    ks.oh = k_head_stride;
    vs.codes = static_cast<uint8_t*>(const_cast<void*>(v_codes));
    vs.scales = const_cast<void*>(v_scales);
    vs.out = static_cast<__nv_bfloat16*>(v_out);
    vs.ot = v_token_stride;
    vs.oh = v_head_stride;
    const int64_t ctas = (total + kTile - 1) / kTile, most = static_cast<int64_t>(sm_count()) * 8;
    const dim3 grid(static_cast<unsigned>(ctas < most ? ctas : most), v_out != nullptr ? 2 : 1);
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    const auto kern = fmt == KV_CACHE_INT8 ? kv_read_kernel<KV_CACHE_INT8> : kv_read_kernel<KV_CACHE_MXFP4>;
    const cudaError_t e = launch(kern, grid, st, ks, vs, table, table_stride, static_cast<int>(max_pages), cu_seqlens, starts, static_cast<int>(seqs),
                                 total, num_pages, static_cast<int>(page_size), static_cast<int>(heads), static_cast<int>(dim));
    return e == cudaSuccess ? W8A8_OK : W8A8_ERR_CUDA;
}

} // extern "C"
