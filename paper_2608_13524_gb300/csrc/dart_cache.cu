// Writes rows of keys and values into the pages of the cache: keys rotated at
// their position, both rounded to bf16 or quantised to e4m3 with one scale
// per token and head.  Contract: include/dart_cache.h.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>

#include "../../include/dart.h"
#include "../../include/dart_cache.h"
#include "dart_cache.cuh"
#include "dart_kernels.h"

namespace dart {

bool valid_cache(const dart_kv_cache* c) {
    if (!c || c->num_pages < 1 || c->Hkv < 1 || c->dh != kHeadDim) return false;
    if (c->page_size != 16 && c->page_size != 32 && c->page_size != 64 && c->page_size != 128) return false;
    if (c->dtype != DART_KV_BF16 && c->dtype != DART_KV_E4M3) return false;
    // rows of dh elements are numbered by 32-bit TMA coordinates
    return static_cast<long long>(c->num_pages) * c->Hkv <= (2147483647ll - 128) / c->page_size;
}

bool valid_cache_pointers(const dart_kv_cache* c) {
    auto ok = [](const void* p) { return p && (reinterpret_cast<uintptr_t>(p) & 15u) == 0; };
    if (!ok(c->k) || !ok(c->v)) return false;
    return c->dtype == DART_KV_BF16 ? !c->k_scale && !c->v_scale : ok(c->k_scale) && ok(c->v_scale);
}

namespace {

constexpr int kAppendThreads = 256;
constexpr int kGroup = 8;  // threads of a token's head: 8 elements of each half of a row are 16 bytes
// Four heads a group (angles once for four) where that still makes this many
// groups, else one: a few tokens are a matter of latency (eight prompts of up to
// 4096 tokens to e4m3 pages 39.8 us with four, 67 % of the copy bandwidth, and 49.9
// with one, to bf16 pages 40.4 and 44.1; below, no difference).
constexpr long long kManyGroups = 9728;  // 152 SMs x 64 groups = 512 threads each
constexpr float kMinScale = 7.52316384526264005e-37f;  // 2^-120: its reciprocal is finite
constexpr float kSmallScale = 8.27180612553027675e-25f, kSmallUp = 1.152921504606846976e18f;  // 2^-80, 2^60

struct AppendArgs {
    int nseq, max_pages, R, Hkv, chunks, page_log2, num_pages;
    const int32_t *table, *lens, *rows, *n_rows;
    const __nv_bfloat16 *k, *v;
    long long k_stride, v_stride;
    uint8_t *pk, *pv;
    float *ks, *vs;
    int* status;
    RopeTurns turns;
};

struct Row {  // elements 8 j .. 8 j + 7 and 64 + 8 j .. of thread j of a group
    float lo[8], hi[8];
};

__device__ __forceinline__ void unpack(const uint4& a, const uint4& b, Row& x) {
    const uint32_t u[4] = {a.x, a.y, a.z, a.w}, w[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
    for (int e = 0; e < 4; e++) {
        x.lo[2 * e] = bf16_lo(u[e]);
        x.lo[2 * e + 1] = bf16_hi(u[e]);
        x.hi[2 * e] = bf16_lo(w[e]);
        x.hi[2 * e + 1] = bf16_hi(w[e]);
    }
}

// x / scale, each quotient rounded once to fp32 (two at a time): the product with the
// rounded reciprocal is at most a unit off, its remainder is exact in one fma, and a
// second fma corrects it (P. Markstein, IBM J. Res. Dev. 34, 1990).  Infinities and NaN
// give NaN.
__device__ __forceinline__ float2 quotients(float a, float b, float scale, float inv) {
    const float2 q = fma2(make_float2(a, b), make_float2(inv, inv), make_float2(-0.0f, -0.0f));
    const float2 r = fma2(q, make_float2(scale, scale), make_float2(-a, -b));
    return fma2(r, make_float2(-inv, -inv), q);  // (in this form -0 stays -0)
}
__device__ __forceinline__ uint2 to_e4m3(const float (&x)[8], float scale, float inv) {
    uint32_t r[2];
#pragma unroll
    for (int h = 0; h < 2; h++) {
        const uint32_t a = __nv_cvt_float2_to_fp8x2(quotients(x[4 * h], x[4 * h + 1], scale, inv), __NV_SATFINITE, __NV_E4M3);
        const uint32_t b = __nv_cvt_float2_to_fp8x2(quotients(x[4 * h + 2], x[4 * h + 3], scale, inv), __NV_SATFINITE, __NV_E4M3);
        r[h] = a | (b << 16);
    }
    return make_uint2(r[0], r[1]);
}

__device__ __forceinline__ void store_bf16(uint8_t* pool, long long row, int j, const Row& x) {
    uint8_t* d = pool + (row * kHeadDim + 8 * j) * 2;
    *reinterpret_cast<uint4*>(d) = make_uint4(pack_bf16x2(x.lo[0], x.lo[1]), pack_bf16x2(x.lo[2], x.lo[3]),
                                              pack_bf16x2(x.lo[4], x.lo[5]), pack_bf16x2(x.lo[6], x.lo[7]));
    *reinterpret_cast<uint4*>(d + 128) = make_uint4(pack_bf16x2(x.hi[0], x.hi[1]), pack_bf16x2(x.hi[2], x.hi[3]),
                                                    pack_bf16x2(x.hi[4], x.hi[5]), pack_bf16x2(x.hi[6], x.hi[7]));
}

// One scale for the 128 values of the group (every thread of the warp calls it).
__device__ __forceinline__ void store_e4m3(uint8_t* pool, float* scales, long long row, int j, Row x, bool use) {
    float amax = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; e++) amax = fmaxf(amax, fmaxf(fabsf(x.lo[e]), fabsf(x.hi[e])));
#pragma unroll
    for (int o = kGroup / 2; o > 0; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(kFull, amax, o));
    const float scale = amax > 0.0f ? fmaxf(__fdiv_rn(amax, 448.0f), kMinScale) : 1.0f;
    if (!use) return;
    float by = scale;
    if (scale < kSmallScale) {  // (rare) a remainder would lie below the floats: both sides times 2^60
        by *= kSmallUp;
#pragma unroll
        for (int e = 0; e < 8; e++) {
            x.lo[e] *= kSmallUp;
            x.hi[e] *= kSmallUp;
        }
    }
    const float inv = __frcp_rn(by);
    uint8_t* d = pool + row * kHeadDim + 8 * j;
    *reinterpret_cast<uint2*>(d) = to_e4m3(x.lo, by, inv);
    *reinterpret_cast<uint2*>(d + 64) = to_e4m3(x.hi, by, inv);
    if (j == 0) scales[row] = scale;
}

// A group of 8 threads takes kHeads heads of one token, so that the angles of
// its position are computed once for all of them and every head's loads are
// in flight together.
template <bool kFp8, int kHeads>
__global__ void __launch_bounds__(kAppendThreads) cache_append_kernel(const __grid_constant__ AppendArgs a) {
    __shared__ uint64_t f[kHeadDim / 2];
    pdl_trigger();
    if (threadIdx.x < kHeadDim / 2) f[threadIdx.x] = a.turns.f[threadIdx.x];
    __syncthreads();
    pdl_wait();
    const int j = threadIdx.x % kGroup;
    const long long group = static_cast<long long>(blockIdx.x) * (kAppendThreads / kGroup) + threadIdx.x / kGroup;
    const int chunk = static_cast<int>(group % a.chunks);
    const long long token = group / a.chunks;
    const int s = static_cast<int>(token / a.R), i = static_cast<int>(token % a.R);
    bool use = s < a.nseq && i < ld_plain(a.n_rows + min(s, a.nseq - 1));
    long long src = 0, dst = 0;
    int pos = 0;
    if (use) {
        const int src_row = a.rows ? ld_plain(a.rows + token) : i;
        const long long most = static_cast<long long>(a.max_pages) << a.page_log2;
        const long long p = min(max(static_cast<long long>(ld_plain(a.lens + s)), 0ll), most) + i;
        int page = -1;
        if (p < most) page = ld_plain(a.table + static_cast<long long>(s) * a.max_pages + (p >> a.page_log2));
        if (src_row < 0 || src_row >= a.R || page < 0 || page >= a.num_pages) {
            if (a.status && j == 0) atomicOr(a.status, kDevBounds);
            use = false;
        } else {
            pos = static_cast<int>(p);
            src = static_cast<long long>(s) * a.R + src_row;
            dst = ((static_cast<long long>(page) * a.Hkv) << a.page_log2) + (p & ((1 << a.page_log2) - 1));
        }
    }
    if (!__any_sync(kFull, use)) return;
    const int h0 = chunk * kHeads;
    uint4 kv[kHeads][4];
#pragma unroll
    for (int h = 0; h < kHeads; h++) {
        const bool in = use && h0 + h < a.Hkv;
        const __nv_bfloat16* k = a.k + src * a.k_stride + (h0 + h) * kHeadDim + 8 * j;
        const __nv_bfloat16* v = a.v + src * a.v_stride + (h0 + h) * kHeadDim + 8 * j;
        const uint4 zero = make_uint4(0, 0, 0, 0);
        kv[h][0] = in ? __ldcs(reinterpret_cast<const uint4*>(k)) : zero;
        kv[h][1] = in ? __ldcs(reinterpret_cast<const uint4*>(k + 64)) : zero;
        kv[h][2] = in ? __ldcs(reinterpret_cast<const uint4*>(v)) : zero;
        kv[h][3] = in ? __ldcs(reinterpret_cast<const uint4*>(v + 64)) : zero;
    }
    float sn[8], cs[8];
#pragma unroll
    for (int e = 0; e < 8; e++) rope_sincos(f[8 * j + e], pos, &sn[e], &cs[e]);
#pragma unroll
    for (int h = 0; h < kHeads; h++) {
        Row x;
        unpack(kv[h][0], kv[h][1], x);
#pragma unroll
        for (int e = 0; e < 8; e++) {
            const float lo = x.lo[e], hi = x.hi[e];
            x.lo[e] = lo * cs[e] - hi * sn[e];
            x.hi[e] = hi * cs[e] + lo * sn[e];
        }
        Row y;
        unpack(kv[h][2], kv[h][3], y);
        const long long row = dst + (static_cast<long long>(h0 + h) << a.page_log2);
        const bool in = use && h0 + h < a.Hkv;
        if (kFp8) {
            store_e4m3(a.pk, a.ks, row, j, x, in);
            store_e4m3(a.pv, a.vs, row, j, y, in);
        } else if (in) {
            store_bf16(a.pk, row, j, x);
            store_bf16(a.pv, row, j, y);
        }
    }
}

template <bool kFp8>
cudaError_t launch_append(const AppendArgs& a, int heads, long long groups, cudaStream_t st) {
    const long long per = kAppendThreads / kGroup;
    const dim3 grid(static_cast<unsigned>((groups + per - 1) / per));
    return heads == 4 ? launch_pdl(cache_append_kernel<kFp8, 4>, grid, dim3(kAppendThreads), 0, st, a)
                      : launch_pdl(cache_append_kernel<kFp8, 1>, grid, dim3(kAppendThreads), 0, st, a);
}

}  // namespace
}  // namespace dart

using namespace dart;

extern "C" int dart_cache_append(const dart_kv_cache* cache, int nseq, int max_pages, const int32_t* page_table,
                                 const int32_t* lens, int R, const void* k, int64_t k_stride, const void* v,
                                 int64_t v_stride, const int32_t* rows, const int32_t* n_rows, float rope_theta,
                                 int* status, void* stream) {
    if (!valid_cache(cache) || !valid_cache_pointers(cache)) return DART_ERR_INVALID;
    auto al = [](const void* p, uintptr_t n) { return p && (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; };
    if (nseq < 1 || max_pages < 1 || R < 1 || !(rope_theta > 1.0f) || !std::isfinite(rope_theta)) return DART_ERR_INVALID;
    if (!al(page_table, 4) || !al(lens, 4) || !al(n_rows, 4) || !al(k, 16) || !al(v, 16)) return DART_ERR_INVALID;
    if ((rows && !al(rows, 4)) || (status && !al(status, 4))) return DART_ERR_INVALID;
    const int64_t width = static_cast<int64_t>(cache->Hkv) * kHeadDim;
    if (k_stride < width || v_stride < width || k_stride % 8 || v_stride % 8) return DART_ERR_INVALID;
    // positions and the number of blocks are 32-bit
    if (static_cast<long long>(max_pages) * cache->page_size > 2147483647ll) return DART_ERR_INVALID;
    if (static_cast<long long>(nseq) * R > 2147483647ll / cache->Hkv) return DART_ERR_INVALID;
    int dev = 0, major = 0, minor = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&minor, cudaDevAttrComputeCapabilityMinor, dev) != cudaSuccess)
        return DART_ERR_CUDA;
    if (major != 10 || minor != 3) return DART_ERR_UNSUPPORTED;
    AppendArgs a{};
    a.nseq = nseq;
    a.max_pages = max_pages;
    a.R = R;
    a.Hkv = cache->Hkv;
    a.num_pages = cache->num_pages;
    while ((1 << a.page_log2) < cache->page_size) a.page_log2++;
    a.table = page_table;
    a.lens = lens;
    a.rows = rows;
    a.n_rows = n_rows;
    a.k = static_cast<const __nv_bfloat16*>(k);
    a.v = static_cast<const __nv_bfloat16*>(v);
    a.k_stride = k_stride;
    a.v_stride = v_stride;
    a.pk = static_cast<uint8_t*>(cache->k);
    a.pv = static_cast<uint8_t*>(cache->v);
    a.ks = cache->k_scale;
    a.vs = cache->v_scale;
    a.status = status;
    a.turns = rope_turns(rope_theta);
    const long long tokens = static_cast<long long>(nseq) * R;
    const int heads = cache->Hkv >= 4 && tokens * ((cache->Hkv + 3) / 4) >= kManyGroups ? 4 : 1;
    a.chunks = (cache->Hkv + heads - 1) / heads;
    const long long groups = tokens * a.chunks;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const cudaError_t e = cache->dtype == DART_KV_E4M3 ? launch_append<true>(a, heads, groups, st)
                                                       : launch_append<false>(a, heads, groups, st);
    return e == cudaSuccess ? DART_OK : DART_ERR_CUDA;
}
