// Writes rows of keys and values into the pages of the cache: keys rotated at
// their position, both rounded to bf16 or quantised to e4m3 with one scale
// per token and head or to e2m1 with a scale for every 16 elements beside it;
// and reads rows back.  Contract: include/dart_cache.h.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
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
    if (c->dtype != DART_KV_BF16 && c->dtype != DART_KV_E4M3 && c->dtype != DART_KV_E2M1) return false;
    // rows of dh elements are numbered by 32-bit TMA coordinates
    return static_cast<long long>(c->num_pages) * c->Hkv <= (2147483647ll - 128) / c->page_size;
}

bool valid_cache_pointers(const dart_kv_cache* c) {
    auto ok = [](const void* p) { return p && (reinterpret_cast<uintptr_t>(p) & 15u) == 0; };
    if (!ok(c->k) || !ok(c->v)) return false;
    if (c->dtype == DART_KV_BF16) return !c->k_scale && !c->v_scale;
    return ok(c->k_scale) && ok(c->v_scale) && (c->dtype != DART_KV_E2M1 || (ok(c->k_block) && ok(c->v_block)));
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
    uint8_t *kb, *vb;
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

__device__ __forceinline__ float max3_abs_nan(float a, float b, float c) {  // NaN if one is
    float r;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
// Eight codes, element 2 i in the low half of byte i; `up` a power of two.
__device__ __forceinline__ uint32_t to_e2m1(const float (&x)[8], float up, float block, float inv) {
    uint32_t b[4];
#pragma unroll
    for (int e = 0; e < 4; e++) {
        const float2 z = quotients(x[2 * e] * up, x[2 * e + 1] * up, block, inv);
        asm("{\n .reg .b8 t;\n cvt.rn.satfinite.e2m1x2.f32 t, %1, %2;\n cvt.u32.u8 %0, t;\n}" : "=r"(b[e]) : "f"(z.y), "f"(z.x));
    }
    return __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
}
// Thread j of a group has half of block j / 2 and half of block 4 + j / 2 (every
// thread of the warp calls it).
__device__ __forceinline__ void store_e2m1(uint8_t* pool, uint8_t* blocks, float* scales, long long row, int j, const Row& x, bool use) {
    float lo = max3_abs_nan(max3_abs_nan(max3_abs_nan(x.lo[0], x.lo[1], x.lo[2]), x.lo[3], x.lo[4]), max3_abs_nan(x.lo[5], x.lo[6], x.lo[7]), 0.0f);
    float hi = max3_abs_nan(max3_abs_nan(max3_abs_nan(x.hi[0], x.hi[1], x.hi[2]), x.hi[3], x.hi[4]), max3_abs_nan(x.hi[5], x.hi[6], x.hi[7]), 0.0f);
    lo = max3_abs_nan(lo, __shfl_xor_sync(kFull, lo, 1), 0.0f);
    hi = max3_abs_nan(hi, __shfl_xor_sync(kFull, hi, 1), 0.0f);
    const bool lo_ok = lo < INFINITY, hi_ok = hi < INFINITY;
    float top = fmaxf(lo_ok ? lo : 0.0f, hi_ok ? hi : 0.0f);
    top = fmaxf(top, __shfl_xor_sync(kFull, top, 2));
    top = fmaxf(top, __shfl_xor_sync(kFull, top, 4));
    const int ex = top > 0.0f ? max(static_cast<int>(__float_as_uint(top) >> 23) - 137, -120) : 0;
    const float scale = __uint_as_float(static_cast<uint32_t>(127 + ex) << 23), up = __uint_as_float(static_cast<uint32_t>(127 - ex) << 23);
    const float2 sixth = quotients(lo_ok ? lo * up : 0.0f, hi_ok ? hi * up : 0.0f, 6.0f, 1.0f / 6.0f);
    const uint32_t pair = __nv_cvt_float2_to_fp8x2(sixth, __NV_SATFINITE, __NV_E4M3);
    const uint32_t wide = e4m3_f16(pair);
    const float2 block = __half22float2(*reinterpret_cast<const __half2*>(&wide));
    // (a block scale of 0: codes of 0)
    const uint32_t code_lo = to_e2m1(x.lo, up, block.x, block.x > 0.0f ? __frcp_rn(block.x) : 0.0f);
    const uint32_t code_hi = to_e2m1(x.hi, up, block.y, block.y > 0.0f ? __frcp_rn(block.y) : 0.0f);
    // the block scales of the row in one word each half
    uint32_t b_lo = (lo_ok ? pair & 0xFFu : 0x7Fu) << (4 * (j & 6)), b_hi = (hi_ok ? pair >> 8 : 0x7Fu) << (4 * (j & 6));
    b_lo |= __shfl_xor_sync(kFull, b_lo, 2);
    b_hi |= __shfl_xor_sync(kFull, b_hi, 2);
    b_lo |= __shfl_xor_sync(kFull, b_lo, 4);
    b_hi |= __shfl_xor_sync(kFull, b_hi, 4);
    if (!use) return;
    uint32_t* d = reinterpret_cast<uint32_t*>(pool + row * row_bytes(DART_KV_E2M1));
    d[j] = code_lo;
    d[8 + j] = code_hi;
    if (j == 0) {
        *reinterpret_cast<uint2*>(blocks + row * kBlocks) = make_uint2(b_lo, b_hi);
        scales[row] = scale;
    }
}

// A group of 8 threads takes kHeads heads of one token, so that the angles of
// its position are computed once for all of them and every head's loads are
// in flight together.
template <int kType, int kHeads>
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
        if (kType == DART_KV_E4M3) {
            store_e4m3(a.pk, a.ks, row, j, x, in);
            store_e4m3(a.pv, a.vs, row, j, y, in);
        } else if (kType == DART_KV_E2M1) {
            store_e2m1(a.pk, a.kb, a.ks, row, j, x, in);
            store_e2m1(a.pv, a.vb, a.vs, row, j, y, in);
        } else if (in) {
            store_bf16(a.pk, row, j, x);
            store_bf16(a.pv, row, j, y);
        }
    }
}

template <int kType>
cudaError_t launch_append(const AppendArgs& a, int heads, long long groups, cudaStream_t st) {
    const long long per = kAppendThreads / kGroup;
    const dim3 grid(static_cast<unsigned>((groups + per - 1) / per));
    return heads == 4 ? launch_pdl(cache_append_kernel<kType, 4>, grid, dim3(kAppendThreads), 0, st, a)
                      : launch_pdl(cache_append_kernel<kType, 1>, grid, dim3(kAppendThreads), 0, st, a);
}

// ------------------------------------------------------------ rows back

struct ReadArgs {
    int nseq, max_pages, R, Hkv, page_log2, num_pages;
    const int32_t *table, *lens, *n_rows;
    __nv_bfloat16 *k, *v;
    long long k_stride, v_stride;
    const uint8_t *pk, *pv, *kb, *vb;
    const float *ks, *vs;
    int* status;
};

// The 16 elements that thread j of a group of 8 reads of a row: 16 j .. 16 j + 15.
template <int kType>
struct Raw {
    uint4 a, b;   // bf16: all of it; e4m3: a; e2m1: a.x, a.y
    uint32_t block;
    float scale;
    __device__ __forceinline__ void load(const uint8_t* pool, const uint8_t* blocks, const float* scales, long long row, int j) {
        const uint8_t* src = pool + row * row_bytes(kType) + j * (row_bytes(kType) / 8);
        if (kType == DART_KV_BF16) {
            a = *reinterpret_cast<const uint4*>(src);
            b = *reinterpret_cast<const uint4*>(src + 16);
        } else {
            if (kType == DART_KV_E4M3) {
                a = *reinterpret_cast<const uint4*>(src);
            } else {
                const uint2 x = *reinterpret_cast<const uint2*>(src);
                a = make_uint4(x.x, x.y, 0u, 0u);
                block = ld_plain(blocks + row * kBlocks + j);
            }
            scale = ld_plain(scales + row);
        }
    }
    __device__ __forceinline__ void store(__nv_bfloat16* dst) const {
        uint4 y[2];
        if (kType == DART_KV_BF16) {
            y[0] = a;
            y[1] = b;
        } else {
            uint32_t x[8];
            if (kType == DART_KV_E4M3) {
                const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    x[2 * e] = e4m3_f16(w[e]);
                    x[2 * e + 1] = e4m3_f16(w[e] >> 16);
                }
            } else {
                uint32_t lo[4], hi[4];
                e2m1_f16(a.x, lo);
                e2m1_f16(a.y, hi);
                const uint32_t by = e4m3_f16(block | block << 8);
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    x[e] = mul_f16x2(lo[e], by);
                    x[4 + e] = mul_f16x2(hi[e], by);
                }
            }
            uint32_t r[8];
#pragma unroll
            for (int e = 0; e < 8; e++) {
                const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&x[e]));
                r[e] = pack_bf16x2(f.x * scale, f.y * scale);
            }
            y[0] = make_uint4(r[0], r[1], r[2], r[3]);
            y[1] = make_uint4(r[4], r[5], r[6], r[7]);
        }
        reinterpret_cast<uint4*>(dst)[0] = y[0];
        reinterpret_cast<uint4*>(dst)[1] = y[1];
    }
};

// A group of 8 threads takes the keys and values of one head of one token.
template <int kType>
__global__ void __launch_bounds__(kAppendThreads) cache_read_kernel(const __grid_constant__ ReadArgs a) {
    pdl_trigger();
    pdl_wait();
    const int j = threadIdx.x % kGroup;
    const long long group = static_cast<long long>(blockIdx.x) * (kAppendThreads / kGroup) + threadIdx.x / kGroup;
    const int head = static_cast<int>(group % a.Hkv);
    const long long token = group / a.Hkv;
    const int s = static_cast<int>(token / a.R), i = static_cast<int>(token % a.R);
    if (s >= a.nseq || i >= ld_plain(a.n_rows + s)) return;
    const long long most = static_cast<long long>(a.max_pages) << a.page_log2;
    const long long p = min(max(static_cast<long long>(ld_plain(a.lens + s)), 0ll), most) + i;
    int page = -1;
    if (p < most) page = ld_plain(a.table + static_cast<long long>(s) * a.max_pages + (p >> a.page_log2));
    if (page < 0 || page >= a.num_pages) {
        if (a.status && j == 0) atomicOr(a.status, kDevBounds);
        return;
    }
    const long long row = ((static_cast<long long>(page) * a.Hkv + head) << a.page_log2) + (p & ((1 << a.page_log2) - 1));
    Raw<kType> k, v;
    k.load(a.pk, a.kb, a.ks, row, j);
    v.load(a.pv, a.vb, a.vs, row, j);
    k.store(a.k + token * a.k_stride + head * kHeadDim + kBlockDim * j);
    v.store(a.v + token * a.v_stride + head * kHeadDim + kBlockDim * j);
}

// ------------------------------------------------------------ whole pages

constexpr int kCopyThreads = 256, kCopyVecs = 4;  // 16-byte vectors of a thread on their way at a time
constexpr int kSlice = kCopyThreads * kCopyVecs;   // vectors of a unit of work, 16 KB

struct CopyArgs {
    int max_pairs, num_pages, slices;
    const int2* pairs;
    const int32_t* count;
    uint4* base[6];     // pages of keys and values, their scales, their block scales
    int page_vecs[6];   // 16-byte vectors of a page in each; 0: none
    int* status;
};

// A unit is 16 KB of a page's arrays, one after the other, so that a few copies of
// large pages and many of small ones load every SM alike.
__global__ void __launch_bounds__(kCopyThreads) cache_copy_kernel(const __grid_constant__ CopyArgs a) {
    pdl_trigger();
    pdl_wait();
    const int n = min(max(ld_plain(a.count), 0), a.max_pairs);
    const long long units = static_cast<long long>(n) * a.slices;
    for (long long u = blockIdx.x; u < units; u += gridDim.x) {
        const int pair = static_cast<int>(u / a.slices), slice = static_cast<int>(u - static_cast<long long>(pair) * a.slices);
        const int2 p = ld_plain(a.pairs + pair);
        if (p.x < 0 || p.x >= a.num_pages || p.y < 0 || p.y >= a.num_pages) {
            if (a.status && slice == 0 && threadIdx.x == 0) atomicOr(a.status, kDevBounds);
            continue;
        }
        uint4 x[kCopyVecs];
        uint4* to[kCopyVecs];
#pragma unroll
        for (int e = 0; e < kCopyVecs; e++) {
            int v = slice * kSlice + e * kCopyThreads + static_cast<int>(threadIdx.x);
            to[e] = nullptr;
#pragma unroll
            for (int i = 0; i < 6; i++) {
                if (to[e] == nullptr && v < a.page_vecs[i]) {
                    x[e] = __ldcs(a.base[i] + static_cast<long long>(p.x) * a.page_vecs[i] + v);
                    to[e] = a.base[i] + static_cast<long long>(p.y) * a.page_vecs[i] + v;
                }
                v -= to[e] == nullptr ? a.page_vecs[i] : 0;
            }
        }
#pragma unroll
        for (int e = 0; e < kCopyVecs; e++)
            if (to[e]) *to[e] = x[e];
    }
}

// 0: an sm_103a device is the current one.
int check_device() {
    int dev = 0, major = 0, minor = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&minor, cudaDevAttrComputeCapabilityMinor, dev) != cudaSuccess)
        return DART_ERR_CUDA;
    return major == 10 && minor == 3 ? DART_OK : DART_ERR_UNSUPPORTED;
}
bool aligned(const void* p, uintptr_t n) { return p && (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

}  // namespace
}  // namespace dart

using namespace dart;

extern "C" int dart_cache_append(const dart_kv_cache* cache, int nseq, int max_pages, const int32_t* page_table,
                                 const int32_t* lens, int R, const void* k, int64_t k_stride, const void* v,
                                 int64_t v_stride, const int32_t* rows, const int32_t* n_rows, float rope_theta,
                                 int* status, void* stream) {
    if (!valid_cache(cache) || !valid_cache_pointers(cache)) return DART_ERR_INVALID;
    auto al = aligned;
    if (nseq < 1 || max_pages < 1 || R < 1 || !(rope_theta > 1.0f) || !std::isfinite(rope_theta)) return DART_ERR_INVALID;
    if (!al(page_table, 4) || !al(lens, 4) || !al(n_rows, 4) || !al(k, 16) || !al(v, 16)) return DART_ERR_INVALID;
    if ((rows && !al(rows, 4)) || (status && !al(status, 4))) return DART_ERR_INVALID;
    const int64_t width = static_cast<int64_t>(cache->Hkv) * kHeadDim;
    if (k_stride < width || v_stride < width || k_stride % 8 || v_stride % 8) return DART_ERR_INVALID;
    // positions and the number of blocks are 32-bit
    if (static_cast<long long>(max_pages) * cache->page_size > 2147483647ll) return DART_ERR_INVALID;
    if (static_cast<long long>(nseq) * R > 2147483647ll / cache->Hkv) return DART_ERR_INVALID;
    if (const int rc = check_device()) return rc;
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
    a.kb = static_cast<uint8_t*>(cache->k_block);
    a.vb = static_cast<uint8_t*>(cache->v_block);
    a.status = status;
    a.turns = rope_turns(rope_theta);
    const long long tokens = static_cast<long long>(nseq) * R;
    const int heads = cache->Hkv >= 4 && tokens * ((cache->Hkv + 3) / 4) >= kManyGroups ? 4 : 1;
    a.chunks = (cache->Hkv + heads - 1) / heads;
    const long long groups = tokens * a.chunks;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const cudaError_t e = cache->dtype == DART_KV_E2M1   ? launch_append<DART_KV_E2M1>(a, heads, groups, st)
                          : cache->dtype == DART_KV_E4M3 ? launch_append<DART_KV_E4M3>(a, heads, groups, st)
                                                         : launch_append<DART_KV_BF16>(a, heads, groups, st);
    return e == cudaSuccess ? DART_OK : DART_ERR_CUDA;
}

extern "C" int dart_cache_read(const dart_kv_cache* cache, int nseq, int max_pages, const int32_t* page_table, const int32_t* lens,
                               int R, void* k, int64_t k_stride, void* v, int64_t v_stride, const int32_t* n_rows, int* status,
                               void* stream) {
    if (!valid_cache(cache) || !valid_cache_pointers(cache)) return DART_ERR_INVALID;
    if (nseq < 1 || max_pages < 1 || R < 1) return DART_ERR_INVALID;
    if (!aligned(page_table, 4) || !aligned(lens, 4) || !aligned(n_rows, 4) || !aligned(k, 16) || !aligned(v, 16)) return DART_ERR_INVALID;
    if (status && !aligned(status, 4)) return DART_ERR_INVALID;
    const int64_t width = static_cast<int64_t>(cache->Hkv) * kHeadDim;
    if (k_stride < width || v_stride < width || k_stride % 8 || v_stride % 8) return DART_ERR_INVALID;
    if (static_cast<long long>(max_pages) * cache->page_size > 2147483647ll) return DART_ERR_INVALID;
    if (static_cast<long long>(nseq) * R > 2147483647ll / cache->Hkv) return DART_ERR_INVALID;
    if (const int rc = check_device()) return rc;
    ReadArgs a{};
    a.nseq = nseq;
    a.max_pages = max_pages;
    a.R = R;
    a.Hkv = cache->Hkv;
    while ((1 << a.page_log2) < cache->page_size) a.page_log2++;
    a.num_pages = cache->num_pages;
    a.table = page_table;
    a.lens = lens;
    a.n_rows = n_rows;
    a.k = static_cast<__nv_bfloat16*>(k);
    a.v = static_cast<__nv_bfloat16*>(v);
    a.k_stride = k_stride;
    a.v_stride = v_stride;
    a.pk = static_cast<const uint8_t*>(cache->k);
    a.pv = static_cast<const uint8_t*>(cache->v);
    a.kb = static_cast<const uint8_t*>(cache->k_block);
    a.vb = static_cast<const uint8_t*>(cache->v_block);
    a.ks = cache->k_scale;
    a.vs = cache->v_scale;
    a.status = status;
    const long long groups = static_cast<long long>(nseq) * R * cache->Hkv, per = kAppendThreads / kGroup;
    const dim3 grid(static_cast<unsigned>((groups + per - 1) / per)), block(kAppendThreads);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const cudaError_t e = cache->dtype == DART_KV_E2M1   ? launch_pdl(cache_read_kernel<DART_KV_E2M1>, grid, block, 0, st, a)
                          : cache->dtype == DART_KV_E4M3 ? launch_pdl(cache_read_kernel<DART_KV_E4M3>, grid, block, 0, st, a)
                                                         : launch_pdl(cache_read_kernel<DART_KV_BF16>, grid, block, 0, st, a);
    return e == cudaSuccess ? DART_OK : DART_ERR_CUDA;
}

extern "C" int dart_cache_copy_pages(const dart_kv_cache* cache, const int32_t* pairs, int max_pairs, const int32_t* count, int* status,
                                     void* stream) {
    if (!valid_cache(cache) || !valid_cache_pointers(cache)) return DART_ERR_INVALID;
    if (max_pairs < 1 || !aligned(pairs, 8) || !aligned(count, 4) || (status && !aligned(status, 4))) return DART_ERR_INVALID;
    CopyArgs a{};
    a.max_pairs = max_pairs;
    a.num_pages = cache->num_pages;
    a.pairs = reinterpret_cast<const int2*>(pairs);
    a.count = count;
    a.status = status;
    const int rows = cache->Hkv * cache->page_size;  // (of a page: a multiple of 16)
    void* const base[6] = {cache->k, cache->v, cache->k_scale, cache->v_scale, cache->k_block, cache->v_block};
    long long vecs = 0;
    for (int i = 0; i < 6; i++) {
        const int bytes = i < 2 ? row_bytes(cache->dtype) : i < 4 ? (cache->dtype == DART_KV_BF16 ? 0 : 4) : cache->dtype == DART_KV_E2M1 ? kBlocks : 0;
        const long long all = static_cast<long long>(rows) * bytes / 16;
        a.base[i] = static_cast<uint4*>(base[i]);
        a.page_vecs[i] = static_cast<int>(all);
        vecs += all;
    }
    if (vecs > 2147483647ll - kSlice) return DART_ERR_INVALID;
    if (const int rc = check_device()) return rc;
    a.slices = static_cast<int>((vecs + kSlice - 1) / kSlice);
    // every SM with as many blocks as it holds, fewer where there cannot be that many units
    const long long units = static_cast<long long>(max_pairs) * a.slices;
    const dim3 grid(static_cast<unsigned>(std::min(units, 8ll * 152)));
    return launch_pdl(cache_copy_kernel, grid, dim3(kCopyThreads), 0, static_cast<cudaStream_t>(stream), a) == cudaSuccess ? DART_OK : DART_ERR_CUDA;
}
