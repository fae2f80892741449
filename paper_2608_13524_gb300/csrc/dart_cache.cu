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
#include <atomic>
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

int check_device() {
    static std::atomic<int> known[64];  // 1: sm_103a, 2: another
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return DART_ERR_CUDA;
    int k = known[dev].load(std::memory_order_relaxed);
    if (k == 0) {
        int major = 0, minor = 0;
        if (cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess ||
            cudaDeviceGetAttribute(&minor, cudaDevAttrComputeCapabilityMinor, dev) != cudaSuccess)
            return DART_ERR_CUDA;
        k = major == 10 && minor == 3 ? 1 : 2;
        known[dev].store(k, std::memory_order_relaxed);
    }
    return k == 1 ? DART_OK : DART_ERR_UNSUPPORTED;
}

namespace {

constexpr int kAppendThreads = 256;
constexpr int kGroup = 8;  // threads of a token's head: 8 elements of each half of a row are 16 bytes
// Four heads a group (angles once for four) where that still makes this many
// groups, else one: a few tokens are a matter of latency (eight prompts of up to
// 4096 tokens to e4m3 pages 39.8 us with four, 67 % of the copy bandwidth, and 49.9
// with one, to bf16 pages 40.4 and 44.1, to e2m1 pages and read back 78 and 103; below, no
// difference or, for the rows that eight rounds kept, 9.3 us with one and 12.4 with four).
constexpr long long kManyGroups = 9728;  // 152 SMs x 64 groups = 512 threads each
constexpr float kMinScale = 7.52316384526264005e-37f;  // 2^-120: its reciprocal is finite
constexpr float kSmallScale = 8.27180612553027675e-25f, kSmallUp = 1.152921504606846976e18f;  // 2^-80, 2^60

struct AppendArgs {
    int nseq, max_pages, R, Hkv, heads, chunks, page_log2, num_pages;  // heads of a group, groups of a token
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
// Eight codes, element 2 i in the low half of byte i, of pairs z of quotients.
__device__ __forceinline__ uint32_t to_e2m1(const float2 (&z)[4]) {
    uint32_t r;
    asm("{\n .reg .b8 a, b, c, d;\n cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n"
        " cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n mov.b32 %0, {a, b, c, d};\n}"
        : "=r"(r)
        : "f"(z[0].x), "f"(z[0].y), "f"(z[1].x), "f"(z[1].y), "f"(z[2].x), "f"(z[2].y), "f"(z[3].x), "f"(z[3].y));
    return r;
}
__device__ __forceinline__ uint32_t to_e2m1(const float2 (&z)[4], float add) {
    float2 x[4];
#pragma unroll
    for (int e = 0; e < 4; e++) x[e] = add2(z[e], make_float2(add, add));
    return to_e2m1(x);
}
// 16 of a row's elements as pairs: 8 j .. 8 j + 7 and 64 + 8 j .. of thread j of a group.
struct Pairs {
    float2 lo[4], hi[4];
};
__device__ __forceinline__ Pairs pairs_of(const uint4& a, const uint4& b) {
    const uint32_t u[4] = {a.x, a.y, a.z, a.w}, w[4] = {b.x, b.y, b.z, b.w};
    Pairs x;
#pragma unroll
    for (int e = 0; e < 4; e++) {
        x.lo[e] = make_float2(bf16_lo(u[e]), bf16_hi(u[e]));
        x.hi[e] = make_float2(bf16_lo(w[e]), bf16_hi(w[e]));
    }
    return x;
}
__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }
__device__ __forceinline__ float largest_of(const float2 (&x)[4]) {
    return max3_abs_nan(max3_abs_nan(max3_abs_nan(x[0].x, x[0].y, x[1].x), x[1].y, x[2].x), max3_abs_nan(x[2].y, x[3].x, x[3].y), 0.0f);
}
// Every thread of the warp calls it.  kRotated: x is off by 2^-21.2 of the row's largest
// element at most (a pair's length is at most 1.42 of that; its angle is off by 2^-23.3,
// sine and cosine by a unit, product and sum by half a unit), quotients by 2^-23 more; true
// where that may decide a rounding of this thread's.  What is stored then is to be stored again.
constexpr float kOff = 7e-7f;
constexpr float kTinyRow = 7.88860905221011805e-31f;  // 2^-100
template <bool kRotated>
__device__ __forceinline__ bool store_e2m1(uint8_t* pool, uint8_t* blocks, float* scales, long long row, int j, const Pairs& x, bool use) {
    float lo = largest_of(x.lo), hi = largest_of(x.hi);
    lo = max3_abs_nan(lo, __shfl_xor_sync(kFull, lo, 1), 0.0f);
    hi = max3_abs_nan(hi, __shfl_xor_sync(kFull, hi, 1), 0.0f);
    const bool lo_ok = lo < INFINITY, hi_ok = hi < INFINITY;
    lo = lo_ok ? lo : 0.0f;
    hi = hi_ok ? hi : 0.0f;
    float top = fmaxf(lo, hi);
    top = fmaxf(top, __shfl_xor_sync(kFull, top, 2));
    top = fmaxf(top, __shfl_xor_sync(kFull, top, 4));
    const int ex = top > 0.0f ? max(static_cast<int>(__float_as_uint(top) >> 23) - 137, -120) : 0;
    const float scale = __uint_as_float(static_cast<uint32_t>(127 + ex) << 23), up = __uint_as_float(static_cast<uint32_t>(127 - ex) << 23);
    const float2 sixth = quotients(lo * up, hi * up, 6.0f, 1.0f / 6.0f);
    const uint32_t pair = __nv_cvt_float2_to_fp8x2(sixth, __NV_SATFINITE, __NV_E4M3);
    const uint32_t wide = e4m3_f16(pair);
    const float2 block = __half22float2(*reinterpret_cast<const __half2*>(&wide));
    // (a block scale of 0: codes of 0)
    const float inv_lo = block.x > 0.0f ? __frcp_rn(block.x) : 0.0f, inv_hi = block.y > 0.0f ? __frcp_rn(block.y) : 0.0f;
    uint32_t code_lo, code_hi;
    bool unsure = false;
    float2 z[4];
    if constexpr (kRotated) {
        // what could be as well: the largest element on the other side of a power of two, block scales
        // and codes of numbers that far off (a code of 0 has either sign)
        const float off = top * up * kOff, off_6 = off * (1.0f / 6.0f), off_lo = off * inv_lo, off_hi = off * inv_hi;
        const uint32_t less = __nv_cvt_float2_to_fp8x2(make_float2(fmaxf(sixth.x - off_6, 0.0f), fmaxf(sixth.y - off_6, 0.0f)), __NV_SATFINITE, __NV_E4M3);
        const uint32_t more = __nv_cvt_float2_to_fp8x2(make_float2(sixth.x + off_6, sixth.y + off_6), __NV_SATFINITE, __NV_E4M3);
        uint32_t away;
#pragma unroll
        for (int e = 0; e < 4; e++) z[e] = mul2(x.lo[e], both(up * inv_lo));
        code_lo = to_e2m1(z, off_lo);
        away = code_lo ^ to_e2m1(z, -off_lo);
#pragma unroll
        for (int e = 0; e < 4; e++) z[e] = mul2(x.hi[e], both(up * inv_hi));
        code_hi = to_e2m1(z, off_hi);
        away |= code_hi ^ to_e2m1(z, -off_hi);
        unsure = less != more || (away & 0x77777777u) || (__float_as_uint(top * (1.0f - kOff)) >> 23) != (__float_as_uint(top * (1.0f + kOff)) >> 23);
        unsure = unsure || (top < kTinyRow && top > 0.0f);  // (up * inv may have left the floats, and products lie below them)
    } else {
        // quotients rounded once, as in `quotients` (-x * up is exact, and in this form -0 stays -0)
        auto divided = [&](const float2 (&v)[4], float by, float inv) {
#pragma unroll
            for (int e = 0; e < 4; e++) {
                const float2 y = mul2(v[e], both(-up)), q = mul2(y, both(-inv));
                z[e] = fma2(fma2(q, both(by), y), both(-inv), q);
            }
        };
        divided(x.lo, block.x, inv_lo);
        code_lo = to_e2m1(z);
        divided(x.hi, block.y, inv_hi);
        code_hi = to_e2m1(z);
    }
    // the block scales of the row in one word each half
    uint32_t b_lo = (lo_ok ? pair & 0xFFu : 0x7Fu) << (4 * (j & 6)), b_hi = (hi_ok ? pair >> 8 : 0x7Fu) << (4 * (j & 6));
    b_lo |= __shfl_xor_sync(kFull, b_lo, 2);
    b_hi |= __shfl_xor_sync(kFull, b_hi, 2);
    b_lo |= __shfl_xor_sync(kFull, b_lo, 4);
    b_hi |= __shfl_xor_sync(kFull, b_hi, 4);
    if (!use) return false;
    uint32_t* d = reinterpret_cast<uint32_t*>(pool + row * row_bytes(DART_KV_E2M1));
    d[j] = code_lo;
    d[8 + j] = code_hi;
    if (j == 0) {
        *reinterpret_cast<uint2*>(blocks + row * kBlocks) = make_uint2(b_lo, b_hi);
        scales[row] = scale;
    }
    return unsure;
}

// ---- numbers as sums of two floats, of which the second is at most half a unit of the
// first: for what a rounding depends on (64-bit floats would cost ten times as much here)

struct Two {
    float hi, lo;
};
__device__ __forceinline__ bool above(const Two& x, float t) { return x.hi > t || (x.hi == t && x.lo > 0.0f); }
__device__ __forceinline__ bool equal(const Two& x, float t) { return x.hi == t && x.lo == 0.0f; }
__device__ __forceinline__ Two larger(const Two& a, const Two& b) { return a.hi > b.hi || (a.hi == b.hi && a.lo > b.lo) ? a : b; }
// a * c + b * s, c and s sums of two.
__device__ __forceinline__ Two turned(float a, const Two& c, float b, const Two& s) {
    const float p = __fmul_rn(a, c.hi), q = __fmul_rn(b, s.hi), sum = __fadd_rn(p, q), bb = __fadd_rn(sum, -p);
    float rest = __fadd_rn(__fadd_rn(p, -__fadd_rn(sum, -bb)), __fadd_rn(q, -bb));  // (of the sum, exact: D. E. Knuth)
    rest += fmaf(a, c.hi, -p) + fmaf(b, s.hi, -q) + fmaf(a, c.lo, b * s.lo);
    const float hi = __fadd_rn(sum, rest);
    return Two{hi, __fadd_rn(rest, -__fadd_rn(hi, -sum))};
}
__device__ __forceinline__ Two fixed_to_two(uint64_t x, bool minus) {  // x * 2^-62, x <= 2^62
    const float hi = __ull2float_rn(x), lo = __ll2float_rn(static_cast<long long>(x) - static_cast<long long>(__float2ull_rn(hi)));
    const float by = minus ? -2.168404344971009e-19f : 2.168404344971009e-19f;  // 2^-62
    return Two{hi * by, lo * by};
}
// cos and sin of a position at frequency f to 2^-45: Taylor's series of the octant's
// angle in 64-bit fixed point (units of 2^-64, coefficients 2^64 / n!).
constexpr int kTerms = 7;
__constant__ uint64_t kSeries[kTerms][2] = {{~0ull / 1307674368000ull, ~0ull / 87178291200ull}, {~0ull / 6227020800ull, ~0ull / 479001600ull},
                                            {~0ull / 39916800ull, ~0ull / 3628800ull}, {~0ull / 362880ull, ~0ull / 40320ull},
                                            {~0ull / 5040ull, ~0ull / 720ull}, {~0ull / 120ull, ~0ull / 24ull}, {~0ull / 6ull, ~0ull / 2ull}};
__device__ __forceinline__ void rope_sincos_two(uint64_t f, int pos, Two* sn, Two* cs) {
    const uint64_t turn = static_cast<uint64_t>(static_cast<int64_t>(pos)) * f;
    const uint32_t octant = static_cast<uint32_t>(turn >> 61);
    const uint64_t part = octant & 1u ? ~(turn << 3) : turn << 3;
    const uint64_t x = __umul64hi(part, 0xC90FDAA22168C235ull), y = __umul64hi(x, x);  // pi / 4
    uint64_t p = 0, q = 0;
#pragma unroll 1
    for (int i = 0; i < kTerms; i++) {
        p = kSeries[i][0] - __umul64hi(p, y);
        q = kSeries[i][1] - __umul64hi(q, y);
    }
    uint64_t s = (x - __umul64hi(x, __umul64hi(p, y))) >> 2, c = (1ull << 62) - (__umul64hi(q, y) >> 2);
    if (((octant + 1u) & 2u) != 0u) {  // octants 1, 2, 5, 6: the other axis is nearer
        const uint64_t z = s;
        s = c;
        c = z;
    }
    *sn = fixed_to_two(s, octant >= 4u);
    *cs = fixed_to_two(c, octant >= 2u && octant < 6u);
}
// The code of |x| / block: by the halves between codes, ties to the even one.
__device__ __forceinline__ uint32_t e2m1_of(const Two& x, float block) {
    const bool minus = x.hi < 0.0f;
    const Two m{fabsf(x.hi), minus ? -x.lo : x.lo};
    constexpr float kHalf[7] = {0.25f, 0.75f, 1.25f, 1.75f, 2.5f, 3.5f, 5.0f};
    uint32_t n = 0;
#pragma unroll
    for (int i = 0; i < 7; i++) n += above(m, kHalf[i] * block) || ((i & 1) && equal(m, kHalf[i] * block));
    return block > 0.0f ? n | (minus ? 8u : 0u) : 0u;
}
__device__ __forceinline__ float e4m3_value(uint32_t code) {
    const uint32_t wide = e4m3_f16(code);
    return __low2float(*reinterpret_cast<const __half2*>(&wide));
}
// A row once more from its elements before the rotation, each to 2^-44 of its pair (at the frequencies in f), by a
// warp: a lane has elements lane, lane + 32, + 64 and + 96.  It takes 2 us of latencies and of
// fetching its instructions (in 64-bit floats 25: those run at a 64th of the rate).
__device__ __noinline__ void store_e2m1_exact(uint8_t* pool, uint8_t* blocks, float* scales, long long row, const __nv_bfloat16* src, int pos, const uint64_t* f) {
    const int lane = threadIdx.x & 31;
    Two x[4], most[4];
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; e++) v[e] = __bfloat162float(src[lane + 32 * e]);
    // rows below 2^-60 times 2^60: the remainders of smaller ones would lie below the floats
    uint32_t any = 0;
#pragma unroll
    for (int e = 0; e < 4; e++) any = max(any, fabsf(v[e]) < INFINITY ? __float_as_uint(fabsf(v[e])) : 0u);
    const int lift = __reduce_max_sync(kFull, any) < __float_as_uint(8.673617379884035e-19f) ? 60 : 0;
#pragma unroll
    for (int e = 0; e < 4; e++) v[e] *= lift ? kSmallUp : 1.0f;
#pragma unroll
    for (int e = 0; e < 2; e++) {
        Two sn, cs;
        rope_sincos_two(f[lane + 32 * e], pos, &sn, &cs);
        x[e] = turned(v[e], cs, -v[e + 2], sn);
        x[e + 2] = turned(v[e + 2], cs, v[e], sn);
    }
    // largest of a block's 16 lanes, of the row
    bool fine[4];
    Two top{0.0f, 0.0f};
#pragma unroll
    for (int e = 0; e < 4; e++) {
        most[e] = x[e].hi < 0.0f ? Two{-x[e].hi, -x[e].lo} : x[e];
        fine[e] = most[e].hi < INFINITY;
#pragma unroll
        for (int o = 1; o < 16; o <<= 1) {
            fine[e] = __shfl_xor_sync(kFull, static_cast<int>(fine[e]), o) && fine[e];
            most[e] = larger(most[e], Two{__shfl_xor_sync(kFull, most[e].hi, o), __shfl_xor_sync(kFull, most[e].lo, o)});
        }
        if (!fine[e]) most[e] = Two{0.0f, 0.0f};
        top = larger(top, most[e]);
    }
    top = larger(top, Two{__shfl_xor_sync(kFull, top.hi, 16), __shfl_xor_sync(kFull, top.lo, 16)});
    const uint32_t bits = __float_as_uint(top.hi);
    // (a power of two less something has the exponent below)
    const int ex = top.hi > 0.0f ? max(static_cast<int>(bits >> 23) - ((bits & 0x7FFFFFu) == 0u && top.lo < 0.0f ? 1 : 0) - 137 - lift, -120) : 0;
    const float up = __uint_as_float(static_cast<uint32_t>(127 - ex - lift) << 23);
#pragma unroll
    for (int e = 0; e < 4; e++) {
        const Two m{most[e].hi * up, most[e].lo * up}, y{x[e].hi * up, x[e].lo * up};
        uint32_t b = __nv_cvt_float_to_fp8(m.hi / 6.0f, __NV_SATFINITE, __NV_E4M3);  // or one beside it
        const float over = 3.0f * (e4m3_value(b) + e4m3_value(b + 1u)), under = b > 0u ? 3.0f * (e4m3_value(b) + e4m3_value(b - 1u)) : -1.0f;
        if (above(m, over) || (equal(m, over) && (b & 1u)))
            b++;
        else if (!above(m, under) && !(equal(m, under) && !(b & 1u)))
            b--;
        const uint32_t code = e2m1_of(y, e4m3_value(b)), next = __shfl_xor_sync(kFull, code, 1);
        if ((lane & 1) == 0) pool[row * row_bytes(DART_KV_E2M1) + 16 * e + lane / 2] = static_cast<uint8_t>(code | next << 4);
        if (lane % 16 == 0) blocks[row * kBlocks + 2 * e + lane / 16] = static_cast<uint8_t>(fine[e] ? b : 0x7Fu);
    }
    if (lane == 0) scales[row] = __uint_as_float(static_cast<uint32_t>(127 + ex) << 23);
}

int heads_of_group(int Hkv, long long tokens) { return Hkv >= 4 && tokens * ((Hkv + 3) / 4) >= kManyGroups ? 4 : 1; }

// Where row i of sequence s comes from and goes to (of head 0).
struct Place {
    bool use;
    int pos;
    long long src, dst;
};
__device__ __forceinline__ Place place_of(const AppendArgs& a, int s, int i, bool reports) {
    Place r{s < a.nseq && i < ld_plain(a.n_rows + min(s, a.nseq - 1)), 0, 0, 0};
    if (!r.use) return r;
    const int src_row = a.rows ? ld_plain(a.rows + static_cast<long long>(s) * a.R + i) : i;
    const long long most = static_cast<long long>(a.max_pages) << a.page_log2;
    const long long p = min(max(static_cast<long long>(ld_plain(a.lens + s)), 0ll), most) + i;
    int page = -1;
    if (p < most) page = ld_plain(a.table + static_cast<long long>(s) * a.max_pages + (p >> a.page_log2));
    if (src_row < 0 || src_row >= a.R || page < 0 || page >= a.num_pages) {
        if (a.status && reports) atomicOr(a.status, kDevBounds);
        r.use = false;
        return r;
    }
    r.pos = static_cast<int>(p);
    r.src = static_cast<long long>(s) * a.R + src_row;
    r.dst = ((static_cast<long long>(page) * a.Hkv) << a.page_log2) + (p & ((1 << a.page_log2) - 1));
    return r;
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
    const Place at = place_of(a, s, i, j == 0);
    const bool use = at.use;
    const long long src = at.src, dst = at.dst;
    const int pos = at.pos;
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
        } else if (in) {
            store_bf16(a.pk, row, j, x);
            store_bf16(a.pv, row, j, y);
        }
    }
}

// The same for e2m1.  2^-20 of a row's largest element decides a code or a block scale of a
// rotated key in a row of 400 or so, which is formed again from longer numbers, so that all
// codes are those of the definition (7 us of the 77 for eight prompts of up to 4096 tokens,
// written and read back; without, the error is 0.00014 instead of 0).  The heads of a group one
// after the other, the next one's rows on their way: a warp's 2300 instructions in a row,
// for four heads, are bound by their fetch (94 us).
constexpr int kNear = 32 / kGroup;  // tokens of a warp, whose rows are neighbours in a page
__global__ void __launch_bounds__(kAppendThreads, 3) cache_append4_kernel(const __grid_constant__ AppendArgs a) {
    __shared__ uint64_t f[kHeadDim / 2];
    pdl_trigger();
    if (threadIdx.x < kHeadDim / 2) f[threadIdx.x] = a.turns.f[threadIdx.x];
    __syncthreads();
    pdl_wait();
    const int j = threadIdx.x % kGroup;
    const long long group = static_cast<long long>(blockIdx.x) * (kAppendThreads / kGroup) + threadIdx.x / kGroup, four = group / kNear;
    const int chunk = static_cast<int>(four % a.chunks);
    const long long token = four / a.chunks * kNear + group % kNear;
    const bool there = token < static_cast<long long>(a.nseq) * a.R;  // (the last four may be fewer)
    const Place at = place_of(a, there ? static_cast<int>(token / a.R) : a.nseq, static_cast<int>(token % a.R), j == 0);
    if (!__any_sync(kFull, at.use)) return;
    const int h0 = chunk * a.heads, h1 = min(h0 + a.heads, a.Hkv);
    uint4 next[4];
    auto fetch = [&](int head) {
        const __nv_bfloat16* k = a.k + at.src * a.k_stride + head * kHeadDim + 8 * j;
        const __nv_bfloat16* v = a.v + at.src * a.v_stride + head * kHeadDim + 8 * j;
        const uint4 zero = make_uint4(0, 0, 0, 0);
        next[0] = at.use ? __ldcs(reinterpret_cast<const uint4*>(k)) : zero;
        next[1] = at.use ? __ldcs(reinterpret_cast<const uint4*>(k + 64)) : zero;
        next[2] = at.use ? __ldcs(reinterpret_cast<const uint4*>(v)) : zero;
        next[3] = at.use ? __ldcs(reinterpret_cast<const uint4*>(v + 64)) : zero;
    };
    fetch(h0);
    float sn[8], cs[8];
#pragma unroll
    for (int e = 0; e < 8; e++) rope_sincos(f[8 * j + e], at.pos, &sn[e], &cs[e]);
#pragma unroll 1
    for (int head = h0; head < h1; head++) {
        const uint4 kv[4] = {next[0], next[1], next[2], next[3]};
        if (head + 1 < h1) fetch(head + 1);
        const long long row = at.dst + (static_cast<long long>(head) << a.page_log2);
        Pairs x = pairs_of(kv[0], kv[1]);
#pragma unroll
        for (int e = 0; e < 4; e++) {
            const float2 lo = x.lo[e], hi = x.hi[e], c = make_float2(cs[2 * e], cs[2 * e + 1]), n = make_float2(sn[2 * e], sn[2 * e + 1]);
            x.lo[e] = fma2(lo, c, mul2(hi, mul2(n, both(-1.0f))));
            x.hi[e] = fma2(hi, c, mul2(lo, n));
        }
        bool unsure = store_e2m1<true>(a.pk, a.kb, a.ks, row, j, x, at.use);
        store_e2m1<false>(a.pv, a.vb, a.vs, row, j, pairs_of(kv[2], kv[3]), at.use);
        if (__any_sync(kFull, unsure && at.pos == 0)) {  // not turned at all: ties are common there, and decided as values' are
            store_e2m1<false>(a.pk, a.kb, a.ks, row, j, x, at.use && at.pos == 0);
            unsure = unsure && at.pos != 0;
        }
        for (unsigned again = __ballot_sync(kFull, unsure); again;) {
            const int lane = (__ffs(again) - 1) & ~(kGroup - 1);
            again &= ~(0xFFu << lane);
            __syncwarp();  // (after the stores above)
            store_e2m1_exact(a.pk, a.kb, a.ks, __shfl_sync(kFull, row, lane), a.k + __shfl_sync(kFull, at.src, lane) * a.k_stride + head * kHeadDim,
                             __shfl_sync(kFull, at.pos, lane), f);
        }
    }
}

cudaError_t launch_append(AppendArgs a, int type, long long tokens, cudaStream_t st) {
    a.heads = heads_of_group(a.Hkv, tokens);
    a.chunks = (a.Hkv + a.heads - 1) / a.heads;
    const bool four = type == DART_KV_E2M1;
    const long long groups = (four ? (tokens + kNear - 1) / kNear * kNear : tokens) * a.chunks, per = kAppendThreads / kGroup;
    const dim3 grid(static_cast<unsigned>((groups + per - 1) / per));
    auto launch = [&](auto* kernel) { return launch_pdl(kernel, grid, dim3(kAppendThreads), 0, st, a); };
    if (four) return launch(cache_append4_kernel);
    if (type == DART_KV_E4M3) return launch(a.heads == 4 ? cache_append_kernel<DART_KV_E4M3, 4> : cache_append_kernel<DART_KV_E4M3, 1>);
    return launch(a.heads == 4 ? cache_append_kernel<DART_KV_BF16, 4> : cache_append_kernel<DART_KV_BF16, 1>);
}

// ------------------------------------------------------------ rows back

struct ReadArgs {
    int nseq, max_pages, R, Hkv, chunks, page_log2, num_pages;
    const int32_t *table, *lens, *n_rows;
    __nv_bfloat16 *k, *v;
    long long k_stride, v_stride;
    const uint8_t *pk, *pv, *kb, *vb;
    const float *ks, *vs;
    int* status;
};

// The 16 elements that thread j of a group of 8 reads of a row: 8 j .. 8 j + 7 and
// 64 + 8 j .., so that each of its accesses lies beside its neighbours'.
template <int kType>
struct Raw {
    uint4 a, b;  // bf16: all of each; e4m3: x, y; e2m1: x
    uint2 block;
    float scale;
    __device__ __forceinline__ void load(const uint8_t* pool, const uint8_t* blocks, const float* scales, long long row, int j) {
        const uint8_t* src = pool + row * row_bytes(kType);
        if (kType == DART_KV_BF16) {
            a = reinterpret_cast<const uint4*>(src)[j];
            b = reinterpret_cast<const uint4*>(src)[8 + j];
        } else {
            if (kType == DART_KV_E4M3) {
                const uint2 x = reinterpret_cast<const uint2*>(src)[j], y = reinterpret_cast<const uint2*>(src)[8 + j];
                a = make_uint4(x.x, x.y, 0u, 0u);
                b = make_uint4(y.x, y.y, 0u, 0u);
            } else {
                a.x = reinterpret_cast<const uint32_t*>(src)[j];
                b.x = reinterpret_cast<const uint32_t*>(src)[8 + j];
                block = ld_plain(reinterpret_cast<const uint2*>(blocks) + row);
            }
            scale = ld_plain(scales + row);
        }
    }
    __device__ __forceinline__ uint4 rows_of(const uint4& c, uint32_t by) const {
        if (kType == DART_KV_BF16) return c;
        uint32_t x[4];
        if (kType == DART_KV_E4M3) {
            x[0] = e4m3_f16(c.x);
            x[1] = e4m3_f16(c.x >> 16);
            x[2] = e4m3_f16(c.y);
            x[3] = e4m3_f16(c.y >> 16);
        } else {
            e2m1_f16(c.x, x);
#pragma unroll
            for (int e = 0; e < 4; e++) x[e] = mul_f16x2(x[e], by);
        }
#pragma unroll
        for (int e = 0; e < 4; e++) {
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&x[e]));
            x[e] = pack_bf16x2(f.x * scale, f.y * scale);
        }
        return make_uint4(x[0], x[1], x[2], x[3]);
    }
    __device__ __forceinline__ void store(__nv_bfloat16* dst, int j) const {
        const uint32_t by_lo = kType == DART_KV_E2M1 ? e4m3_f16(__byte_perm(block.x, 0u, (j >> 1) * 0x11)) : 0u;
        const uint32_t by_hi = kType == DART_KV_E2M1 ? e4m3_f16(__byte_perm(block.y, 0u, (j >> 1) * 0x11)) : 0u;
        reinterpret_cast<uint4*>(dst)[j] = rows_of(a, by_lo);
        reinterpret_cast<uint4*>(dst)[8 + j] = rows_of(b, by_hi);
    }
};

// A group of 8 threads takes the keys and values of kHeads heads of one token: the same
// prompts 25 us, 6.0 TB/s, 88 % of the measured copy bandwidth (one head a group and 16
// neighbouring elements a thread 35: half of each store's sectors).
template <int kType, int kHeads>
__global__ void __launch_bounds__(kAppendThreads) cache_read_kernel(const __grid_constant__ ReadArgs a) {
    pdl_trigger();
    pdl_wait();
    const int j = threadIdx.x % kGroup;
    const long long group = static_cast<long long>(blockIdx.x) * (kAppendThreads / kGroup) + threadIdx.x / kGroup;
    const int h0 = static_cast<int>(group % a.chunks) * kHeads;
    const long long token = group / a.chunks;
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
    const long long row = ((static_cast<long long>(page) * a.Hkv + h0) << a.page_log2) + (p & ((1 << a.page_log2) - 1));
    Raw<kType> k[kHeads], v[kHeads];
#pragma unroll
    for (int h = 0; h < kHeads; h++) {
        if (h0 + h >= a.Hkv) break;
        k[h].load(a.pk, a.kb, a.ks, row + (static_cast<long long>(h) << a.page_log2), j);
        v[h].load(a.pv, a.vb, a.vs, row + (static_cast<long long>(h) << a.page_log2), j);
    }
#pragma unroll
    for (int h = 0; h < kHeads; h++) {
        if (h0 + h >= a.Hkv) break;
        k[h].store(a.k + token * a.k_stride + (h0 + h) * kHeadDim, j);
        v[h].store(a.v + token * a.v_stride + (h0 + h) * kHeadDim, j);
    }
}

template <int kType>
cudaError_t launch_read(const ReadArgs& a, int heads, long long groups, cudaStream_t st) {
    const long long per = kAppendThreads / kGroup;
    const dim3 grid(static_cast<unsigned>((groups + per - 1) / per));
    return heads == 4 ? launch_pdl(cache_read_kernel<kType, 4>, grid, dim3(kAppendThreads), 0, st, a)
                      : launch_pdl(cache_read_kernel<kType, 1>, grid, dim3(kAppendThreads), 0, st, a);
}

// ------------------------------------------------------------ whole pages

constexpr int kCopyThreads = 256, kCopyVecs = 8;  // 16-byte vectors of a thread on their way at a time
constexpr int kSlice = kCopyThreads * kCopyVecs;   // vectors of a unit of work, 32 KB

struct CopyArgs {
    int max_pairs, num_pages, slices;  // slices of a page: of its arrays, one after the other
    const int2* pairs;
    const int32_t* count;
    uint4* base[6];     // pages of keys and values, their scales, their block scales
    int page_vecs[6];   // 16-byte vectors of a page in each; 0: none
    int slices_to[6];   // slices up to and with this array
    int* status;
};

// A unit is up to 32 KB of one of a page's arrays, so that a few copies of
// large pages and many of small ones load every SM alike.  507 MB of copies take 79 us, 6.4 TB/s,
// 94 % of the measured copy bandwidth (with compaction around them 104 to 107 us; four vectors
// a thread on their way instead of eight 108, units that go across the arrays 111).
__global__ void __launch_bounds__(kCopyThreads) cache_copy_kernel(const __grid_constant__ CopyArgs a) {
    pdl_trigger();
    pdl_wait();
    const int n = min(max(ld_plain(a.count), 0), a.max_pairs);
    const long long units = static_cast<long long>(n) * a.slices;
    for (long long u = blockIdx.x; u < units; u += gridDim.x) {
        const int pair = static_cast<int>(u / a.slices);
        int slice = static_cast<int>(u - static_cast<long long>(pair) * a.slices), i = 0;
        const int2 p = ld_plain(a.pairs + pair);
        if (p.x < 0 || p.x >= a.num_pages || p.y < 0 || p.y >= a.num_pages) {
            if (a.status && slice == 0 && threadIdx.x == 0) atomicOr(a.status, kDevBounds);
            continue;
        }
#pragma unroll
        for (int k = 0; k < 5; k++) i += slice >= a.slices_to[k];
        if (i > 0) slice -= a.slices_to[i - 1];
        const int vecs = a.page_vecs[i], v0 = slice * kSlice + static_cast<int>(threadIdx.x);
        const uint4* from = a.base[i] + static_cast<long long>(p.x) * vecs + v0;
        uint4* to = a.base[i] + static_cast<long long>(p.y) * vecs + v0;
        uint4 x[kCopyVecs];
#pragma unroll
        for (int e = 0; e < kCopyVecs; e++)
            if (v0 + e * kCopyThreads < vecs) x[e] = __ldcs(from + e * kCopyThreads);
#pragma unroll
        for (int e = 0; e < kCopyVecs; e++)
            if (v0 + e * kCopyThreads < vecs) to[e * kCopyThreads] = x[e];
    }
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
    const cudaError_t e = launch_append(a, cache->dtype, tokens, static_cast<cudaStream_t>(stream));
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
    const long long tokens = static_cast<long long>(nseq) * R;
    const int heads = heads_of_group(cache->Hkv, tokens);
    a.chunks = (cache->Hkv + heads - 1) / heads;
    const long long groups = tokens * a.chunks;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const cudaError_t e = cache->dtype == DART_KV_E2M1   ? launch_read<DART_KV_E2M1>(a, heads, groups, st)
                          : cache->dtype == DART_KV_E4M3 ? launch_read<DART_KV_E4M3>(a, heads, groups, st)
                                                         : launch_read<DART_KV_BF16>(a, heads, groups, st);
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
        a.slices += static_cast<int>((all + kSlice - 1) / kSlice);
        a.slices_to[i] = a.slices;
    }
    if (vecs > 2147483647ll - kSlice) return DART_ERR_INVALID;
    if (const int rc = check_device()) return rc;
    // every SM with as many blocks as it holds, fewer where there cannot be that many units
    const long long units = static_cast<long long>(max_pairs) * a.slices;
    const dim3 grid(static_cast<unsigned>(std::min(units, 8ll * 152)));
    return launch_pdl(cache_copy_kernel, grid, dim3(kCopyThreads), 0, static_cast<cudaStream_t>(stream), a) == cudaSuccess ? DART_OK : DART_ERR_CUDA;
}
