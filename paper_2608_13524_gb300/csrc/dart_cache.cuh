// Device code shared by the paged cache's kernels: rotary angles, words of two
// bf16 values, two fp32 operations in one instruction.
#pragma once

#include <cmath>
#include <cstdint>

#include "../../include/dart_cache.h"
#include "dart_device.cuh"

namespace dart {

int check_device();  // DART_OK: the current device is an sm_103a one

constexpr int kHeadDim = 128;
constexpr int kBlockDim = 16, kBlocks = kHeadDim / kBlockDim;  // elements of a block scale (e2m1), block scales of a row

// Bytes of a row of head elements in pages of type DART_KV_*.
__host__ __device__ constexpr int row_bytes(int type) {
    return type == DART_KV_BF16 ? 2 * kHeadDim : type == DART_KV_E4M3 ? kHeadDim : kHeadDim / 2;
}

// RoPE frequencies as fractions of a turn in units of 2^-64: the integer part of
// theta^(-2t/dh) / (2 pi) * 2^64, computed in fp64.  pos * f modulo 2^64 is the
// exact fraction of a turn of that frequency, so far positions lose nothing but
// pos * 2^-54 of a turn of the frequency's own (an fp32 product is off by
// pos * 2^-24 radians).
struct RopeTurns {
    uint64_t f[kHeadDim / 2];
};
inline const RopeTurns& rope_turns(float theta) {
    thread_local RopeTurns r;  // 64 powers cost microseconds of every call
    thread_local float of = 0.0f;
    if (of != theta) {
        for (int t = 0; t < kHeadDim / 2; t++)
            r.f[t] = static_cast<uint64_t>(
                std::ldexp(std::pow(static_cast<double>(theta), -2.0 * t / kHeadDim) / 6.283185307179586477, 64));
        of = theta;
    }
    return r;
}

// cos and sin of position pos at frequency f: the top 32 bits of the turn, as
// half turns in [-1, 1), rounded to fp32 (2^-26 of a turn at most, which moves a
// rotated pair by 2^-23.3 of its length).
__device__ __forceinline__ void rope_sincos(uint64_t f, int pos, float* sn, float* cs) {
    const int32_t top = static_cast<int32_t>((static_cast<uint64_t>(static_cast<int64_t>(pos)) * f) >> 32);
    sincospif(static_cast<float>(top) * 4.656612873077392578e-10f, sn, cs);  // 2^-31
}

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t pack_bf16x2(float a, float b) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
    return r;
}

// The eight e2m1 codes of a word as f16 pairs, elements 2 i, 2 i + 1 in x[i]: exact.
__device__ __forceinline__ void e2m1_f16(uint32_t word, uint32_t (&x)[4]) {
    asm("{\n .reg .b8 a, b, c, d;\n mov.b32 {a, b, c, d}, %4;\n cvt.rn.f16x2.e2m1x2 %0, a;\n cvt.rn.f16x2.e2m1x2 %1, b;\n"
        " cvt.rn.f16x2.e2m1x2 %2, c;\n cvt.rn.f16x2.e2m1x2 %3, d;\n}"
        : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3])
        : "r"(word));
}
// Elements 4 half .. 4 half + 3 alone.
__device__ __forceinline__ void e2m1_f16(uint32_t word, int half, uint32_t (&x)[2]) {
    asm("{\n .reg .b8 a, b, c, d;\n mov.b32 {a, b, c, d}, %2;\n cvt.rn.f16x2.e2m1x2 %0, a;\n cvt.rn.f16x2.e2m1x2 %1, b;\n}"
        : "=r"(x[0]), "=r"(x[1])
        : "r"(half ? word >> 16 : word));
}
// Two e4m3 codes as an f16 pair: exact.
__device__ __forceinline__ uint32_t e4m3_f16(uint32_t two) {
    uint32_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"(static_cast<uint16_t>(two)));
    return r;
}
// Whether a row of codes has an element that is not 0, as far as that can be seen at little
// cost: from an e2m1 row's block scales, from all e4m3 codes (bits of some, or'ed).  A row of
// zeros may have any scale (1 where the cache writes left it), so it must have no part in
// what other rows are measured by: beside values of 2^-13 it would leave their f16 weights 2^-23.
__device__ __forceinline__ bool e2m1_in_use(const uint2& blocks) { return ((blocks.x | blocks.y) & 0x7F7F7F7Fu) != 0u; }
__device__ __forceinline__ uint32_t e4m3_bits(const uint4& x) { return (x.x | x.y | x.z | x.w) & 0x7F7F7F7Fu; }
// Products of f16 pairs (of an e2m1 code and a block scale: at most 6 significant
// bits between 2^-10 and 2688, exact).
__device__ __forceinline__ uint32_t mul_f16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

// Two fp32 operations in one instruction.
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(*reinterpret_cast<uint64_t*>(&a)), "l"(*reinterpret_cast<uint64_t*>(&b)));
    return *reinterpret_cast<float2*>(&r);
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(*reinterpret_cast<uint64_t*>(&a)), "l"(*reinterpret_cast<uint64_t*>(&b)));
    return *reinterpret_cast<float2*>(&r);
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(*reinterpret_cast<uint64_t*>(&a)), "l"(*reinterpret_cast<uint64_t*>(&b)),
        "l"(*reinterpret_cast<uint64_t*>(&c)));
    return *reinterpret_cast<float2*>(&r);
}

}  // namespace dart
