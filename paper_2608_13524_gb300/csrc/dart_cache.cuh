// Device code shared by the paged cache's kernels: rotary angles, words of two
// bf16 values, two fp32 operations in one instruction.
#pragma once

#include <cmath>
#include <cstdint>

#include "dart_device.cuh"

namespace dart {

constexpr int kHeadDim = 128;

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

// Two fp32 operations in one instruction.
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(*reinterpret_cast<uint64_t*>(&a)), "l"(*reinterpret_cast<uint64_t*>(&b)));
    return *reinterpret_cast<float2*>(&r);
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(*reinterpret_cast<uint64_t*>(&a)), "l"(*reinterpret_cast<uint64_t*>(&b)),
        "l"(*reinterpret_cast<uint64_t*>(&c)));
    return *reinterpret_cast<float2*>(&r);
}

}  // namespace dart
