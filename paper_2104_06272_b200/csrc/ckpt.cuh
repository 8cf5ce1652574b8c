// The format of 8-bit activation checkpoints (see ckpt.cu), as its readers decode it.
#pragma once
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "common.cuh"

namespace anakin {
namespace ckpt {

constexpr int kMinExp = -117, kMaxExp = 120;  // exponents of a block's scale: every kept value is a normal number or zero in fp32 and bf16

// n / d and n % d for n < 2^31 by a multiplication (d >= 1; Granlund and Montgomery 1994): q = (n mul) >> (32 + shift).
struct FastDiv {
    uint32_t d, mul, shift;
    explicit FastDiv(uint32_t div = 1) : d(div) {
        shift = 0;
        while ((1ull << shift) < div) ++shift;
        // ceil(2^(31 + shift) / d) < 2^32, error below 2^shift: exact for n < 2^31
        mul = (uint32_t)(((1ull << (31 + shift)) + div - 1) / div);
    }
    __device__ __forceinline__ uint32_t div(uint32_t n) const { return (uint32_t)(((unsigned long long)n * mul) >> (31 + shift)); }
};

// Eight codes and their block's scale byte as floats (exact: 4 bits of fraction at most).  e4m3 numbers are fp16 numbers.
__device__ __forceinline__ void decode8(const uint2& c, uint32_t scale, float2 (&f)[4]) {
    // 2^(scale - 127): bytes 10 .. 247 (others are nobody's checkpoint; the number is then wrong, nothing else)
    const float2 up = make_float2(__uint_as_float(scale << 23), __uint_as_float(scale << 23));
    const uint32_t w[2] = {c.x, c.y};
#pragma unroll
    for (int h = 0; h < 4; ++h) {
        const __half2_raw q = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w[h >> 1] >> (16 * (h & 1))), __NV_E4M3);
        f[h] = __fmul2_rn(__half22float2(__half2(q)), up);
    }
}
__device__ __forceinline__ void decode8(const uint2& c, uint32_t scale, float (&f)[8]) {
    float2 v[4];
    decode8(c, scale, v);
#pragma unroll
    for (int h = 0; h < 4; ++h) { f[2 * h] = v[h].x; f[2 * h + 1] = v[h].y; }
}
// Where `on` has all bits, negative codes to zero (by their sign bits; the one NaN code that is written has none).
__device__ __forceinline__ uint32_t relu_codes(uint32_t w, uint32_t on) {
    uint32_t sign;  // all bits of every byte that is negative
    asm("prmt.b32 %0, %1, 0, 0xBA98;" : "=r"(sign) : "r"(w));
    return w & ~(sign & on);
}

// Host: checks of what every call on a checkpoint has in common.
int check(int dtype, int act, int64_t rows, int64_t cols, const uint8_t* codes, const uint8_t* scales);

}  // namespace ckpt
}  // namespace anakin
