// The format of 8-bit activation checkpoints (see ckpt.cu), as its readers decode it.
#pragma once
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "common.cuh"

namespace anakin {
namespace ckpt {

constexpr int kMinExp = -117, kMaxExp = 120;  // exponents of a block's scale: every kept value is a normal number or zero in fp32 and bf16

// Eight codes and their block's scale byte as floats (exact: 4 bits of fraction at most).  e4m3 numbers are fp16 numbers.
__device__ __forceinline__ void decode8(const uint2& c, uint32_t scale, float (&f)[8]) {
    // 2^(scale - 127): bytes 10 .. 247 (others are nobody's checkpoint; the number is then wrong, nothing else)
    const float up = __uint_as_float(scale << 23);
    const uint32_t w[2] = {c.x, c.y};
#pragma unroll
    for (int h = 0; h < 4; ++h) {
        const __half2_raw q = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w[h >> 1] >> (16 * (h & 1))), __NV_E4M3);
        const float2 v = __half22float2(__half2(q));
        f[2 * h] = v.x * up;
        f[2 * h + 1] = v.y * up;
    }
}

// Host: checks of what every call on a checkpoint has in common.
int check(int dtype, int act, int64_t rows, int64_t cols, const uint8_t* codes, const uint8_t* scales);

}  // namespace ckpt
}  // namespace anakin
