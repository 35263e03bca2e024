// The packed matrices of adasum_fp8_pack.cu and adasum_fp8_linear.cu: e4m3 codes with a power of two for every 128
// columns of a row (or 128 x 128 block).
#pragma once

#include <cuda_fp8.h>

#include "adasum_operators.cuh"

namespace adasum {

constexpr int kFp8Block = 128;             // columns that share a step (rows too, in weights); rows of a block of step bytes
constexpr int kFp8StepBytes = 512;         // step bytes of 128 rows x 128 columns

__host__ __device__ inline int64_t fp8_blocks(int64_t n) { return (n + kFp8Block - 1) / kFp8Block; }
__host__ __device__ inline int64_t fp8_width(int64_t columns) { return fp8_blocks(columns) * kFp8Block; }
inline size_t fp8_bytes(int64_t rows, int64_t columns)
{
    const int64_t blocks = fp8_blocks(columns);
    return (size_t)rows * (size_t)(blocks * kFp8Block) + (size_t)fp8_blocks(rows) * (size_t)blocks * kFp8StepBytes;
}

// Place of a row's step bytes inside the step bytes of 128 columns.
__device__ __forceinline__ int64_t fp8_step_at(int64_t row, int64_t column_block, int64_t column_blocks)
{
    return ((row >> 7) * column_blocks + column_block) * kFp8StepBytes + ((row & 31) << 4) + (((row & 127) >> 5) << 2);
}

// Step byte of a block from the bits of its largest magnitude: 448 = 1.75 * 2^8, so the exponent less 8, one more
// where the significand exceeds 1.75.
__device__ __forceinline__ uint32_t fp8_step_byte(uint32_t top_bits)
{
    const int exponent = (int)(top_bits >> 23);              // E + 127 (0: zero or subnormal)
    return exponent == 255 ? 255u : (uint32_t)max(exponent - 8 + ((top_bits & 0x7fffffu) > 0x600000u ? 1 : 0), 1);
}
// 2^(byte - 127); Inf for 255, whose codes are 0, so that code * step is NaN.
__device__ __forceinline__ float fp8_step_value(uint32_t byte) { return __uint_as_float(byte << 23); }

// Four codes to floats, and back.
__device__ __forceinline__ void fp8_decode(uint32_t packed, float (&x)[4])
{
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(packed >> (16 * i)), __NV_E4M3);
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
        x[2 * i] = f.x;
        x[2 * i + 1] = f.y;
    }
}
__device__ __forceinline__ uint32_t fp8_encode(float a, float b, float c, float d)
{
    const uint32_t low = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
    const uint32_t high = __nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, __NV_E4M3);
    return low | high << 16;
}

}  // namespace adasum
