// Matrices held in 8 bits with a scale for each block of 128 columns (tt.h, tt_quantize_fp8): what the kernels that write
// them and the products that read them share.
#pragma once

#include "contract.hip.h"

namespace tt {

constexpr int kFp8Block = TT_FP8_BLOCK;
TT_HD int64_t fp8_blocks(int64_t cols) { return (cols + kFp8Block - 1) / kFp8Block; }

// The largest magnitude of a block is found on the bits of |x|: as unsigned integers they are in the order of the magnitudes,
// infinity above the finite values and NaN above infinity, where fmaxf would drop a NaN.
__device__ __forceinline__ uint32_t magnitude_bits(float x) { return __float_as_uint(x) & 0x7fffffffu; }
constexpr uint32_t kFp8Smallest = (127u - 100u) << 23; // 2^-100: below it 448 / a would leave float32's range
// scale = a / 448 and the factor of the values, 448 / a, each rounded once (the two divisions are per block of 128 or more).
struct Fp8Scale {
    float scale, factor;
};
__device__ __forceinline__ Fp8Scale fp8_scale(uint32_t largest)
{
    const float a = __uint_as_float(max(largest, kFp8Smallest));
    return {a / 448.0f, 448.0f / a};
}
// Four values to nearest even.  |x| <= a keeps x * factor within 448 * (1 + 2^-23), which rounds to 448: nothing overflows.
__device__ __forceinline__ uint32_t pack_fp8x4(float a, float b, float c, float d)
{
    const int low = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, low, true);
}

} // namespace tt
