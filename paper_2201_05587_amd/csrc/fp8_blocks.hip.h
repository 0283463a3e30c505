// Matrices held in 8 bits with a scale for each block of 128 columns (tt.h, tt_quantize_fp8): what the kernels that write
// them and the products that read them share.
#pragma once

#include "contract.hip.h"

namespace tt {

constexpr int kFp8Block = TT_FP8_BLOCK;
TT_HD int64_t fp8_blocks(int64_t cols) { return (cols + kFp8Block - 1) / kFp8Block; }

// The largest magnitude of a block is found on the bits of |x|: as unsigned integers they are in the order of the magnitudes,
// infinity above the finite values and NaN above infinity, where fmaxf would drop a NaN.
constexpr uint32_t kFp8Smallest = (127u - 100u) << 23; // 2^-100: what is smaller is held with its scale, and 448 / a stays in range
// scale = a / 448 and the factor of the values, 448 / a, each rounded once.  All lanes of a block form both, so that two of the
// compiler's divisions (some 24 instructions) would cost a lane of eight values as much as its values; from an approximate reciprocal
// and the remainder of the quotient they are nine.  Checked for every mantissa of a: both are the rounded quotients.
struct Fp8Scale {
    float scale, factor;
    float rest; // 448 / a - factor, to 24 bits
    // x * 448 / a, to be rounded to e4m3 as if it had never been rounded before.
    // bf16 x: rounded to float32 once, instead of factor and product each.  An 8-bit by 3-bit product over an 8-bit one that is no
    // midpoint of e4m3 is 2^-13 of itself away from one, so that no second rounding lands there.
    // float32 x: rounded to the odd neighbour where it is not exact, which no midpoint is.  (What is left over is itself off by some
    // 2^-47 of y; where y is a midpoint and not exact it is at least 2^-30 of it, a 24-bit product's distance from a 29-bit one.)
    template <int DT> __device__ __forceinline__ float value(float x) const
    {
#pragma clang fp contract(off) // (v is the rounded product, also where it is added to)
        const float v = x * factor, e = fmaf(x, rest, fmaf(x, factor, -v)), y = v + e;
        if constexpr (DT == TT_BF16) return y;
        const float over = e - (y - v);
        const uint32_t b = __float_as_uint(y), away = (b ^ __float_as_uint(over)) >> 31;
        return fabsf(over) > fabsf(y) * 0x1p-40f && (b & 1u) == 0u ? __uint_as_float(b + 1u - 2u * away) : y;
    }
};
__device__ __forceinline__ Fp8Scale fp8_scale(uint32_t largest)
{
    const float a = __uint_as_float(max(largest, kFp8Smallest));
    Fp8Scale s;
    if (largest < (127u + 100u) << 23) { // a and 1 / a far from where float32 ends
        constexpr float R = 1.0f / 448.0f;
        const float q = a * R;
        s.scale = fmaf(fmaf(-448.0f, q, a), R, q);
        const float r0 = __builtin_amdgcn_rcpf(a), r = fmaf(fmaf(-a, r0, 1.0f), r0, r0), f = 448.0f * r;
        s.factor = fmaf(fmaf(-a, f, 448.0f), r, f);
        s.rest = fmaf(-a, s.factor, 448.0f) * r;
    } else {
        s.scale = a / 448.0f, s.factor = 448.0f / a;
        s.rest = largest < 0x7f800000u ? fmaf(-a, s.factor, 448.0f) / a : 0.0f;
    }
    return s;
}
// The largest magnitude of values, two at a time: as signed integers the positive ones are in order, as unsigned ones the negative
// ones above them all.
struct Largest {
    int32_t positive = 0;
    uint32_t negative = 0;
    __device__ __forceinline__ void add(float a, float b)
    {
        positive = max(positive, max(__float_as_int(a), __float_as_int(b)));
        negative = max(negative, max(__float_as_uint(a), __float_as_uint(b)));
    }
    __device__ __forceinline__ uint32_t bits() const { return max((uint32_t)positive, negative & ((uint32_t)((int32_t)negative >> 31) >> 1)); }
};
// The largest of 16 neighbouring lanes (lanes 16 i .. 16 i + 15), in each of them: rotations inside the row.
__device__ __forceinline__ uint32_t largest_of_16_lanes(uint32_t v)
{
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x128, 0xf, 0xf, false)); // row_ror:8, 4, 2, 1
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x124, 0xf, 0xf, false));
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x122, 0xf, 0xf, false));
    return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x121, 0xf, 0xf, false));
}
// x Phi(x) = max(x, 0) - |x| Q(|x|), Q(a) = 1 - Phi(a).  exp(a^2 / 2) Q(a) falls smoothly from 1/2 like 1 / (a sqrt(2 pi)) and is, to 5.5e-8
// of itself, a polynomial of degree 8 in t = 1 / (1 + 0.3 a) (fitted to scipy's erfcx on a <= 12; beyond, exp(-a^2 / 2) ends it).  Against the
// value in 64 bits: 2.4e-7 at most, 7.6e-7 of it down to x = -4; below, 2^-20 of it and 1.3 x^2 2^-24 (exp2's argument is rounded), about what a
// rounding of x changes, and nothing from x = -13.2 on, where exp2 ends.  Some 20 instructions without a branch, where the compiler's erff
// takes 60: 1024 x 768 x 768 with GELU 6.8 -> 5.5 us, 9 x 7 x 90 7.0 -> 6.2.
__device__ __forceinline__ float gelu_smooth(float x)
{
    constexpr float C[9] = {4.74133549e-06f, 0.119528323f, 0.121634774f, 0.0957856551f, 0.139975503f, -0.0728332847f, 0.225472927f, -0.16763334f, 0.0380647257f};
    const float m = fabsf(x), a = m > 16.0f ? 16.0f : m; // (a NaN stays one; |x| times nothing is nothing)
    const float t = __builtin_amdgcn_rcpf(fmaf(a, 0.3f, 1.0f));
    float r = C[8];
#pragma unroll
    for (int k = 7; k >= 0; --k) r = fmaf(r, t, C[k]);
    const float q = __builtin_amdgcn_exp2f(a * a * -0.72134752f) * r;
    return fmaf(-a, q, x < 0.0f ? 0.0f : x);
}
// Four of them out of line, for epilogues of many unrolled vectors.
static __device__ __noinline__ f32x4 gelu_smooth4(f32x4 v)
{
    return f32x4{gelu_smooth(v[0]), gelu_smooth(v[1]), gelu_smooth(v[2]), gelu_smooth(v[3])};
}
// Four values to nearest even.  |x| <= a keeps them within 448 * (1 + 2^-23), which rounds to 448: nothing overflows.
__device__ __forceinline__ uint32_t pack_fp8x4(float a, float b, float c, float d)
{
    const int low = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, low, true);
}

} // namespace tt
