// Matrix-core products of matrices held in 8 bits with a scale for each block of 128 (tt.h, tt_dense_fp8).
//
// One step of the reduction is one column block: the matrix cores sum the 128 products of a block (bf16 results: one
// v_mfma_f32_16x16x128_f8f6f4), and the sum goes into the float32 accumulators times the two scales, by vector FMAs.
//
// The matrix cores' rows are B's rows (n) and their columns A's rows (m): a lane then holds four consecutive n of one m, so
// that its scale of A is one register, the scale of B is the same for the whole tile (b_rows = 128), and what it stores is
// contiguous.
//
// The order of the 128 elements inside a step is the same permutation for both operands, which leaves the sum unchanged.
#pragma once

#include "fp8_blocks.hip.h"

namespace tt {

typedef __attribute__((ext_vector_type(8))) int i32x8;

struct ProductArgs {
    const uint8_t *a, *b;
    const float *a_scale, *b_scale;
    const void *bias; // may be null
    void *out;
    float *ws;
    int32_t batch, M, N, kb;
    int32_t b_rows, b_scale_row; // rows of B that share a scale; scales of one column block of B
    int32_t act;
};

// The two 16-byte pieces of a row's 128 bytes that a lane multiplies: pieces g and g + 4 of the eight, g = lane / 16.
struct Fragment {
    u32x4 lo, hi;
};

// The sums of 128 products, 16 rows of B by 16 rows of A.
template <int DT> struct BlockProduct;
template <> struct BlockProduct<TT_BF16> {
    static __device__ __forceinline__ f32x4 run(const Fragment &b, const Fragment &a)
    {
        const i32x8 x = __builtin_shufflevector(__builtin_bit_cast(__attribute__((ext_vector_type(4))) int, b.lo),
                                                __builtin_bit_cast(__attribute__((ext_vector_type(4))) int, b.hi), 0, 1, 2, 3, 4, 5, 6, 7);
        const i32x8 y = __builtin_shufflevector(__builtin_bit_cast(__attribute__((ext_vector_type(4))) int, a.lo),
                                                __builtin_bit_cast(__attribute__((ext_vector_type(4))) int, a.hi), 0, 1, 2, 3, 4, 5, 6, 7);
        const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, zero, 0, 0, 0, 0, 0, 0);
    }
};
// Eight e4m3 values as bf16, exactly.
__device__ __forceinline__ bf16x8 widen_fp8(uint32_t lo, uint32_t hi)
{
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
template <> struct BlockProduct<TT_F32> {
    static __device__ __forceinline__ f32x4 run(const Fragment &b, const Fragment &a)
    {
        f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const u32x4 &x = s < 2 ? b.lo : b.hi, &y = s < 2 ? a.lo : a.hi;
            sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen_fp8(x[s % 2 * 2], x[s % 2 * 2 + 1]),
                                                          widen_fp8(y[s % 2 * 2], y[s % 2 * 2 + 1]), sum, 0, 0, 0);
        }
        return sum;
    }
};

// 16 x 16 outputs a wave, operands from memory straight into the fragments.
template <int DT> __global__ void __launch_bounds__(64) product_direct_kernel(const ProductArgs g)
{
    const int lane = threadIdx.x, r = lane % 16, part = lane / 16;
    const int tiles_n = (g.N + 15) / 16, n0 = (int)(blockIdx.x % tiles_n) * 16, m0 = (int)(blockIdx.x / tiles_n) * 16;
    const int64_t kp = (int64_t)g.kb * kFp8Block, batch = blockIdx.y;
    // rows past a matrix read its last row; what they give is not stored
    const uint8_t *const a = g.a + (batch * g.M + min(m0 + r, g.M - 1)) * kp + part * 16;
    const uint8_t *const b = g.b + (batch * g.N + min(n0 + r, g.N - 1)) * kp + part * 16;
    const float *const a_scale = g.a_scale + batch * g.kb * g.M + min(m0 + r, g.M - 1);
    const float *const b_scale = g.b_scale + batch * g.kb * g.b_scale_row;
    f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int j = 0; j < g.kb; ++j) {
        Fragment x, y;
        load16(x.lo, b + j * kFp8Block), load16(x.hi, b + j * kFp8Block + 64);
        load16(y.lo, a + j * kFp8Block), load16(y.hi, a + j * kFp8Block + 64);
        const f32x4 p = BlockProduct<DT>::run(x, y);
        const float sa = a_scale[(int64_t)j * g.M];
#pragma unroll
        for (int e = 0; e < 4; ++e)
            sum[e] = fmaf(p[e], sa * b_scale[(int64_t)j * g.b_scale_row + min(n0 + part * 4 + e, g.N - 1) / g.b_rows], sum[e]);
    }
    if (m0 + r >= g.M) return;
    for (int e = 0; e < 4; ++e) {
        const int n = n0 + part * 4 + e;
        if (n >= g.N) continue;
        const float v = sum[e] + (g.bias ? load_as_float<DT>(g.bias, n) : 0.0f);
        store_from_float<DT>(g.out, (batch * g.M + m0 + r) * g.N + n, apply_act(v, g.act));
    }
}

} // namespace tt
