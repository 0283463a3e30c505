// Products of matrices held in 8 bits, entry points and launch rule.
#include <hip/hip_runtime.h>

#include "fp8_block.hip.h"

namespace tt {
namespace {

int plan_of(const tt_fp8_shape &s, tt_fp8_launch *l)
{
    if (s.batch < 1 || s.m < 1 || s.n < 1 || s.k < 1 || (s.b_rows != 1 && s.b_rows != kFp8Block)) return TT_ERR_BAD_ARG;
    if (s.dtype != TT_F32 && s.dtype != TT_BF16) return TT_ERR_BAD_ARG;
    *l = tt_fp8_launch{};
    if (s.k > kFp8LargestK || s.batch > 65535) return TT_ERR_UNSUPPORTED;
    const int64_t blocks_m = (s.m + 255ll) / 256, blocks_n = (s.n + 255ll) / 256;
    if (s.dtype == TT_BF16 && blocks_m * blocks_n * s.batch >= compute_units() / 2) {
        l->kernel = TT_FP8_BLOCKS;
        l->tile_m = l->tile_n = 256;
        l->split_k = 1;
        if (blocks_m * blocks_n > INT32_MAX) return TT_ERR_UNSUPPORTED;
        l->grid = (int32_t)(blocks_m * blocks_n);
        l->block = Fp8Block::THREADS;
        l->lds_bytes = Fp8Block::LDS;
        return TT_OK;
    }
    l->kernel = TT_FP8_DIRECT;
    l->tile_m = l->tile_n = 16;
    l->split_k = 1;
    const int64_t grid = ((s.m + 15ll) / 16) * ((s.n + 15ll) / 16);
    if (grid > INT32_MAX) return TT_ERR_UNSUPPORTED;
    l->grid = (int32_t)grid;
    l->block = 64;
    return TT_OK;
}

template <int B_ROWS> int launch_blocks(const ProductArgs &g, const tt_fp8_launch &l, void *stream)
{
    auto kern = product_block_kernel<B_ROWS>;
    static DynamicLdsLimit limit;
    if (const int rc = limit.raise_to(reinterpret_cast<const void *>(kern), l.lds_bytes); rc != TT_OK) return rc;
    hipLaunchKernelGGL(kern, dim3(l.grid, g.batch), dim3(l.block), l.lds_bytes, static_cast<hipStream_t>(stream), g, (g.M + 255) / 256, (g.N + 255) / 256);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? TT_OK : note_hip_error((int)e, "product_block_kernel launch");
}

template <int DT> int launch(const ProductArgs &g, const tt_fp8_launch &l, void *stream)
{
    if constexpr (DT == TT_BF16)
        if (l.kernel == TT_FP8_BLOCKS) return g.b_rows == 1 ? launch_blocks<1>(g, l, stream) : launch_blocks<kFp8Block>(g, l, stream);
    hipLaunchKernelGGL((product_direct_kernel<DT>), dim3(l.grid, g.batch), dim3(l.block), 0, static_cast<hipStream_t>(stream), g);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? TT_OK : note_hip_error((int)e, "product_direct_kernel launch");
}

int run(const void *a, const float *a_scale, const void *b, const float *b_scale, const void *bias, void *c,
        const tt_fp8_shape *shape, int act, void *ws, size_t ws_bytes, void *stream)
{
    if (!shape || !a || !a_scale || !b || !b_scale || !c) return TT_ERR_BAD_ARG;
    for (const void *p : {a, (const void *)a_scale, b, (const void *)b_scale, bias, (const void *)c})
        if (!aligned16(p)) return TT_ERR_BAD_ARG;
    tt_fp8_launch l;
    if (const int rc = plan_of(*shape, &l); rc != TT_OK) return rc;
    if (l.workspace_bytes > 0 && (!ws || !aligned16(ws) || (int64_t)ws_bytes < l.workspace_bytes)) return TT_ERR_WORKSPACE;
    ProductArgs g{};
    g.a = static_cast<const uint8_t *>(a), g.b = static_cast<const uint8_t *>(b);
    g.a_scale = a_scale, g.b_scale = b_scale;
    g.bias = bias, g.out = c;
    g.batch = shape->batch, g.M = shape->m, g.N = shape->n, g.kb = (int32_t)fp8_blocks(shape->k);
    g.b_rows = shape->b_rows, g.act = act;
    g.b_scale_row = (shape->n + shape->b_rows - 1) / shape->b_rows;
    return shape->dtype == TT_F32 ? launch<TT_F32>(g, l, stream) : launch<TT_BF16>(g, l, stream);
}

} // namespace
} // namespace tt

using namespace tt;

extern "C" int tt_fp8_plan(const tt_fp8_shape *shape, tt_fp8_launch *launch)
{
    return shape && launch ? plan_of(*shape, launch) : TT_ERR_BAD_ARG;
}

extern "C" int tt_dense_fp8(const void *x, const float *x_scale, const void *w, const float *w_scale, const void *bias, void *y,
                            const tt_fp8_shape *shape, int cls, void *ws, size_t ws_bytes, void *stream)
{
    if (!is_dense_class(cls) || !shape || shape->batch != 1) return TT_ERR_BAD_ARG;
    return run(x, x_scale, w, w_scale, bias, y, shape, act_of_class(cls), ws, ws_bytes, stream);
}

extern "C" int tt_batch_matmul_fp8(const void *a, const float *a_scale, const void *b, const float *b_scale, void *c,
                                   const tt_fp8_shape *shape, void *ws, size_t ws_bytes, void *stream)
{
    return run(a, a_scale, b, b_scale, nullptr, c, shape, ACT_NONE, ws, ws_bytes, stream);
}
