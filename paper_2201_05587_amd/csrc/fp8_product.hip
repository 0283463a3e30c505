// Products of matrices held in 8 bits, entry points and launch rule.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "fp8_block.hip.h"

namespace tt {
namespace {

// Estimated time (us) of a launch of `tiles` workgroups over `steps` steps of the reduction, from launches of 4096 x 4096 x 4096, 8192^3
// and m x 4096 x 4096, m = 16 .. 2048, and 1024 and 4096 x 768 x 768 (bf16, a scale in 128 rows of B; us, tiles of 64 | 128 | blocks):
//   m = 256  13.3 | 24.3 | 47     512  17.5 | 24.8 | 47     1024  31 | 26.4 | 48     2048  62 | 58 | 50     4096  129 | 100 | 62
//   4096 x 768 x 768  8.5 | 9.5 | 15.4     1024 x 768 x 768  4.8 | 8.4 | 14.7     8192^3  903 | 716 | 454
// A step of a block takes 1.8 us, of 128 x 128 0.8, a workgroup on a CU at a time; of 64 x 64 a CU takes three together, a quarter of a
// microsecond each where it has many.
double estimate(int tile, int64_t tiles, int64_t steps, int64_t cus)
{
    const double rounds = (double)((tiles + cus - 1) / cus);
    switch (tile) {
    case 64: return 3.2 + (double)steps * (tiles <= cus ? 0.28 + 0.11 * (double)tiles / (double)cus : std::max(0.2 + 0.19 * rounds, 0.25 * rounds));
    case 128: return 4.0 + (double)steps * 0.8 * rounds;
    default: return 6.0 + (double)steps * 1.8 * rounds;
    }
}

// Rows of A at most for the streaming kernel: it reads A once for 16 rows of B (24 x 1000 x 2048 fp32 5.2 us, in tiles 8.0; 32 x 4096 x 4096
// 9.0 and 9.9; 64 x 4096 x 4096 13.3 and 11.1).
constexpr int kStreamRows = 32;

int plan_of(const tt_fp8_shape &s, tt_fp8_launch *l)
{
    if (s.batch < 1 || s.m < 1 || s.n < 1 || s.k < 1 || (s.b_rows != 1 && s.b_rows != kFp8Block)) return TT_ERR_BAD_ARG;
    if (s.dtype != TT_F32 && s.dtype != TT_BF16) return TT_ERR_BAD_ARG;
    *l = tt_fp8_launch{};
    if (s.k > kFp8LargestK || s.batch > 65535) return TT_ERR_UNSUPPORTED;
    if ((double)s.batch * std::max(s.m, s.n) * s.k > 0x1p46 || (double)s.batch * s.m * s.n > 0x1p44) return TT_ERR_UNSUPPORTED;
    const int64_t kb = fp8_blocks(s.k), cus = compute_units();
    auto tiles = [&](int64_t tm, int64_t tn) { return ((s.m + tm - 1) / tm) * ((s.n + tn - 1) / tn); };
    auto in = [&](int kernel, int tm, int tn, int block, int lds) {
        l->kernel = kernel, l->tile_m = tm, l->tile_n = tn, l->split_k = 1, l->block = block, l->lds_bytes = lds;
    };
    if (s.m <= kStreamRows) {
        in(TT_FP8_STREAM, s.m <= 16 ? 16 : 32, 16, 512, 0);
    } else {
        in(TT_FP8_TILES, 64, 64, 256, Tiles<64, 64>::LDS);
        double best = estimate(64, tiles(64, 64) * s.batch, kb, cus);
        // fp32 with a scale per row of B holds too much for the larger tile's registers
        if (s.dtype == TT_BF16 || s.b_rows > 1)
            if (const double us = estimate(128, tiles(128, 128) * s.batch, kb, cus); us < best) best = us, in(TT_FP8_TILES, 128, 128, 256, Tiles<128, 128>::LDS);
        if (s.dtype == TT_BF16)
            if (const double us = estimate(256, tiles(256, 256) * s.batch, kb, cus); us < best) best = us, in(TT_FP8_BLOCKS, 256, 256, Fp8Block::THREADS, Fp8Block::LDS);
        // Few tiles and a long reduction: splits of it, whose sums a second launch adds (3.5 us, and a third of one for every split).
        // 100 x 512 x 8192: 21 us, 4 splits 11.1, 8 10.6, 16 13.5; 300 x 1000 x 1000 7.8 us, 2 splits 8.9.
        int splits = 1;
        for (int n = 2; n <= 16 && n * 2 <= kb; n *= 2) {
            const double us = estimate(64, tiles(64, 64) * s.batch * n, (kb + n - 1) / n, cus) + 3.5 + 0.35 * n;
            if (us < best) best = us, splits = n;
        }
        if (splits > 1) {
            in(TT_FP8_TILES, 64, 64, 256, Tiles<64, 64>::LDS);
            const int64_t steps = (kb + splits - 1) / splits;
            l->split_k = (int32_t)((kb + steps - 1) / steps);
            l->workspace_bytes = (int64_t)l->split_k * s.batch * s.m * s.n * 4;
        }
    }
    const int64_t grid = tiles(l->tile_m, l->tile_n);
    if (grid * l->block > INT32_MAX) return TT_ERR_UNSUPPORTED;
    l->grid = (int32_t)grid;
    return TT_OK;
}

int launched(const char *what)
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? TT_OK : note_hip_error((int)e, what);
}

// (a kernel per instance, so that its limit is raised once)
template <auto KERNEL> int launch_kernel(const ProductArgs &g, const tt_fp8_launch &l, void *stream)
{
    static DynamicLdsLimit limit;
    if (const int rc = limit.raise_to(reinterpret_cast<const void *>(KERNEL), l.lds_bytes); rc != TT_OK) return rc;
    hipLaunchKernelGGL(KERNEL, dim3(l.grid, g.batch, l.split_k), dim3(l.block), l.lds_bytes, static_cast<hipStream_t>(stream), g);
    return launched("8-bit product launch");
}

template <int DT, int B_ROWS> int launch(ProductArgs &g, const tt_fp8_launch &l, void *stream)
{
    g.tiles_m = (g.M + l.tile_m - 1) / l.tile_m, g.tiles_n = (g.N + l.tile_n - 1) / l.tile_n;
    g.splits = l.split_k, g.split_steps = (g.kb + l.split_k - 1) / l.split_k;
    if (l.kernel == TT_FP8_STREAM)
        return l.tile_m == 16 ? launch_kernel<product_stream_kernel<DT, 1>>(g, l, stream) : launch_kernel<product_stream_kernel<DT, 2>>(g, l, stream);
    if constexpr (DT == TT_BF16)
        if (l.kernel == TT_FP8_BLOCKS) return launch_kernel<product_block_kernel<B_ROWS>>(g, l, stream);
    if constexpr (DT == TT_BF16 || B_ROWS > 1)
        if (l.tile_m == 128) return launch_kernel<product_tile_kernel<DT, 128, 128, B_ROWS>>(g, l, stream);
    const int rc = launch_kernel<product_tile_kernel<DT, 64, 64, B_ROWS>>(g, l, stream);
    if (rc != TT_OK || l.split_k == 1) return rc;
    const int64_t threads = (int64_t)g.batch * g.M * ((g.N + 7) / 8);
    hipLaunchKernelGGL((product_reduce_kernel<DT>), dim3((uint32_t)((threads + 255) / 256)), dim3(256), 0, static_cast<hipStream_t>(stream), g);
    return launched("product_reduce_kernel launch");
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
    g.ws = static_cast<float *>(ws);
    if (g.b_rows == 1) return shape->dtype == TT_F32 ? launch<TT_F32, 1>(g, l, stream) : launch<TT_BF16, 1>(g, l, stream);
    return shape->dtype == TT_F32 ? launch<TT_F32, kFp8Block>(g, l, stream) : launch<TT_BF16, kFp8Block>(g, l, stream);
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
