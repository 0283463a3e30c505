// Products of matrices held in 8 bits, entry points and launch rule.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "fp8_block.hip.h"

namespace tt {
namespace {

// Estimated times (us) of a launch, fitted to launches of 1 .. 8192 rows by 64 .. 32768 columns by 64 .. 16384, 1 to 256 in a batch.
//
// bf16, a scale in 128 rows of B, tiles of 64 | 128 | blocks:
//   m x 4096 x 4096, m = 256  13.2 | 24.5 | 49     512  18 | 24.9 | 49     1024  33 | 26.9 | 50     2048  57 | 51 | 52     4096  122 | 102 | 61
//   4096 x 768 x 768  7.9 | 9.2 | 15.8     1024 x 768 x 768  4.7 | 8.5 | 15.1     8192^3  852 | 715 | 448     8192 x 8192 x 64  54 | 69 | 36
// Rounds of workgroups over the CUs; of 64 x 64 a CU takes three together, and one alone is no faster than its loads.  Further:
//   fp32 widens its operands, which costs the smaller tile more: m x 4096 x 4096, m = 512  28 | 38     1024  49 | 41     4096  176 | 152;
//   a scale in every row of B is a product more for each output: 3012 x 2982 x 1601  31 | 43 | 34;
//   rows of bf16 that start at odd elements are stored by halves, 64 KB of a block by one CU: 302 x 247 x 467  4.1 | 7.3 | 15.5 (248: 11.1).
double estimate_tiles(int tile, const tt_fp8_shape &s, int64_t tiles, int64_t steps, int64_t cus)
{
    const double full = (double)tiles / (double)cus, rounds = (double)((tiles + cus - 1) / cus), k = (double)steps;
    const bool f32 = s.dtype == TT_F32, each = s.b_rows == 1, odd = !f32 && s.n % 2;
    switch (tile) {
    case 64: return 2.6 + std::max(k * ((f32 ? 0.44 : 0.28) + 0.03 * full), rounds * (odd ? 0.8 : 0.55) + rounds * k * (f32 ? 0.36 : 0.21));
    case 128: return 2.3 + rounds * ((odd ? 5.2 : 3.0) + k * (f32 ? 1.02 : each ? 0.72 : 0.66));
    default: {
        const double store = odd ? 9.0 : 0.0, step = each ? 1.6 : 1.2;
        return full < 1.0 ? 7.3 + store + 2.0 * full + k * (step + 0.45 * full * full) : 2.3 + rounds * (7.0 + store + k * (step + 0.45));
    }
    }
}

// The streaming kernel reads A again for 16 rows of B, so that it leads while its workgroups are few (us, stream | tiles, their
// reduction split where that is faster):
//   1 x 4096 x 4096  5.6 | 8.3     12 x 4096 x 4096  6.6 | 8.7     32 x 4096 x 4096  9.1 | 9.5     24 x 1000 x 2048 fp32  5.3 | 7.8
//   1 x 8192 x 8192  16.1 | 14.3   32 x 8192 x 8192  28.7 | 15.3   1 x 32768 x 1024  15.6 | 7.3    16 batches of 32 x 512 x 512  5.6 | 3.9
// The estimates count no bytes from memory: all of these found their weights in the memory-side cache.
constexpr int kStreamRows = 32;
double estimate_stream(int64_t rows, int64_t workgroups, int64_t steps, int64_t cus)
{
    const double full = workgroups <= cus ? (double)workgroups / (double)cus : (double)((workgroups + cus - 1) / cus), k = (double)steps;
    const double one = rows <= 16 ? 0.09 + 0.002 * (double)rows : 0.19; // a step of a workgroup that has its CU alone
    return 2.3 + std::max(one * k, full * (rows <= 16 ? 0.75 + (0.1 + 0.0015 * (double)rows) * k : 1.3 + 0.18 * k));
}

int plan_of(const tt_fp8_shape &s, tt_fp8_launch *l)
{
    if (s.batch < 1 || s.m < 1 || s.n < 1 || s.k < 1 || (s.b_rows != 1 && s.b_rows != kFp8Block)) return TT_ERR_BAD_ARG;
    if (s.dtype != TT_F32 && s.dtype != TT_BF16) return TT_ERR_BAD_ARG;
    *l = tt_fp8_launch{};
    if (s.k > kFp8LargestK || s.batch > 65535) return TT_ERR_UNSUPPORTED;
    if ((double)s.batch * std::max(s.m, s.n) * s.k > 0x1p46 || (double)s.batch * s.m * s.n > 0x1p44) return TT_ERR_UNSUPPORTED;
    const int64_t kb = fp8_blocks(s.k), cus = compute_units();
    auto tiles = [&](int64_t tm, int64_t tn) { return ((s.m + tm - 1) / tm) * ((s.n + tn - 1) / tn); };
    const bool f32 = s.dtype == TT_F32;
    double best = INFINITY;
    // The fastest of those whose workgroups a launch can have.
    auto consider = [&](double us, int kernel, int tm, int tn, int block, int lds) {
        if (us >= best || tiles(tm, tn) * block > INT32_MAX) return false;
        best = us;
        l->kernel = kernel, l->tile_m = tm, l->tile_n = tn, l->split_k = 1, l->block = block, l->lds_bytes = lds;
        return true;
    };
    consider(estimate_tiles(64, s, tiles(64, 64) * s.batch, kb, cus), TT_FP8_TILES, 64, 64, 256, Tiles<64, 64>::LDS);
    // fp32 with a scale per row of B holds too much for the larger tile's registers
    if (!f32 || s.b_rows > 1) consider(estimate_tiles(128, s, tiles(128, 128) * s.batch, kb, cus), TT_FP8_TILES, 128, 128, 256, Tiles<128, 128>::LDS);
    if (!f32) consider(estimate_tiles(256, s, tiles(256, 256) * s.batch, kb, cus), TT_FP8_BLOCKS, 256, 256, Fp8Block::THREADS, Fp8Block::LDS);
    if (s.m <= kStreamRows) consider(estimate_stream(s.m, tiles(kStreamRows, 16) * s.batch, kb, cus), TT_FP8_STREAM, s.m <= 16 ? 16 : 32, 16, 512, 0);
    // Few tiles and a long reduction: splits of it, whose sums a second launch adds, from a workspace written and read.
    // 100 x 512 x 8192: 21 us, 4 splits 10.9, 8 9.7, 16 11.0; 300 x 1000 x 1000 5.2 us, 2 splits 7.6; 200 x 8192 x 4096 17.5 us, 8 splits 38.
    int splits = 1;
    for (int n = 2; n <= 16 && n * 2 <= kb; n *= 2) {
        const double sums = 2.5 + 0.35 * n + (double)n * s.batch * s.m * s.n * 4 / 2.5e6;
        if (consider(estimate_tiles(64, s, tiles(64, 64) * s.batch * n, (kb + n - 1) / n, cus) + sums, TT_FP8_TILES, 64, 64, 256, Tiles<64, 64>::LDS)) splits = n;
    }
    if (best == INFINITY) return TT_ERR_UNSUPPORTED;
    if (splits > 1) {
        const int64_t steps = (kb + splits - 1) / splits;
        l->split_k = (int32_t)((kb + steps - 1) / steps);
        l->workspace_bytes = (int64_t)l->split_k * s.batch * s.m * s.n * 4;
    }
    l->grid = (int32_t)tiles(l->tile_m, l->tile_n);
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
