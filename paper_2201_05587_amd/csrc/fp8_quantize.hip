// Tensors into matrices held in 8 bits.
#include <hip/hip_runtime.h>

#include "fp8_blocks.hip.h"

namespace tt {
namespace {

constexpr int64_t kFp8LargestRows = 1ll << 26; // a launch has less than 2^32 threads

struct QuantizeArgs {
    const void *x;
    uint8_t *q;
    float *scale;
    int32_t rows, cols, kb;
};

// One block a workgroup: GROUP rows (1 or 128) by 128 columns.
template <int DT, int GROUP> __global__ void __launch_bounds__(GROUP == 1 ? 64 : 256) quantize_block_kernel(const QuantizeArgs g)
{
    constexpr int THREADS = GROUP == 1 ? 64 : 256;
    __shared__ uint32_t tops[THREADS / 64];
    const int tid = threadIdx.x;
    const int row_blocks = (g.rows + GROUP - 1) / GROUP;
    const int64_t row_block = blockIdx.x % row_blocks, batch = blockIdx.x / row_blocks;
    const int col0 = blockIdx.y * kFp8Block, row0 = (int)row_block * GROUP, rows = min(GROUP, g.rows - row0);
    const int64_t first = batch * g.rows + row0;
    uint32_t top = 0;
    for (int i = tid; i < rows * kFp8Block; i += THREADS) {
        const int col = col0 + i % kFp8Block;
        if (col < g.cols) top = max(top, magnitude_bits(load_as_float<DT>(g.x, (first + i / kFp8Block) * g.cols + col)));
    }
    for (int d = 1; d < 64; d *= 2) top = max(top, (uint32_t)__shfl_xor((int)top, d));
    if (tid % 64 == 0) tops[tid / 64] = top;
    __syncthreads();
    for (int w = 0; w < THREADS / 64; ++w) top = max(top, tops[w]);
    const Fp8Scale s = fp8_scale(top);
    if (tid == 0) g.scale[(batch * g.kb + blockIdx.y) * row_blocks + row_block] = s.scale;
    for (int i = tid; i < rows * (kFp8Block / 4); i += THREADS) {
        const int64_t row = first + i / (kFp8Block / 4);
        const int col = col0 + i % (kFp8Block / 4) * 4;
        float v[4];
        for (int e = 0; e < 4; ++e) v[e] = col + e < g.cols ? load_as_float<DT>(g.x, row * g.cols + col + e) * s.factor : 0.0f;
        *reinterpret_cast<uint32_t *>(g.q + row * g.kb * kFp8Block + col) = pack_fp8x4(v[0], v[1], v[2], v[3]);
    }
}

template <int DT> int launch(const QuantizeArgs &g, const tt_quant_shape &s, void *stream)
{
    const int64_t row_blocks = (s.rows + s.block_rows - 1) / s.block_rows;
    const dim3 grid((uint32_t)(row_blocks * s.batch), (uint32_t)g.kb);
    if (s.block_rows == 1)
        hipLaunchKernelGGL((quantize_block_kernel<DT, 1>), grid, dim3(64), 0, static_cast<hipStream_t>(stream), g);
    else
        hipLaunchKernelGGL((quantize_block_kernel<DT, 128>), grid, dim3(256), 0, static_cast<hipStream_t>(stream), g);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? TT_OK : note_hip_error((int)e, "quantize_block_kernel launch");
}

} // namespace

int check_quant_shape(const tt_quant_shape &s)
{
    if (s.batch < 1 || s.rows < 1 || s.cols < 1 || (s.block_rows != 1 && s.block_rows != kFp8Block)) return TT_ERR_BAD_ARG;
    if (s.dtype != TT_F32 && s.dtype != TT_BF16) return TT_ERR_BAD_ARG;
    return (int64_t)s.batch * s.rows >= kFp8LargestRows || s.cols > kFp8LargestK ? TT_ERR_UNSUPPORTED : TT_OK;
}

} // namespace tt

using namespace tt;

extern "C" int tt_quantize_fp8(const void *x, void *q, float *scale, const tt_quant_shape *shape, void *stream)
{
    if (!shape || !x || !q || !scale || !aligned16(x) || !aligned16(q) || !aligned16(scale)) return TT_ERR_BAD_ARG;
    const tt_quant_shape &s = *shape;
    if (const int rc = check_quant_shape(s); rc != TT_OK) return rc;
    const QuantizeArgs g = {x, static_cast<uint8_t *>(q), scale, s.rows, s.cols, (int32_t)fp8_blocks(s.cols)};
    return s.dtype == TT_F32 ? launch<TT_F32>(g, s, stream) : launch<TT_BF16>(g, s, stream);
}
