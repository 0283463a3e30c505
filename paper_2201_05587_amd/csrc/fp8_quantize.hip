// Tensors into matrices held in 8 bits.
#include <hip/hip_runtime.h>

#include "fp8_blocks.hip.h"

namespace tt {
namespace {

constexpr int64_t kFp8LargestRows = 1ll << 26; // of all batches: a launch has less than 2^32 threads

struct QuantizeArgs {
    const void *x;
    uint8_t *q;
    float *scale;
    int32_t rows, cols, kb;
    int64_t all_rows; // of all batches
};

// A lane holds eight consecutive columns and sixteen lanes a block's 128, whose largest magnitude they find among themselves.  It is
// all memory traffic: every load of a thread is in flight before the first is used, and x is read once.
template <int DT> struct EightColumns {
    static constexpr int W = 8 / ElemOf<DT>::CH;
    u32x4 raw[W];
    __device__ __forceinline__ void load(const void *x, int64_t at, int count)
    {
#pragma unroll
        for (int w = 0; w < W; ++w) {
            constexpr int CH = ElemOf<DT>::CH;
            raw[w] = u32x4{0u, 0u, 0u, 0u};
            if (count >= 8)
                load16(raw[w], static_cast<const typename ElemOf<DT>::type *>(x) + at + w * CH);
            else if (count > w * CH)
                raw[w] = load_piece<DT>(x, at + w * CH, count - w * CH);
        }
    }
    __device__ __forceinline__ float operator[](int e) const { return element_of<DT>(raw[e / ElemOf<DT>::CH], e % ElemOf<DT>::CH); }
    __device__ __forceinline__ void largest(Largest &top) const
    {
#pragma unroll
        for (int e = 0; e < 8; e += 2) top.add((*this)[e], (*this)[e + 1]);
    }
    __device__ __forceinline__ void store(uint8_t *to, const Fp8Scale &s) const
    {
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = s.value<DT>((*this)[e]);
        *reinterpret_cast<uint2 *>(to) = uint2{pack_fp8x4(v[0], v[1], v[2], v[3]), pack_fp8x4(v[4], v[5], v[6], v[7])};
    }
};

// A scale per row.  A wave covers 4 blocks at a time, `across` (1, 2 or 4) of one row side by side, and R times that many further
// down; the workgroup's scales go out through the LDS, a run of rows of each column block.
template <int DT, int R> __global__ void __launch_bounds__(256) quantize_rows_kernel(const QuantizeArgs g, int across_bits)
{
    __shared__ float scales[16 * R][4]; // (at most 16 R rows)
    const int tid = threadIdx.x, sixteen = tid % 64 / 16, wave = tid / 64;
    const int across = 1 << across_bits, down = 4 >> across_bits, tile_rows = 4 * R * down;
    const int64_t row0 = (int64_t)blockIdx.x * tile_rows; // of all batches together
    const int block0 = (int)blockIdx.y * across, block = block0 + (sixteen & (across - 1));
    const int row = wave * down + (sixteen >> across_bits), col = block * kFp8Block + tid % 16 * 8;
    const int count = g.cols - col;
    EightColumns<DT> x[R];
#pragma unroll
    for (int i = 0; i < R; ++i)
        if (block < g.kb) x[i].load(g.x, min(row0 + row + i * 4 * down, g.all_rows - 1) * g.cols + col, count);
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int r = row + i * 4 * down;
        if (block >= g.kb || row0 + r >= g.all_rows) break;
        Largest top;
        x[i].largest(top);
        const Fp8Scale s = fp8_scale(largest_of_16_lanes(top.bits()));
        x[i].store(g.q + (row0 + r) * g.kb * kFp8Block + col, s);
        if (tid % 16 == 0) scales[r][block - block0] = s.scale;
    }
    __syncthreads();
    for (int i = tid; i < tile_rows * across; i += 256) {
        const int b = block0 + i / tile_rows;
        const int64_t r = row0 + i % tile_rows;
        if (b >= g.kb || r >= g.all_rows) continue;
        const int64_t batch = g.rows == g.all_rows ? 0 : r / g.rows;
        g.scale[(batch * g.kb + b) * g.rows + (r - batch * g.rows)] = scales[i % tile_rows][b - block0];
    }
}

// A scale per 128 x 128: a block a workgroup, four rows a thread.
template <int DT> __global__ void __launch_bounds__(512) quantize_squares_kernel(const QuantizeArgs g)
{
    constexpr int R = 4;
    __shared__ uint32_t tops[8];
    const int tid = threadIdx.x;
    const int row_blocks = (g.rows + kFp8Block - 1) / kFp8Block;
    const int64_t batch = blockIdx.x / row_blocks, row_block = blockIdx.x % row_blocks;
    const int row = (int)row_block * kFp8Block + tid / 16, col = (int)blockIdx.y * kFp8Block + tid % 16 * 8;
    EightColumns<DT> x[R];
#pragma unroll
    for (int i = 0; i < R; ++i) x[i].load(g.x, (batch * g.rows + min(row + i * 32, g.rows - 1)) * g.cols + col, g.cols - col);
    Largest largest; // (rows past the end are the last one again)
#pragma unroll
    for (int i = 0; i < R; ++i) x[i].largest(largest);
    uint32_t top = largest_of_16_lanes(largest.bits());
    top = max(top, (uint32_t)__shfl_xor((int)top, 16));
    top = max(top, (uint32_t)__shfl_xor((int)top, 32));
    if (tid % 64 == 0) tops[tid / 64] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 8; ++w) top = max(top, tops[w]);
    const Fp8Scale s = fp8_scale(top);
    if (tid == 0) g.scale[(batch * g.kb + blockIdx.y) * row_blocks + row_block] = s.scale;
#pragma unroll
    for (int i = 0; i < R; ++i)
        if (row + i * 32 < g.rows) x[i].store(g.q + (batch * g.rows + row + i * 32) * g.kb * kFp8Block + col, s);
}

template <int DT> int launch(const QuantizeArgs &g, const tt_quant_shape &s, void *stream)
{
    hipStream_t on = static_cast<hipStream_t>(stream);
    if (s.block_rows == 1) {
        const int bits = g.kb >= 4 ? 2 : g.kb >= 2 ? 1 : 0, down = 4 >> bits;
        const int64_t columns = (g.kb + (1 << bits) - 1) >> bits;
        // Two rows a thread: with eight the workgroups at work together are spread over more of the memory than it likes (16384 x 4096
        // bf16 51 us, four rows 40, two 38; 8192 x 8192 fp32 76, 75, 69).
        constexpr int MANY = 2;
        // one row a thread where that leaves CUs without work
        const bool many = (g.all_rows + 4 * MANY * down - 1) / (4 * MANY * down) * columns >= compute_units();
        const int rows = 4 * down * (many ? MANY : 1);
        const dim3 grid((uint32_t)((g.all_rows + rows - 1) / rows), (uint32_t)columns);
        if (many)
            hipLaunchKernelGGL((quantize_rows_kernel<DT, MANY>), grid, dim3(256), 0, on, g, bits);
        else
            hipLaunchKernelGGL((quantize_rows_kernel<DT, 1>), grid, dim3(256), 0, on, g, bits);
    } else {
        const dim3 grid((uint32_t)((s.rows + kFp8Block - 1) / kFp8Block * s.batch), (uint32_t)g.kb);
        hipLaunchKernelGGL((quantize_squares_kernel<DT>), grid, dim3(512), 0, on, g);
    }
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? TT_OK : note_hip_error((int)e, "quantize kernel launch");
}

} // namespace

int check_quant_shape(const tt_quant_shape &s)
{
    if (s.batch < 1 || s.rows < 1 || s.cols < 1 || (s.block_rows != 1 && s.block_rows != kFp8Block)) return TT_ERR_BAD_ARG;
    if (s.dtype != TT_F32 && s.dtype != TT_BF16) return TT_ERR_BAD_ARG;
    const int64_t squares = (int64_t)s.batch * (((int64_t)s.rows + kFp8Block - 1) / kFp8Block); // of a column block, 512 threads each
    if (s.block_rows == kFp8Block && squares >= 1ll << 23) return TT_ERR_UNSUPPORTED;
    return (int64_t)s.batch * s.rows >= kFp8LargestRows || s.cols > kFp8LargestK ? TT_ERR_UNSUPPORTED : TT_OK;
}

} // namespace tt

using namespace tt;

extern "C" int tt_quantize_fp8(const void *x, void *q, float *scale, const tt_quant_shape *shape, void *stream)
{
    if (!shape || !x || !q || !scale || !aligned16(x) || !aligned16(q) || !aligned16(scale)) return TT_ERR_BAD_ARG;
    const tt_quant_shape &s = *shape;
    if (const int rc = check_quant_shape(s); rc != TT_OK) return rc;
    const QuantizeArgs g = {x, static_cast<uint8_t *>(q), scale, s.rows, s.cols, (int32_t)fp8_blocks(s.cols), (int64_t)s.batch * s.rows};
    return s.dtype == TT_F32 ? launch<TT_F32>(g, s, stream) : launch<TT_BF16>(g, s, stream);
}
