// Group norm + activation over channels-last activations (tt.h, tt_group_norm_act).
#include <hip/hip_runtime.h>

#include "fp8_blocks.hip.h"

namespace tt {
namespace {

struct NormArgs {
    const void *x, *gamma, *beta; // gamma, beta: may be null
    void *y;                      // or the values of the matrix held in 8 bits
    float *scale, *ws;            // ws: mean and sum of squared differences of every (image, group)
    int64_t pixels;               // of an image
    int32_t n, c, groups, act;
    float eps;
};

__device__ __forceinline__ float norm_act(float v, int act)
{
    return act == TT_ACT_SILU ? v / (1.0f + expf(-v)) : apply_act(v, act);
}

__device__ __forceinline__ float sum_of_workgroup(float v, float *shared)
{
    for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d);
    __syncthreads();
    if (threadIdx.x % 64 == 0) shared[threadIdx.x / 64] = v;
    __syncthreads();
    return shared[0] + shared[1] + shared[2] + shared[3];
}

// One (image, group) a workgroup: the mean first, then the squared differences to it.
template <int DT> __global__ void __launch_bounds__(256) norm_statistics_kernel(const NormArgs g)
{
    __shared__ float shared[4];
    const int wide = g.c / g.groups;
    const int64_t image = blockIdx.x / g.groups, group = blockIdx.x % g.groups;
    const int64_t first = image * g.pixels * g.c + group * wide, count = g.pixels * wide;
    float sum = 0.0f;
    for (int64_t i = threadIdx.x; i < count; i += 256) sum += load_as_float<DT>(g.x, first + i / wide * g.c + i % wide);
    const float mean = sum_of_workgroup(sum, shared) / (float)count;
    float squares = 0.0f;
    for (int64_t i = threadIdx.x; i < count; i += 256) {
        const float d = load_as_float<DT>(g.x, first + i / wide * g.c + i % wide) - mean;
        squares = fmaf(d, d, squares);
    }
    squares = sum_of_workgroup(squares, shared);
    if (threadIdx.x == 0) g.ws[2 * blockIdx.x] = mean, g.ws[2 * blockIdx.x + 1] = squares;
}

template <int DT> __device__ __forceinline__ float normalised(const NormArgs &g, int64_t image, int64_t pixel, int c)
{
    const int wide = g.c / g.groups;
    const float *const stat = g.ws + 2 * (image * g.groups + c / wide);
    const float rstd = 1.0f / sqrtf(stat[1] / (float)(g.pixels * wide) + g.eps);
    const float gamma = g.gamma ? load_as_float<DT>(g.gamma, c) : 1.0f, beta = g.beta ? load_as_float<DT>(g.beta, c) : 0.0f;
    const float x = load_as_float<DT>(g.x, (image * g.pixels + pixel) * g.c + c);
    return norm_act(fmaf(x - stat[0], rstd * gamma, beta), g.act);
}

template <int DT> __global__ void __launch_bounds__(256) norm_apply_kernel(const NormArgs g)
{
    const int64_t per_image = g.pixels * g.c;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < g.n * per_image; i += (int64_t)gridDim.x * 256) {
        const int64_t image = i / per_image, at = i % per_image;
        store_from_float<DT>(g.y, i, normalised<DT>(g, image, at / g.c, (int)(at % g.c)));
    }
}

// One pixel's 128 channels a wave.
template <int DT> __global__ void __launch_bounds__(64) norm_apply_fp8_kernel(const NormArgs g)
{
    const int kb = (int)fp8_blocks(g.c), lane = threadIdx.x;
    const int64_t rows = g.n * g.pixels, row = blockIdx.x / kb;
    const int block = (int)(blockIdx.x % kb), c = block * kFp8Block + lane * 2;
    float v[2];
    for (int e = 0; e < 2; ++e) v[e] = c + e < g.c ? normalised<DT>(g, row / g.pixels, row % g.pixels, c + e) : 0.0f;
    uint32_t top = max(magnitude_bits(v[0]), magnitude_bits(v[1]));
    for (int d = 1; d < 64; d *= 2) top = max(top, (uint32_t)__shfl_xor((int)top, d));
    const Fp8Scale s = fp8_scale(top);
    if (lane == 0) g.scale[block * rows + row] = s.scale;
    reinterpret_cast<uint16_t *>(g.y)[(row * kb + block) * (kFp8Block / 2) + lane] = (uint16_t)pack_fp8x4(v[0] * s.factor, v[1] * s.factor, 0.0f, 0.0f);
}

int plan_of(const tt_norm_shape &s, int fp8, tt_norm_launch *l)
{
    if (s.n < 1 || s.h < 1 || s.w < 1 || s.c < 1 || s.groups < 1 || s.c % s.groups != 0) return TT_ERR_BAD_ARG;
    if (s.dtype != TT_F32 && s.dtype != TT_BF16) return TT_ERR_BAD_ARG;
    *l = tt_norm_launch{};
    const int64_t rows = (int64_t)s.n * s.h * s.w;
    if ((int64_t)s.n * s.groups > INT32_MAX || (int64_t)s.h * s.w > INT32_MAX || rows > INT32_MAX / fp8_blocks(s.c)) return TT_ERR_UNSUPPORTED;
    l->kernel = TT_NORM_TWO_PASS;
    l->chunks = 1;
    l->grid = fp8 ? (int32_t)(rows * fp8_blocks(s.c)) : (int32_t)std::min<int64_t>((rows * s.c + 255) / 256, 1 << 16);
    l->block = fp8 ? 64 : 256;
    l->workspace_bytes = (int64_t)s.n * s.groups * 8;
    return TT_OK;
}

template <int DT> int launch(const NormArgs &g, const tt_norm_launch &l, bool fp8, void *stream)
{
    hipLaunchKernelGGL((norm_statistics_kernel<DT>), dim3(g.n * g.groups), dim3(256), 0, static_cast<hipStream_t>(stream), g);
    if (fp8)
        hipLaunchKernelGGL((norm_apply_fp8_kernel<DT>), dim3(l.grid), dim3(l.block), 0, static_cast<hipStream_t>(stream), g);
    else
        hipLaunchKernelGGL((norm_apply_kernel<DT>), dim3(l.grid), dim3(l.block), 0, static_cast<hipStream_t>(stream), g);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? TT_OK : note_hip_error((int)e, "group norm launch");
}

int run(const void *x, const void *gamma, const void *beta, void *y, float *scale, const tt_norm_shape *shape, int act, float eps,
        void *ws, size_t ws_bytes, bool fp8, void *stream)
{
    if (!shape || !x || !y || (fp8 && !scale)) return TT_ERR_BAD_ARG;
    for (const void *p : {x, gamma, beta, (const void *)y, (const void *)scale})
        if (!aligned16(p)) return TT_ERR_BAD_ARG;
    if (act < TT_ACT_NONE || act > TT_ACT_SILU || !(eps >= 0.0f)) return TT_ERR_BAD_ARG;
    tt_norm_launch l;
    if (const int rc = plan_of(*shape, fp8, &l); rc != TT_OK) return rc;
    if (l.workspace_bytes > 0 && (!ws || !aligned16(ws) || (int64_t)ws_bytes < l.workspace_bytes)) return TT_ERR_WORKSPACE;
    NormArgs g{};
    g.x = x, g.gamma = gamma, g.beta = beta, g.y = y, g.scale = scale, g.ws = static_cast<float *>(ws);
    g.pixels = (int64_t)shape->h * shape->w;
    g.n = shape->n, g.c = shape->c, g.groups = shape->groups, g.act = act, g.eps = eps;
    return shape->dtype == TT_F32 ? launch<TT_F32>(g, l, fp8, stream) : launch<TT_BF16>(g, l, fp8, stream);
}

} // namespace
} // namespace tt

using namespace tt;

extern "C" int tt_norm_plan(const tt_norm_shape *shape, int fp8, tt_norm_launch *launch)
{
    return shape && launch ? plan_of(*shape, fp8, launch) : TT_ERR_BAD_ARG;
}

extern "C" int tt_group_norm_act(const void *x, const void *gamma, const void *beta, void *y, const tt_norm_shape *shape, int act,
                                 float eps, void *ws, size_t ws_bytes, void *stream)
{
    return run(x, gamma, beta, y, nullptr, shape, act, eps, ws, ws_bytes, false, stream);
}

extern "C" int tt_group_norm_act_fp8(const void *x, const void *gamma, const void *beta, void *q, float *scale, const tt_norm_shape *shape,
                                     int act, float eps, void *ws, size_t ws_bytes, void *stream)
{
    return run(x, gamma, beta, q, scale, shape, act, eps, ws, ws_bytes, true, stream);
}
