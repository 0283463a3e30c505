// Group norm + activation over channels-last activations (tt.h, tt_group_norm_act).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <numeric>

#include "fp8_blocks.hip.h"

namespace tt {
namespace {

// How a launch is laid out over an image: `tiles` column tiles of tx vectors, and parts of part_pixels pixels that ty rows of
// threads walk down.
struct NormTiles {
    int32_t columns, tx, ty, tiles, parts, part_pixels; // columns: vectors of a row
    FastDiv div_tx, div_tiles;
};

struct NormArgs {
    const void *x, *gamma, *beta; // gamma, beta: may be null
    void *y;                      // or the values of the matrix held in 8 bits
    float *scale;
    float2 *ws;                   // mean and sum of squared differences to it, [image][group][part][column tile, where a group has several]
    int32_t n, pixels, c, groups, wide; // pixels: of an image; wide: channels of a group
    float eps, top;                     // top: of the clamp
    NormTiles t;                        // of this launch
    int32_t stat_parts, stat_pixels, stat_tiles, stat_width; // of the first pass: column tiles of a group, channels of one
    FastDiv div_wide, div_wide_vectors, div_stat_tiles;      // div_wide_vectors: by the vectors of a group, where they are whole
    bool past;                                               // see store_channels
    double each;                                             // 1 / values of an (image, group)
};

// The activations a kernel is compiled for: one with a clamp to [0, top] for both ReLUs.  (With the activation a switch inside, 64
// unrolled copies of all five made a kernel of some 80 KB, and fetching it took most of a small launch: 13 us.)
enum NormAct { NORM_NONE, NORM_CLAMP, NORM_GELU, NORM_SILU };

// v / (1 + exp(-v)).  exp2's argument is rounded once: off by |v| 2^-24 of the exponential, which counts where v < 0.
__device__ __forceinline__ float silu(float v)
{
    return v * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(v * -1.44269504088896341f));
}

// A NaN stays one.
template <int ACT, int V> __device__ __forceinline__ void norm_act(float (&v)[V], float top)
{
    if constexpr (ACT == NORM_CLAMP) {
#pragma unroll
        for (int e = 0; e < V; ++e) {
            v[e] = v[e] < 0.0f ? 0.0f : v[e];
            v[e] = v[e] > top ? top : v[e];
        }
    } else if constexpr (ACT == NORM_GELU) {
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = gelu_smooth(v[e]);
    } else if constexpr (ACT == NORM_SILU) {
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = silu(v[e]);
    }
}

// V consecutive channels, `count` of them (at least one) in their row of c: whole 16-byte items at any element's address.  An item that is
// cut off by the row's end is loaded as the row's last 16 bytes, and settle() moves its channels to the front once they are wanted: loads
// of single elements under their conditions wait for one another (48 x 17 x 95 x 330 bf16 59 -> 46 us, 336 channels 43).  What
// lies behind `count` is anything.
template <int DT, int V> struct Channels {
    static constexpr int CH = ElemOf<DT>::CH, W = V / CH;
    u32x4 raw[W];
    __device__ __forceinline__ void load_whole(const void *p, int64_t at)
    {
#pragma unroll
        for (int w = 0; w < W; ++w) load16(raw[w], static_cast<const typename ElemOf<DT>::type *>(p) + at + w * CH);
    }
    __device__ __forceinline__ void load(const void *p, int64_t at, int count, int c)
    {
        using E = typename ElemOf<DT>::type;
        const E *const from = static_cast<const E *>(p) + at;
        if (c >= CH) { // (an item with no channel at all, too: it is in the row)
#pragma unroll
            for (int w = 0; w < W; ++w) load16(raw[w], from + w * CH - max(0, (w + 1) * CH - count));
        } else { // the row is shorter than an item
#pragma unroll
            for (int w = 0; w < W; ++w) raw[w] = u32x4{0u, 0u, 0u, 0u};
#pragma unroll
            for (int e = 0; e < CH - 1; ++e) {
                const E x = from[min(e, count - 1)];
                if constexpr (DT == TT_F32)
                    raw[0][e] = __float_as_uint(x);
                else
                    raw[0][e / 2] |= (uint32_t)x << (16 * (e % 2));
            }
        }
    }
    __device__ __forceinline__ void settle(int count, int c)
    {
        if (count >= V || c < CH) return;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            const int by = (w + 1) * CH - count; // elements
            u32x4 &r = raw[w];
            if (by <= 0 || by >= CH) continue;
            const int dwords = DT == TT_F32 ? by : by / 2;
            if (dwords & 2) r[0] = r[2], r[1] = r[3];
            if (dwords & 1) r[0] = r[1], r[1] = r[2], r[2] = r[3];
            if (DT == TT_BF16 && (by & 1))
                r[0] = r[0] >> 16 | r[1] << 16, r[1] = r[1] >> 16 | r[2] << 16, r[2] = r[2] >> 16 | r[3] << 16, r[3] >>= 16;
        }
    }
    __device__ __forceinline__ float operator[](int e) const { return element_of<DT>(raw[e / ElemOf<DT>::CH], e % ElemOf<DT>::CH); }
};
// `past`: the results are more than the caches hold, and are written past them, so that x is still there for the second pass
// (16 x 128 x 128 x 256 bf16, 134 MB in and out: 82 -> 71 us; 32 images: 152 -> 126).
template <int DT, int V> __device__ __forceinline__ void store_channels(void *p, int64_t at, const float (&v)[V], int count, bool past)
{
    constexpr int CH = ElemOf<DT>::CH;
    static_assert(V == CH, "one 16-byte item");
    u32x4 r;
#pragma unroll
    for (int h = 0; h < 4; ++h)
        if constexpr (DT == TT_F32)
            r[h] = __float_as_uint(v[h]);
        else
            r[h] = pack_bf16x2(v[(2 * h) % V], v[(2 * h + 1) % V]);
    if (past)
        __builtin_nontemporal_store(r, reinterpret_cast<u32x4 *>(static_cast<typename ElemOf<DT>::type *>(p) + at));
    else
        store_piece<DT>(p, at, r, count);
}

// v of another lane of the row of 16, or of the lane 16 or 32 further: without the LDS, whose lane permutations cost some 130 cycles
// each.
template <int CONTROL> __device__ __forceinline__ double lane_of_row(double v)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)b, CONTROL, 0xf, 0xf, false);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(b >> 32), CONTROL, 0xf, 0xf, false);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
template <bool HALVES> __device__ __forceinline__ double sum_of_rows(double v) // with the lane 32 (HALVES) or 16 further
{
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint32_t l = (uint32_t)b, h = (uint32_t)(b >> 32);
    u32x2 lo, hi; // (both operands of a swap the same: it leaves one row's value in both rows, and the other's)
    if constexpr (HALVES)
        lo = __builtin_amdgcn_permlane32_swap(l, l, false, false), hi = __builtin_amdgcn_permlane32_swap(h, h, false, false);
    else
        lo = __builtin_amdgcn_permlane16_swap(l, l, false, false), hi = __builtin_amdgcn_permlane16_swap(h, h, false, false);
    return __builtin_bit_cast(double, (uint64_t)hi[0] << 32 | lo[0]) + __builtin_bit_cast(double, (uint64_t)hi[1] << 32 | lo[1]);
}
// The sum over `lanes` (a power of two up to 64) neighbouring lanes, in each of them.
__device__ __forceinline__ double sum_of_lanes(double v, int lanes)
{
    if (lanes > 1) v += lane_of_row<0xb1>(v);  // quad_perm: the other of two lanes
    if (lanes > 2) v += lane_of_row<0x4e>(v);  // quad_perm: two lanes further
    if (lanes > 4) v += lane_of_row<0x141>(v); // row_half_mirror: the other four of eight
    if (lanes > 8) v += lane_of_row<0x140>(v); // row_mirror: the other eight
    if (lanes > 16) v = sum_of_rows<false>(v);
    if (lanes > 32) v = sum_of_rows<true>(v);
    return v;
}

// Sums of n values with mean `mean` and squared differences `squares` to it, relative to a value `origin` of their size, in 64 bits:
// the squares about the joint mean are what is left of them, and 29 bits may cancel before float32's are touched.
struct JointSums {
    double sum = 0.0, squares = 0.0;
    __device__ __forceinline__ void add(float mean, float squares_, double n, float origin)
    {
        const double d = (double)mean - (double)origin, nd = n * d;
        sum += nd;
        squares += fma(nd, d, (double)squares_);
    }
    __device__ __forceinline__ void add_lanes(int lanes) // of `lanes` neighbours, a power of two up to 64
    {
        sum = sum_of_lanes(sum, lanes), squares = sum_of_lanes(squares, lanes);
    }
    // (each: 1 / how many values there are)
    __device__ __forceinline__ float mean(float origin, double each) const { return (float)((double)origin + sum * each); }
    __device__ __forceinline__ double squares_about_mean(double each) const { return fmax(squares - sum * sum * each, squares * 0.0); }
};
struct JointSumsOfWave {
    double sum, squares, each;
    float origin;
};
// The threads of a workgroup that share a group's sums: a power of two up to `most`.
__device__ __forceinline__ int lanes_per_group(int groups, int most)
{
    int lanes = most;
    while (lanes > 1 && lanes * groups > (int)blockDim.x) lanes /= 2;
    return lanes;
}

// A workgroup's place: tx vectors of channels side by side in ty rows of threads, each of which walks down its column of pixels.
struct NormPlace {
    int tile, part, image;
    int tx, ty;                            // of this thread; ty >= g.t.ty: it has no column
    int channel, count;                    // its first channel, and how many of its V there are (at most 0: none)
    int tile_begin, tile_end;              // channels of the tile
    int first_group, groups;               // of the tile
    int begin, end;                        // pixels
    int64_t base;                          // element of the thread's first channel in the image's first pixel
    template <int V> __device__ __forceinline__ void init(const NormArgs &g)
    {
        part = (int)fast_div(blockIdx.x, g.t.div_tiles);
        tile = (int)blockIdx.x - part * g.t.tiles;
        image = (int)blockIdx.y;
        ty = (int)fast_div(threadIdx.x, g.t.div_tx);
        tx = (int)threadIdx.x - ty * g.t.tx;
        if (tile * g.t.tx + tx >= g.t.columns) ty = g.t.ty; // (the last tile may be narrower)
        tile_begin = tile * g.t.tx * V;
        tile_end = min(tile_begin + g.t.tx * V, g.c);
        channel = tile_begin + tx * V;
        count = ty < g.t.ty ? g.c - channel : 0;
        first_group = (int)fast_div((uint32_t)tile_begin, g.div_wide);
        groups = (int)fast_div((uint32_t)(tile_end - 1), g.div_wide) - first_group + 1;
        begin = part * g.t.part_pixels;
        end = min(begin + g.t.part_pixels, g.pixels);
        base = (int64_t)image * g.pixels * g.c + channel;
    }
};

// R pixels of a thread, all loads in flight together (pixels past the end: the last one again).
template <int DT, int V, int R> struct Pixels {
    Channels<DT, V> x[R];
    template <bool WHOLE> __device__ __forceinline__ void request(const NormArgs &g, const NormPlace &at, int first)
    {
        if (at.count <= 0) return;
        auto from = [&](int i) { return at.base + (int64_t)min(first + i * g.t.ty, at.end - 1) * g.c; };
        if constexpr (WHOLE) {
#pragma unroll
            for (int i = 0; i < R; ++i) x[i].load_whole(g.x, from(i));
        } else {
#pragma unroll
            for (int i = 0; i < R; ++i) x[i].load(g.x, from(i), at.count, g.c);
        }
    }
    template <bool WHOLE> __device__ __forceinline__ void settle(const NormArgs &g, const NormPlace &at)
    {
        if constexpr (WHOLE) return;
#pragma unroll
        for (int i = 0; i < R; ++i) x[i].settle(at.count, g.c);
    }
};

// Mean and squared differences to it of each of a thread's channels, from the registers that hold a batch (the squares of values far
// from zero would cancel).  Batches are joined by
//   mean += (mean' - mean) n' / (n + n'),   squares += squares' + (mean' - mean)^2 n n' / (n + n').
template <int DT, int V, int R> struct ChannelStatistics {
    float mean[V] = {}, squares[V] = {};
    int seen = 0;
    template <bool WHOLE> __device__ __forceinline__ void join(const Pixels<DT, V, R> &p, int rows)
    {
        const float r = 1.0f / (float)rows, share = (float)rows / (float)(seen + rows);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            float sum = 0.0f, sq = 0.0f;
#pragma unroll
            for (int i = 0; i < R; ++i) sum += WHOLE || i < rows ? p.x[i][e] : 0.0f;
            const float m = sum * r;
#pragma unroll
            for (int i = 0; i < R; ++i) {
                const float d = WHOLE || i < rows ? p.x[i][e] - m : 0.0f;
                sq = fmaf(d, d, sq);
            }
            const float step = m - mean[e];
            mean[e] = fmaf(step, share, mean[e]);
            squares[e] += fmaf(step * (share * (float)seen), step, sq);
        }
        seen += rows;
    }
    __device__ __forceinline__ void join(const Pixels<DT, V, R> &p, int rows)
    {
        if (rows == R)
            join<true>(p, R);
        else
            join<false>(p, rows);
    }
};

// The workgroup's channels and rows of threads joined to groups, through the LDS; one thread a group k of the tile calls
// done(k, mean, squares about it).
template <int V, int DT, int R, class F>
__device__ __forceinline__ void join_groups(const NormArgs &g, const NormPlace &at, const ChannelStatistics<DT, V, R> &mine, float2 *joined, F &&done)
{
    __shared__ int row_counts[512];
    __shared__ JointSumsOfWave waves[8];
    // one entry a channel, or where groups are whole vectors one a vector
    const bool vectors = g.wide % V == 0;
    const int unit = vectors ? V : 1, width = (at.tile_end - at.tile_begin) / unit;
    if (at.ty < g.t.ty) {
        if (vectors) {
            float mean = 0.0f, squares = 0.0f, apart = 0.0f;
#pragma unroll
            for (int e = 0; e < V; ++e) mean += mine.mean[e], squares += mine.squares[e];
            mean *= 1.0f / V;
#pragma unroll
            for (int e = 0; e < V; ++e) apart = fmaf(mine.mean[e] - mean, mine.mean[e] - mean, apart);
            if (at.count > 0) joined[at.ty * width + at.tx] = float2{mean, fmaf(apart, (float)mine.seen, squares)};
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (e < at.count) joined[at.ty * width + at.tx * V + e] = float2{mine.mean[e], mine.squares[e]};
        }
        if (at.tx == 0) row_counts[at.ty] = mine.seen * unit; // (a row's first thread always has channels)
    }
    __syncthreads();
    const int lanes = lanes_per_group(at.groups, 512), lane = (int)threadIdx.x % lanes;
    for (int k = (int)threadIdx.x / lanes; k < at.groups; k += (int)blockDim.x / lanes) {
        const int group = at.first_group + k;
        const int begin = max(group * g.wide, at.tile_begin), channels = min((group + 1) * g.wide, at.tile_end) - begin;
        const int from = (begin - at.tile_begin) / unit, wide = channels / unit, entries = g.t.ty * wide;
        const double each = 1.0 / ((double)(at.end - at.begin) * (double)channels);
        const float origin = joined[from].x;
        JointSums sums;
        constexpr int BATCH = 4; // (rows without pixels count nothing: entries past the end are one's)
        for (int first = lane; first < entries; first += BATCH * lanes) {
            float2 v[BATCH];
            int n[BATCH];
#pragma unroll
            for (int b = 0; b < BATCH; ++b) {
                const int i = min(first + b * lanes, entries - 1);
                const int row = channels == g.wide ? (int)fast_div((uint32_t)i, vectors ? g.div_wide_vectors : g.div_wide) : i / wide;
                v[b] = joined[row * width + from + i - row * wide];
                n[b] = first + b * lanes < entries ? row_counts[row] : 0;
            }
#pragma unroll
            for (int b = 0; b < BATCH; ++b) sums.add(v[b].x, n[b] > 0 ? v[b].y : 0.0f, (double)n[b], n[b] > 0 ? origin : v[b].x);
        }
        sums.add_lanes(min(lanes, 64));
        if (lanes <= 64) {
            if (lane == 0) done(k, sums.mean(origin, each), (float)sums.squares_about_mean(each));
        } else if (threadIdx.x % 64 == 0)
            waves[threadIdx.x / 64] = {sums.sum, sums.squares, each, origin};
    }
    if (lanes > 64) { // (at most one group a thread)
        __syncthreads();
        const int k = (int)threadIdx.x / lanes;
        if (lane == 0 && k < at.groups) {
            const JointSumsOfWave first = waves[threadIdx.x / 64];
            JointSums sums;
            for (int w = 0; w < lanes / 64; ++w) sums.sum += waves[threadIdx.x / 64 + w].sum, sums.squares += waves[threadIdx.x / 64 + w].squares;
            done(k, sums.mean(first.origin, first.each), (float)sums.squares_about_mean(first.each));
        }
    }
}

// First pass: the statistics of a part of an image.  The next batch is requested before the present one is summed.
template <int DT, int V, int R, bool WHOLE> __global__ void __launch_bounds__(512) norm_statistics_kernel(const NormArgs g)
{
    extern __shared__ float2 joined[]; // [row of threads][channel of the tile]
    NormPlace at;
    at.init<V>(g);
    ChannelStatistics<DT, V, R> mine;
    if (at.count > 0) {
        const int step = g.t.ty * R;
        Pixels<DT, V, R> now, next;
        int first = at.begin + at.ty;
        if (first < at.end) now.template request<WHOLE>(g, at, first);
        while (first < at.end) {
            const int rows = min(R, (at.end - first + g.t.ty - 1) / g.t.ty);
            const bool more = first + step < at.end;
            if (more) next.template request<WHOLE>(g, at, first + step);
            now.template settle<WHOLE>(g, at);
            mine.join(now, rows);
            if (more) now = next;
            first += step;
        }
    }
    join_groups<V>(g, at, mine, joined, [&](int k, float mean, float squares) {
        g.ws[((int64_t)at.image * g.groups + at.first_group + k) * (g.t.parts * g.stat_tiles) + at.part * g.stat_tiles + at.tile % g.stat_tiles] = float2{mean, squares};
    });
}

// Mean and 1 / sqrt(var + eps) of the tile's groups into the LDS, from the statistics of all parts; four loads of a lane in flight.
__device__ __forceinline__ void join_statistics(const NormArgs &g, const NormPlace &at, float2 *stat)
{
    constexpr int BATCH = 4;
    const int lanes = lanes_per_group(at.groups, 64), lane = (int)threadIdx.x % lanes;
    const int entries = g.stat_parts * g.stat_tiles;
    const double each = g.each;
    for (int k = (int)threadIdx.x / lanes; k < at.groups; k += (int)blockDim.x / lanes) {
        const int group = at.first_group + k, begin = group * g.wide, end = begin + g.wide;
        const float2 *const part = g.ws + ((int64_t)at.image * g.groups + group) * entries;
        const float origin = part[g.stat_tiles > 1 ? begin / g.stat_width : 0].x; // of the first part, in the tile where the group begins
        JointSums sums;
        for (int first = lane; first < entries; first += BATCH * lanes) {
            float2 v[BATCH];
            int n[BATCH], wide[BATCH]; // pixels and channels behind an entry
#pragma unroll
            for (int b = 0; b < BATCH; ++b) {
                n[b] = 0;
                if (b * lanes >= entries) continue; // (the same for all lanes)
                const int i = min(first + b * lanes, entries - 1);
                const int chunk = (int)fast_div((uint32_t)i, g.div_stat_tiles), tile = i - chunk * g.stat_tiles;
                n[b] = first + b * lanes < entries ? min(g.stat_pixels, g.pixels - chunk * g.stat_pixels) : 0;
                wide[b] = g.stat_tiles > 1 ? min(end, (tile + 1) * g.stat_width) - max(begin, tile * g.stat_width) : g.wide;
                v[b] = part[i];
            }
#pragma unroll
            for (int b = 0; b < BATCH; ++b) // (what the first pass has not written is not looked at)
                if (b * lanes < entries && n[b] > 0 && wide[b] > 0) sums.add(v[b].x, v[b].y, (double)n[b] * (double)wide[b], origin);
        }
        sums.add_lanes(lanes);
        if (lane == 0) stat[k] = float2{sums.mean(origin, each), 1.0f / sqrtf((float)(sums.squares_about_mean(each) * each) + g.eps)};
    }
    __syncthreads();
}

// What turns a thread's channels into the results: act((x - mean) * factor + shift).
template <int DT, int V, int R, bool FP8, int ACT> struct Apply {
    float mean[V], factor[V], shift[V];
    __device__ __forceinline__ void init(const NormArgs &g, const NormPlace &at, const float2 *stat, const Channels<DT, V> &gamma, const Channels<DT, V> &beta)
    {
#pragma unroll
        for (int e = 0; e < V; ++e) {
            mean[e] = factor[e] = shift[e] = 0.0f;
            if (e < at.count) {
                const float2 s = stat[(int)fast_div((uint32_t)(at.channel + e), g.div_wide) - at.first_group];
                mean[e] = s.x;
                factor[e] = s.y * (g.gamma ? gamma[e] : 1.0f);
                shift[e] = g.beta ? beta[e] : 0.0f;
            }
        }
    }
    __device__ __forceinline__ void run(const NormArgs &g, const NormPlace &at, const Pixels<DT, V, R> &p, int first) const
    {
        const int64_t rows = (int64_t)g.n * g.pixels;
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int pixel = first + i * g.t.ty;
            if (pixel >= at.end) break;
            float v[V];
#pragma unroll
            for (int e = 0; e < V; ++e) v[e] = fmaf(p.x[i][e] - mean[e], factor[e], shift[e]);
            norm_act<ACT, V>(v, g.top);
            if constexpr (!FP8) {
                store_channels<DT, V>(g.y, at.base + (int64_t)pixel * g.c, v, at.count, g.past);
            } else {
                // the largest magnitude of 16 lanes' 128 channels (those behind the last one are zeros)
                if (at.count < V) {
#pragma unroll
                    for (int e = 0; e < V; ++e) v[e] = e < at.count ? v[e] : 0.0f;
                }
                Largest top;
#pragma unroll
                for (int e = 0; e < V; e += 2) top.add(v[e], v[e + 1]);
                const Fp8Scale s = fp8_scale(largest_of_16_lanes(top.bits()));
                const int64_t row = (int64_t)at.image * g.pixels + pixel;
                const uint2 q = {pack_fp8x4(v[0] * s.factor, v[1] * s.factor, v[2] * s.factor, v[3] * s.factor),
                                 pack_fp8x4(v[4 % V] * s.factor, v[5 % V] * s.factor, v[6 % V] * s.factor, v[7 % V] * s.factor)};
                *reinterpret_cast<uint2 *>(static_cast<uint8_t *>(g.y) + row * (g.t.columns * 8) + at.channel) = q;
                if (at.tx % 16 == 0) g.scale[at.channel / kFp8Block * rows + row] = s.scale;
            }
        }
    }
};
template <bool WHOLE, int DT, int V> __device__ __forceinline__ void request_weights(const NormArgs &g, const NormPlace &at, Channels<DT, V> &gamma, Channels<DT, V> &beta)
{
    if (at.count <= 0) return;
    if (g.gamma) WHOLE ? gamma.load_whole(g.gamma, at.channel) : gamma.load(g.gamma, at.channel, at.count, g.c);
    if (g.beta) WHOLE ? beta.load_whole(g.beta, at.channel) : beta.load(g.beta, at.channel, at.count, g.c);
}

// Second pass.  The first batch of pixels is requested before the statistics are joined.
template <int DT, int V, int R, bool FP8, int ACT, bool WHOLE> __global__ void __launch_bounds__(512) norm_apply_kernel(const NormArgs g)
{
    extern __shared__ float2 stat[]; // of the tile's groups
    NormPlace at;
    at.init<V>(g);
    Pixels<DT, V, R> p;
    int first = at.begin + at.ty;
    p.template request<WHOLE>(g, at, first);
    Channels<DT, V> gamma, beta;
    request_weights<WHOLE>(g, at, gamma, beta);
    join_statistics(g, at, stat);
    if (FP8 ? at.ty >= g.t.ty : at.count <= 0) return;
    Apply<DT, V, R, FP8, ACT> apply;
    if constexpr (!WHOLE) gamma.settle(at.count, g.c), beta.settle(at.count, g.c);
    apply.init(g, at, stat, gamma, beta);
    for (;;) {
        p.template settle<WHOLE>(g, at);
        apply.run(g, at, p, first);
        first += g.t.ty * R;
        if (first >= at.end) break;
        p.template request<WHOLE>(g, at, first);
    }
}

// Both in one: an image's pixels of whole groups in the registers of a workgroup.
template <int DT, int V, int R, bool FP8, int ACT, bool WHOLE> __global__ void __launch_bounds__(512) norm_one_pass_kernel(const NormArgs g)
{
    extern __shared__ float2 joined[]; // [row of threads][channel of the tile], behind them mean and 1 / sqrt(var + eps) of the groups
    NormPlace at;
    at.init<V>(g);
    float2 *const stat = joined + g.t.ty * (at.tile_end - at.tile_begin);
    Pixels<DT, V, R> p;
    p.template request<WHOLE>(g, at, at.ty);
    Channels<DT, V> gamma, beta;
    request_weights<WHOLE>(g, at, gamma, beta);
    ChannelStatistics<DT, V, R> mine;
    p.template settle<WHOLE>(g, at);
    if (at.count > 0) mine.join(p, min(R, (g.pixels - at.ty + g.t.ty - 1) / g.t.ty));
    join_groups<V>(g, at, mine, joined, [&](int k, float mean, float squares) {
        stat[k] = float2{mean, 1.0f / sqrtf(squares * (float)g.each + g.eps)};
    });
    __syncthreads();
    if (FP8 ? at.ty >= g.t.ty : at.count <= 0) return;
    Apply<DT, V, R, FP8, ACT> apply;
    if constexpr (!WHOLE) gamma.settle(at.count, g.c), beta.settle(at.count, g.c);
    apply.init(g, at, stat, gamma, beta);
    apply.run(g, at, p, at.ty);
}

// ---- geometry ----------------------------------------------------------------------------------------------------------
// Pixels of a thread in flight together: in the first pass and in one pass, and in the second pass where there are many
// workgroups or few.
constexpr int kNormBatch = 4, kNormFew = 2;
constexpr int kNormJoined = 128; // batches that a thread of the first pass joins at most
constexpr int norm_held(int dtype, bool fp8) { return dtype == TT_F32 && fp8 ? 8 : 16; } // of a thread in one pass, at most
constexpr int norm_many(int dtype, bool fp8) { return dtype == TT_F32 && fp8 ? 4 : 8; }
constexpr int norm_vector(int dtype, bool fp8) { return fp8 || dtype == TT_BF16 ? 8 : 4; }
constexpr int kNormWidest = 256; // vectors of a column tile
constexpr int64_t kNormPast = 32 << 20; // bytes of results (the L2s together hold so much) from which on they are written past the caches

// Column tiles of at most `tx` vectors (a multiple of `unit`), and workgroups of some `threads`.
NormTiles tiles_of(int columns, int tx, int threads, int64_t pixels)
{
    NormTiles t{};
    t.columns = columns;
    t.tx = tx;
    t.tiles = (columns + tx - 1) / tx;
    t.ty = (int32_t)std::min<int64_t>(std::max(1, threads / tx), pixels);
    t.div_tx = make_fastdiv((uint32_t)tx);
    t.div_tiles = make_fastdiv((uint32_t)t.tiles);
    return t;
}
// ... with an image in at most `parts` parts of at least `batch` pixels a thread.
void set_parts(NormTiles &t, int64_t parts, int batch, int64_t pixels)
{
    const int64_t most = (pixels + (int64_t)t.ty * batch - 1) / ((int64_t)t.ty * batch);
    parts = std::max<int64_t>(1, std::min(parts, most));
    t.part_pixels = (int32_t)((pixels + parts - 1) / parts);
    t.parts = (int32_t)((pixels + t.part_pixels - 1) / t.part_pixels);
}
int block_of(const NormTiles &t) { return (t.tx * t.ty + 63) / 64 * 64; }

struct NormLayout {
    NormArgs args;          // without pointers; t: of the second (or only) launch
    NormTiles first;        // of the first pass
    int one_pass;           // pixels a thread holds; 0: two passes
    bool few;               // in the second pass: kNormFew pixels a thread at a time
};

int lay_out(const tt_norm_shape &s, bool fp8, NormLayout *lay, tt_norm_launch *l)
{
    if (s.n < 1 || s.h < 1 || s.w < 1 || s.c < 1 || s.groups < 1 || s.c % s.groups != 0) return TT_ERR_BAD_ARG;
    if (s.dtype != TT_F32 && s.dtype != TT_BF16) return TT_ERR_BAD_ARG;
    *l = tt_norm_launch{};
    const int64_t pixels = (int64_t)s.h * s.w, cus = compute_units();
    if (s.n > 65535 || s.c > (1 << 20) || pixels > (1 << 30) || pixels > INT32_MAX / s.n) return TT_ERR_UNSUPPORTED;
    *lay = NormLayout{};
    NormArgs &g = lay->args;
    g.n = s.n, g.pixels = (int32_t)pixels, g.c = s.c, g.groups = s.groups, g.wide = s.c / s.groups;
    g.div_wide = make_fastdiv((uint32_t)g.wide);
    g.div_stat_tiles = make_fastdiv(1);
    g.each = 1.0 / ((double)pixels * g.wide);
    // vectors of a row; rows of 8-bit blocks are whole blocks of 16 vectors
    const int V = norm_vector(s.dtype, fp8), unit = fp8 ? 16 : 1;
    g.div_wide_vectors = make_fastdiv((uint32_t)std::max(1, g.wide / V));
    const int columns = (int32_t)(fp8 ? fp8_blocks(s.c) * 16 : (s.c + V - 1) / V);

    // One pass: column tiles of whole groups whose pixels the registers of a workgroup hold, kNormBatch pixels a thread.  The fewest
    // groups that are whole vectors make the most workgroups, but an image's rows in pieces of 16 bytes; where that many
    // workgroups are not needed, tiles are wider, up to 256 bytes, and up to 128 with more pixels a thread (64 x 28 x 28 x 256 bf16 in
    // pieces of 16 bytes 50 us, 32 bytes 25, two passes 22, 128 bytes 16; 256 x 14 x 14 x 256 50, two passes 22, here 17; 8 x 14 x 14 x 512
    // 5.9, two passes 9.2).
    const int held = norm_held(s.dtype, fp8);
    const int64_t group_tile = (int64_t)g.wide / std::gcd(g.wide, V * unit) * (V * unit); // channels
    int tile = s.c % group_tile == 0 ? (int)std::min<int64_t>(group_tile / V, columns) : columns;
    auto fits = [&](int tx, int rows) { return tx <= kNormWidest && pixels <= (512 / tx) * (int64_t)rows; };
    auto many_workgroups = [&](int tx) { return (int64_t)s.n * ((columns + tx - 1) / tx) >= cus; };
    if (fits(tile, kNormBatch))
        lay->one_pass = kNormBatch;
    else if (fits(tile, held) && many_workgroups(tile))
        lay->one_pass = held;
    if (lay->one_pass) {
        while (tile < 16 && columns % (2 * tile) == 0 && many_workgroups(2 * tile)) {
            if (!fits(2 * tile, lay->one_pass)) {
                if (tile >= 8 || !fits(2 * tile, held)) break;
                lay->one_pass = held;
            }
            tile *= 2;
        }
        g.t = tiles_of(columns, tile, 512, pixels);
        g.t.parts = 1, g.t.part_pixels = (int32_t)pixels;
        l->kernel = TT_NORM_ONE_PASS;
        l->chunks = 0;
    } else {
        // Two passes.  The first in column tiles of whole groups (of some 256 bytes, so that an image makes many workgroups and
        // still few parts) where one has room for a group; every workgroup of the second reads the statistics of all parts of its
        // groups, so that there are at most 64 of them (more where a thread's float32 sums would run over more than kNormJoined
        // batches), and its tiles are 16 vectors wide.
        const int SV = norm_vector(s.dtype, false); // (vectors of eight fp32 channels would hold too many registers: 129)
        const int64_t whole = (int64_t)g.wide / std::gcd(g.wide, SV); // vectors of the fewest whole groups
        const int channels = (s.c + SV - 1) / SV; // vectors that hold any
        const int even = (channels + kNormWidest - 1) / kNormWidest; // column tiles of equal width
        const bool aligned = whole <= kNormWidest || channels <= kNormWidest;
        const int first_tx = whole <= kNormWidest ? (int)std::min<int64_t>(channels, whole * ((15 + whole) / whole)) : aligned ? channels : (channels + even - 1) / even;
        lay->first = tiles_of(channels, first_tx, 512, pixels);
        const int64_t others = (int64_t)s.n * lay->first.tiles;
        const int64_t longest = (int64_t)lay->first.ty * kNormBatch * kNormJoined; // pixels of a part
        set_parts(lay->first, std::max(std::min<int64_t>(64, (2 * cus + others - 1) / others), (pixels + longest - 1) / longest), kNormBatch, pixels);
        g.stat_parts = lay->first.parts, g.stat_pixels = lay->first.part_pixels;
        g.stat_tiles = aligned ? 1 : lay->first.tiles, g.stat_width = lay->first.tx * SV;
        g.div_stat_tiles = make_fastdiv((uint32_t)g.stat_tiles);
        // The second in at most four workgroups a CU, which run together (16 x 32 x 32 x 1280 into 8 bits 33.6 -> 32.1 us for 4.4 of
        // them), with many pixels a thread at a time where it has so many.
        const int many = norm_many(s.dtype, fp8);
        const int threads = (int64_t)s.n * columns * pixels < 4 * cus * 512 * kNormFew ? 256 : 512;
        g.t = tiles_of(columns, std::min(columns, 16), threads, pixels);
        const int64_t besides = (int64_t)s.n * g.t.tiles;
        set_parts(g.t, 4 * cus / besides, kNormFew, pixels);
        lay->few = g.t.part_pixels < (int64_t)g.t.ty * many;
        const int64_t bytes = (int64_t)s.n * pixels * s.c * (s.dtype == TT_F32 ? 4 : 2);
        g.past = !fp8 && s.c % V == 0 && bytes >= kNormPast;
        l->kernel = TT_NORM_TWO_PASS;
        l->chunks = g.stat_parts;
        l->workspace_bytes = (int64_t)s.n * s.groups * g.stat_parts * g.stat_tiles * (int64_t)sizeof(float2);
    }
    if ((int64_t)g.t.parts * g.t.tiles * block_of(g.t) > INT32_MAX) return TT_ERR_UNSUPPORTED;
    l->grid = g.t.parts * g.t.tiles;
    l->block = block_of(g.t);
    return TT_OK;
}

// (WHOLE: rows of c are whole vectors)
template <int DT, bool FP8, int ACT, bool WHOLE> void launch_last(const NormLayout &lay, void *stream)
{
    constexpr int V = norm_vector(DT, FP8);
    const NormArgs &g = lay.args;
    const int width = std::min(g.t.tx * V, g.c);
    const int stat_bytes = std::min(g.groups, width / g.wide + 2) * (int)sizeof(float2);
    const dim3 grid(g.t.parts * g.t.tiles, g.n), block(block_of(g.t));
    hipStream_t s = static_cast<hipStream_t>(stream);
    const int lds = g.t.ty * width * (int)sizeof(float2) + stat_bytes;
    if (lay.one_pass == kNormBatch)
        hipLaunchKernelGGL((norm_one_pass_kernel<DT, V, kNormBatch, FP8, ACT, WHOLE>), grid, block, lds, s, g);
    else if (lay.one_pass)
        hipLaunchKernelGGL((norm_one_pass_kernel<DT, V, norm_held(DT, FP8), FP8, ACT, WHOLE>), grid, block, lds, s, g);
    else if (lay.few)
        hipLaunchKernelGGL((norm_apply_kernel<DT, V, kNormFew, FP8, ACT, WHOLE>), grid, block, stat_bytes, s, g);
    else
        hipLaunchKernelGGL((norm_apply_kernel<DT, V, norm_many(DT, FP8), FP8, ACT, WHOLE>), grid, block, stat_bytes, s, g);
}

template <int DT, bool FP8, bool WHOLE> int launch(NormLayout &lay, int act, void *stream)
{
    if (!lay.one_pass) {
        constexpr int V = norm_vector(DT, false);
        NormArgs g = lay.args;
        g.t = lay.first;
        g.div_wide_vectors = make_fastdiv((uint32_t)std::max(1, g.wide / V));
        const int lds = g.t.ty * std::min(g.t.tx * V, g.c) * (int)sizeof(float2);
        // (fp32 rows of whole vectors of eight are rows of whole vectors of four)
        hipLaunchKernelGGL((norm_statistics_kernel<DT, V, kNormBatch, WHOLE>), dim3(g.t.parts * g.t.tiles, g.n), dim3(block_of(g.t)), lds, static_cast<hipStream_t>(stream), g);
        if (const hipError_t e = hipGetLastError(); e != hipSuccess) return note_hip_error((int)e, "norm_statistics_kernel launch");
    }
    lay.args.top = act == TT_ACT_RELU6 ? 6.0f : INFINITY;
    switch (act) {
    case TT_ACT_NONE: launch_last<DT, FP8, NORM_NONE, WHOLE>(lay, stream); break;
    case TT_ACT_GELU: launch_last<DT, FP8, NORM_GELU, WHOLE>(lay, stream); break;
    case TT_ACT_SILU: launch_last<DT, FP8, NORM_SILU, WHOLE>(lay, stream); break;
    default: launch_last<DT, FP8, NORM_CLAMP, WHOLE>(lay, stream); break;
    }
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? TT_OK : note_hip_error((int)e, "group norm launch");
}

template <bool FP8> int launch(NormLayout &lay, int dtype, int act, void *stream)
{
    const bool whole = lay.args.c % norm_vector(dtype, FP8) == 0;
    if (dtype == TT_F32) return whole ? launch<TT_F32, FP8, true>(lay, act, stream) : launch<TT_F32, FP8, false>(lay, act, stream);
    return whole ? launch<TT_BF16, FP8, true>(lay, act, stream) : launch<TT_BF16, FP8, false>(lay, act, stream);
}

int run(const void *x, const void *gamma, const void *beta, void *y, float *scale, const tt_norm_shape *shape, int act, float eps,
        void *ws, size_t ws_bytes, bool fp8, void *stream)
{
    if (!shape || !x || !y || (fp8 && !scale)) return TT_ERR_BAD_ARG;
    for (const void *p : {x, gamma, beta, (const void *)y, (const void *)scale})
        if (!aligned16(p)) return TT_ERR_BAD_ARG;
    if (act < TT_ACT_NONE || act > TT_ACT_SILU || !(eps >= 0.0f)) return TT_ERR_BAD_ARG;
    tt_norm_launch l;
    NormLayout lay;
    if (const int rc = lay_out(*shape, fp8, &lay, &l); rc != TT_OK) return rc;
    if (l.workspace_bytes > 0 && (!ws || !aligned16(ws) || (int64_t)ws_bytes < l.workspace_bytes)) return TT_ERR_WORKSPACE;
    NormArgs &g = lay.args;
    g.x = x, g.gamma = gamma, g.beta = beta, g.y = y, g.scale = scale, g.ws = static_cast<float2 *>(ws), g.eps = eps;
    return fp8 ? launch<true>(lay, shape->dtype, act, stream) : launch<false>(lay, shape->dtype, act, stream);
}

} // namespace
} // namespace tt

using namespace tt;

extern "C" int tt_norm_plan(const tt_norm_shape *shape, int fp8, tt_norm_launch *launch)
{
    NormLayout lay;
    return shape && launch ? lay_out(*shape, fp8 != 0, &lay, launch) : TT_ERR_BAD_ARG;
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
