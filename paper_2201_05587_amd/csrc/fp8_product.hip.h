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
    int32_t tiles_m, tiles_n, splits, split_steps; // of a launch in tiles: splits of the reduction, steps of one
};

// The two 16-byte pieces of a row's 128 bytes that a lane multiplies: pieces g and g + 4 of the eight, g = lane / 16.
struct Fragment {
    u32x4 lo, hi;
};

// The sums of 128 products, 16 rows of B by 16 rows of A, of operands in the form that the matrix cores take (Held: as they wait in
// registers).
typedef __attribute__((ext_vector_type(4))) int i32x4;
template <int DT> struct BlockProduct;
template <> struct BlockProduct<TT_BF16> {
    using Operand = i32x8;
    using Held = i32x8;
    static __device__ __forceinline__ Operand operand(const Held &h) { return h; }
    static __device__ __forceinline__ Held hold(const Fragment &f)
    {
        return __builtin_shufflevector(__builtin_bit_cast(i32x4, f.lo), __builtin_bit_cast(i32x4, f.hi), 0, 1, 2, 3, 4, 5, 6, 7);
    }
    static __device__ __forceinline__ f32x4 run(const Operand &b, const Operand &a)
    {
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a, f32x4{0.0f, 0.0f, 0.0f, 0.0f}, 0, 0, 0, 0, 0, 0);
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
    struct Operand {
        bf16x8 v[4];
    };
    using Held = Fragment;
    static __device__ __forceinline__ Held hold(const Fragment &f) { return f; }
    static __device__ __forceinline__ Operand operand(const Fragment &f)
    {
        return {{widen_fp8(f.lo[0], f.lo[1]), widen_fp8(f.lo[2], f.lo[3]), widen_fp8(f.hi[0], f.hi[1]), widen_fp8(f.hi[2], f.hi[3])}};
    }
    static __device__ __forceinline__ f32x4 run(const Operand &b, const Operand &a)
    {
        f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int s = 0; s < 4; ++s) sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b.v[s], a.v[s], sum, 0, 0, 0);
        return sum;
    }
};

// A block's sum p counts p * sa * sb.  p is 0 or between 2^-18 and 2^25 (128 products of e4m3 values), and scales go from 2^-109 to 2^119 (a / 448,
// a from 2^-100 on), so that p * sa * sb may be an ordinary float32 number where a part of it is not: two scales of 2^-70 leave
// ten bits of their product, and two of 2^70 an infinity, which makes a NaN of a sum of 0.
//   rows of B that share a scale: sa * sb is formed once for all sums of a row of A, times 2^92, which makes the smallest (2^-218, zeros beside
//   zeros) a normal number, and the sums are taken back by 2^-92 at the end: the same bits;
//   a scale for each row of B: (p * sa) * sb, as many instructions as p * (sa * sb), where p * sa is 2^-127 at least.
// What overflows that way (results from 2^36 on, or scales beyond any use) leaves a sum that is not finite.  A wave that has one computes its sums
// again, from memory, the smaller scale first where sa * sb or p * sa is no ordinary number: p * smaller overflows only where both are
// above 2^100 and the result is infinite too.  (Where every wave does, 4096^3 takes 1.4 ms for 63 us; with both ways in the loop the
// accumulators do not fit the registers, and looking at every scale there costs a tenth.)
constexpr float kRaised = 0x1p92f;
// x * 0 added up: a NaN once one of the values is not finite
__device__ __forceinline__ void note_not_finite(float &none, f32x4 v)
{
#pragma unroll
    for (int e = 0; e < 4; ++e) none = fmaf(v[e], 0.0f, none);
}
__device__ __forceinline__ bool wave_sums_again(float none) { return __builtin_amdgcn_ballot_w64(none != none) != 0; }
template <int B_ROWS> __device__ __forceinline__ float add_near(float p, float sa, float sb, float both, float sum) // both: sa * sb, raised or not
{
    return B_ROWS > 1 ? fmaf(p, both, sum) : fmaf(p * sa, sb, sum);
}
template <int B_ROWS> __device__ __forceinline__ float add_any(float p, float sa, float sb, float sum)
{
    const float both = sa * sb, first = B_ROWS > 1 ? both : p * sa;
    const bool swap = fabsf(sa) > fabsf(sb);
    const bool near = B_ROWS > 1 ? __builtin_isnormal(first) : __builtin_isfinite(first);
    return near ? add_near<B_ROWS>(p, sa, sb, both, sum) : fmaf(p * (swap ? sb : sa), swap ? sa : sb, sum);
}
// The sums of one lane over steps begin, begin + by ..: a, b: its row's piece of step 0; a_scale: of its row, b_scale: of four rows of B.
template <int DT, int B_ROWS>
__device__ __forceinline__ f32x4 sums_of_any_scales(const ProductArgs &g, const uint8_t *a, const uint8_t *b, const float *a_scale, const float *b_scale,
                                                    const int (&b_row)[4], int begin, int end, int by)
{
    using P = BlockProduct<DT>;
    f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 1
    for (int t = begin; t < end; t += by) {
        Fragment x, y;
        load16(x.lo, a + t * kFp8Block), load16(x.hi, a + t * kFp8Block + 64);
        load16(y.lo, b + t * kFp8Block), load16(y.hi, b + t * kFp8Block + 64);
        const f32x4 p = P::run(P::operand(P::hold(y)), P::operand(P::hold(x)));
        const float sa = a_scale[(int64_t)t * g.M];
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] = add_any<B_ROWS>(p[e], sa, b_scale[(int64_t)t * g.b_scale_row + b_row[e]], sum[e]);
    }
    return sum;
}

// Position of a row's 16-byte pieces in the LDS: piece c of row r lies at c ^ swizzle(r).  A fragment's 16 lanes read one piece of
// 16 rows, which the swizzle spreads over all banks (256 bytes, two rows).
//   rows of A: r, r + 1, ... r + 15;   rows of B: 8 (i / 4) + i % 4 (+ 4), i = 0 .. 15, so that the matrix cores leave eight
//   consecutive columns of the result in a lane.
__device__ __forceinline__ int a_swizzle(int r) { return (r >> 1) & 7; }
__device__ __forceinline__ int b_swizzle(int r) { return ((r >> 1) & 1) | ((r >> 2) & 6); }

__device__ __forceinline__ void load4_to_lds(__amdgpu_buffer_rsrc_t rsrc, uint32_t byte_offset, uint32_t lds_addr)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds"
                 :
                 : "s"(lds_addr), "v"(byte_offset), "s"(rsrc)
                 : "memory", "m0");
}

// Eight consecutive columns of one row of the result.
template <int DT> __device__ __forceinline__ void store_eight(void *out, int64_t at, const float (&v)[8], int count);
template <> __device__ __forceinline__ void store_eight<TT_BF16>(void *out, int64_t at, const float (&v)[8], int count)
{
    const u32x4 r = {pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
    store_piece<TT_BF16>(out, at, r, count);
}
template <> __device__ __forceinline__ void store_eight<TT_F32>(void *out, int64_t at, const float (&v)[8], int count)
{
    store_piece<TT_F32>(out, at, u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])}, min(count, 4));
    if (count > 4)
        store_piece<TT_F32>(out, at + 4, u32x4{__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7])}, count - 4);
}
template <int DT> __device__ __forceinline__ void load_eight(float (&v)[8], const void *p, int64_t at, int count)
{
#pragma unroll
    for (int h = 0; h < 8; h += ElemOf<DT>::CH) {
        const u32x4 r = count > h ? load_piece<DT>(p, at + h, count - h) : u32x4{0u, 0u, 0u, 0u};
#pragma unroll
        for (int e = 0; e < ElemOf<DT>::CH; ++e) v[h + e] = element_of<DT>(r, e);
    }
}

// Bias and activation of N (a multiple of 4) results.  A NaN stays one.
template <int N> __device__ __forceinline__ void finish_results(float (&v)[N], const float (&bias)[N], int act)
{
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] += bias[e];
    if (act == ACT_RELU) {
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = v[e] < 0.0f ? 0.0f : v[e];
    } else if (act == ACT_GELU) {
#pragma unroll
        for (int e = 0; e < N; e += 4) {
            const f32x4 r = gelu_smooth4(f32x4{v[e], v[e + 1], v[e + 2], v[e + 3]});
            v[e] = r[0], v[e + 1] = r[1], v[e + 2] = r[2], v[e + 3] = r[3];
        }
    }
}

// Pieces of 16 rows of A by 32 of B, stored: a_row(i), b_row(j): the rows that the lane multiplies, of B the first of two, 4 apart; n(j): the first of
// the eight outputs that it then holds.
template <int DT, int B_ROWS, class RowOfA, class RowOfB, class N>
__device__ __forceinline__ void store_with_any_scales(const ProductArgs &g, int pieces_of_a, int pieces_of_b, int begin, int end, RowOfA &&a_row, RowOfB &&b_row, N &&n_of)
{
    const int64_t batch = blockIdx.y, kp = (int64_t)g.kb * kFp8Block;
    const int piece = (int)(threadIdx.x & 63) / 16 * 16;
#pragma unroll 1
    for (int i = 0; i < pieces_of_a; ++i)
#pragma unroll 1
        for (int j = 0; j < pieces_of_b; ++j) {
            const int m = a_row(i), n = n_of(j), m_in = min(m, g.M - 1); // rows past a matrix read its last row; what they give is not stored
            float v[8];
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                int scale_row[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) scale_row[e] = min(n + half * 4 + e, g.N - 1) / B_ROWS;
                const f32x4 sum = sums_of_any_scales<DT, B_ROWS>(
                    g, g.a + (batch * g.M + m_in) * kp + piece, g.b + (batch * g.N + min(b_row(j) + half * 4, g.N - 1)) * kp + piece,
                    g.a_scale + batch * g.kb * g.M + m_in, g.b_scale + batch * g.kb * g.b_scale_row, scale_row, begin, end, 1);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[half * 4 + e] = sum[e];
            }
            if (m >= g.M || n >= g.N) continue;
            const int64_t at = (batch * g.M + m) * g.N + n;
            if (g.splits > 1)
                store_eight<TT_F32>(g.ws + (int64_t)blockIdx.z * g.batch * g.M * g.N, at, v, g.N - n);
            else {
                float bias[8] = {};
                if (g.bias) load_eight<DT>(bias, g.bias, n, g.N - n);
                finish_results<8>(v, bias, g.act);
                store_eight<DT>(g.out, at, v, g.N - n);
            }
        }
}

// Tile `wg` of tiles_m x tiles_n: a contiguous run of tiles per XCD, walked in bands of `band` tile rows, so that the tiles an XCD
// works on at a time form a rectangle and its L2 serves each operand row to several of them.
__device__ __forceinline__ void place_of_tile(int wg, int tiles_m, int tiles_n, int band_rows, int *im, int *in)
{
    const int total = tiles_m * tiles_n, per = total / kXcds, rem = total % kXcds, x = wg % kXcds;
    const int L = x * per + min(x, rem) + wg / kXcds;
    const int band = L / (band_rows * tiles_n), at = L - band * band_rows * tiles_n, high = min(band_rows, tiles_m - band * band_rows);
    *in = at / high;
    *im = band * band_rows + at - *in * high;
}

// ---- few rows of A: B streams past them ----------------------------------------------------------------------------------
// A workgroup has 16 rows of B and all of A's (16 MS of them), its eight waves every eighth step of the reduction; fragments come from memory as
// they are, UNROLL steps of loads in flight, and the waves' sums meet in the LDS.  What is read is B, once, and A by every
// workgroup (from the L2): the kernel for a token or a few, whose time is B's bytes, up to two workgroups a CU (1 x 4096 x 4096 5.6 us, 3.0 TB/s).
template <int MS> struct Stream {
    static constexpr int WAVES = 8, UNROLL = 4;
};
template <int DT, int MS> __global__ void __launch_bounds__(512) product_stream_kernel(const ProductArgs g)
{
    using S = Stream<MS>;
    using P = BlockProduct<DT>;
    __shared__ f32x4 sums[S::WAVES][MS][64];
    const int tid = threadIdx.x, lane = tid % 64, wave = __builtin_amdgcn_readfirstlane(tid / 64), r = lane % 16, part = lane / 16;
    const int n0 = (int)blockIdx.x * 16;
    const int64_t kp = (int64_t)g.kb * kFp8Block, batch = blockIdx.y;
    // rows past a matrix read its last row; what they give is not stored
    const uint8_t *const b = g.b + (batch * g.N + min(n0 + r, g.N - 1)) * kp + part * 16;
    const float *const b_scale = g.b_scale + batch * g.kb * g.b_scale_row;
    const float *const a_scale = g.a_scale + batch * g.kb * g.M;
    const uint8_t *a[MS];
    int row[MS], b_row[4];
#pragma unroll
    for (int i = 0; i < MS; ++i) {
        row[i] = min(i * 16 + r, g.M - 1);
        a[i] = g.a + (batch * g.M + row[i]) * kp + part * 16;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) b_row[e] = min(n0 + part * 4 + e, g.N - 1) / g.b_rows;
    f32x4 sum[MS] = {};
    for (int first = wave; first < g.kb; first += S::WAVES * S::UNROLL) {
        Fragment x[S::UNROLL], y[S::UNROLL][MS];
        float sa[S::UNROLL][MS], sb[S::UNROLL][4];
#pragma unroll
        for (int u = 0; u < S::UNROLL; ++u) {
            const int j = first + u * S::WAVES;
            if (j >= g.kb) break; // (the same for the whole wave)
            load16(x[u].lo, b + j * kFp8Block), load16(x[u].hi, b + j * kFp8Block + 64);
#pragma unroll
            for (int i = 0; i < MS; ++i) {
                load16(y[u][i].lo, a[i] + j * kFp8Block), load16(y[u][i].hi, a[i] + j * kFp8Block + 64);
                sa[u][i] = a_scale[(int64_t)j * g.M + row[i]];
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) sb[u][e] = b_scale[(int64_t)j * g.b_scale_row + b_row[e]];
        }
#pragma unroll
        for (int u = 0; u < S::UNROLL; ++u) {
            if (first + u * S::WAVES >= g.kb) break;
            const typename P::Operand bx = P::operand(P::hold(x[u]));
#pragma unroll
            for (int i = 0; i < MS; ++i) {
                const f32x4 p = P::run(bx, P::operand(P::hold(y[u][i])));
                const float raised = sa[u][i] * kRaised;
#pragma unroll
                for (int e = 0; e < 4; ++e) sum[i][e] = fmaf(p[e], raised * sb[u][e], sum[i][e]);
            }
        }
    }
    float none = 0.0f;
#pragma unroll
    for (int i = 0; i < MS; ++i) {
        note_not_finite(none, sum[i]);
        sum[i] *= 1.0f / kRaised; // (the scales are multiplied with each other first, whatever b_rows)
    }
    if (__builtin_expect(wave_sums_again(none), 0)) {
#pragma unroll
        for (int i = 0; i < MS; ++i) sum[i] = sums_of_any_scales<DT, kFp8Block>(g, a[i], b, a_scale + row[i], b_scale, b_row, wave, g.kb, S::WAVES);
    }
#pragma unroll
    for (int i = 0; i < MS; ++i) sums[wave][i][lane] = sum[i];
    __syncthreads();
    if (wave >= MS) return;
    const int m = wave * 16 + r, n = n0 + part * 4;
    if (m >= g.M || n >= g.N) return;
    float v[4] = {}, bias[4] = {};
#pragma unroll
    for (int w = 0; w < S::WAVES; ++w)
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += sums[w][wave][lane][e];
    if (g.bias)
#pragma unroll
        for (int e = 0; e < 4; ++e) bias[e] = load_as_float<DT>(g.bias, min(n + e, g.N - 1));
    finish_results<4>(v, bias, g.act);
    const int64_t at = (batch * g.M + m) * g.N + n;
    if constexpr (DT == TT_F32)
        store_piece<TT_F32>(g.out, at, u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])}, g.N - n);
    else if (g.N - n >= 4) {
        const uint2 q = {pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
        __builtin_memcpy(static_cast<uint16_t *>(g.out) + at, &q, 8);
    } else
        store_piece<TT_BF16>(g.out, at, u32x4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), 0u, 0u}, g.N - n);
}

// ---- tiles -----------------------------------------------------------------------------------------------------------
// TM x TN outputs a workgroup of four waves (2 x 2), steps of the reduction through a ring of LDS buffers that asynchronous loads
// fill two to three steps ahead, one barrier a step.  A workgroup of 128 x 128 has a CU to itself, and its waves read the next step's
// fragments before they multiply the present one's; of 64 x 64 a CU has three, which run past each other.
// Both float32 and bf16 results, and splits of the reduction where the tiles are too few for the chip: their sums go to the
// workspace, and product_reduce_kernel adds them.
template <int TM, int TN> struct Tiles {
    static constexpr bool AHEAD = TM * TN > 64 * 64; // fragments of the next step are read before the present one is multiplied
    static constexpr int THREADS = 256, RING = AHEAD ? 4 : 3, WM = TM / 2, WN = TN / 2, MI = WM / 16, NJ = WN / 16;
    static constexpr int A_BYTES = TM * kFp8Block, B_BYTES = TN * kFp8Block, SCALES = 1024, STAGE = A_BYTES + B_BYTES + SCALES;
    static constexpr int LOADS = (TM + TN) / 32 + 1; // of a thread and step: 16-byte items, and one scale
    static constexpr int LDS = RING * STAGE, BAND = 8;
    static_assert(TM + TN <= THREADS && WN % 32 == 0, "");
};
template <int DT, int TM, int TN, int B_ROWS> __global__ void __launch_bounds__(256, 2) product_tile_kernel(const ProductArgs g)
{
    using S = Tiles<TM, TN>;
    using P = BlockProduct<DT>;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const uint32_t lds0 = lds_address(smem);
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave & 1, wn = wave >> 1;
    int im, in;
    place_of_tile((int)blockIdx.x, g.tiles_m, g.tiles_n, S::BAND, &im, &in);
    const int m0 = im * TM, n0 = in * TN;
    const int64_t batch = blockIdx.y;
    const int begin = (int)blockIdx.z * g.split_steps, end = min(begin + g.split_steps, g.kb);
    const uint32_t kp = (uint32_t)g.kb * kFp8Block;
    const __amdgpu_buffer_rsrc_t a_rsrc = make_rsrc(g.a + (batch * g.M + m0) * kp, (uint32_t)min(TM, g.M - m0) * kp);
    const __amdgpu_buffer_rsrc_t b_rsrc = make_rsrc(g.b + (batch * g.N + n0) * kp, (uint32_t)min(TN, g.N - n0) * kp);
    // this thread's piece of its first row; its others lie 32 rows apart (rows past the matrix are past the end of the buffer)
    const int first = tid / 8;
    const uint32_t a_at = first * kp + ((tid % 8) ^ a_swizzle(first)) * 16, b_at = first * kp + ((tid % 8) ^ b_swizzle(first)) * 16;
    const float *const a_scales = g.a_scale + batch * g.kb * g.M + m0, *const b_scales = g.b_scale + batch * g.kb * g.b_scale_row + n0 / B_ROWS;
    auto request = [&](int t) {
        const uint32_t to = lds0 + (uint32_t)((t % S::RING) * S::STAGE);
        const uint32_t k0 = t < end ? (uint32_t)t * kFp8Block : kOutOfRange; // (the other offsets are below 2^30)
#pragma unroll
        for (int i = 0; i < TM / 32; ++i) load16_to_lds(a_rsrc, a_at + (uint32_t)(i * 32) * kp + k0, to + (uint32_t)((i * 256 + wave * 64) * 16));
#pragma unroll
        for (int i = 0; i < TN / 32; ++i) load16_to_lds(b_rsrc, b_at + (uint32_t)(i * 32) * kp + k0, to + (uint32_t)(S::A_BYTES + (i * 256 + wave * 64) * 16));
        // waves of A's rows, of B's, and (small tiles) waves without a row: a load each, so that all count alike
        const int at = min(t, g.kb - 1);
        const int row = tid - (wave * 64 < TM ? 0 : TM);
        const __amdgpu_buffer_rsrc_t rsrc = wave * 64 < TM ? make_rsrc(a_scales + (int64_t)at * g.M, 4u * (uint32_t)min(TM, g.M - m0))
                                                           : make_rsrc(b_scales + (int64_t)at * g.b_scale_row, 4u * (uint32_t)((min(TN, g.N - n0) + B_ROWS - 1) / B_ROWS));
        load4_to_lds(rsrc, wave * 64 < TM ? 4u * (uint32_t)row : row < TN ? 4u * (uint32_t)(row / B_ROWS) : kOutOfRange, to + (uint32_t)(S::A_BYTES + S::B_BYTES + wave * 256));
    };
    f32x4 acc[S::MI][S::NJ];
#pragma unroll
    for (int i = 0; i < S::MI; ++i)
#pragma unroll
        for (int j = 0; j < S::NJ; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const int lane_r = lane % 16, lane_g = lane / 16;
    const int a_row = wm * S::WM + lane_r, b_row = wn * S::WN + lane_r / 4 * 8 + lane_r % 4;
    const int a_from = a_row * kFp8Block + (lane_g ^ a_swizzle(a_row)) * 16, b_from = S::A_BYTES + b_row * kFp8Block + (lane_g ^ b_swizzle(b_row)) * 16;
    // what a wave multiplies in a step
    struct Step {
        typename P::Held a[S::MI], b[S::NJ];
    };
    auto fragment = [&](const unsigned char *from, int at) {
        return P::hold({*reinterpret_cast<const u32x4 *>(from + at), *reinterpret_cast<const u32x4 *>(from + (at ^ 64))});
    };
    auto read = [&](Step &s, int t) {
        const unsigned char *const from = smem + (t % S::RING) * S::STAGE;
#pragma unroll
        for (int i = 0; i < S::MI; ++i) s.a[i] = fragment(from + i * 16 * kFp8Block, a_from);
#pragma unroll
        for (int j = 0; j < S::NJ; ++j) s.b[j] = fragment(from + (j / 2 * 32 + j % 2 * 4) * kFp8Block, b_from); // (the same swizzle)
    };
    // the scales of step t: of the lane's rows of A (times that of B, where it is one), and of its four rows of B's block j
    const int a_scale_at = S::A_BYTES + S::B_BYTES + 4 * a_row, b_scale_at = S::A_BYTES + S::B_BYTES + 4 * (TM + wn * S::WN + lane_g * 8);
    auto read_scales = [&](float (&sa)[S::MI], f32x4 &sb, int t) {
        const unsigned char *const from = smem + (t % S::RING) * S::STAGE;
#pragma unroll
        for (int i = 0; i < S::MI; ++i) sa[i] = *reinterpret_cast<const float *>(from + a_scale_at + i * 64);
        if constexpr (B_ROWS == 1)
            sb = *reinterpret_cast<const f32x4 *>(from + b_scale_at);
        else
            sb[0] = *reinterpret_cast<const float *>(from + b_scale_at);
    };
    auto multiply = [&](const Step &s, float (&sa)[S::MI], f32x4 sb, int t) {
        constexpr int COUNT = S::MI * S::NJ, LAG = COUNT < 8 ? 2 : 3; // matrix instructions issued before the first one's products are used
        const unsigned char *const from = smem + (t % S::RING) * S::STAGE + b_scale_at;
        if constexpr (B_ROWS > 1) {
            const float raised = sb[0] * kRaised;
#pragma unroll
            for (int i = 0; i < S::MI; ++i) sa[i] *= raised;
        }
        f32x4 part[COUNT], sb_next = sb;
        auto accumulate = [&](int x) {
            const int i = x % S::MI, j = x / S::MI;
            if (B_ROWS == 1 && i == 0) { // the next four rows' scales a block ahead
                sb = sb_next;
                if (j + 1 < S::NJ) sb_next = *reinterpret_cast<const f32x4 *>(from + 4 * ((j + 1) / 2 * 32 + (j + 1) % 2 * 4));
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[i][j][e] = add_near<B_ROWS>(part[x][e], sa[i], sb[e], sa[i], acc[i][j][e]);
            asm volatile("" : "+v"(acc[i][j])); // (keeps the FMAs here, between the matrix instructions)
        };
        if constexpr (DT == TT_BF16) {
#pragma unroll
            for (int x = 0; x < COUNT; ++x) {
                part[x] = P::run(P::operand(s.b[x / S::MI]), P::operand(s.a[x % S::MI]));
                __builtin_amdgcn_sched_barrier(0);
                if (x >= LAG) accumulate(x - LAG);
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int x = COUNT - LAG; x < COUNT; ++x) accumulate(x);
        } else {
            typename P::Operand a[S::MI];
#pragma unroll
            for (int i = 0; i < S::MI; ++i) a[i] = P::operand(s.a[i]);
#pragma unroll
            for (int j = 0; j < S::NJ; ++j) {
                const typename P::Operand b = P::operand(s.b[j]);
#pragma unroll
                for (int i = 0; i < S::MI; ++i) part[j * S::MI + i] = P::run(b, a[i]);
#pragma unroll
                for (int i = 0; i < S::MI; ++i) accumulate(j * S::MI + i);
            }
        }
    };
#pragma unroll
    for (int t = 0; t < S::RING - 1; ++t) request(begin + t);
    if constexpr (S::AHEAD) {
        wait_loads_outstanding<(S::RING - 2) * S::LOADS>();
        __syncthreads();
        Step now, next;
        read(now, begin);
        auto step = [&](int t, const Step &now, Step &next) {
            float sa[S::MI];
            f32x4 sb;
            wait_loads_outstanding<(S::RING - 3) * S::LOADS>(); // step t + 1 has landed
            __syncthreads();                                    // ... for every wave, and all have multiplied step t - 1
            request(t + S::RING - 1);
            read_scales(sa, sb, t);
            read(next, t + 1); // (past the end: what the requests past the end left, zeros)
            multiply(now, sa, sb, t);
        };
        for (int t = begin; t < end; t += 2) {
            step(t, now, next);
            if (t + 1 < end) step(t + 1, next, now);
        }
    } else
        for (int t = begin; t < end; ++t) {
            Step now;
            float sa[S::MI];
            f32x4 sb;
            wait_loads_outstanding<(S::RING - 2) * S::LOADS>(); // step t has landed
            __syncthreads();                                    // ... for every wave, and all have multiplied step t - 1
            request(t + S::RING - 1);
            read_scales(sa, sb, t);
            read(now, t);
            multiply(now, sa, sb, t);
        }
    wait_loads_outstanding<0>(); // the requests past the end: nothing may still write the LDS when the workgroup ends
    float none = 0.0f;
#pragma unroll
    for (int i = 0; i < S::MI; ++i)
#pragma unroll
        for (int j = 0; j < S::NJ; ++j) {
            note_not_finite(none, acc[i][j]);
            if constexpr (B_ROWS > 1) acc[i][j] *= 1.0f / kRaised;
        }
    if (__builtin_expect(wave_sums_again(none), 0))
        return store_with_any_scales<DT, B_ROWS>(g, S::MI, S::NJ / 2, begin, end, [&](int i) { return m0 + a_row + i * 16; },
                                                 [&](int j) { return n0 + b_row + j * 32; }, [&](int j) { return n0 + wn * S::WN + lane_g * 8 + j * 32; });
#pragma unroll
    for (int jj = 0; jj < S::NJ / 2; ++jj) {
        const int n = n0 + wn * S::WN + jj * 32 + lane_g * 8;
        float bias[8] = {};
        if (g.bias && g.splits == 1 && n < g.N) load_eight<DT>(bias, g.bias, n, g.N - n);
#pragma unroll
        for (int i = 0; i < S::MI; ++i) {
            const int m = m0 + a_row + i * 16;
            if (m >= g.M || n >= g.N) continue;
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = acc[i][jj * 2 + e / 4][e % 4];
            const int64_t at = (batch * g.M + m) * g.N + n;
            if (g.splits > 1)
                store_eight<TT_F32>(g.ws + (int64_t)blockIdx.z * g.batch * g.M * g.N, at, v, g.N - n);
            else {
                finish_results<8>(v, bias, g.act);
                store_eight<DT>(g.out, at, v, g.N - n);
            }
        }
    }
}

// The sums of the splits, in their order, bias, activation: eight columns a thread.
template <int DT> __global__ void __launch_bounds__(256) product_reduce_kernel(const ProductArgs g)
{
    const int per_row = (g.N + 7) / 8;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, row = i / per_row;
    const int n = (int)(i - row * per_row) * 8;
    if (row >= (int64_t)g.batch * g.M) return;
    const int64_t at = row * g.N + n, apart = (int64_t)g.batch * g.M * g.N;
    float v[8], bias[8] = {};
    load_eight<TT_F32>(v, g.ws, at, g.N - n);
#pragma unroll 4
    for (int s = 1; s < g.splits; ++s) {
        float more[8];
        load_eight<TT_F32>(more, g.ws + s * apart, at, g.N - n);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += more[e];
    }
    if (g.bias) load_eight<DT>(bias, g.bias, n, g.N - n);
    finish_results<8>(v, bias, g.act);
    store_eight<DT>(g.out, at, v, g.N - n);
}

} // namespace tt
