// Products of matrices held in 8 bits in 256 x 256 blocks (bf16 results), for launches with enough outputs to give every CU one.
//
// The order of work is that of contract_block.hip.h, whose slices of 64 bf16 elements are as many bytes as a step of 128 here:
// eight waves in two teams take turns at the matrix cores, a step is four phases of one quadrant (64 rows of A by 32 of B a
// wave) each, and every phase requests one region of a later step:
//
//   phase      0            1            2            3
//   multiply   A0 . B0      A0 . B1      A1 . B1      A1 . B0
//   read       A0           B1           A1           B0 of the next step
//   request    B1 (t + 1)   A1 (t + 1)   A0 (t + 2)   B0 (t + 2), scales (t + 2)          (step t, buffer t mod 2)
//
// What is new is the scaling.  A matrix instruction starts from zero, and its four sums a lane go into the accumulators by FMAs
// three instructions later, in issue slots that the matrix cores leave free (32 cycles an instruction, 16 of FMAs); the last three
// of a turn are taken in the next reading turn, so that no wave waits for a product's latency.
// A step's scales, 256 of A and as many of B, come into the LDS with the operands, in a ring of four.
//
// 8192^3: 472 us called in turn on three sets of operands (2.33 PFLOP/s), a scale per row of B 20 % more (eight FMAs and products an
// instruction for four).  The card's power sets its clock, so that the time depends on what ran before: 448 us at best, 500 where launches
// are traced apart, and 374 on operands of zeros, in as many cycles.  Before the scales were raised (454 us for 462 now) it took 416 us
// without the operands' requests and 455 without the stores of the results; fragments read a turn ahead, and two quadrants a turn with
// half the barriers, took the same time to a percent.
#pragma once

#include "fp8_product.hip.h"

namespace tt {

struct Fp8Block {
    static constexpr int BM = 256, BN = 256, THREADS = 512, STEP = 64, NL = 2; // STEP: rows between the NL loads of a thread
    static constexpr int ROW = kFp8Block, REGION = 128 * ROW, SLICE = 4 * REGION;
    static constexpr int SCALES = 512 * 4, RING = 4, LDS = 2 * SLICE + RING * SCALES;
    static constexpr int BAND = 4;
};

template <int B_ROWS> __global__ void __launch_bounds__(512) product_block_kernel(const ProductArgs g)
{
    using S = Fp8Block;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const uint32_t lds0 = lds_address(smem);
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int team = wave >> 2;
    const int wm = team, wn = wave & 3; // 64-row strip of every region of A, 32-row strip of every region of B

    int m0, n0;
    place_of_tile((int)blockIdx.x, g.tiles_m, g.tiles_n, S::BAND, &m0, &n0);
    m0 *= S::BM, n0 *= S::BN;
    const int64_t batch = blockIdx.y;
    const int kb = g.kb;
    const uint32_t kp = (uint32_t)kb * kFp8Block;
    const __amdgpu_buffer_rsrc_t a_rsrc = make_rsrc(g.a + (batch * g.M + m0) * kp, (uint32_t)min(S::BM, g.M - m0) * kp);
    const __amdgpu_buffer_rsrc_t b_rsrc = make_rsrc(g.b + (batch * g.N + n0) * kp, (uint32_t)min(S::BN, g.N - n0) * kp);
    // this thread's piece of its first row of a region: rows past the matrix are past the end of the buffer
    const int first = tid / 8;
    const uint32_t a_at = first * kp + ((tid % 8) ^ a_swizzle(first)) * 16, b_at = first * kp + ((tid % 8) ^ b_swizzle(first)) * 16;
    auto request = [&](__amdgpu_buffer_rsrc_t rsrc, uint32_t at, int region, int h, int t, int buffer) {
        const uint32_t to = lds0 + (uint32_t)(buffer * S::SLICE + region * S::REGION + wave * 64 * 16);
#pragma unroll
        for (int i = 0; i < S::NL; ++i) // (at is below 2^30)
            load16_to_lds(rsrc, at + (t < kb ? (uint32_t)(h * 128 + i * S::STEP) * kp + (uint32_t)t * kFp8Block : kOutOfRange),
                          to + (uint32_t)(i * S::THREADS * 16));
    };
    auto request_a = [&](int h, int t, int buffer) { request(a_rsrc, a_at, h, h, t, buffer); };
    auto request_b = [&](int h, int t, int buffer) { request(b_rsrc, b_at, 2 + h, h, t, buffer); };
    // waves 0-3: the scales of the block's rows of A; waves 4-7: of B (one in 128 rows: the same scale for each of them)
    const float *const scales = team == 0 ? g.a_scale + batch * kb * g.M + m0 : g.b_scale + batch * kb * g.b_scale_row + n0 / B_ROWS;
    const int64_t scale_row = team == 0 ? g.M : g.b_scale_row;
    const uint32_t scale_bytes = 4u * (uint32_t)(team == 0 ? min(S::BM, g.M - m0) : min(S::BN / B_ROWS, g.b_scale_row - n0 / B_ROWS));
    const uint32_t scale_at = 4u * (uint32_t)(team == 0 ? tid : (tid - 256) / B_ROWS);
    auto request_scales = [&](int t) {
        const __amdgpu_buffer_rsrc_t rsrc = make_rsrc(scales + min(t, kb - 1) * scale_row, t < kb ? scale_bytes : 0u);
        load4_to_lds(rsrc, scale_at, lds0 + (uint32_t)(2 * S::SLICE + (t % S::RING) * S::SCALES + wave * 256));
    };

    f32x4 acc[2][2][4][2]; // [A region][B region][16 rows of A][16 rows of B]
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) acc[h][k][i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    const int lane_r = lane % 16, lane_g = lane / 16;
    const int a_row = wm * 64 + lane_r, b_row = wn * 32 + lane_r / 4 * 8 + lane_r % 4;
    // (rows 16 further have A's swizzle unchanged, rows 4 further B's)
    const int a_from = a_row * S::ROW + (lane_g ^ a_swizzle(a_row)) * 16, b_from = b_row * S::ROW + (lane_g ^ b_swizzle(b_row)) * 16;
    using P = BlockProduct<TT_BF16>;
    P::Operand af[4], bf[2][2];
    auto fragment = [&](const unsigned char *from, int at) {
        return P::hold({*reinterpret_cast<const u32x4 *>(from + at), *reinterpret_cast<const u32x4 *>(from + (at ^ 64))});
    };
    auto read_a = [&](int h, int buffer) {
#pragma unroll
        for (int i = 0; i < 4; ++i) af[i] = fragment(smem + buffer * S::SLICE + h * S::REGION + i * 16 * S::ROW, a_from);
    };
    auto read_b = [&](P::Operand (&to)[2], int h, int buffer) {
#pragma unroll
        for (int j = 0; j < 2; ++j) to[j] = fragment(smem + buffer * S::SLICE + (2 + h) * S::REGION + j * 4 * S::ROW, b_from);
    };
    auto swap_teams = [&]() {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("" ::: "memory");
    };
    // the scales of quadrant (h, k) of step t: of A (times that of B, where it is one), and of B's rows
    float sa[4], sb[B_ROWS == 1 ? 8 : 1];
    struct Scales {
        float a[4], b[B_ROWS == 1 ? 8 : 1];
    };
    auto read_scales = [&](int h, int k, int t) {
        const float *const from = reinterpret_cast<const float *>(smem + 2 * S::SLICE + (t % S::RING) * S::SCALES);
        Scales s;
#pragma unroll
        for (int e = 0; e < (B_ROWS == 1 ? 8 : 1); ++e) s.b[e] = from[256 + k * 128 + (B_ROWS == 1 ? wn * 32 + lane_g * 8 + e : 0)];
#pragma unroll
        for (int i = 0; i < 4; ++i) s.a[i] = from[h * 128 + a_row + i * 16];
        return s;
    };
    auto take_scales = [&](const Scales &s) {
        __builtin_amdgcn_sched_barrier(0); // (waits for them behind the FMAs of finish)
        const float raised = s.b[0] * kRaised;
#pragma unroll
        for (int i = 0; i < 4; ++i) sa[i] = B_ROWS == 1 ? s.a[i] : s.a[i] * raised;
#pragma unroll
        for (int e = 0; e < (B_ROWS == 1 ? 8 : 1); ++e) sb[e] = s.b[e];
    };
    f32x4 part[8]; // products of the matrix instructions of a quadrant, 2 i + j
    auto accumulate = [&](f32x4 (&c)[4][2], int x) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            c[x / 2][x % 2][e] = add_near<B_ROWS>(part[x][e], sa[x / 2], sb[(x % 2 * 4 + e) % (B_ROWS == 1 ? 8 : 1)], sa[x / 2], c[x / 2][x % 2][e]);
    };
    constexpr int LAG = 3; // matrix instructions issued before the first one's products are used
    auto multiply = [&](f32x4 (&c)[4][2], const P::Operand (&b)[2]) {
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int x = 0; x < 8; ++x) {
            part[x] = P::run(b[x % 2], af[x / 2]);
            __builtin_amdgcn_sched_barrier(0);
            if (x >= LAG) accumulate(c, x - LAG);
            __builtin_amdgcn_sched_barrier(0);
        }
        __builtin_amdgcn_s_setprio(0);
    };
    auto finish = [&](f32x4 (&c)[4][2]) {
#pragma unroll
        for (int x = 8 - LAG; x < 8; ++x) accumulate(c, x);
    };

    // steps 0 and 1, in the order the loop would have requested them: all but the last two regions of step 1
    request_a(0, 0, 0), request_b(0, 0, 0), request_scales(0), request_b(1, 0, 0), request_a(1, 0, 0);
    request_a(0, 1, 1), request_b(0, 1, 1), request_scales(1);
    wait_loads_outstanding<9>(); // A0, B0 and scales of step 0
    __syncthreads();
    read_b(bf[0], 0, 0);
    if (team == 1) swap_teams(); // team 1 runs one turn behind

    // `buffer`: t mod 2, a constant
    auto step = [&](int t, int buffer, P::Operand (&b0)[2], P::Operand (&b1)[2]) {
        // phase 0
        read_a(0, buffer);
        request_b(1, t + 1, buffer ^ 1);
        const Scales s00 = read_scales(0, 0, t);
        if (t > 0) finish(acc[1][0]);
        take_scales(s00);
        wait_loads_outstanding<9>(); // B1 of this step has landed (the other team reads it a turn later)
        swap_teams();
        multiply(acc[0][0], b0);
        swap_teams();
        // phase 1
        read_b(b1, 1, buffer);
        request_a(1, t + 1, buffer ^ 1);
        const Scales s01 = read_scales(0, 1, t);
        finish(acc[0][0]);
        take_scales(s01);
        wait_loads_outstanding<9>(); // A1 of this step
        swap_teams();
        multiply(acc[0][1], b1);
        swap_teams();
        // phase 2
        read_a(1, buffer);
        request_a(0, t + 2, buffer);
        const Scales s11 = read_scales(1, 1, t);
        finish(acc[0][1]);
        take_scales(s11);
        wait_loads_outstanding<6>(); // A0, B0 and scales of the next step
        swap_teams();
        multiply(acc[1][1], b1);
        swap_teams();
        // phase 3
        read_b(b1, 0, buffer ^ 1);
        request_b(0, t + 2, buffer);
        request_scales(t + 2);
        const Scales s10 = read_scales(1, 0, t);
        finish(acc[1][1]);
        take_scales(s10);
        swap_teams();
        multiply(acc[1][0], b0);
        swap_teams();
    };
    for (int t = 0; t < kb; t += 2) {
        step(t, 0, bf[0], bf[1]);
        if (t + 1 < kb) step(t + 1, 1, bf[1], bf[0]);
    }
    finish(acc[1][0]);
    if (team == 0) swap_teams(); // team 1 is one turn behind
    wait_loads_outstanding<0>(); // the requests past the end: nothing may still write the LDS when the workgroup ends
    float none = 0.0f;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int x = 0; x < 16; ++x) {
            f32x4 &sum = acc[h][x / 8][x / 2 % 4][x % 2];
            note_not_finite(none, sum);
            if constexpr (B_ROWS > 1) sum *= 1.0f / kRaised;
        }
    if (__builtin_expect(wave_sums_again(none), 0))
        return store_with_any_scales<TT_BF16, B_ROWS>(g, 8, 2, 0, kb, [&](int i) { return m0 + i / 4 * 128 + a_row + i % 4 * 16; },
                                                      [&](int j) { return n0 + j * 128 + b_row; }, [&](int j) { return n0 + j * 128 + wn * 32 + lane_g * 8; });

#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int n = n0 + k * 128 + wn * 32 + lane_g * 8;
        float bias[8] = {};
        if (g.bias && n < g.N) load_eight<TT_BF16>(bias, g.bias, n, g.N - n);
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int m = m0 + h * 128 + a_row + i * 16;
                if (m >= g.M || n >= g.N) continue;
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = acc[h][k][i][e / 4][e % 4];
                finish_results<8>(v, bias, g.act);
                store_eight<TT_BF16>(g.out, (batch * g.M + m) * g.N + n, v, g.N - n);
            }
    }
}

} // namespace tt
