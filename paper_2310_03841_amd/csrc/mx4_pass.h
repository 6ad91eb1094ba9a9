// The pass over 4-bit A of a protected product over groups, as group_passes.h has it for other types: e^T A, max|A| and the row prediction A b from one read.
//
// Items of the product's own launch: eight rows to a wave at a time, and a window of 1 KB along K, a block of 32 elements of each row to a lane.  The additions of items to the same
// words are served one after the other, some 45 ns each, so items of large groups make several trips (mx4_plan).  Within a window
// sums are added up in a fixed order; items add theirs by fp32 additions in any order, which moves a prediction by some 2^-24 of itself, four orders below
// the tolerance it is held against.
#pragma once
#include "group_args.h"
#include "group_passes.h"
#include "mx4_device.h"

namespace abft {

// LDS: each wave's sums of the window's columns (SUMS: e^T A is wanted too), and a maximum to a wave
template <int WAVES, bool SUMS = true> constexpr int mx4_pass_lds() { return (SUMS ? WAVES * PASS_BYTES * 2 * 4 : 0) + WAVES * 4; }

// Rows row0 .. of group e (which has `rows` from `first` on), 2^log2 times WAVES * PASS_ROWS of them at most, ROWS of a wave on their way together.
template <int WAVES, bool SUMS = true, int ROWS = PASS_ROWS> __device__ __forceinline__ void mx4_pass(const Mx4Args &g, int e, int first, int rows, int row0, int log2, int win, uint8_t *smem)
{
    constexpr int COLS = PASS_BYTES * 2;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int nb = g.K / 16, K2 = 2 * g.K, upto = min(rows, row0 + (WAVES * PASS_ROWS << log2));
    float *const red = reinterpret_cast<float *>(smem);
    float *const tops = red + (SUMS ? WAVES * COLS : 0);
    const int block = win * 64 + lane, at = min(block, nb - 1);
    const bool in = block < nb;
    float col[32], b[32];
#pragma unroll
    for (int q = 0; q < 32; ++q) col[q] = 0.f;
    float top = 0.f;
    const uint32_t *bs = g.b_sum + (long)e * K2 + at * 32;
#pragma unroll
    for (int q4 = 0; q4 < 8; ++q4) {
        const i32x4_word v = *reinterpret_cast<const i32x4_word *>(bs + 4 * q4);
#pragma unroll
        for (int i = 0; i < 4; ++i) b[4 * q4 + i] = __uint_as_float((uint32_t)v[i]);
    }
    for (int r0 = row0 + wave * ROWS; r0 < upto; r0 += WAVES * ROWS) {
        i32x4 x[ROWS];
        uint32_t s[ROWS];
        float dot[ROWS];
#pragma unroll
        for (int u = 0; u < ROWS; ++u) {
            const long r = first + min(r0 + u, rows - 1);
            x[u] = *reinterpret_cast<const i32x4 *>(g.A + r * g.lda + at * 16);
            s[u] = g.sa[r * g.ld_sa + at];
            dot[u] = 0.f;
        }
#pragma unroll
        for (int u = 0; u < ROWS; ++u) {
            if (!in || r0 + u >= rows) continue;
            float v[32];
            mx4_values(x[u], mx4_unit(s[u]), v);
#pragma unroll
            for (int q = 0; q < 32; ++q) {
                dot[u] = __builtin_fmaf(v[q], b[q], dot[u]);
                if constexpr (SUMS) col[q] += v[q];
                top = fmaxf(top, fabsf(v[q]));
            }
            __builtin_amdgcn_sched_barrier(0);                   // (a row's 32 values at a time: all eight's do not fit)
        }
        float mine = 0.f;
#pragma unroll
        for (int u = 0; u < ROWS; ++u) {
            const float t = wave_sum(dot[u]);
            mine = lane == u ? t : mine;
        }
        if (lane < ROWS && r0 + lane < rows) atomic_add_word(g.rc_pred + first + r0 + lane, mine);
    }
#pragma unroll
    for (int q4 = 0; q4 < 8 && SUMS; ++q4)
        *reinterpret_cast<f32x4 *>(red + wave * COLS + lane * 32 + 4 * q4) = f32x4{col[4 * q4], col[4 * q4 + 1], col[4 * q4 + 2], col[4 * q4 + 3]};
    top = wave_max(top);
    if (lane == 0) tops[wave] = top;
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");       // (over LDS alone: not for the additions above)
#pragma unroll
    for (int c = tid; c < COLS && SUMS; c += 64 * WAVES) {
        if (win * COLS + c < K2) {
            float s = red[c];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) s += red[w * COLS + c];
            atomic_add_word(g.a_sum + (long)e * K2 + win * COLS + c, s);
        }
    }
    if (tid == 0) {
        float m = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) m = fmaxf(m, tops[w]);
        if (m > 0.f) atomicMax(g.a_max + e, __float_as_uint(m));
    }
}

}  // namespace abft
