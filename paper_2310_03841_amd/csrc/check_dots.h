// What the kernels share that compare checksums: the dots of an operand's rows with a vector, and the report of what disagrees.
#pragma once
#include "abft_device.h"

namespace abft {

// A wave found n rows (side 0) or n columns (side 1) that disagree.  counts[side] gains them; counts[2] and
// counts[4] become the status: localised once both sides have flags, suspect while one has.  Only the
// first wave of a side writes it.  It adds first and looks at the other side second, so of the two first
// waves at least one sees both; "localised" goes in whatever is there, "suspect" only replaces "clean".
// (With every wave looking and writing, a bf16 12608 x 3072 x 768 whose every row and column flags took 137 us;
// so 84, and 78 clean: atomics on one line are served one after the other.)
// fix_count: after a correction (counts[4] is the status before it; counts[2] stays where the list was too long).
__device__ __forceinline__ void report_flags(uint32_t *counts, int side, unsigned n, const uint32_t *fix_count = nullptr)
{
    if (atomicAdd(counts + side, n) != 0u) return;
    if (fix_count && fix_count[1]) return;
    if (atomicAdd(counts + (side ^ 1), 0u) != 0u) {
        atomicExch(counts + 2, 1u);
        if (!fix_count) atomicExch(counts + 4, 1u);
    } else {
        atomicCAS(counts + 2, 0u, 2u);
        if (!fix_count) atomicCAS(counts + 4, 0u, 2u);
    }
}

// Dots of RW rows of a K-contiguous operand with a vector of K words: lanes along K, two chunks per
// lane and trip, everything of a trip in flight.  split: this wave takes every fourth run of 128
// chunks.  Every lane returns the wave's share of all RW dots.
// Loads without a lane's branch (around one the compiler waits for those before it): lanes and rows past the end ask for the last
// whole chunk and the last row.  What lies behind the last whole chunk is asked for first, an element a lane.  The vector may
// start on any word: batch items of a ragged K do, and a caller's may.  (The kernel, with a branch around each load / with a path of loads
// without them for whole chunks and aligned vectors, word by word otherwise / so: int8 10624 x 221 x 2360 14.8 / 20.6 / 11.8 us; 570 x 570 x 48, 48
// items, where the second 64 lanes of a trip have nothing, 19.1 / 21.8 / 11.7; bf16 640 x 2880 x 1535 4.7 / 6.6 / 4.8.)
template <int DT, int RW>
__device__ __forceinline__ void row_dots(const uint8_t *X, long ld, int row0, int rows, int K, const uint32_t *vec,
                                         bool split, typename Traits<DT>::acc_t (&dot)[RW])
{
    using T = Traits<DT>;
    typedef typename T::acc_t acc_t;
    constexpr int ES = T::ES, CE = 16 / ES;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int nch = K / CE, tail = nch * CE + lane;              // whole chunks; this lane's element behind them
    uint32_t xt[RW], vt;
    if (nch * CE < K) {
        const int k = min(tail, K - 1);
        vt = vec[k];
#pragma unroll
        for (int j = 0; j < RW; ++j) {
            const uint8_t *at = X + ((long)min(row0 + j, rows - 1) * ld + k) * ES;
            if constexpr (ES == 2) xt[j] = *reinterpret_cast<const uint16_t *>(at);
            else xt[j] = *at;
        }
    }
#pragma unroll
    for (int j = 0; j < RW; ++j) dot[j] = T::zero();
    for (int ch0 = split ? wave * 128 : 0; ch0 < nch; ch0 += split ? 512 : 128) {
        i32x4 v[RW][2];
        i32x4_word aw[2][CE / 4];
        auto load = [&](int h) __attribute__((always_inline)) {
            const int ch = min(ch0 + 64 * h + lane, nch - 1);
#pragma unroll
            for (int j = 0; j < RW; ++j)
                v[j][h] = *reinterpret_cast<const i32x4 *>(X + ((long)min(row0 + j, rows - 1) * ld + (long)ch * CE) * ES);
#pragma unroll
            for (int q4 = 0; q4 < CE / 4; ++q4) aw[h][q4] = *reinterpret_cast<const i32x4_word *>(vec + ch * CE + 4 * q4);
        };
        auto add = [&](int h) __attribute__((always_inline)) {
            if (ch0 + 64 * h + lane < nch) {
#pragma unroll
                for (int j = 0; j < RW; ++j)
#pragma unroll
                    for (int q = 0; q < CE; ++q)
                        dot[j] = add_t(dot[j], mul_t(T::elem(v[j][h], q), from_word<acc_t>((uint32_t)aw[h][q >> 2][q & 3])));
            }
        };
        const bool two = ch0 + 64 < nch;
        load(0);
        if (two) load(1);
        add(0);
        if (two) add(1);
    }
    if (tail < K && (!split || wave == 0)) {
#pragma unroll
        for (int j = 0; j < RW; ++j)
            dot[j] = add_t(dot[j], mul_t(T::elem(i32x4{(int)xt[j], 0, 0, 0}, 0), from_word<acc_t>(vt)));
    }
#pragma unroll
    for (int j = 0; j < RW; ++j) dot[j] = wave_sum(dot[j]);
}

}  // namespace abft
