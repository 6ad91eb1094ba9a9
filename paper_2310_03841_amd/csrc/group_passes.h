// The pass over A of a protected product over groups: one read of A gives e^T A and max|A| of each group and, with b = B e of the row's
// group at hand, the row prediction A b (Sec. III-B.1 "Checksums").  Items of the product's own launch, beside its tiles.
//
// An item is eight rows of a group to a wave and a window of 1 KB along K, a lane 16 bytes of each row.  The waves' column sums meet in LDS and go out
// together.  Bound by the latency of its loads, all of which are on their way at once, and by the additions at its end, where items meet in the same
// lines.  (us, a launch of its own: a wave to 32 rows, with additions of its own, int8 12608 x 768 126, bf16 12608 x 768 in 16 groups 31,
// int8 6304 x 3072 in 8 groups 56; 256 rows and 128 bytes of each to a workgroup, 7.0, 12.6 and 9.9.)
#pragma once
#include "group_args.h"

namespace abft {

constexpr int PASS_ROWS = 8;                 // rows of a wave
constexpr int PASS_BYTES = 1024;             // of a row

// LDS: each wave's sums of the window's columns, and a maximum to a wave
template <int DT, int WAVES> constexpr int group_pass_lds() { return WAVES * PASS_BYTES / Traits<DT>::ES * 4 + WAVES * 4; }

// Rows row0 .. of group e (which has `rows` from `first` on), WAVES * PASS_ROWS at most; window win.  SUMS: e^T A is wanted too.
template <int DT, int WAVES, bool SUMS = true> __device__ __forceinline__ void group_pass(const GroupArgs &g, int e, int first, int rows, int row0, int win, uint8_t *smem)
{
    using T = Traits<DT>;
    typedef typename T::acc_t acc_t;
    constexpr int ES = T::ES, CE = 16 / ES, COLS = PASS_BYTES / ES;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int K = g.K, r0 = row0 + wave * PASS_ROWS;
    acc_t *red = reinterpret_cast<acc_t *>(smem);
    float *tops = reinterpret_cast<float *>(smem + WAVES * COLS * 4);
    const int k0 = win * COLS, k = k0 + lane * CE, keep = (K - k) * ES;      // bytes of the lane's chunk that hold data
    const uint8_t *src = g.A + ((long)first * g.lda + (keep > 0 ? k : 0)) * ES;
    acc_t dot[PASS_ROWS], col[CE];
#pragma unroll
    for (int u = 0; u < PASS_ROWS; ++u) dot[u] = T::zero();
#pragma unroll
    for (int q = 0; q < CE; ++q) col[q] = T::zero();
    float top = 0.f;
    if (r0 < rows) {
        i32x4 x[PASS_ROWS];
        acc_t b[CE];
#pragma unroll
        for (int u = 0; u < PASS_ROWS; ++u) x[u] = *reinterpret_cast<const i32x4 *>(src + (long)min(r0 + u, rows - 1) * g.lda * ES);
        // b starts on any word: a group's of a ragged K does
        const uint32_t *bs = g.b_sum + (long)e * K;
        if (k + CE <= K) {
#pragma unroll
            for (int q4 = 0; q4 < CE / 4; ++q4) {
                const i32x4_word v = *reinterpret_cast<const i32x4_word *>(bs + k + 4 * q4);
#pragma unroll
                for (int i = 0; i < 4; ++i) b[4 * q4 + i] = from_word<acc_t>((uint32_t)v[i]);
            }
        } else {
#pragma unroll
            for (int q = 0; q < CE; ++q) b[q] = from_word<acc_t>(bs[min(k + q, K - 1)]);
        }
        // NARROW: |b| <= 128 N is below 2^23, and products take one instruction instead of one at a quarter of the rate
        auto add = [&](auto narrow_c) __attribute__((always_inline)) {
#pragma unroll
            for (int u = 0; u < PASS_ROWS; ++u) {
                const i32x4 w = r0 + u < rows ? mask_chunk(x[u], keep) : i32x4{0, 0, 0, 0};
#pragma unroll
                for (int q = 0; q < CE; ++q) {
                    const acc_t v = T::elem(w, q);
                    if constexpr (decltype(narrow_c)::value) dot[u] += __mul24((int)v, (int)b[q]);
                    // (past the end of K nothing is multiplied: b may hold what is not finite)
                    else if (T::IS_INT || q * ES < keep) dot[u] = add_t(dot[u], mul_t(v, b[q]));
                    if constexpr (!SUMS) {}
                    else if constexpr (T::IS_INT) col[q] = __builtin_amdgcn_sdot4(w[q >> 2], 1 << (8 * (q & 3)), col[q], false);
                    else col[q] = add_t(col[q], v);
                    if constexpr (!T::IS_INT) top = fmaxf(top, fabsf((float)v));
                }
            }
        };
        if (T::IS_INT && g.N < 65536) add(std::integral_constant<bool, T::IS_INT>{});
        else add(std::false_type{});
    }
#pragma unroll
    for (int q4 = 0; q4 < CE / 4 && SUMS; ++q4)
        *reinterpret_cast<i32x4 *>(red + wave * COLS + lane * CE + 4 * q4) =
            i32x4{(int)as_word(col[4 * q4]), (int)as_word(col[4 * q4 + 1]), (int)as_word(col[4 * q4 + 2]), (int)as_word(col[4 * q4 + 3])};
    if constexpr (!T::IS_INT) {
        top = wave_max(top);
        if (lane == 0) tops[wave] = top;
    }
    acc_t mine = T::zero();
#pragma unroll
    for (int u = 0; u < PASS_ROWS; ++u) {
        const acc_t s = wave_sum(dot[u]);
        mine = lane == u ? s : mine;
    }
    if (lane < PASS_ROWS && r0 + lane < rows) atomic_add_word(g.rc_pred + first + r0 + lane, mine);
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");       // (over LDS alone: not for the additions above)
#pragma unroll
    for (int c = tid; c < COLS && SUMS; c += 64 * WAVES) {
        if (k0 + c < K) {
            acc_t s = red[c];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) s = add_t(s, red[w * COLS + c]);
            atomic_add_word(g.a_sum + (long)e * K + k0 + c, s);
        }
    }
    if constexpr (!T::IS_INT) {
        if (tid == 0) {
            float m = 0.f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) m = fmaxf(m, tops[w]);
            if (m > 0.f) atomicMax(g.a_max + e, __float_as_uint(m));
        }
    }
}

}  // namespace abft
