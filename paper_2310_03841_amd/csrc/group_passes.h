// The pass over A of a protected product over groups: one read of A gives e^T A and max|A| of each group and, with b = B e of the row's
// group at hand, the row prediction A b (Sec. III-B.1 "Checksums").  Workgroups of the product's own launch ahead of its tiles, or a launch of their
// own ahead of tiles that leave no room beside them.
//
// A workgroup takes 256 rows of a group and 128 bytes of each, eight lanes to a row.  Bound by the latency of its loads, all of which are on their way at once,
// and by the additions at its end, where workgroups meet in the same lines: a word of e^T A takes one from every 256 rows.  (A wave to 32 rows and 1 KB of
// each, with additions of its own: int8 12608 x 768 126 us, bf16 12608 x 768 in 16 groups 31.)
#pragma once
#include "group_args.h"

namespace abft {

constexpr int PASS_ROWS = 256, PASS_CHUNKS = 8;

// LDS: 32 rows' sums of the window's columns, and four maxima
template <int DT> constexpr int group_pass_lds() { return 32 * SLAB_BYTES / Traits<DT>::ES * 4 + 16; }

// Workgroup `unit` of the pass, 256 threads.
template <int DT> __device__ __forceinline__ void group_pass(const GroupArgs &g, int unit, uint8_t *smem)
{
    using T = Traits<DT>;
    typedef typename T::acc_t acc_t;
    constexpr int ES = T::ES, CE = 16 / ES, U = PASS_ROWS / 32, COLS = PASS_CHUNKS * CE;
    GroupTile t;
    if (!find_tile<PASS_ROWS>(g, g.pass_win, g.pass_inv, unit, &t)) return;
    const int tid = threadIdx.x, lane = tid & 63, cx = tid & (PASS_CHUNKS - 1), ry = tid / PASS_CHUNKS;
    const int K = g.K, chunk = t.tn * PASS_CHUNKS + cx, k0 = chunk * CE;
    const int keep = K * ES - chunk * 16;                        // bytes of the lane's chunk that hold data
    const int row0 = t.tm * PASS_ROWS + ry, rows = t.rows;
    const uint8_t *src = g.A + ((long)t.first * g.lda) * ES + (keep > 0 ? (long)chunk * 16 : 0);
    i32x4 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) x[u] = *reinterpret_cast<const i32x4 *>(src + (long)min(row0 + 32 * u, rows - 1) * g.lda * ES);
    acc_t b[CE], col[CE];
#pragma unroll
    for (int q = 0; q < CE; ++q) {
        b[q] = from_word<acc_t>(g.b_sum[(long)t.e * K + min(k0 + q, K - 1)]);
        col[q] = T::zero();
    }
    float top = 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const bool in = row0 + 32 * u < rows;
        const i32x4 w = in ? mask_chunk(x[u], keep) : i32x4{0, 0, 0, 0};
        acc_t dot = T::zero();
#pragma unroll
        for (int q = 0; q < CE; ++q) {
            const acc_t v = T::elem(w, q);
            // (past the end of K nothing is multiplied: b may hold what is not finite)
            if (T::IS_INT || q * ES < keep) dot = add_t(dot, mul_t(v, b[q]));
            col[q] = add_t(col[q], v);
            if constexpr (!T::IS_INT) top = fmaxf(top, fabsf((float)v));
        }
        dot = seg_sum(dot, PASS_CHUNKS);
        if (cx == 0 && in) atomic_add_word(g.rc_pred + t.first + row0 + 32 * u, dot);
    }
    acc_t *red = reinterpret_cast<acc_t *>(smem);
    float *top4 = reinterpret_cast<float *>(smem + 32 * COLS * 4);
#pragma unroll
    for (int q = 0; q < CE; ++q) red[ry * COLS + cx * CE + q] = col[q];
    if constexpr (!T::IS_INT) {
        top = wave_max(top);
        if (lane == 0) top4[tid >> 6] = top;
    }
    __syncthreads();
    const int k = t.tn * COLS + tid;
    if (tid < COLS && k < K) {
        acc_t s = red[tid];
#pragma unroll
        for (int y = 1; y < 32; ++y) s = add_t(s, red[y * COLS + tid]);
        atomic_add_word(g.a_sum + (long)t.e * K + k, s);
    }
    if constexpr (!T::IS_INT) {
        if (tid == 0) {
            const float m = fmaxf(fmaxf(top4[0], top4[1]), fmaxf(top4[2], top4[3]));
            if (m > 0.f) atomicMax(g.a_max + t.e, __float_as_uint(m));
        }
    }
}

}  // namespace abft
