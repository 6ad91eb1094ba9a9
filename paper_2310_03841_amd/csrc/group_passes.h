// The pass over A of a protected product over groups: one read of A gives e^T A and max|A| of each group and, with b = B e of the row's
// group at hand, the row prediction A b (Sec. III-B.1 "Checksums").  Workgroups of the product's own launch, ahead of its tiles.
#pragma once
#include "group_args.h"

namespace abft {

constexpr int PASS_ROWS = 8;                 // rows of a wave on their way at once

// Wave `unit` of the pass: window of 64 chunks along K, g.pass_rows rows.  Rows are sorted, so a wave meets its groups one after the other: it
// keeps b and the column sums of one in registers and hands the sums over at the group's end.
template <int DT> __device__ __forceinline__ void group_pass(const GroupArgs &g, int unit)
{
    using T = Traits<DT>;
    typedef typename T::acc_t acc_t;
    constexpr int ES = T::ES, CE = 16 / ES;
    const int lane = threadIdx.x & 63;
    const int win = unit % g.pass_win, run = unit / g.pass_win;
    const int nch = (g.K * ES + 15) / 16, ch = win * 64 + lane;
    const bool in = ch < nch;
    const int k0 = ch * CE, keep = g.K * ES - ch * 16;           // bytes of the lane's chunk that hold data
    const uint8_t *src = g.A + (long)(in ? ch : 0) * 16;
    const int stop = min(g.M, (run + 1) * g.pass_rows);
    int r = run * g.pass_rows;
    while (r < stop) {
        int end;
        const int e = __builtin_amdgcn_readfirstlane(group_of(g.offsets, g.M, g.groups, r, &end));
        if (e < 0) { ++r; continue; }                            // a row of no group
        end = min(__builtin_amdgcn_readfirstlane(end), stop);
        acc_t b[CE], col[CE];
#pragma unroll
        for (int q = 0; q < CE; ++q) {
            const int k = min(k0 + q, g.K - 1);
            b[q] = from_word<acc_t>(g.b_sum[(long)e * g.K + k]);
            col[q] = T::zero();
        }
        float top = 0.f;
        for (; r < end; r += PASS_ROWS) {
            i32x4 x[PASS_ROWS];
#pragma unroll
            for (int u = 0; u < PASS_ROWS; ++u) x[u] = *reinterpret_cast<const i32x4 *>(src + (long)min(r + u, end - 1) * g.lda * ES);
            acc_t mine = T::zero();
#pragma unroll
            for (int u = 0; u < PASS_ROWS; ++u) {
                const i32x4 w = r + u < end ? mask_chunk(x[u], in ? keep : 0) : i32x4{0, 0, 0, 0};
                acc_t dot = T::zero();
#pragma unroll
                for (int q = 0; q < CE; ++q) {
                    const acc_t v = T::elem(w, q);
                    // (past the end of K and of the rows nothing is multiplied: b may hold what is not finite)
                    if (T::IS_INT || q * ES < keep) dot = add_t(dot, mul_t(v, b[q]));
                    col[q] = add_t(col[q], v);
                    if constexpr (!T::IS_INT) top = fmaxf(top, fabsf((float)v));
                }
                if (!in || r + u >= end) dot = T::zero();
                dot = wave_sum(dot);
                mine = lane == u ? dot : mine;
            }
            if (lane < PASS_ROWS && r + lane < end) atomic_add_word(g.rc_pred + r + lane, mine);
        }
        r = end;
        if (in) {
#pragma unroll
            for (int q = 0; q < CE; ++q)
                if (k0 + q < g.K) atomic_add_word(g.a_sum + (long)e * g.K + k0 + q, col[q]);
        }
        if constexpr (!T::IS_INT) {
            top = wave_max(top);
            if (lane == 0 && top > 0.f) atomicMax(g.a_max + e, __float_as_uint(top));
        }
    }
}

}  // namespace abft
