// Products over groups of few rows for gfx950 (group_args.h; single tokens, a few to an expert): sixteen rows of a group and 16 or 32 columns to a
// workgroup, B stored N x K.
//
// What bounds these products is reading the groups' matrices, once, or, where those are small, the chain of latencies of a call.  The four waves of a workgroup
// share out K, 128 bytes of each of its rows of B to a wave at a time, straight into the registers of 16 x 16 MFMAs: nothing is staged, so nothing is
// waited for but the loads, up to 16 KB of which a wave has on their way.  The waves' sums meet in LDS, in a fixed order.
//
// Protected, the check of the columns is the workgroup's own: it sums its rows of A first (e^T A of sixteen rows at most) and multiplies that vector
// with the elements of B it holds, by vector instructions beside the MFMAs, for which the loads leave time; so B is read once, and not again by the check
// kernel.  Its tolerance goes by its rows' max|A|.  A column that disagrees leaves a mark in cc_obs for the check kernel, which writes the flags.  Rows: the
// check kernel adds up the workgroups' shares of the observed sums, which lie side by side (added by atomics, all columns' in the same few words, they took int8
// 24 rows in 8 groups, 3072 x 768, 17.9 us, 8.4 so); the predictions come from the pass over A (group_passes.h), as for the other tiles.
#include <algorithm>

#include "abft_device.h"
#include "block_out.h"
#include "group_args.h"
#include "group_passes.h"

namespace abft {

constexpr int FEW_PAIRS = 4;                // pieces of 128 bytes of a row that a wave has on their way

struct FewArgs {
    GroupArgs g;
    const uint32_t *b_max;                  // max|B| of each group
    float tau_cols;                         // > 0: instead of 1e-3 K max|A| max|B|
    uint32_t *shares;                       // [tiles_n * NB][M]: observed sums of rows, a workgroup's columns each
    int sums_off;                           // where the column sums of A lie in LDS, behind what the waves exchange
};

// NB: blocks of sixteen columns
template <int DT, int NB> constexpr int few_part_bytes() { return 4 * NB * 64 * 16 + 4 * NB * 16 * 4 + 16; }

template <int DT, int OT, bool PROT, int NB>
__global__ __launch_bounds__(256) void gemm_group_few_kernel(FewArgs f)
{
    using T = Traits<DT>;
    typedef typename T::acc_t acc_t;
    typedef typename Acc4<DT>::type acc4_t;
    constexpr bool SCALED = OT != DT;
    constexpr int ES = T::ES, OS = Traits<OT>::OS, CE = 16 / ES, BN = 16 * NB, U = FEW_PAIRS;
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    fetch_args<FewArgs>();
    const GroupArgs &g = f.g;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    if constexpr (PROT) {
        if (blockIdx.x == 0 && tid < 5) g.counts[tid] = 0u;
        if ((int)blockIdx.x < g.n_pass) {
            GroupTile t;
            if (find_tile<4 * PASS_ROWS>(g, g.pass_win, g.pass_inv, (int)blockIdx.x, &t))
                group_pass<DT, 4, false>(g, t.e, t.first, t.rows, t.tm * 4 * PASS_ROWS, t.tn, smem);
            return;
        }
    }
    GroupTile t;
    if (!find_tile<16>(g, g.tiles_n, g.group_inv, (int)blockIdx.x - (PROT ? g.n_pass : 0), &t)) return;
    const int m0 = t.tm * 16, n0 = t.tn * BN, N = g.N, K = g.K;
    const int rows = min(t.rows - m0, 16);                       // of this tile
    const int nch = (K * ES + 15) / 16, pairs = (nch + 7) / 8;   // 16-byte chunks of a row, pieces of 128 bytes
    const int i16 = lane & 15, piece = lane >> 4;
    const uint8_t *At = g.A + (long)(t.first + m0) * g.lda * ES;
    const uint8_t *arow = At + (long)min(i16, rows - 1) * g.lda * ES;
    const uint8_t *brow[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) brow[nb] = g.B + ((long)t.e * g.sB + (long)min(n0 + 16 * nb + i16, N - 1) * g.ldb) * ES;

    // ---- e^T A of the tile's rows: integers, |sum| <= 2^11, as two digits of 8 bits, a chunk's sixteen side by side; else words.  Four threads to a
    // chunk, every fourth row to each.
    uint8_t *const sums = smem + f.sums_off;
    float *const tops = reinterpret_cast<float *>(smem + few_part_bytes<DT, NB>() - 16);
    i32x4 ax[4];
    float top = 0.f;
    auto load_rows = [&](int c) __attribute__((always_inline)) {
        const uint8_t *at = At + (long)min(c, nch - 1) * 16;
#pragma unroll
        for (int j = 0; j < 4; ++j) ax[j] = *reinterpret_cast<const i32x4 *>(at + (long)min(4 * j + (tid & 3), rows - 1) * g.lda * ES);
    };
    auto sum_rows = [&](int c) __attribute__((always_inline)) {
        const int keep = K * ES - c * 16;
        if constexpr (T::IS_INT) {
            // 16-bit fields: bytes plus 128, so that no sum is negative
            uint32_t even[4] = {0, 0, 0, 0}, odd[4] = {0, 0, 0, 0};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const i32x4 w = mask_chunk(ax[j], keep);
                const bool in = 4 * j + (tid & 3) < rows;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t x = in ? (uint32_t)w[i] ^ 0x80808080u : 0u;
                    even[i] += x & 0x00FF00FFu;
                    odd[i] += x >> 8 & 0x00FF00FFu;
                }
            }
            // s + 128 + 2^12 in a field: its low byte is the low digit plus 128, what is left the high one plus 16
            const uint32_t back = (uint32_t)(4096 + 128 - 128 * rows) * 0x10001u;
            i32x4 lo, hi;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t digits[2][2];
#pragma unroll
                for (int o = 0; o < 2; ++o) {
                    int v = (int)(o ? odd[i] : even[i]);
                    v += dpp_mov<0xB1>(v);                       // lane ^ 1
                    v += dpp_mov<0x4E>(v);                       // lane ^ 2
                    const uint32_t u = (uint32_t)v + back;
                    digits[o][0] = (u & 0x00FF00FFu) ^ 0x00800080u;
                    digits[o][1] = ((u >> 8 & 0x00FF00FFu) + 0x00F000F0u) & 0x00FF00FFu;
                }
                lo[i] = (int)(digits[0][0] | digits[1][0] << 8);
                hi[i] = (int)(digits[0][1] | digits[1][1] << 8);
            }
            if ((tid & 3) == 0 && c < nch) {
                *reinterpret_cast<i32x4 *>(sums + c * 32) = lo;
                *reinterpret_cast<i32x4 *>(sums + c * 32 + 16) = hi;
            }
        } else {
            acc_t s[CE];
#pragma unroll
            for (int q = 0; q < CE; ++q) s[q] = T::zero();
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const i32x4 w = 4 * j + (tid & 3) < rows ? mask_chunk(ax[j], keep) : i32x4{0, 0, 0, 0};
#pragma unroll
                for (int q = 0; q < CE; ++q) {
                    const acc_t v = T::elem(w, q);
                    s[q] = add_t(s[q], v);
                    if (c < nch) top = fmaxf(top, fabsf((float)v));
                }
            }
#pragma unroll
            for (int q = 0; q < CE; ++q) {
                s[q] = add_t(s[q], dpp_get<0xB1>(s[q]));
                s[q] = add_t(s[q], dpp_get<0x4E>(s[q]));
            }
            if ((tid & 3) == 0 && c < nch) {
#pragma unroll
                for (int q4 = 0; q4 < CE / 4; ++q4)
                    *reinterpret_cast<i32x4 *>(sums + c * 32 + 16 * q4) =
                        i32x4{(int)as_word(s[4 * q4]), (int)as_word(s[4 * q4 + 1]), (int)as_word(s[4 * q4 + 2]), (int)as_word(s[4 * q4 + 3])};
            }
        }
    };

    // scales of what this wave stores in the end (lane: row lane & 15, columns 4 (lane >> 4) + i of block `wave`), on their way meanwhile
    const int c0 = n0 + 16 * wave + 4 * piece;
    float rscale = 1.f, cscale[4] = {1.f, 1.f, 1.f, 1.f}, bias[4] = {0.f, 0.f, 0.f, 0.f};
    if constexpr (SCALED) {
        if (wave < NB) {
            if (g.row_scale) rscale = g.row_scale[t.first + m0 + min(i16, rows - 1)];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int c = min(c0 + i, N - 1);
                if (g.col_scale) cscale[i] = g.col_scale[(long)t.e * N + c];
                if (g.bias) bias[i] = g.bias[c];
            }
        }
    }

    // ---- this wave's pieces: every fourth
    acc4_t acc[NB];
    acc_t pred[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) { acc[nb] = acc4_zero<DT>(); pred[nb] = T::zero(); }
    i32x4 a[U][2], b[U][2][NB];
    auto load = [&](int p0) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (u && p0 + 4 * u >= pairs) break;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const long at = (long)min((p0 + 4 * u) * 8 + 4 * h + piece, nch - 1) * 16;
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) b[u][h][nb] = *reinterpret_cast<const i32x4 *>(brow[nb] + at);
                a[u][h] = *reinterpret_cast<const i32x4 *>(arow + at);
            }
        }
    };
    // the loads of the last sums and of the first pieces go out together
    if constexpr (PROT) {
        int c = tid >> 2;
        for (; c + 64 < nch + (tid >> 2); c += 64) {
            load_rows(c);
            sum_rows(c);
        }
        load_rows(c);
        load(wave);
        sum_rows(c);
        if constexpr (!T::IS_INT) {
            top = wave_max(top);
            if (lane == 0) tops[wave] = top;
        }
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    } else {
        load(wave);
    }
    for (int p0 = wave; p0 < pairs; p0 += 4 * U) {
        if (p0 != wave) load(p0);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (u && p0 + 4 * u >= pairs) break;
            // past the end of K nothing is multiplied, whatever both hold there
            if ((p0 + 4 * u) * 8 + 8 > K * ES / 16) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int keep = K * ES - ((p0 + 4 * u) * 8 + 4 * h + piece) * 16;
                    a[u][h] = mask_chunk(a[u][h], keep);
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) b[u][h][nb] = mask_chunk(b[u][h][nb], keep);
                }
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) acc[nb] = mfma16<DT>(b[u][h][nb], a[u][h], acc[nb]);
                if constexpr (PROT) {
                    const int ch = min((p0 + 4 * u) * 8 + 4 * h + piece, nch - 1);
                    const i32x4 s0 = *reinterpret_cast<const i32x4 *>(sums + ch * 32), s1 = *reinterpret_cast<const i32x4 *>(sums + ch * 32 + 16);
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) {
                        if constexpr (T::IS_INT) {
                            int lo = 0, hi = 0;
#pragma unroll
                            for (int w = 0; w < 4; ++w) {
                                lo = __builtin_amdgcn_sdot4(b[u][h][nb][w], s0[w], lo, false);
                                hi = __builtin_amdgcn_sdot4(b[u][h][nb][w], s1[w], hi, false);
                            }
                            pred[nb] += lo + (int)((uint32_t)hi << 8);
                        } else {
#pragma unroll
                            for (int q = 0; q < CE; ++q)
                                pred[nb] = __builtin_fmaf((float)T::elem(b[u][h][nb], q), __uint_as_float((uint32_t)(q < 4 ? s0[q & 3] : s1[q & 3])), pred[nb]);
                        }
                    }
                }
            }
        }
    }

    // ---- the waves' sums, in LDS: [wave][nb][lane] of four, then [wave][nb][column] predictions
    acc_t *const ppart = reinterpret_cast<acc_t *>(smem + 4 * NB * 64 * 16);
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        *reinterpret_cast<acc4_t *>(smem + ((wave * NB + nb) * 64 + lane) * 16) = acc[nb];
        if constexpr (PROT) {
            const acc_t s = add_xor32(add_xor16(pred[nb]));
            if (lane < 16) ppart[(wave * NB + nb) * 16 + lane] = s;
        }
    }
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    if (wave >= NB) return;
    const int nb = wave;
    acc_t v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = T::zero();
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const acc4_t x = *reinterpret_cast<const acc4_t *>(smem + ((w * NB + nb) * 64 + lane) * 16);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = add_t(v[i], (acc_t)x[i]);
    }
    const bool in = i16 < rows;
    if (g.inj_b == t.e && g.inj_row == m0 + i16 && in) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (c0 + i == g.inj_col) v[i] = from_word<acc_t>(as_word(v[i]) ^ (1u << g.inj_bit));
    }
    if (in && c0 < N) {
        uint8_t *dst = g.C + ((long)(t.first + m0 + i16) * g.ldc + c0) * OS;
        const int n = min(N - c0, 4);
        if constexpr (T::IS_INT && !SCALED) {
            const i32x4 w = {(int)v[0], (int)v[1], (int)v[2], (int)v[3]};
            if (n == 4) *reinterpret_cast<i32x4 *>(dst) = w;
            else
#pragma unroll
                for (int i = 0; i < 3; ++i)
                    if (i < n) reinterpret_cast<int *>(dst)[i] = w[i];
        } else {
            float x[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[i] = (float)v[i];
                if constexpr (SCALED) x[i] = __builtin_fmaf(x[i] * rscale, cscale[i], bias[i]);
            }
            const uint2 w = make_uint2(pack2<OT>(x[0], x[1]), pack2<OT>(x[2], x[3]));
            if (n == 4) *reinterpret_cast<uint2 *>(dst) = w;
            else
#pragma unroll
                for (int i = 0; i < 3; ++i)
                    if (i < n) reinterpret_cast<uint16_t *>(dst)[i] = (uint16_t)((i < 2 ? w.x : w.y) >> (16 * (i & 1)));
        }
    }
    if constexpr (PROT) {
        acc_t rsum = T::zero();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (!in || c0 + i >= N) v[i] = T::zero();
            rsum = add_t(rsum, v[i]);
        }
        rsum = add_xor32(add_xor16(rsum));
        if (lane < rows && 16 * nb + n0 < N) f.shares[(long)(t.tn * NB + nb) * g.M + t.first + m0 + lane] = as_word(rsum);
        // a column's sum over the sixteen lanes of its rows, against its prediction
        float tol = 0.f;
        if constexpr (!T::IS_INT) {
            const float top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
            tol = f.tau_cols > 0.f ? f.tau_cols : (1e-3f * (float)K) * top * __uint_as_float(f.b_max[t.e]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const acc_t obs = row16_sum(v[i]);
            acc_t p = T::zero();
#pragma unroll
            for (int w = 0; w < 4; ++w) p = add_t(p, ppart[(w * NB + nb) * 16 + 4 * piece + i]);
            if (i16 == 0 && c0 + i < N && mismatch<T::IS_INT>(as_word(obs), as_word(p), tol)) atomicOr(g.cc_obs + (long)t.e * N + c0 + i, 1u);
        }
    }
}

// ------------------------------------------------------------------------------------------
constexpr int FEW_MAX_SUMS = 64 * 1024;      // bytes of LDS for the column sums of A

bool group_few_fits(int dt, bool protect, const GroupArgs &g)
{
    return !protect || (g.M <= 32L * g.groups && ((long)g.K * elem_size(dt) + 15) / 16 * 32 <= FEW_MAX_SUMS);
}

// 32 columns to a workgroup, which reads its rows of A once for both halves, unless that leaves compute units without one.  (16 / 32, protected, us: fewer rows
// than groups, 4096 x 1024, bf16 31 rows in 32 groups 59.4 / 53.6, 63 in 64 112.6 / 98.8, int8 33.5 / 29.5 and 59.3 / 51.0; unprotected the same.)
int group_few_columns(const GroupArgs &g)
{
    const long rows = ((long)g.M + g.groups - 1) / g.groups;                 // of a group on average
    return std::min(g.M, g.groups) * ((rows + 15) / 16) * ((g.N + 31) / 32) >= 512 ? 32 : 16;
}

long group_few_workgroups(const GroupArgs &g)
{
    const int bn = group_few_columns(g);
    return ((g.groups == 1 ? (g.M + 15) / 16 : g.M / 16 + std::min(g.M, g.groups)) * (long)((g.N + bn - 1) / bn) + 7) / 8 * 8;
}

template <int DT, int OT, bool PROT, int NB> static hipError_t launch_few_one(FewArgs &f, hipStream_t st)
{
    GroupArgs &g = f.g;
    auto kern = gemm_group_few_kernel<DT, OT, PROT, NB>;
    f.sums_off = (few_part_bytes<DT, NB>() + 15) & ~15;
    int smem = f.sums_off;
    if (PROT) smem = std::max(smem + (g.K * Traits<DT>::ES + 15) / 16 * 32, group_pass_lds<DT, 4>());
    const hipError_t e = ensure_max_lds(reinterpret_cast<const void *>(kern), FEW_MAX_SUMS + 32 * 1024);
    if (e != hipSuccess) return e;
    g.tiles_n = (g.N + 16 * NB - 1) / (16 * NB);
    g.group_inv = map_inverse(g.tiles_n);
    const long wgs = (PROT ? g.n_pass : 0) + group_few_workgroups(g);
    hipLaunchKernelGGL(kern, dim3((unsigned)wgs), dim3(256), smem, st, f);
    return hipGetLastError();
}

template <int DT, int OT> static hipError_t launch_few_type(bool protect, FewArgs &f, hipStream_t st)
{
    const bool wide = group_few_columns(f.g) == 32;
    if (protect) return wide ? launch_few_one<DT, OT, true, 2>(f, st) : launch_few_one<DT, OT, true, 1>(f, st);
    return wide ? launch_few_one<DT, OT, false, 2>(f, st) : launch_few_one<DT, OT, false, 1>(f, st);
}

hipError_t launch_group_few(int dt, int ot, bool protect, GroupArgs &g, const uint32_t *b_max, float tau_cols, hipStream_t st)
{
    FewArgs f = {g, b_max, tau_cols, group_few_shares(g), 0};
    if (dt == DT_I8)
        return ot == DT_I8   ? launch_few_type<DT_I8, DT_I8>(protect, f, st)
               : ot == DT_BF16 ? launch_few_type<DT_I8, DT_BF16>(protect, f, st)
                               : launch_few_type<DT_I8, DT_F16>(protect, f, st);
    return dt == DT_BF16 ? launch_few_type<DT_BF16, DT_BF16>(protect, f, st) : launch_few_type<DT_F16, DT_F16>(protect, f, st);
}

}  // namespace abft
