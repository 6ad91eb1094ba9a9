// Products over groups of few rows of 4-bit operands (single tokens, a few to an expert): sixteen rows of a group and 16, 32 or, protected, 64 columns to a workgroup, as
// gemm_group_few.hip has it for other types.
//
// What bounds these products is reading the groups' matrices, once, or, where those are small, the chain of latencies of a call.  The four waves share out K, 128
// bytes (eight blocks) of each of their rows of B at a time, straight into the registers of 16 x 16 MFMAs, whose lanes each take a block and its power
// of two.  The waves' sums meet in LDS, in a fixed order.
//
// Protected, a workgroup sums its rows of A first and multiplies that vector with the elements of B it holds, so that B is read once.  MFMAs do it too: a block
// of the vector is split into five terms of 8 bits (mx4_put_terms), and a term is a row of the other operand.  A
// column that disagrees leaves a mark in cc_obs for the check kernel; the workgroups' shares of the rows' sums lie side by side for it.
//
// 32 tokens, 32 experts of 4096 x 1024 (us on the card): 10.1, protected 12.9 by 64 columns, for fewer of those sums, and 13.2 by 32; with the vector multiplied by vector instructions
// and 132 registers, three waves to a SIMD, 16.5.  A chain of latencies to a workgroup (its place among the groups, rows of A, their sums, B, the waves' sums), one to two
// rounds of workgroups: the 33 MB of the fifteen matrices whose groups have rows would take 6.6 at a large copy's rate.
#include <algorithm>

#include "block_out.h"
#include "gemm_mx4.h"
#include "mx4_pass.h"

namespace abft {

struct Mx4FewArgs {
    Mx4Args g;
    const uint32_t *b_max;
    float tau_k, tau_cols;                  // 1e-3 K; > 0: instead of tau_k max|A| max|B|
    uint32_t *shares;                       // [tiles_n * NB][M]
    int sums_off;                           // where the terms of the column sums of A lie in LDS, behind what the waves exchange
};

template <int NB> constexpr int mx4_few_part_bytes() { return 4 * NB * 64 * 16 + 4 * NB * 16 * 4 + 16; }

// Waves of a SIMD that there are to be registers for.
constexpr int few_waves(bool protect, int nb, int u) { return !protect || u == 4 ? 1 : nb == 4 ? 4 : u == 1 ? 5 : 4; }

// U: pieces of 128 bytes of a row that a wave has on their way
template <int OT, bool PROT, int NB, int U> __global__ __launch_bounds__(256, few_waves(PROT, NB, U)) void gemm_mx4_few_kernel(Mx4FewArgs f)
{
    constexpr int BN = 16 * NB;
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    fetch_args<Mx4FewArgs>();
    const Mx4Args &g = f.g;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    if constexpr (PROT) {
        if (blockIdx.x == 0 && tid < 5) g.counts[tid] = 0u;
        if ((int)blockIdx.x < g.n_pass) {
            GroupTile t;
            if (find_tile<4 * PASS_ROWS>(g, g.pass_win, g.pass_inv, (int)blockIdx.x, &t, g.pass_log2))
                mx4_pass<4, false, 2>(g, t.e, t.first, t.rows, t.tm * 4 * PASS_ROWS << g.pass_log2, g.pass_log2, t.tn, smem);
            return;
        }
    }
    GroupTile t;
    if (!find_tile<16>(g, g.tiles_n, g.group_inv, (int)blockIdx.x - (PROT ? g.n_pass : 0), &t)) return;
    const int m0 = t.tm * 16, n0 = t.tn * BN, N = g.N;
    const int rows = min(t.rows - m0, 16);                       // of this tile
    const int nch = g.K / 16, pairs = (nch + 7) / 8;             // blocks of a row, pieces of 128 bytes
    const int i16 = lane & 15, piece = lane >> 4;
    const uint8_t *At = g.A + (long)(t.first + m0) * g.lda, *St = g.sa + (long)(t.first + m0) * g.ld_sa;
    const uint8_t *arow = At + (long)min(i16, rows - 1) * g.lda, *asc = St + (long)min(i16, rows - 1) * g.ld_sa;
    const uint8_t *brow[NB], *bsc[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        const long c = min(n0 + 16 * nb + i16, N - 1);
        brow[nb] = g.B + (long)t.e * g.sB + c * g.ldb;
        bsc[nb] = g.sb + (long)t.e * g.stride_sb + c * g.ld_sb;
    }

    // ---- this wave's pieces: every fourth
    f32x4 acc[NB], pred[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) { acc[nb] = pred[nb] = f32x4{0.f, 0.f, 0.f, 0.f}; }
    i32x4 a[U][2], b[U][2][NB];
    uint2 as[U], bs[U][NB];
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
            // (rows of powers of two are whole 16 bytes)
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) bs[u][nb] = *reinterpret_cast<const uint2 *>(bsc[nb] + (p0 + 4 * u) * 8);
            as[u] = *reinterpret_cast<const uint2 *>(asc + (p0 + 4 * u) * 8);
        }
    };
    // (what the sums of A below begin with is asked for first: loads come back in the order they were asked for)
    uint32_t ax[4], as4[4];
    auto load_rows = [&](int i, int r0) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const long r = min(r0 + j, rows - 1);
            ax[j] = *reinterpret_cast<const uint32_t *>(At + r * g.lda + (i >> 3) * 16 + ((i & 7) >> 1) * 4);
            as4[j] = St[r * g.ld_sa + (i >> 3)];
        }
    };
    if (PROT && tid < nch * 8) load_rows(tid, 0);
    const float b_top = PROT && f.tau_cols <= 0.f ? __uint_as_float(f.b_max[t.e]) : 0.f;
    if (wave < pairs) load(wave);

    // ---- e^T A of the tile's rows, in fp32, as eight-bit terms: a thread to four columns of a block
    uint8_t *const terms = smem + f.sums_off, *const powers = terms + nch * TERMS * 32;
    float *const tops = reinterpret_cast<float *>(smem + mx4_few_part_bytes<NB>() - 16);
    if constexpr (PROT) {
        float top = 0.f;
        for (int i = tid; i < nch * 8; i += 256) {
            const int c = i >> 3, half = i & 1;
            f32x4 sum = {0.f, 0.f, 0.f, 0.f};
            for (int r0 = 0; r0 < rows; r0 += 4) {
                if (i != tid || r0) load_rows(i, r0);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t v = half ? ax[j] >> 16 : ax[j];
                    const f32x2 p = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(v, mx4_unit(as4[j]), 0), q = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(v, mx4_unit(as4[j]), 1);
                    if (r0 + j < rows) {
                        sum += f32x4{p[0], p[1], q[0], q[1]};
                        top = fmaxf(fmaxf(fmaxf(top, fabsf(p[0])), fmaxf(fabsf(p[1]), fabsf(q[0]))), fabsf(q[1]));
                    }
                }
            }
            mx4_put_terms(sum, i & 7, terms + c * TERMS * 32, powers + c * 8);
        }
        top = wave_max(top);
        if (lane == 0) tops[wave] = top;
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    }
    for (int p0 = wave; p0 < pairs; p0 += 4 * U) {
        if constexpr (U > 1)                                     // (one piece is all there is for U = 1)
            if (p0 != wave) load(p0);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (u && p0 + 4 * u >= pairs) break;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int ch = (p0 + 4 * u) * 8 + 4 * h + piece;
                // past the last block nothing is multiplied, whatever both hold there
                const bool in = ch < nch;
                const i32x4 av = in ? a[u][h] : i32x4{0, 0, 0, 0};
                const uint32_t asv = in ? ((h ? as[u].y : as[u].x) >> (8 * piece)) & 0xFFu : 0u;
                i32x8 ev;
                uint32_t esv;
                if constexpr (PROT) mx4_get_terms(terms, powers, ch - piece, nch, lane, ev, esv);
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    const i32x4 bv = in ? b[u][h][nb] : i32x4{0, 0, 0, 0};
                    const uint32_t bsv = in ? ((h ? bs[u][nb].y : bs[u][nb].x) >> (8 * piece)) & 0xFFu : 0u;
                    acc[nb] = mfma16_mx4<0>(bv, av, acc[nb], bsv, asv);
                    if constexpr (PROT) pred[nb] = mfma16_mx4_f8(bv, ev, pred[nb], bsv, esv);
                }
            }
        }
    }

    // ---- the waves' sums, in LDS: [wave][nb][lane] of four, then [wave][nb][column] predictions
    float *const ppart = reinterpret_cast<float *>(smem + 4 * NB * 64 * 16);
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        *reinterpret_cast<f32x4 *>(smem + ((wave * NB + nb) * 64 + lane) * 16) = acc[nb];
        if constexpr (PROT) {
            f32x4 p;
#pragma unroll
            for (int i = 0; i < 4; ++i) p[i] = row16_sum(pred[nb][i]);           // (of the terms)
            if (i16 == 0) *reinterpret_cast<f32x4 *>(ppart + (wave * NB + nb) * 16 + 4 * piece) = p;
        }
    }
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    if (wave >= NB) return;
    const int nb = wave, c0 = n0 + 16 * nb + 4 * piece;
    float v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const f32x4 x = *reinterpret_cast<const f32x4 *>(smem + ((w * NB + nb) * 64 + lane) * 16);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] += x[i];
    }
    const bool in = i16 < rows;
    if (g.inj_b == t.e && g.inj_row == m0 + i16 && in) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (c0 + i == g.inj_col) v[i] = __uint_as_float(__float_as_uint(v[i]) ^ (1u << g.inj_bit));
    }
    if (in && c0 < N) {
        uint8_t *dst = g.C + ((long)(t.first + m0 + i16) * g.ldc + c0) * 2;
        const int n = min(N - c0, 4);
        float x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = v[i] + (g.bias ? g.bias[min(c0 + i, N - 1)] : 0.f);
        const uint2 w = make_uint2(pack2<OT>(x[0], x[1]), pack2<OT>(x[2], x[3]));
        if (n == 4) *reinterpret_cast<uint2 *>(dst) = w;
        else
#pragma unroll
            for (int i = 0; i < 3; ++i)
                if (i < n) reinterpret_cast<uint16_t *>(dst)[i] = (uint16_t)((i < 2 ? w.x : w.y) >> (16 * (i & 1)));
    }
    if constexpr (PROT) {
        float rsum = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (!in || c0 + i >= N) v[i] = 0.f;
            rsum += v[i];
        }
        rsum = add_xor32(add_xor16(rsum));
        if (lane < rows && 16 * nb + n0 < N) f.shares[(long)(t.tn * NB + nb) * g.M + t.first + m0 + lane] = as_word(rsum);
        // a column's sum over the sixteen lanes of its rows, against its prediction
        const float top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
        const float tol = f.tau_cols > 0.f ? f.tau_cols : f.tau_k * top * b_top;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float obs = row16_sum(v[i]);
            float p = 0.f;
#pragma unroll
            for (int w = 0; w < 4; ++w) p += ppart[(w * NB + nb) * 16 + 4 * piece + i];
            if (i16 == 0 && c0 + i < N && mismatch<false>(as_word(obs), as_word(p), tol)) atomicOr(g.cc_obs + (long)t.e * N + c0 + i, 1u);
        }
    }
}

// ------------------------------------------------------------------------------------------
constexpr int MX4_FEW_MAX_K = 8 * 1024;           // bytes of a row, protected: the column sums of A are kept in LDS

bool mx4_few_fits(bool protect, const Mx4Args &g) { return !protect || (g.M <= 32L * g.groups && g.K <= MX4_FEW_MAX_K); }

static int few_pieces(const Mx4Args &g) { return (g.K + 4 * SLAB_BYTES - 1) / (4 * SLAB_BYTES); }       // of a wave
// 32 columns to a workgroup, which reads its rows of A once for both halves, unless that leaves compute units without one; protected 64, while their
// registers leave room for several workgroups on a compute unit.
int mx4_few_columns(bool protect, const Mx4Args &g)
{
    const long rows = ((long)g.M + g.groups - 1) / g.groups, tiles = std::min(g.M, g.groups) * ((rows + 15) / 16);     // rows: of a group on average
    if (protect && few_pieces(g) == 1 && tiles * ((g.N + 63) / 64) >= 512) return 64;
    return tiles * ((g.N + 31) / 32) >= 512 ? 32 : 16;
}

long mx4_few_workgroups(bool protect, const Mx4Args &g)
{
    const int bn = mx4_few_columns(protect, g);
    return ((g.groups == 1 ? (g.M + 15) / 16 : g.M / 16 + std::min(g.M, g.groups)) * (long)((g.N + bn - 1) / bn) + 7) / 8 * 8;
}

template <int OT, bool PROT, int NB, int U> static hipError_t launch_few_of(Mx4FewArgs &f, hipStream_t st)
{
    Mx4Args &g = f.g;
    auto kern = gemm_mx4_few_kernel<OT, PROT, NB, U>;
    f.sums_off = (mx4_few_part_bytes<NB>() + 15) & ~15;
    int smem = f.sums_off;
    if (PROT) smem = std::max(smem + g.K / 16 * TERM_BYTES, mx4_pass_lds<4, false>());
    const hipError_t e = ensure_max_lds(reinterpret_cast<const void *>(kern), MX4_FEW_MAX_K / 16 * TERM_BYTES + 32 * 1024);
    if (e != hipSuccess) return e;
    g.tiles_n = (g.N + 16 * NB - 1) / (16 * NB);
    g.group_inv = map_inverse(g.tiles_n);
    const long wgs = (PROT ? g.n_pass : 0) + mx4_few_workgroups(PROT, g);
    hipLaunchKernelGGL(kern, dim3((unsigned)wgs), dim3(256), smem, st, f);
    return hipGetLastError();
}

// Registers for no more pieces than a wave has: with few, more waves share a SIMD, and they have more on their way together.
template <int OT, bool PROT, int NB> static hipError_t launch_few_one(Mx4FewArgs &f, hipStream_t st)
{
    const int pieces = few_pieces(f.g);
    return pieces <= 1 ? launch_few_of<OT, PROT, NB, 1>(f, st) : pieces <= 2 ? launch_few_of<OT, PROT, NB, 2>(f, st) : launch_few_of<OT, PROT, NB, 4>(f, st);
}

template <int OT> static hipError_t launch_few_type(bool protect, Mx4FewArgs &f, hipStream_t st)
{
    const int columns = mx4_few_columns(protect, f.g);
    if (!protect) return columns == 32 ? launch_few_one<OT, false, 2>(f, st) : launch_few_one<OT, false, 1>(f, st);
    if (columns == 64) return launch_few_of<OT, true, 4, 1>(f, st);
    return columns == 32 ? launch_few_one<OT, true, 2>(f, st) : launch_few_one<OT, true, 1>(f, st);
}

hipError_t launch_mx4_few(int ot, bool protect, Mx4Args &g, const uint32_t *b_max, float tau_k, float tau_cols, hipStream_t st)
{
    Mx4FewArgs f = {g, b_max, tau_k, tau_cols, group_few_shares(g), 0};
    return ot == DT_BF16 ? launch_few_type<DT_BF16>(protect, f, st) : launch_few_type<DT_F16>(protect, f, st);
}

}  // namespace abft
