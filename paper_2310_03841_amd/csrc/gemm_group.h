// Products over groups of rows for gfx950 (group_args.h): C_e = A_e B_e for every group e of the rows of A, with the scales of quantised operands
// (C = row scale x column scale x integer product + bias) or without, protected or not; and the gradient of the B_e, G_e = Y_e^T X_e,
// whose depth is a group's rows.
//
// Tile: BM x BN by four waves of (BM/2) x (BN/2), 32 x 32 MFMA blocks; slabs of 128 bytes of K straight from memory into LDS, NS buffers deep, one barrier
// per slab; the fragments of slab s are read while the MFMAs of slab s - 1 run.  An operand that is contiguous along K keeps rows of
// 128 bytes in LDS; one that is not (B stored K x N; both operands of the gradient) keeps rows of k, which the LDS transpose reads of gfx950 turn
// on the way to the matrix cores.  Every swizzle is applied by choosing which chunk of memory a lane fetches.
//
// Edges: rows, columns and k past the end fetch the last valid ones.  What they produce is never stored or summed, or cleared in registers ahead of
// the MFMAs (k: of both operands, as either may hold what is not finite).
#pragma once
#include <algorithm>

#include "abft_device.h"
#include "block_out.h"
#include "group_args.h"
#include "group_passes.h"

namespace abft {

typedef const __attribute__((address_space(1))) void *grp_gas_ptr;
typedef __attribute__((address_space(3))) void *grp_las_ptr;
typedef int i32x2_t __attribute__((ext_vector_type(2)));

// One operand of a tile: W rows of A (or columns of B) from `first` on.  KM: rows of k in memory, W of whose elements are the tile's.
template <int DT, int W, bool KM> struct GroupOperand {
    static constexpr int ES = Traits<DT>::ES, KE = SLAB_BYTES / ES, G = W / 32, BYTES = W * SLAB_BYTES;
    static constexpr int ROWB = W * ES;                          // KM: bytes of a row of k
    static constexpr int NB = W / 64;                            // 32-wide blocks of a wave
    const uint8_t *src[KM ? 1 : G];
    int chunk, kk[KM ? G : 1], at[KM ? G : 1];
    long ldb;

    // base: of the group's operand; n: its rows (KM: columns)
    __device__ __forceinline__ void setup(const uint8_t *base, long ld, int first, int n, int wave, int lane)
    {
        ldb = ld * ES;
        if constexpr (KM) {
            constexpr int LPR = ROWB / 16, RPG = 64 / LPR;       // lanes to a row of k, rows to a load
            src[0] = base;
            const int last = ((n - 1) * ES) / 16 * 16;           // last chunk that holds an element
#pragma unroll
            for (int p = 0; p < G; ++p) {
                kk[p] = (4 * p + wave) * RPG + lane / LPR;
                const int cb = first * ES + (((lane % LPR) ^ kn_swizzle<ES, ROWB>(kk[p])) * 16);
                at[p] = cb < last ? cb : last;
            }
        } else {
            const int lrow = lane >> 3;
            chunk = (lane & 7) ^ (((wave & 1) << 2) + (lrow >> 1));
#pragma unroll
            for (int p = 0; p < G; ++p) {
                const int r = first + (4 * p + wave) * 8 + lrow;
                src[p] = base + (long)(r < n ? r : n - 1) * ldb;
            }
        }
    }
    __device__ __forceinline__ void issue(int s, uint8_t *to, int K, int wave) const
    {
        const int nch = (K * ES + 15) / 16;
#pragma unroll
        for (int p = 0; p < G; ++p) {
            const uint8_t *from;
            if constexpr (KM) {
                const int k = s * KE + kk[p];
                from = src[0] + (long)(k < K ? k : K - 1) * ldb + at[p];
            } else {
                const int ch = s * 8 + chunk;
                from = src[p] + (long)(ch < nch ? ch : nch - 1) * 16;
            }
            __builtin_amdgcn_global_load_lds((grp_gas_ptr)from, (grp_las_ptr)(to + (4 * p + wave) * 8 * SLAB_BYTES), 16, 0, 0);
        }
    }
    // the four steps' fragments of a wave whose blocks begin at `w0`
    __device__ __forceinline__ static void read(i32x4 (&f)[4][NB], const uint8_t *sm, int w0, int lane)
    {
        const int l32 = lane & 31, lh = lane >> 5;
        if constexpr (!KM) {
#pragma unroll
            for (int s4 = 0; s4 < 4; ++s4)
#pragma unroll
                for (int i = 0; i < NB; ++i)
                    f[s4][i] = *reinterpret_cast<const i32x4 *>(sm + (w0 + i * 32 + l32) * SLAB_BYTES + ((2 * s4 + lh) ^ ((lane >> 1) & 7)) * 16);
        } else {
            // Sixteen lanes read 4 (8) rows of k of sixteen columns; each gets one column.  Instructions with their own wait: in front of the
            // built-in the compiler waits for every outstanding load.
            constexpr int HALF = (ES == 2 ? 4 : 8) * ROWB, STEP = (ES == 2 ? 16 : 32) * ROWB;
            const int i16 = lane & 15;
            const int k = ES == 2 ? 8 * lh + (i16 >> 2) : 16 * lh + (i16 >> 1);
#pragma unroll
            for (int i = 0; i < NB; ++i) {
                const int cb = (w0 + i * 32 + 16 * ((lane >> 4) & 1)) * ES + (ES == 2 ? (i16 & 3) : (i16 & 1)) * 8;
                const uint32_t a = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const uint8_t *)(
                    sm + k * ROWB + (((cb >> 4) ^ kn_swizzle<ES, ROWB>(k)) * 16) + (cb & 15));
                i32x2_t h[8];
#define GROUP_TR(T) \
                asm volatile(T " %0, %8\n\t" T " %1, %8 offset:%9\n\t" T " %2, %8 offset:%10\n\t" T " %3, %8 offset:%11\n\t" \
                             T " %4, %8 offset:%12\n\t" T " %5, %8 offset:%13\n\t" T " %6, %8 offset:%14\n\t" T " %7, %8 offset:%15\n\t" \
                             "s_waitcnt lgkmcnt(0)" \
                             : "=&v"(h[0]), "=&v"(h[1]), "=&v"(h[2]), "=&v"(h[3]), "=&v"(h[4]), "=&v"(h[5]), "=&v"(h[6]), "=&v"(h[7]) \
                             : "v"(a), "n"(HALF), "n"(STEP), "n"(STEP + HALF), "n"(2 * STEP), "n"(2 * STEP + HALF), "n"(3 * STEP), \
                               "n"(3 * STEP + HALF) : "memory")
                if constexpr (ES == 2) GROUP_TR("ds_read_b64_tr_b16");
                else GROUP_TR("ds_read_b64_tr_b8");
#undef GROUP_TR
#pragma unroll
                for (int s4 = 0; s4 < 4; ++s4) f[s4][i] = i32x4{h[2 * s4][0], h[2 * s4][1], h[2 * s4 + 1][0], h[2 * s4 + 1][1]};
            }
        }
    }
};

// What a kernel computes: C over groups of rows, or the gradient over groups along the depth.
enum { GROUP_ROWS, GROUP_DEPTH };

__host__ __device__ constexpr int group_loop_bytes(int BM, int BN, int ns)
{
    const int loop = ns * (BM + BN) * SLAB_BYTES, epi = 2 * (BM + BN) * 4;
    return loop > epi ? loop : epi;
}
// behind the buffers: scales of the tile's rows and columns, bias of its columns
__host__ __device__ constexpr int group_lds_bytes(int BM, int BN, int ns, bool scaled) { return group_loop_bytes(BM, BN, ns) + (scaled ? (BM + 2 * BN) * 4 : 0); }

// DT: of the operands; OT: of C, the same or, of scaled int8, a 16-bit type.
template <int DT, int OT, int BM, int BN, int NS, bool PROT, int GROUP, bool TRANSB>
__global__ __launch_bounds__(256) void gemm_group_kernel(GroupArgs g)
{
    using T = Traits<DT>;
    typedef typename T::acc_t acc_t;
    typedef typename T::accv_t accv_t;
    constexpr bool SCALED = OT != DT, DEPTH = GROUP == GROUP_DEPTH;
    constexpr int ES = T::ES, OS = Traits<OT>::OS, KE = SLAB_BYTES / ES;
    constexpr int TM = BM / 2, TN = BN / 2, MI = TM / 32, NI = TN / 32;
    constexpr int BUF = (BM + BN) * SLAB_BYTES;
    typedef GroupOperand<DT, BM, DEPTH> OpA;
    typedef GroupOperand<DT, BN, DEPTH || !TRANSB> OpB;
    constexpr int NLD = OpA::G + OpB::G;
    static_assert((NS - 2) * NLD < 64, "the wait count is an immediate");

    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    fetch_args<GroupArgs>();
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    if constexpr (PROT) {
        if (blockIdx.x == 0 && tid < 5) g.counts[tid] = 0u;
        if ((int)blockIdx.x < g.n_pass) {
            GroupTile t;
            if (find_tile<4 * PASS_ROWS>(g, g.pass_win, g.pass_inv, (int)blockIdx.x, &t))
                group_pass<DT, 4>(g, t.e, t.first, t.rows, t.tm * 4 * PASS_ROWS, t.tn, smem);
            return;
        }
    }
    const int wm = wave >> 1, wn = wave & 1;
    const int l32 = lane & 31, lh = lane >> 5;
    const int bid = (int)blockIdx.x - (PROT ? g.n_pass : 0);
    GroupTile t;
    int M, K;                                                    // of the group
    const int N = g.N;
    const uint8_t *Ab, *Bb;
    uint8_t *Cb;
    if constexpr (DEPTH) {
        // A: rows of the depth, K of the launch elements of each are the product's rows
        M = g.K;
        const int tiles_m = (M + BM - 1) / BM, per = tiles_m * g.tiles_n, nb = per * g.groups;
        const int q = nb >> 3, r = nb & 7, xcd = bid & 7, i = bid >> 3;
        if (i >= q + (xcd < r ? 1 : 0)) return;
        const int L = xcd * q + (xcd < r ? xcd : r) + i;
        t.e = L / per;
        tile_at(L - t.e * per, tiles_m, g.tiles_n, g.group_inv, &t.tm, &t.tn);
        group_rows(g.offsets, g.M, t.e, &t.first, &t.rows);
        K = t.rows;
        Ab = g.A + (long)t.first * g.lda * ES;
        Bb = g.B + (long)t.first * g.ldb * ES;
        Cb = g.C + (long)t.e * g.sB * OS;
    } else {
        if (!find_tile<BM>(g, g.tiles_n, g.group_inv, bid, &t)) return;
        M = t.rows;
        K = g.K;
        Ab = g.A + (long)t.first * g.lda * ES;
        Bb = g.B + (long)t.e * g.sB * ES;
        Cb = g.C + (long)t.first * g.ldc * OS;
    }
    const int m0 = t.tm * BM, n0 = t.tn * BN;
    const int nslab = (int)(((long)K + KE - 1) / KE);

    accv_t acc[MI][NI];
#pragma unroll
    for (int mi = 0; mi < MI; ++mi)
#pragma unroll
        for (int ni = 0; ni < NI; ++ni)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[mi][ni][i] = T::zero();

    float *const srow = reinterpret_cast<float *>(smem + group_loop_bytes(BM, BN, NS)), *const scol = srow + BM, *const sbias = scol + BN;
    if constexpr (SCALED) {
        // (absent: ones, and a bias of zeros)
        for (int i = tid; i < BM; i += 256) srow[i] = g.row_scale ? g.row_scale[t.first + min(m0 + i, M - 1)] : 1.f;
        for (int i = tid; i < BN; i += 256) {
            const int c = min(n0 + i, N - 1);
            scol[i] = g.col_scale ? g.col_scale[(long)t.e * N + c] : 1.f;
            sbias[i] = g.bias ? g.bias[c] : 0.f;
        }
    }
    if (!DEPTH || nslab > 0) {
        OpA oa;
        OpB ob;
        oa.setup(Ab, g.lda, m0, M, wave, lane);
        ob.setup(Bb, g.ldb, n0, N, wave, lane);
        i32x4 fa[2][4][MI], fb[2][4][NI];
        auto issue = [&](int s) __attribute__((always_inline)) {
            uint8_t *d = smem + (s % NS) * BUF;
            oa.issue(s, d, K, wave);
            ob.issue(s, d + OpA::BYTES, K, wave);
        };
        auto read = [&](int s, auto set_c) __attribute__((always_inline)) {
            const uint8_t *d = smem + (s % NS) * BUF;
            OpA::read(fa[decltype(set_c)::value], d, wm * TM, lane);
            OpB::read(fb[decltype(set_c)::value], d + OpA::BYTES, wn * TN, lane);
        };
        auto clear_tail = [&](auto set_c) __attribute__((always_inline)) {
            constexpr int set = decltype(set_c)::value;
            const int base = (K - (nslab - 1) * KE) * ES;        // bytes of K in the last slab
#pragma unroll
            for (int s4 = 0; s4 < 4; ++s4) {
                const int keep = base - (2 * s4 + lh) * 16;
#pragma unroll
                for (int mi = 0; mi < MI; ++mi) fa[set][s4][mi] = mask_chunk(fa[set][s4][mi], keep);
#pragma unroll
                for (int ni = 0; ni < NI; ++ni) fb[set][s4][ni] = mask_chunk(fb[set][s4][ni], keep);
            }
        };
        auto mfmas = [&](auto set_c) __attribute__((always_inline)) {
            constexpr int set = decltype(set_c)::value;
#pragma unroll
            for (int s4 = 0; s4 < 4; ++s4)
#pragma unroll
                for (int mi = 0; mi < MI; ++mi)
#pragma unroll
                    for (int ni = 0; ni < NI; ++ni) acc[mi][ni] = T::mfma(fb[set][s4][ni], fa[set][s4][mi], acc[mi][ni]);
        };
        typedef std::integral_constant<int, 0> set0;
        typedef std::integral_constant<int, 1> set1;
        // Slab s is in place behind "at most the slabs issued after it outstanding" (a wave's loads complete in order) and the barrier; the same
        // barrier says that every wave has its fragments of slab s - 1 in registers, so that buffer takes slab s + NS - 1.
        for (int s = 0; s < NS - 1; ++s)
            if (s < nslab) issue(s);
        auto arrive = [&](int s) __attribute__((always_inline)) {
            const int ahead = nslab - 1 - s;                     // slabs issued after s: min(ahead, NS - 2)
            if (ahead >= NS - 2) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" :: "n"((NS - 2) * NLD) : "memory");
            else if (NS > 3 && ahead == 1) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" :: "n"(NLD) : "memory");
            else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
            if (s + NS - 1 < nslab) issue(s + NS - 1);
        };
        static_assert(NS == 3 || NS == 4, "what arrive() tells apart");
        const bool ragged = K % KE != 0;
        arrive(0);
        read(0, set0{});
        int s = 1;
        for (; s + 1 < nslab; s += 2) {
            arrive(s);
            read(s, set1{});
            mfmas(set0{});
            arrive(s + 1);
            read(s + 1, set0{});
            mfmas(set1{});
        }
        if (s < nslab) {
            arrive(s);
            read(s, set1{});
            mfmas(set0{});
            if (ragged) clear_tail(set1{});
            mfmas(set1{});
        } else {
            if (ragged) clear_tail(set0{});
            mfmas(set0{});
        }
    }

    // ---- epilogue, from the registers (block_out.h): lane l holds row l & 31 of a block and in register i column
    // 8 (i >> 2) + 4 (l >> 5) + (i & 3)
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");       // every wave is done with the operand buffers; the scales are in place
    acc_t *rs_part = reinterpret_cast<acc_t *>(smem);                     // [2][BM] by wave column
    acc_t *cs_part = rs_part + 2 * BM;                                    // [2][BN] by wave row
    const bool inj_here = g.inj_b == t.e && g.inj_row >= m0 && g.inj_row < m0 + BM && g.inj_col >= n0 && g.inj_col < n0 + BN;
    const bool inside = m0 + BM <= M && n0 + BN <= N;
    constexpr bool QUADS = Traits<OT>::IS_INT && !PROT;
    constexpr int NP = out_passes<OT>(), RPP = out_step<OT, QUADS>();
    const int orow = m0 + wm * TM + out_row<OT, QUADS>(lane), ocol = n0 + wn * TN + out_col<OT, QUADS>(lane);
    // (a gradient's rows are ldc apart too: the host passes the weights' leading dimension)
    uint8_t *const dst0 = Cb + ((long)orow * g.ldc + ocol) * OS;
    const long pass_bytes = (long)RPP * g.ldc * OS;
    const int left = (N * OS) & 15;
    acc_t cs[NI][16];
    if (PROT) {
#pragma unroll
        for (int ni = 0; ni < NI; ++ni)
#pragma unroll
            for (int i = 0; i < 16; ++i) cs[ni][i] = T::zero();
    }
    static_for<0, MI>([&](auto mi_c) {
        constexpr int mi = decltype(mi_c)::value;
        const int row = m0 + wm * TM + mi * 32 + l32;
        acc_t rsum = T::zero();
        float rscale = 1.f;
        if constexpr (SCALED) rscale = srow[wm * TM + mi * 32 + l32];
        static_for<0, NI>([&](auto ni_c) {
            constexpr int ni = decltype(ni_c)::value;
            const int c0 = n0 + wn * TN + ni * 32;
            acc_t v[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = acc[mi][ni][i];
            if (inj_here && row == g.inj_row) {
                // the armed flip: one bit of one accumulator, before scales, rounding and sums
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (c0 + 8 * (i >> 2) + 4 * lh + (i & 3) == g.inj_col) v[i] = from_word<acc_t>(as_word(v[i]) ^ (1u << g.inj_bit));
            }
            if (PROT && !inside) {
#pragma unroll
                for (int i = 0; i < 16; ++i) v[i] = row < M && c0 + 8 * (i >> 2) + 4 * lh + (i & 3) < N ? v[i] : T::zero();
            }
            if (PROT) {
#pragma unroll
                for (int i = 0; i < 16; ++i) cs[ni][i] = add_t(cs[ni][i], v[i]);
                rsum = add_t(rsum, sum16<acc_t>(v));
            }
            i32x4 out[NP];
            if constexpr (SCALED) {
                // each step one rounding of fp32: the sum, times the row's scale, times the column's, the bias with it
                float f[16];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const i32x4 c4 = *reinterpret_cast<const i32x4 *>(scol + wn * TN + ni * 32 + 8 * q + 4 * lh);
                    const i32x4 b4 = *reinterpret_cast<const i32x4 *>(sbias + wn * TN + ni * 32 + 8 * q + 4 * lh);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        f[4 * q + e] = __builtin_fmaf((float)v[4 * q + e] * rscale, __uint_as_float((uint32_t)c4[e]), __uint_as_float((uint32_t)b4[e]));
                }
                uint32_t w[8];
                pack_block<OT>(f, w);
                turn_block<OT>(w, out);
            } else if constexpr (T::IS_INT) {
                uint32_t w[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) w[i] = (uint32_t)v[i];
                if constexpr (QUADS) turn_quads(w, out, lane);
                else turn_block<DT>(w, out);
            } else {
                uint32_t w[8];
                pack_block<DT>(v, w);
                turn_block<DT>(w, out);
            }
            uint8_t *dst = dst0 + (long)(mi * 32) * g.ldc * OS + ni * 32 * OS;
            if (inside) {
#pragma unroll
                for (int p = 0; p < NP; ++p) *reinterpret_cast<i32x4 *>(dst + p * pass_bytes) = out[p];
            } else {
                const int gc = ocol + ni * 32, rows = M - (orow + mi * 32);      // valid rows from this lane's first on
                if (gc + 16 / OS <= N) {
#pragma unroll
                    for (int p = 0; p < NP; ++p)
                        if (p * RPP < rows) *reinterpret_cast<i32x4 *>(dst + p * pass_bytes) = out[p];
                } else if (gc < N) {
                    // in falling powers of two, all passes of a size together: few branches
                    if (left & 8) {
#pragma unroll
                        for (int p = 0; p < NP; ++p)
                            if (p * RPP < rows) *reinterpret_cast<i32x2_t *>(dst + p * pass_bytes) = i32x2_t{out[p][0], out[p][1]};
                    }
                    if (left & 4) {
                        const int at = left & 8;
#pragma unroll
                        for (int p = 0; p < NP; ++p)
                            if (p * RPP < rows) *reinterpret_cast<int *>(dst + p * pass_bytes + at) = at ? out[p][2] : out[p][0];
                    }
                    if (left & 2) {
                        const int at = left & 12;
#pragma unroll
                        for (int p = 0; p < NP; ++p)
                            if (p * RPP < rows)
                                *reinterpret_cast<uint16_t *>(dst + p * pass_bytes + at) =
                                    (uint16_t)(at & 8 ? (at & 4 ? out[p][3] : out[p][2]) : (at & 4 ? out[p][1] : out[p][0]));
                    }
                }
            }
        });
        if (PROT) {
            const acc_t r = add_xor32(rsum);
            if (lane < 32) rs_part[wn * BM + wm * TM + mi * 32 + lane] = r;
        }
    });
    if (PROT) {
#pragma unroll
        for (int ni = 0; ni < NI; ++ni) {
            const acc_t s = fold16<acc_t>(cs[ni], lane);
            if ((lane & 1) == 0) cs_part[wm * BN + wn * TN + ni * 32 + fold16_column(lane)] = s;
        }
        // over LDS traffic only: a full barrier would also wait for every store of C
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        for (int i = tid; i < BM + BN; i += 256) {
            const bool isrow = i < BM;
            const int q = isrow ? i : i - BM, gi = (isrow ? m0 : n0) + q;
            if (gi < (isrow ? M : N)) {
                const acc_t *src = isrow ? rs_part + q : cs_part + q;
                const long o = isrow ? (long)t.first + gi : (long)t.e * N + gi;
                const acc_t sum = add_t(src[0], src[isrow ? BM : BN]);
                if constexpr (T::IS_INT) atomic_add_word((isrow ? g.rc_obs : g.cc_obs) + o, sum);
                else unsafeAtomicAdd((isrow ? g.rc_acc : g.cc_acc) + o, (double)sum);
            }
        }
    }
}

// ------------------------------------------------------------------------------------------
inline long ceil_div(long a, long b) { return (a + b - 1) / b; }

// Most tiles along the rows, whatever their split: a tile that is not full for each group that has rows.
inline long row_tiles(int M, int groups, int BM) { return groups == 1 ? ceil_div(M, BM) : M / BM + std::min(M, groups); }

template <int DT, int OT, int BM, int BN, int NS, bool PROT, int GROUP, bool TRANSB>
static hipError_t launch_one(GroupArgs &g, hipStream_t st)
{
    constexpr int smem = group_lds_bytes(BM, BN, NS, OT != DT);
    static_assert(smem >= group_pass_lds<DT, 4>(), "the pass over A runs in the LDS of a tile");
    auto kern = gemm_group_kernel<DT, OT, BM, BN, NS, PROT, GROUP, TRANSB>;
    hipError_t e = ensure_max_lds(reinterpret_cast<const void *>(kern), smem);
    if (e != hipSuccess) return e;
    g.tiles_n = (int)ceil_div(g.N, BN);
    g.group_inv = map_inverse(g.tiles_n);
    const long tiles_m = GROUP == GROUP_DEPTH ? ceil_div(g.K, BM) * g.groups : row_tiles(g.M, g.groups, BM);
    const long wgs = (PROT ? g.n_pass : 0) + ceil_div(tiles_m * g.tiles_n, 8) * 8;
    hipLaunchKernelGGL(kern, dim3((unsigned)wgs), dim3(256), smem, st, g);
    return hipGetLastError();
}

template <int DT, int OT, int BM, int BN, int NS>
static hipError_t launch_rows(bool protect, bool transB, GroupArgs &g, hipStream_t st)
{
    if (protect) return transB ? launch_one<DT, OT, BM, BN, NS, true, GROUP_ROWS, true>(g, st)
                               : launch_one<DT, OT, BM, BN, NS, true, GROUP_ROWS, false>(g, st);
    return transB ? launch_one<DT, OT, BM, BN, NS, false, GROUP_ROWS, true>(g, st)
                  : launch_one<DT, OT, BM, BN, NS, false, GROUP_ROWS, false>(g, st);
}


// Tiles of 64 x 64, with four or three buffers, and of 64 x 128.  (Of 128 x 128 they were the best of three shapes for one of 180 random problems, by 1 %.)
enum { TILE_64_4, TILE_64, TILE_64_128 };
template <int DT, int OT> static hipError_t launch_rows_of(int tiles, bool protect, bool transB, GroupArgs &g, hipStream_t st)
{
    switch (tiles) {
    case TILE_64_4:   return launch_rows<DT, OT, 64, 64, 4>(protect, transB, g, st);
    case TILE_64:     return launch_rows<DT, OT, 64, 64, 3>(protect, transB, g, st);
    default:          return launch_rows<DT, OT, 64, 128, 3>(protect, transB, g, st);
    }
}
template <int DT> static hipError_t launch_depth_of(int tiles, GroupArgs &g, hipStream_t st)
{
    switch (tiles) {
    case TILE_64_4:   return launch_one<DT, DT, 64, 64, 4, false, GROUP_DEPTH, false>(g, st);
    case TILE_64:     return launch_one<DT, DT, 64, 64, 3, false, GROUP_DEPTH, false>(g, st);
    default:          return launch_one<DT, DT, 64, 128, 3, false, GROUP_DEPTH, false>(g, st);
    }
}

// Each in a file of its own, for the time it takes to compile them.
hipError_t launch_group_rows_i8(int ot, int tiles, bool protect, bool transB, GroupArgs &g, hipStream_t st);
hipError_t launch_group_rows_bf16(int tiles, bool protect, bool transB, GroupArgs &g, hipStream_t st);
hipError_t launch_group_rows_f16(int tiles, bool protect, bool transB, GroupArgs &g, hipStream_t st);
hipError_t launch_group_depth_bf16(int tiles, GroupArgs &g, hipStream_t st);
hipError_t launch_group_depth_f16(int tiles, GroupArgs &g, hipStream_t st);

}  // namespace abft
