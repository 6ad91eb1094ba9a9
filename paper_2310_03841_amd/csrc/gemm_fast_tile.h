// One tile of the fast GEMM kernels: what gemm_fast.hip and gemm_group_big.h share.  The loop is described in gemm_fast.hip.
#pragma once
#include "abft_device.h"
#include "gemm_args.h"
#include "gemm_epilogue.h"
#include "mx4_device.h"

namespace abft {

typedef const __attribute__((address_space(1))) void *gas_ptr;
typedef __attribute__((address_space(3))) void *las_ptr;

// Unprotected; protected, the tiles reduce A; protected, workgroups beside the tiles do.  A kernel for each: the last
// has no code for owned slabs, the others none for the pass beside them.
enum { FAST_PLAIN, FAST_OWN, FAST_BESIDE };

// LDS of a tile: a slab is MI units of A and 2 NI of B, 64 rows of 128 bytes each: one load instruction of every wave.  Unit mi of A
// holds the rows of block row mi of both wave rows, unit (ni, h) of B those of block column ni of wave columns 2 h and 2 h + 1.
// The first FM units of A and the first 2 FN of B have three buffers, the others two.
template <int BM, int FM, int FN> struct FastLds {
    static constexpr int MI = BM / 64, NI = 2, UNIT = 64 * SLAB_BYTES;
    static constexpr int NLD = MI + 2 * NI;                                // units
    static constexpr int NF = FM + 2 * FN, NR = NLD - NF;                  // those with three buffers, with two
    static constexpr int F_BYTES = NF * UNIT, R_BYTES = NR * UNIT, BYTES = 3 * F_BYTES + 2 * R_BYTES;
    // Load q of a slab: first the units with two buffers, A then B, then those with three.
    static constexpr bool ring3(int q) { return q >= NR; }
    static constexpr bool is_a(int q) { return q < NR ? q < MI - FM : q < NR + FM; }
    static constexpr int unit(int q)                                       // mi, or 2 ni + h
    {
        return q < NR ? (q < MI - FM ? FM + q : 2 * FN + q - (MI - FM)) : q < NR + FM ? q - NR : q - NR - FM;
    }
    // Loads of the four steps from a slab's barrier on: the first of them go where the next barrier needs them.
    static constexpr int by_step(int n) { return n == 0 ? 0 : n == 1 ? (3 * NLD + 7) / 8 : n == 2 ? (5 * NLD + 7) / 8 : n == 3 ? 7 * NLD / 8 : NLD; }
    // where it lies in its buffer
    static constexpr int at(int q) { return (q < NR ? q : q - NR) * UNIT; }
    static constexpr int load_of_a(int mi) { return mi < FM ? NR + mi : mi - FM; }
    static constexpr int load_of_b(int ni) { return ni < FN ? NR + FM + 2 * ni : MI - FM + 2 * (ni - FN); }      // h = 0
};
// 4-bit operands: behind the buffers lie two of the powers of two of a slab, eight bytes to a row, 256 rows of A and of B.
constexpr int FAST_SCALES = 2 * 256 * 8;
template <int DT, int MODE, int BM> struct FastShape;
template <int DT, int MODE> struct FastShape<DT, MODE, 256> { typedef FastLds<256, MODE == FAST_OWN || DT == DT_MX4 ? 3 : 4, 0> lds; };
template <int DT, int MODE> struct FastShape<DT, MODE, 128> { typedef FastLds<128, 2, 2> lds; };
template <int DT, int MODE> constexpr int fast_ring_bytes()
{
    const int b = FastShape<DT, MODE, 256>::lds::BYTES, s = FastShape<DT, MODE, 128>::lds::BYTES;
    return b > s ? b : s;
}
template <int DT, int MODE> constexpr int fast_lds_bytes() { return fast_ring_bytes<DT, MODE>() + (DT == DT_MX4 ? 2 * FAST_SCALES : 0); }

// One BM x 256 tile with origin (m0, n0) of batch item bz.
// What the pass over A keeps lies behind the operand buffers.
// AT, BT (16-bit types): the operand lies as rows of k (A: the transpose; B: K x N).  A unit then is 64 rows of k of 64 rows of A (columns of B), which the
// LDS transpose reads turn; rows of k past the end arrive as zeros, and K need not be whole slabs.  Without: whole slabs, three at least.
template <int DT, int OT, int BM, int MODE, int STO, bool AT, bool BT, typename SRC>
__device__ __forceinline__ void fast_tile(const GemmArgs &g, SRC source, uint8_t *smem, int m0, int n0, int bz, int tn)
{
    using T = Traits<DT>;
    using L = typename FastShape<DT, MODE, BM>::lds;
    typedef typename T::accv_t accv_t;
    typedef __attribute__((address_space(3))) uint8_t *lds_ptr;
    typedef __attribute__((address_space(3))) void *lds_void;
    typedef const __attribute__((address_space(3))) i32x4 *lds_frag;
    constexpr int ES = T::ES;
    constexpr int KE = SLAB_BYTES / ES;
    constexpr int TM = BM / 2, TN = 64;
    constexpr int MI = L::MI, NI = L::NI, NMF = MI * NI, NFR = MI + NI;
    constexpr int NF = L::NF, NR = L::NR, NLD = L::NLD;
    constexpr bool PROT = MODE != FAST_PLAIN, OWN = MODE == FAST_OWN;
    static_assert(!AT || BT, "A's rows of k come with B's");
    static_assert(!(AT || BT) || (ES == 2 && !OWN), "rows of k are turned 16 bits at a time, and not reduced");

    const int tid = tile_thread_index(), lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);      // wave-uniform by construction
    const int wm = wave >> 2, wn = wave & 3;
    const int l32 = lane & 31, lh = lane >> 5;
    const int M = g.M, N = g.N, K = g.K;

    // ---- global sources.  This wave's load of a unit fills its LDS rows 8 wave .. + 8;
    // lane l lands in row + (l >> 3), slot (l & 7), and fetches the chunk for which
    // LDS slot = chunk ^ ((row >> 1) & 7).  (A 16-byte fragment read is served sixteen lanes at a
    // time from 64 banks: sixteen consecutive rows must fall on sixteen different 16-byte bank
    // groups.  Two consecutive 128-byte rows span all 64 banks, so the eight even rows need eight
    // different slots, and so do the eight odd rows; chunk ^ (row & 7) makes rows r and r + 8
    // collide, which the LDS bank-conflict counter showed as half of all LDS cycles.)  Buffer loads: the tile's
    // origin in a descriptor, a lane's offset inside the tile, which never changes, in a register, the slab's in a scalar, so
    // that a load inside the main loop is itself and the word that says where it goes.  Rows of the tile past
    // the end of the matrix fetch the last valid row instead.
    const int lrow = lane >> 3;
    const int lchunk = (lane & 7) ^ (((wave & 1) << 2) + (lrow >> 1));
    constexpr int RSRC_FLAGS = 0x00027000;
    // (rows of k: as many bytes as the matrix has from the tile's first element on, and loads past them bring zeros)
    const __amdgpu_buffer_rsrc_t a_src = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<uint8_t *>(g.A + ((long)bz * g.sA + (AT ? (long)m0 : (long)m0 * g.lda)) * ES), 0, AT ? max((int)((K * g.lda - m0) * ES), 0) : 0x7FFFFFFF, RSRC_FLAGS);
    const __amdgpu_buffer_rsrc_t b_src = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<uint8_t *>(g.B + ((long)bz * g.sB + (BT ? (long)n0 : (long)n0 * g.ldb)) * ES), 0, BT ? max((int)((K * g.ldb - n0) * ES), 0) : 0x7FFFFFFF, RSRC_FLAGS);
    int off[NLD];
    static_for<0, NLD>([&](auto q_c) {
        constexpr int q = decltype(q_c)::value, u = L::unit(q);
        constexpr bool is_a = L::is_a(q), rows_of_k = is_a ? AT : BT;
        const int last = (is_a ? M - m0 : N - n0) - 1;
        if constexpr (rows_of_k) {
            const int k = wave * 8 + lrow, at = u * 128 + ((lane & 7) ^ kn_swizzle<2, 128>(k)) * 16, end = (last * ES) & ~15;
            off[q] = k * (int)((is_a ? g.lda : g.ldb) * ES) + (at < end ? at : end);     // (past the last row or column: the last chunk with one)
        } else {
            const int in = (wave & 3) * 8 + lrow;
            int r = is_a ? (wave >> 2) * TM + u * 32 + in : (2 * (u & 1) + (wave >> 2)) * TN + (u >> 1) * 32 + in;
            r = r < last ? r : last;
            off[q] = r * (int)((is_a ? g.lda : g.ldb) * ES) + lchunk * 16;
        }
    });
    const int a_step = AT ? KE * (int)(g.lda * ES) : SLAB_BYTES, b_step = BT ? KE * (int)(g.ldb * ES) : SLAB_BYTES;      // from slab to slab
    const int a_rows = M - m0;                        // rows of this tile inside A
    const int nslab = AT ? max(3, (K + KE - 1) / KE) : K / KE;      // at least 3 (gemm_fast_eligible)
    EpiScale sc = {1.f, 1.f, 0.f};
    if constexpr (OT != DT) sc = source.scales(m0, n0, tid, M, N);

    // The accumulators are never zero-filled: the first MFMA of every block takes a literal
    // zero as its addend.  Every block is always computed, also where the tile hangs over the
    // edge of the problem: a conditional MFMA would move the accumulators out of their registers.
    accv_t acc[MI][NI];
    accv_t zerov;
#pragma unroll
    for (int i = 0; i < 16; ++i) zerov[i] = T::zero();

    // The buffers of a slab: f of those in rings of three, r of two.
    const lds_ptr lds = (lds_ptr)smem;
    struct Buf { int f, r; };
    auto load = [&](auto q_c, int s, Buf to) __attribute__((always_inline)) {
        constexpr int q = decltype(q_c)::value;
        const lds_ptr dst = lds + ((L::ring3(q) ? to.f : to.r) + wave * 8 * SLAB_BYTES) + L::at(q);
        int at = s * (L::is_a(q) ? a_step : b_step);
        // (4 bits: slabs past the last one begin at the descriptor's end, and cost no memory)
        if constexpr (DT == DT_MX4) at = s < nslab ? at : 0x7FFFFFFF;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(L::is_a(q) ? a_src : b_src, (lds_void)dst, 16, off[q], at, 0, 0);
    };
    // 4 bits: the powers of two of a slab go through LDS as the units with two buffers do, two loads of a wave ahead of those; a lane reads the word of its rows' next four
    // blocks two steps at a time, and bytes 0 and 2 of it, shifted, are those of its own blocks.  (Straight into registers, two steps ahead of their use: loads come back in order, so a
    // wait for these is one for the operands of slabs to come; bf16 out, 12608 x 1024 x 4096 in 8 groups 65 us.)
    constexpr bool MX4 = DT == DT_MX4;
    constexpr int SCALE_LOADS = MX4 ? 2 : 0;
    [[maybe_unused]] uint32_t sa[2][MX4 ? MI : 1], sb[2][MX4 ? NI : 1];
    [[maybe_unused]] int sa_off, sb_off, sa_end, sb_end;
    [[maybe_unused]] __amdgpu_buffer_rsrc_t sa_src, sb_src;
    typedef const __attribute__((address_space(3))) uint32_t *lds_word;
    constexpr int SCALES_AT = fast_ring_bytes<DT, MODE>();
    auto scale_load = [&](int s) __attribute__((always_inline)) {
        if constexpr (MX4) {
            const lds_ptr dst = lds + (SCALES_AT + (s & 1) * FAST_SCALES + wave * 256);
            // (past the last slab at the descriptor's end, not behind it: an offset is held against what the end leaves of that)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(sa_src, (lds_void)dst, 4, sa_off, s < nslab ? s * 8 : sa_end, 0, 0);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(sb_src, (lds_void)(dst + FAST_SCALES / 2), 4, sb_off, s < nslab ? s * 8 : sb_end, 0, 0);
        }
    };
    auto scale_read = [&](auto h_c, int s) __attribute__((always_inline)) {
        if constexpr (MX4) {
            constexpr int h = decltype(h_c)::value;
            const lds_ptr at = lds + (SCALES_AT + (s & 1) * FAST_SCALES + l32 * 8);
#pragma unroll
            for (int mi = 0; mi < MI; ++mi) sa[h][mi] = *(lds_word)(at + wm * TM * 8 + (mi * 32 * 8 + 4 * h));
#pragma unroll
            for (int ni = 0; ni < NI; ++ni) sb[h][ni] = *(lds_word)(at + wn * TN * 8 + (FAST_SCALES / 2 + ni * 32 * 8 + 4 * h));
        }
    };
    // ahead of steps 0 and 2
    auto scale_turn = [&](auto t_c) __attribute__((always_inline)) {
        constexpr int t = decltype(t_c)::value, h = t >> 1;
        if constexpr (MX4 && (t & 1) == 0) {
#pragma unroll
            for (int mi = 0; mi < MI; ++mi) sa[h][mi] >>= 8 * lh;
#pragma unroll
            for (int ni = 0; ni < NI; ++ni) sb[h][ni] >>= 8 * lh;
        }
    };
    if constexpr (MX4) {
        const auto rows = source.scale_rows(m0, n0);
        // (rows past the end bring zeros)
        sa_end = min(M - m0, BM) * rows.lda;
        sb_end = min(N - n0, 256) * rows.ldb;
        sa_src = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(rows.a), 0, sa_end, RSRC_FLAGS);
        sb_src = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(rows.b), 0, sb_end, RSRC_FLAGS);
        sa_off = (wave * 32 + (lane >> 1)) * rows.lda + 4 * (lane & 1);
        sb_off = (wave * 32 + (lane >> 1)) * rows.ldb + 4 * (lane & 1);
    }
    // ---- main loop, software-pipelined by hand.  A slab is four MFMA steps of 32 bytes of K.
    // The fragments of step t+1 are read from LDS while the MFMAs of step t run (two register
    // sets).  The barrier sits between steps 2 and 3: by then every wave has
    // read its step-3 fragments, so nobody reads this slab's buffers any more.  From there on, over the four steps up to the
    // next slab's barrier, the loads into those buffers are issued: the units with two buffers of slab s + 2, then those with
    // three of slab s + 3.
    i32x4 fa[2][MI], fb[2][NI];
    // a lane's place in a unit of A at step 0 (row l32 of this wave's half); at step t chunk 2 t + lh, so bits 5 and 6 change
    const int frag_at = wm * 32 * SLAB_BYTES + l32 * SLAB_BYTES + (lh ^ ((lane >> 1) & 7)) * 16;
    const int b_from_a = (wn - wm) * 32 * SLAB_BYTES; // the same in a unit of B, from unit h = 0 on
    // fragment j of step t: of B, then of A
    auto fragment = [&](auto j_c, auto t_c, Buf b) __attribute__((always_inline)) {
        constexpr int j = decltype(j_c)::value, t = decltype(t_c)::value, set = t & 1;
        constexpr bool isb = j < NI;
        if constexpr (isb ? BT : AT) return;
        constexpr int q = isb ? L::load_of_b(isb ? j : 0) : L::load_of_a(isb ? 0 : j - NI);
        const int base = (L::ring3(q) ? b.f : b.r) + (isb ? b_from_a : 0);
        const i32x4 v = *(lds_frag)(lds + ((frag_at ^ (32 * t)) + base) + L::at(q));
        if constexpr (isb) fb[set][isb ? j : 0] = v;
        else fa[set][isb ? 0 : j - NI] = v;
    };
    // The fragments of step t of operands that lie as rows of k: sixteen lanes read 4 rows of sixteen elements, each gets one's.  A unit is one wave row's (of A: of
    // 256, half of one's) or wave column's; bit 6 of the place tells its two blocks apart.  All reads and their wait are one block: the
    // compiler puts a wait for every outstanding load in front of the built-in.
    typedef int i32x2 __attribute__((ext_vector_type(2)));
    const int i16 = lane & 15, turn_at = (8 * lh + (i16 >> 2)) * SLAB_BYTES + (((2 * ((lane >> 4) & 1) + ((i16 & 3) >> 1)) ^ kn_swizzle<2, 128>(i16 >> 2)) * 16) + (i16 & 1) * 8;
    auto turned = [&](auto t_c, Buf b) __attribute__((always_inline)) {
        constexpr int t = decltype(t_c)::value, set = t & 1, HALF = 4 * SLAB_BYTES, STEP = 16 * SLAB_BYTES * t;
        [[maybe_unused]] const uint32_t base = (uint32_t)(uintptr_t)lds + turn_at;
        auto put = [&](i32x4 &f, const i32x2 &x, const i32x2 &y) __attribute__((always_inline)) { f = i32x4{x[0], x[1], y[0], y[1]}; };
        const uint32_t pb = base + (L::ring3(L::load_of_b(0)) ? b.f : b.r) + L::at(L::load_of_b(0)) + wn * L::UNIT;
        const uint32_t pa = base + (L::ring3(L::load_of_a(0)) ? b.f : b.r) + L::at(L::load_of_a(0)) + wm * (MI / 2) * L::UNIT;
#define FAST_TURN(O, P) "ds_read_b64_tr_b16 %" O ", %" P
        if constexpr (AT && MI == 4) {
            i32x2 h[12];
            asm volatile(FAST_TURN("0", "12") " offset:%18\n\t" FAST_TURN("1", "12") " offset:%19\n\t" FAST_TURN("2", "13") " offset:%18\n\t" FAST_TURN("3", "13") " offset:%19\n\t"
                         FAST_TURN("4", "14") " offset:%18\n\t" FAST_TURN("5", "14") " offset:%19\n\t" FAST_TURN("6", "15") " offset:%18\n\t" FAST_TURN("7", "15") " offset:%19\n\t"
                         FAST_TURN("8", "16") " offset:%18\n\t" FAST_TURN("9", "16") " offset:%19\n\t" FAST_TURN("10", "17") " offset:%18\n\t" FAST_TURN("11", "17") " offset:%19\n\t"
                         "s_waitcnt lgkmcnt(0)"
                         : "=&v"(h[0]), "=&v"(h[1]), "=&v"(h[2]), "=&v"(h[3]), "=&v"(h[4]), "=&v"(h[5]), "=&v"(h[6]), "=&v"(h[7]), "=&v"(h[8]), "=&v"(h[9]), "=&v"(h[10]),
                           "=&v"(h[11])
                         : "v"(pb), "v"(pb ^ 64u), "v"(pa), "v"(pa ^ 64u), "v"(pa + L::UNIT), "v"((pa ^ 64u) + L::UNIT), "n"(STEP), "n"(STEP + HALF) : "memory");
            put(fb[set][0], h[0], h[1]);
            put(fb[set][1], h[2], h[3]);
#pragma unroll
            for (int i = 0; i < 4; ++i) put(fa[set][i], h[4 + 2 * i], h[5 + 2 * i]);
        } else if constexpr (AT) {
            static_assert(MI == 2);
            i32x2 h[8];
            asm volatile(FAST_TURN("0", "8") " offset:%12\n\t" FAST_TURN("1", "8") " offset:%13\n\t" FAST_TURN("2", "9") " offset:%12\n\t" FAST_TURN("3", "9") " offset:%13\n\t"
                         FAST_TURN("4", "10") " offset:%12\n\t" FAST_TURN("5", "10") " offset:%13\n\t" FAST_TURN("6", "11") " offset:%12\n\t" FAST_TURN("7", "11") " offset:%13\n\t"
                         "s_waitcnt lgkmcnt(0)"
                         : "=&v"(h[0]), "=&v"(h[1]), "=&v"(h[2]), "=&v"(h[3]), "=&v"(h[4]), "=&v"(h[5]), "=&v"(h[6]), "=&v"(h[7])
                         : "v"(pb), "v"(pb ^ 64u), "v"(pa), "v"(pa ^ 64u), "n"(STEP), "n"(STEP + HALF) : "memory");
            put(fb[set][0], h[0], h[1]);
            put(fb[set][1], h[2], h[3]);
            put(fa[set][0], h[4], h[5]);
            put(fa[set][1], h[6], h[7]);
        } else {
            i32x2 h[4];
            asm volatile(FAST_TURN("0", "4") " offset:%6\n\t" FAST_TURN("1", "4") " offset:%7\n\t" FAST_TURN("2", "5") " offset:%6\n\t" FAST_TURN("3", "5") " offset:%7\n\t"
                         "s_waitcnt lgkmcnt(0)"
                         : "=&v"(h[0]), "=&v"(h[1]), "=&v"(h[2]), "=&v"(h[3]) : "v"(pb), "v"(pb ^ 64u), "n"(STEP), "n"(STEP + HALF) : "memory");
            put(fb[set][0], h[0], h[1]);
            put(fb[set][1], h[2], h[3]);
        }
#undef FAST_TURN
    };
    // MFMA j of step t (set t & 1)
    auto mfma = [&](auto first_c, auto t_c, auto j_c) __attribute__((always_inline)) {
        constexpr int set = decltype(t_c)::value & 1, mi = decltype(j_c)::value / NI, ni = decltype(j_c)::value % NI;
        if constexpr (MX4) {
            constexpr int t = decltype(t_c)::value;
            acc[mi][ni] = mfma_mx4<2 * (t & 1)>(fb[set][ni], fa[set][mi], decltype(first_c)::value ? zerov : acc[mi][ni], sb[t >> 1][ni], sa[t >> 1][mi]);
        } else {
            acc[mi][ni] = T::mfma(fb[set][ni], fa[set][mi], decltype(first_c)::value ? zerov : acc[mi][ni]);
        }
    };
    // Protected tiles reduce the slabs of A they own (slab s belongs to tile column s mod
    // tiles_n) while those are resident: see gemm_apass.h.
    constexpr int AUX_OFF = fast_lds_bytes<DT, MODE>();    // behind the buffers of the larger tile
    static_assert(epi_total_bytes(BM, 256) <= AUX_OFF, "the epilogue reads the column sums there while it fills the LDS ahead of them");
    EpiProt<DT, MI> ep;
    ep.slab0 = tn; ep.slab_step = g.tiles_n; ep.owned = (OWN && tn < nslab) ? (nslab - tn + g.tiles_n - 1) / g.tiles_n : 0;
    ep.col_lds = reinterpret_cast<uint32_t *>(smem + AUX_OFF);
    ep.back = 1.f;
    {
        int next_own = tn, own_at = 0;                 // the next slab to reduce, and its place among the owned
        // column sums, [owned][KE]; terms of b, [2][3][KE]; zeros; words of b, [2][KE]
        constexpr int TERM = SLAB_BYTES, TERMS = 3 * TERM;
        uint8_t *const terms = smem + AUX_OFF + ep.owned * KE * 4;
        uint32_t *const words = reinterpret_cast<uint32_t *>(terms + 2 * TERMS + TERM);
        // b of the j-th owned slab, straight into LDS, two owned slabs ahead.  (A register would be waited for together
        // with every operand load behind it.)
        auto fetch_b = [&](int j) __attribute__((always_inline)) {
            if (wave < KE / 64 && j < ep.owned)
                __builtin_amdgcn_global_load_lds((gas_ptr)(g.b_sum + (long)bz * K + (tn + j * g.tiles_n) * KE + 64 * wave + lane),
                                                 (las_ptr)(words + (j & 1) * KE + 64 * wave), 4, 0, 0);
        };
        if constexpr (OWN) {
            fetch_b(0);
            fetch_b(1);
#pragma unroll
            for (int mi = 0; mi < MI; ++mi) ep.pass.dot[mi] = acc4_zero<DT>();
            ep.pass.amax = 0u;
            for (int i = tid; i < ep.owned * KE + SLAB_BYTES / 4; i += 64 * FAST_WAVES)
                reinterpret_cast<uint32_t *>(smem + AUX_OFF)[i < ep.owned * KE ? i : i + 2 * TERMS / 4] = 0u;
        }
        // buffers of slabs s, s + 1, s + 2 (three-buffer units; two-buffer units of s + 2: those of s)
        int f0 = 0, f1 = L::F_BYTES, f2 = 2 * L::F_BYTES, r0 = 3 * L::F_BYTES, r1 = r0 + L::R_BYTES;
        auto next = [&]() __attribute__((always_inline)) {
            const int f = f0, r = r0;
            f0 = f1; f1 = f2; f2 = f;
            r0 = r1; r1 = r;
        };
        scale_load(0);
        static_for<0, NLD>([&](auto q_c) { load(q_c, 0, Buf{f0, r0}); });
        scale_load(1);
        static_for<0, NLD>([&](auto q_c) { load(q_c, 1, Buf{f1, r1}); });
        // Start as soon as slab 0 is in place: loads complete in order, so "at most the loads of the
        // slab behind it outstanding" means everything issued before them has landed.
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" :: "n"(NLD + SCALE_LOADS) : "memory");
        scale_read(std::integral_constant<int, 0>{}, 0);
        static_for<0, NFR>([&](auto j_c) { fragment(j_c, std::integral_constant<int, 0>{}, Buf{f0, r0}); });
        if constexpr (AT || BT) turned(std::integral_constant<int, 0>{}, Buf{f0, r0});
        // The barrier of slab s: slab s + 1 is in place; what was requested after it are the units with three buffers of
        // slab s + 2 (or nothing any more).
        auto slab_barrier = [&](auto behind_c) __attribute__((always_inline)) {
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" :: "n"(decltype(behind_c)::value ? NF : 0) : "memory");
        };
        // b of the next slab to reduce in terms of the operand type, a slab ahead of it
        float scale = 1.f;
        if constexpr (OWN && DT == DT_F16) b_scale(N, &scale, &ep.back);
        auto put_terms = [&]() __attribute__((always_inline)) {
            if (wave < KE / 64) {
                typename T::acc_t v = from_word<typename T::acc_t>(words[(own_at & 1) * KE + 64 * wave + lane]);
                if constexpr (DT == DT_F16) v *= scale;
                uint8_t *d = terms + (own_at & 1) * TERMS + (64 * wave + lane) * ES;
#pragma unroll
                for (int e = 0; e < 3; ++e) {
                    const uint32_t h = b_term<DT>(v);
                    if constexpr (ES == 1) d[e * TERM] = (uint8_t)h;
                    else *reinterpret_cast<uint16_t *>(d + e * TERM) = (uint16_t)h;
                }
            }
        };
        if (OWN && tn == 0) {
            put_terms();
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        }
        auto own_ahead = [&](int s) __attribute__((always_inline)) {
            if (OWN && s + 1 == next_own) put_terms();
        };
        auto own_done = [&](int s) __attribute__((always_inline)) {
            if (OWN && s == next_own) {
                next_own += g.tiles_n;
                own_at += 1;
                fetch_b(own_at + 1);
            }
        };
        // The pass over a slab this tile owns, ahead of its MFMAs: a wave takes the fragments of step wn once more, of its rows, two at a
        // time: some ninety instructions, beside which the SIMD's other wave multiplies.  (Dealt out in pieces behind the MFMAs of the slab's
        // first three steps it is no faster: pieces / so, us, bf16 12608 x 768 x 3072 72.7 / 72.2, 20000 x 768 x 2048 66.8 / 65.8, f16 12608 x 768 x
        // 768 30.5 / 30.0, int8 36928 x 1024 x 4096 163.5 / 163.0; 72 problems, 1.006 of the time in pieces.)
        auto reduce = [&](int s) __attribute__((always_inline)) {
            if constexpr (OWN) {
                if (s != next_own) return;
                constexpr int NU = T::IS_INT ? 2 : 1;
                // lane: column c = lane & 15 of the product belongs to the rows of half c >> 2, and to term c & 3
                const int ln = tile_thread_index() & 63, c = ln & 15, term = (c >> 2) == ((ln >> 4) & 1) ? c & 3 : 3;  // (formed here, not kept across the tile)
                const uint8_t *src = terms + (term < 3 ? (own_at & 1) * TERMS + term * TERM : 2 * TERMS);
                const i32x4 b = *reinterpret_cast<const i32x4 *>(src + wn * 32 + (ln >> 5) * 16);
                const i32x4 id0 = turn_operand<DT>(ln, 0), id1 = T::IS_INT ? turn_operand<DT>(ln, 1) : id0;
                typename Acc4<DT>::type sums[NU];
                static_for<0, MI / 2>([&](auto h_c) {
                    constexpr int h = decltype(h_c)::value;
                    i32x4 x[2];
                    TurnSums<DT> ts;
                    static_for<0, 2>([&](auto i_c) {
                        constexpr int i = decltype(i_c)::value, q = L::load_of_a(2 * h + i);
                        x[i] = *(lds_frag)(lds + ((frag_at ^ (32 * wn)) + (L::ring3(q) ? f0 : r0)) + L::at(q));
                        // rows past the end hold the last one's elements
                        if (wm * TM + (2 * h + i) * 32 + l32 >= a_rows) x[i] = i32x4{0, 0, 0, 0};
                    });
                    pass_mfmas<DT>(ep.pass.dot[2 * h], ep.pass.dot[2 * h + 1], ts, x, b, id0, id1);
                    if constexpr (!T::IS_INT) {
                        typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
                        u16x2 m = __builtin_bit_cast(u16x2, ep.pass.amax);
#pragma unroll
                        for (int i = 0; i < 8; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, x[i >> 2][i & 3] & 0x7FFF7FFF));
                        ep.pass.amax = __builtin_bit_cast(uint32_t, m);
                        ts.c[0] += ts.c[1];
                    }
#pragma unroll
                    for (int u = 0; u < NU; ++u) sums[u] = h == 0 ? ts.c[u] : sums[u] + ts.c[u];
                });
#pragma unroll
                for (int u = 0; u < NU; ++u) {
                    typename T::acc_t v = add_t(add_t((typename T::acc_t)sums[u][0], (typename T::acc_t)sums[u][1]),
                                                add_t((typename T::acc_t)sums[u][2], (typename T::acc_t)sums[u][3]));
                    v = add_xor32(add_xor16(v));
                    if (ln < 16) lds_add_word(const_cast<uint32_t *>(ep.col_lds) + own_at * KE + wn * (KE / 4) + 16 * u + ln, v);
                }
            }
        };
        // A slab with loads between its MFMAs, in explicit program order (one group per MFMA, fenced): left
        // alone, the compiler issues all loads in one burst and the matrix pipe waits for them.  first_c: the first slab; all
        // of slab 1 has been requested ahead of it.
        auto slab = [&](auto first_c, int s) __attribute__((always_inline)) {
            constexpr bool FIRST = decltype(first_c)::value;
            if constexpr (FIRST) reduce(s);
            own_ahead(s);
            static_for<0, 4>([&](auto t_c) {
                constexpr int t = decltype(t_c)::value;
                // this step's loads: step 3 begins with those into this slab's buffers, steps 0 to 2 go on with those into the last one's
                constexpr int at = t == 3 ? 0 : t + 1;
                constexpr int q0 = FIRST && t < 3 ? NR + NF * t / 3 : L::by_step(at), q1 = FIRST && t < 3 ? NR + NF * (t + 1) / 3 : L::by_step(at + 1);
                constexpr int RPM = NMF >= NFR ? 1 : 2;                // fragment reads behind an MFMA
                scale_turn(t_c);
                if constexpr (t == 0) scale_read(std::integral_constant<int, 1>{}, s);
                if constexpr (t == 3) {
                    scale_load(s + 2);
                    scale_read(std::integral_constant<int, 0>{}, s + 1);
                }
                __builtin_amdgcn_sched_barrier(0);
                static_for<0, NMF>([&](auto j_c) {
                    constexpr int j = decltype(j_c)::value;
                    mfma(std::integral_constant<bool, FIRST && t == 0>{}, t_c, j_c);
                    static_for<(j * RPM < NFR ? j * RPM : NFR), (j * RPM + RPM < NFR ? j * RPM + RPM : NFR)>([&](auto r_c) {
                        fragment(r_c, std::integral_constant<int, (t + 1) & 3>{}, t < 3 ? Buf{f0, r0} : Buf{f1, r1});
                    });
                    static_for<q0 + (q1 - q0) * j / NMF, q0 + (q1 - q0) * (j + 1) / NMF>([&](auto q_c) {
                        constexpr int q = decltype(q_c)::value;
                        int to = s + (t == 3 ? 1 : 0) + (q < NR ? 1 : 2);
                        if (FIRST && t == 3 && q >= NR) to = to < nslab ? to : nslab - 1;      // of three slabs: bytes nobody reads
                        load(q_c, to, t == 3 ? Buf{f0, r0} : Buf{f2, r1});
                    });
                    if constexpr ((AT || BT) && j == NMF - 1) turned(std::integral_constant<int, (t + 1) & 3>{}, t < 3 ? Buf{f0, r0} : Buf{f1, r1});
                    __builtin_amdgcn_sched_barrier(0);
                });
                if constexpr (t == 2) slab_barrier(std::true_type{});
            });
            own_done(s);
            next();
        };
        // One of the last slabs: the loads that are still to come in groups ahead of a step's MFMAs.
        auto tail_slab = [&](int s) __attribute__((always_inline)) {
            reduce(s);
            own_ahead(s);
            static_for<0, 4>([&](auto t_c) {
                constexpr int t = decltype(t_c)::value;
                constexpr int at = t == 3 ? 0 : t + 1;
                constexpr int q0 = L::by_step(at), q1 = L::by_step(at + 1), qr = q1 < NR ? q1 : NR < q0 ? q0 : NR;
                const int ahead = s + (t == 3 ? 1 : 0);
                if (q0 < qr && ahead + 1 < nslab) static_for<q0, qr>([&](auto q_c) { load(q_c, ahead + 1, Buf{f0, t == 3 ? r0 : r1}); });
                if (qr < q1 && ahead + 2 < nslab) static_for<qr, q1>([&](auto q_c) { load(q_c, ahead + 2, Buf{t == 3 ? f0 : f2, r0}); });
                __builtin_amdgcn_sched_barrier(0);
                static_for<0, NMF>([&](auto j_c) {
                    constexpr int j = decltype(j_c)::value;
                    constexpr int RPM = NMF >= NFR ? 1 : 2;
                    mfma(std::false_type{}, t_c, j_c);
                    // after the last slab: read and never used
                    static_for<(j * RPM < NFR ? j * RPM : NFR), (j * RPM + RPM < NFR ? j * RPM + RPM : NFR)>([&](auto r_c) {
                        fragment(r_c, std::integral_constant<int, (t + 1) & 3>{}, t < 3 ? Buf{f0, r0} : Buf{f1, r1});
                    });
                    if constexpr ((AT || BT) && j == NMF - 1) turned(std::integral_constant<int, (t + 1) & 3>{}, t < 3 ? Buf{f0, r0} : Buf{f1, r1});
                    __builtin_amdgcn_sched_barrier(0);
                });
                if constexpr (t == 2) {
                    if (s + 2 < nslab) slab_barrier(std::true_type{});
                    else slab_barrier(std::false_type{});
                }
            });
            own_done(s);
            next();
        };
        slab(std::true_type{}, 0);
        int s = 1;
        // the middle slabs: runs of slabs that are not this workgroup's, each followed by one that is
        const int mid_end = nslab - 3;
        if constexpr (OWN) {
            while (next_own < mid_end) {                   // next_own >= s here
                for (; s < next_own; ++s) slab(std::false_type{}, s);
                reduce(s);
                slab(std::false_type{}, s);
                ++s;
            }
        }
        if constexpr (MX4) {
            // All alike: a branch around loads lets the compiler move MFMAs with scales, which it does not hold to their block, behind it, and a slab's fragments with them.
            for (; s < nslab; ++s) slab(std::false_type{}, s);
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        } else {
            for (; s < mid_end; ++s) slab(std::false_type{}, s);
            for (; s < nslab; ++s) tail_slab(s);
        }
    }
    __syncthreads();
    gemm_epilogue<DT, OT, BM, PROT, STO>(g, source, acc, smem, m0, n0, bz, ep, sc);
}

}  // namespace abft
