// Fast path of the protected GEMM for gfx950: B stored N x K (both operands K-contiguous) and
// K a whole number (at least three) of 128-byte slabs.  The data movement:
//   * global -> LDS with buffer loads that go straight there (buffer_load_dwordx4 ... lds): no VGPR staging.  One
//     wave instruction fills 8 LDS rows of 128 bytes; the XOR swizzle of the LDS layout is
//     applied by choosing which global 16-byte chunk each lane fetches.
//   * 256 x 256 tiles by eight waves of 128 x 64 (eight 32x32 MFMA blocks per wave), 128 x 256 tiles by eight of 64 x 64;
//     one barrier per slab, loads spread evenly between the MFMAs.
//   * two waves per SIMD: what one wave spends on issuing loads, fragment reads and the epilogue's vector instructions, the other
//     fills with MFMAs.  With one (four waves of 128 x 128, the LDS traffic of a slab 192 instead of 256 KB) every instruction
//     beside an MFMA costs five clocks of the only wave there is.  What bounded that loop was not LDS bandwidth, which a
//     micro-benchmark puts at 256 bytes per clock for 16-byte fragment reads (64 KB of them per 32 KB loaded cost nothing), but issue:
//     the vector memory path takes a load of 1 KB every 18 clocks per compute unit, and all of a slab's loads in one of its four steps
//     held every wave there.  Four waves / eight, clocks per slab (MFMAs alone 2048 and 1024): 256 x 256
//     2388 / 2152, 128 x 256 1526 / 1130; epilogue of a 256 x 256 tile, unprotected 5500 / 3900, protected 12000 / 10200.
//     bf16, unprotected: 6304 x 768 x 768 11.9 -> 10.7 us, 6304 x 768 x 3072 40.9 -> 32.6, 12608 x 3072 x 768 57.9 -> 55.0, 4096 x 4096 x 4096
//     103 -> 100.  The large ones are power-limited: of the 11 % fewer clocks the chip takes back most by its clock (1.73 -> 1.56
//     GHz over 4096 x 4096 x 4096).
//   * MFMAs take the B fragment first, so a lane owns a row of C (see gemm_epilogue.h).
//   * workgroup -> tile mapping keeps the workgroups that share an XCD (and its L2) on a
//     compact group of tiles.
// Rows of the tile beyond the problem are fetched from a valid row instead of being
// zero-filled: a row of A only influences the same row of C, which is discarded, and the pass
// over A's slabs ignores them.
#include <mutex>
#include <queue>
#include <vector>

#include "abft_device.h"
#include "encode_pass.h"
#include "gemm_args.h"
#include "gemm_epilogue.h"
#include "gemm_fast_tile.h"

namespace abft {

// The grid mixes two tile shapes against wave quantisation: 256 x 256 tiles cover the first
// big_rows rows, 128 x 256 tiles the rest; how many of each is chosen by playing the dispatch
// through (choose_big_rows).  (600 big tiles on 256 CUs would be three rounds for 2.34 rounds
// of work.)
template <int DT, int MODE, int STO>
__global__ __launch_bounds__(64 * FAST_WAVES) void gemm_fast_kernel(GemmArgs whole)
{
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    constexpr bool PROT = MODE != FAST_PLAIN;
    fetch_args<GemmArgs>();
    // Persistent workgroups: one per compute unit, each walks the tile list with the grid's stride.
    // The 128-row tiles come first in the list: the compute units that start with one are half a
    // tile ahead of the others from then on, so the two groups store their tiles of C at different
    // times (a round of the machine that stores in step asks for tens of MB at once) and draw on
    // the matrix pipes at different times.  Measured on 12608 x 3072 x 768 (tiles by four waves): 63 -> 60.5 us.
    for (int t = blockIdx.x;;) {
        // (unprotected, there are scalars enough for all of a launch, and one trip to them is less)
        const GemmArgs &g = PROT ? kernel_args<GemmArgs>() : whole;
        if (PROT && t == 0 && threadIdx.x < 5) g.counts[threadIdx.x] = 0u;               // completed by the check kernel
        const int n_tile = MODE == FAST_BESIDE ? (int)gridDim.x - g.beside.n : (int)gridDim.x;
        if constexpr (MODE == FAST_BESIDE) {
            if ((int)blockIdx.x >= n_tile) {
                a_beside<DT>(g, (int)blockIdx.x - n_tile, smem);
                return;
            }
        }
        const int per_item = g.n_small + g.n_big;
        const int bz = t < per_item ? 0 : t / per_item, bid = t - bz * per_item;
        int tm, tn;
        if (STO != STO_128 && bid >= g.n_small) {
            map_tile(bid - g.n_small, g.n_big, g.tiles_m_big, g.tiles_n, g.group_inv, &tm, &tn);
            if constexpr (STO != STO_128) fast_tile<DT, DT, 256, MODE, STO, false, false>(g, LaunchSource{}, smem, tm * 256, tn * 256, bz, tn);
        } else {
            map_tile(bid, g.n_small, g.tiles_m_small, g.tiles_n, g.group_inv, &tm, &tn);
            fast_tile<DT, DT, 128, MODE, STO, false, false>(g, LaunchSource{}, smem, g.tiles_m_big * 256 + tm * 128, tn * 256, bz, tn);
        }
        t += n_tile;
        if (t >= per_item * g.batch) break;
        // the epilogue's last reads of LDS precede the next tile's first writes
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    }
}

// ------------------------------------------------------------------------------------------
// How many tile rows get 256-row tiles (the rest of M gets 128-row tiles).  Workgroups are
// dispatched in index order to whichever CU is free, one per CU; a 128 x 256 tile takes 0.57 of the time of a 256 x 256 tile
// (19.6 k of 34.6 k clocks at 12 slabs), protected 0.66 (29.7 k of 45 k): its prologue is the same.  A few candidate splits are
// played through with those two costs and the one that finishes first wins; the result is remembered per shape.  (The ratio falls
// with depth, to 0.54 and 0.57 at 60 slabs.  Costs by a problem's slabs and owned slabs were
// no better: 1.001 of the time over 120 random problems, single ones within 4 % either way.)
static double play_schedule(int big_rows, int M, int tiles_n, int batch, int ncu, double small)
{
    const int rest = M - big_rows * 256;
    const long nb = (long)big_rows * tiles_n, ns = (long)(rest > 0 ? (rest + 127) / 128 : 0) * tiles_n;
    std::priority_queue<double, std::vector<double>, std::greater<double>> cu;
    for (int i = 0; i < ncu; ++i) cu.push(0.0);
    double end = 0.0;
    for (int z = 0; z < batch; ++z)
        for (long t = 0; t < nb + ns; ++t) {
            const double f = cu.top() + (t < ns ? small : 1.0);     // dispatch order: the half-height tiles first
            cu.pop();
            cu.push(f);
            if (f > end) end = f;
        }
    return end;
}

static int choose_big_rows(int M, int tiles_n, int batch, int ncu, bool protect)
{
    struct Memo { int M, tiles_n, batch, ncu, protect, big_rows; };
    static Memo memo[16];
    static int memo_n = 0;
    static std::mutex memo_lock;                 // contexts may be driven from different host threads
    std::lock_guard<std::mutex> hold(memo_lock);
    for (int i = 0; i < memo_n; ++i)
        if (memo[i].M == M && memo[i].tiles_n == tiles_n && memo[i].batch == batch && memo[i].ncu == ncu && memo[i].protect == protect)
            return memo[i].big_rows;
    const double small = protect ? 0.66 : 0.57;
    const int rows_all_big = (M + 255) / 256;
    const long per_row = (long)tiles_n * batch;
    const long total_big = rows_all_big * per_row;
    int cand[4], nc = 0;
    cand[nc++] = rows_all_big;                                   // big tiles only
    cand[nc++] = 0;                                              // half-height tiles only
    long whole = (total_big / ncu) * ncu / per_row;              // whole rounds of big tiles
    if (whole > rows_all_big) whole = rows_all_big;
    cand[nc++] = (int)whole;
    const long fewer = whole - (ncu + per_row - 1) / per_row;    // one round fewer
    if (fewer > 0) cand[nc++] = (int)fewer;
    int best = cand[0];
    double best_t = play_schedule(cand[0], M, tiles_n, batch, ncu, small);
    for (int i = 1; i < nc; ++i) {
        const double t = play_schedule(cand[i], M, tiles_n, batch, ncu, small);
        if (t < best_t - 1e-9) { best_t = t; best = cand[i]; }
    }
    Memo m = {M, tiles_n, batch, ncu, protect, best};
    memo[memo_n < 16 ? memo_n++ : (M + tiles_n) & 15] = m;
    return best;
}

// Workgroups that reduce A on the `idle` compute units the tiles of a single round leave (a_beside).  Windows of 8
// to 64 chunks along K (least padding, then widest), the rows dealt to as few row blocks as end in 0.85 of the time that the
// tiles take: whatever reads A at once takes from the tiles' loads, and on every idle compute unit the pass cost more than it saved
// where those were many.  us, tiles that own slabs / a workgroup on every idle unit / so: bf16 3775 x 1280 x 1600 33.2 / 33.6 / 30.3, f16 1447 x
// 2752 x 2304 41.2 / 42.2 / 36.0, 8014 x 512 x 1344 31.0 / 33.8 / 28.3, 6304 x 768 x 3072 50.5 / 48.4 / 44.7; bf16 5664 x 768 x 3904 58.3 / 49.6 /
// 49.5, int8 4655 x 1664 x 2688 40.2 / 37.8 / 37.5.  210 random problems that the conditions below let in: 0.957 of the time with owned
// slabs (the worst 1.02, as far as two runs differ), 16-bit types 0.964 and int8 0.993 of that with all idle units.
// Times in us of a workgroup's pass (it reads 64 KB at a time) and of a tile beside one, with what the clock comes down to under load.
static double beside_us(int dt, long bytes) { return 4.0 + (double)bytes / (dt == DT_I8 ? 15e3 : 20e3); }
static double tile_us(bool big, int slabs) { return big ? 8.0 + 1.25 * slabs : 6.0 + 0.7 * slabs; }
static BesideArgs plan_beside(int dt, int M, int K, int batch, int slabs, int tiles_n, int idle, bool big)
{
    const BesideArgs none = {0, 0, 0, 0, 0};
    if (dt == DT_I8 ? slabs < 9 || slabs < tiles_n : slabs < 20 || slabs < 3 * tiles_n) return none;
    const EncPlan w = plan_window(M, K, 16 / elem_size(dt));
    const long per_row_block = (long)w.nwin * batch;
    if (per_row_block > idle) return none;
    BesideArgs b;
    b.cw_log2 = w.cw_log2; b.nwin = w.nwin;
    const int rl = (64 * FAST_WAVES >> w.cw_log2) * 8;                      // rows a workgroup takes at a time
    const double tiles_us = tile_us(big, slabs);
    const int most = (int)(idle / per_row_block);
    double us = 0.0;
    for (int n = 1; n <= most; ++n) {
        b.rpb = ((M + n - 1) / n + 15) / 16 * 16;
        if (b.rpb < rl) b.rpb = rl;
        us = beside_us(dt, (long)b.rpb * (16 << w.cw_log2));
        if (us <= 0.85 * tiles_us || b.rpb == rl) break;
    }
    b.nrb = (M + b.rpb - 1) / b.rpb;
    b.n = (int)(b.nrb * per_row_block);
    return us <= 1.2 * tiles_us ? b : none;
}

template <int DT, bool PROT, bool STO>
static hipError_t launch_fast_one(GemmArgs &g, int batch, hipStream_t st)
{
    constexpr int smem_max = 160 * 1024;
    const int slabs = g.K / (SLAB_BYTES / Traits<DT>::ES);
    hipError_t e;
    const int num_cu = device_cu_count(&e);
    if (e != hipSuccess) return e;
    g.tiles_n = (g.N + 255) / 256;
    g.group_inv = map_inverse(g.tiles_n);
    const int big_rows = choose_big_rows(g.M, g.tiles_n, batch, num_cu, PROT);
    g.tiles_m_big = big_rows;
    g.n_big = big_rows * g.tiles_n;
    const int rest = g.M - big_rows * 256;
    g.tiles_m_small = rest > 0 ? (rest + 127) / 128 : 0;
    g.tiles_m = g.tiles_m_big + g.tiles_m_small;
    g.n_small = g.tiles_m_small * g.tiles_n;
    g.batch = batch;
    const long total = (long)(g.n_big + g.n_small) * batch;
    if (total > 0x7FFFFFFFL) return hipErrorInvalidValue;
    dim3 grid((unsigned)(total < num_cu ? total : num_cu), 1, 1);
    g.beside.n = 0;
    if (PROT && total < num_cu) {
        g.beside = plan_beside(DT, g.M, g.K, batch, slabs, g.tiles_n, num_cu - (int)total, g.n_big != 0);
        grid.x += g.beside.n;
    }
    size_t smem;
    // Stored sums: the mix of tiles of any other call, and a kernel of its own where all have 128 rows (gemm_epilogue.h).  us, protected and
    // stored: all of 128 rows / mixed: bf16 12608 x 768 x 3072 103.4 / 81.7, 12608 x 3072 x 768 95.5 / 85.5, 6304 x 3072 x 768 62.0 / 55.0,
    // fp16 12212 x 3712 x 3904 381 / 344.
    constexpr int ALL = STO ? STO_256 : STO_NO, SMALL = STO ? STO_128 : STO_NO;
    auto kern = STO && !big_rows ? gemm_fast_kernel<DT, PROT ? FAST_OWN : FAST_PLAIN, SMALL> : gemm_fast_kernel<DT, PROT ? FAST_OWN : FAST_PLAIN, ALL>;
    if constexpr (PROT) {
        const size_t aux = fast_aux_bytes(DT, slabs, g.tiles_n);
        smem = fast_lds_bytes<FAST_OWN>() + aux;
        if (g.beside.n) {
            kern = STO && !big_rows ? gemm_fast_kernel<DT, FAST_BESIDE, SMALL> : gemm_fast_kernel<DT, FAST_BESIDE, ALL>;
            smem = fast_lds_bytes<FAST_BESIDE>();
        }
    } else {
        smem = fast_lds_bytes<FAST_PLAIN>();
    }
    if (smem > (size_t)smem_max) return hipErrorInvalidValue;
    e = ensure_max_lds(reinterpret_cast<const void *>(kern), smem_max);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kern, grid, dim3(64 * FAST_WAVES), smem, st, g);
    return hipGetLastError();
}

bool gemm_fast_eligible(int dt, int M, int N, int K, bool transB, long lda, long ldb)
{
    const int ke = SLAB_BYTES / elem_size(dt);
    // whole slabs, at least three of them (the main loop is peeled), and 32-bit row offsets
    // inside a tile
    // (int8: N < 65536 keeps |b| <= 128 N below 2^23, which the pass over A's slabs relies on here)
    return transB && (K % ke) == 0 && K >= 3 * ke && M >= 512 && N >= 512 && (dt != DT_I8 || N < 65536) &&
           lda * elem_size(dt) < (1L << 23) && ldb * elem_size(dt) < (1L << 23) &&
           // what the pass over A's slabs keeps per tile fits behind the operand buffers (protected or
           // not: a problem takes the same kernel in every mode)
           fast_lds_bytes<FAST_OWN>() + fast_aux_bytes(dt, K / ke, (N + 255) / 256) <= 160 * 1024;
}

void gemm_fast_tile(int *tm, int *tn) { *tm = 256; *tn = 256; }

template <int DT> static hipError_t launch_fast_type(bool protect, GemmArgs &g, int batch, hipStream_t st)
{
    if (!protect) return launch_fast_one<DT, false, false>(g, batch, st);
    if constexpr (!Traits<DT>::IS_INT)
        if (g.cc_sto) return launch_fast_one<DT, true, true>(g, batch, st);
    return launch_fast_one<DT, true, false>(g, batch, st);
}

hipError_t launch_gemm_fast(int dt, bool protect, GemmArgs &g, int batch, hipStream_t st)
{
    switch (dt) {
    case DT_I8:   return launch_fast_type<DT_I8>(protect, g, batch, st);
    case DT_BF16: return launch_fast_type<DT_BF16>(protect, g, batch, st);
    case DT_F16:  return launch_fast_type<DT_F16>(protect, g, batch, st);
    }
    return hipErrorInvalidValue;
}

}  // namespace abft
