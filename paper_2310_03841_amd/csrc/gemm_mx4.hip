// Products over groups of rows of 4-bit operands: tiles by four waves, and which kernel a call takes.
#include "gemm_group.h"
#include "gemm_mx4.h"

namespace abft {

template <int OT> static hipError_t launch_of(int tiles, bool protect, Mx4Args &g, hipStream_t st)
{
    if (tiles == TILE_64) return protect ? launch_one<DT_MX4, OT, 64, 64, 3, true, GROUP_ROWS, true>(g, st) : launch_one<DT_MX4, OT, 64, 64, 3, false, GROUP_ROWS, true>(g, st);
    return protect ? launch_one<DT_MX4, OT, 64, 128, 3, true, GROUP_ROWS, true>(g, st) : launch_one<DT_MX4, OT, 64, 128, 3, false, GROUP_ROWS, true>(g, st);
}

hipError_t launch_mx4(const GroupKernel &k, int ot, bool protect, Mx4Args &g, const uint32_t *b_max, float tau_k, float tau_cols, hipStream_t st)
{
    if (k.kind == GROUP_KERNEL_FEW) return launch_mx4_few(ot, protect, g, b_max, tau_k, tau_cols, st);
    if (k.kind == GROUP_KERNEL_BIG) {
        g.cc_acc = g.rc_acc = nullptr;                           // these tiles add to the sums themselves
        return launch_mx4_big(ot, protect, g, st);
    }
    return ot == DT_BF16 ? launch_of<DT_BF16>(k.tiles, protect, g, st) : launch_of<DT_F16>(k.tiles, protect, g, st);
}

// ---- The kernel of a problem is the one of the least estimated time, of groups of average rows, as for other types (gemm_group.hip); us.  Against the best of the kernels, each
// forced, it takes on average 1.02 (320 random problems, 1 to 64 groups, sizes 64 to 4096, uneven rows; the worst 1.5).  Both sides (tiles of 64 x 64 / of 64 x 128 / of the fast
// kernel / few rows): 12608 x 4096 x 1024 in 16 groups 104.7 / 96.3 / 48.9 / -; 12608 x 1024 x 4096 in 8 78.0 / 74.5 / 34.2 / -; 2304 x 704 x 1280 7.5 / 6.6 / 9.3 / -; 64 x 1730 x 3200
// 8.1 / 9.6 / 17.4 / 6.2; protected 64 x 4012 x 768 in 26 28.4 / 29.2 / 32.9 / 22.0; 4608 x 2816 x 768 34.6 / 33.4 / 22.6 / -.
struct Mx4Problem { long rows, N, groups; int slabs; double row; bool protect; };      // row: bytes of one of A or B

static double mx4_tile_us(const Mx4Problem &p, int bn)
{
    const bool wide = bn == 128;
    const double slab = wide ? 0.505 : 0.27, alone = wide ? 0.505 : 0.33, end = (wide ? 0.73 : 0.62) * (p.protect ? 1.8 : 1.0), matrices = p.groups * p.N * p.row;
    const long n = ceil_div(ceil_div(p.rows, 64) * ceil_div(p.N, bn) * p.groups, 256);
    return (wide ? 3.6 : 4.0) + std::max(n > 1 ? n * (p.slabs * slab + end) : p.slabs * alone + end, matrices / 5e6) + (p.protect ? (wide ? 5.7 : 5.3) + matrices / 5e6 : 0.0);
}
static double mx4_big_us(const Mx4Problem &p)
{
    const long over = p.rows & 255, tall = ((p.rows >> 8) + (over > 128)) * ceil_div(p.N, 256) * p.groups, small = ((over + 127) >> 7 & 1) * ceil_div(p.N, 256) * p.groups;
    const double rounds = ((double)tall + (p.protect ? 0.66 : 0.57) * small) / 256, least = tall ? 1.0 : 0.9;
    const double n = rounds < least ? least : rounds + 1.6;
    return 0.8 + n * ((p.protect ? 9.2 : 4.3) + (p.N % 64 ? 20.0 / ceil_div(p.N, 256) : 0.0) + 0.77 * p.slabs) + (p.protect ? 2.1 + p.groups * p.N * p.row / 5e6 : 0.0);
}
static double mx4_few_us(const Mx4Problem &p)
{
    const double tiles = p.groups * (ceil_div(p.rows, 16) + (p.groups > 1 && p.rows > 4 ? 0.3 : 0.0)) * ceil_div(p.N, 32);
    return 5.1 + (p.protect ? 5.2 + 1e-3 * tiles : 0.0) + std::max(tiles * 48 * p.row / 14.6e6, p.groups * p.N * p.row / 15.2e6);
}

void mx4_tile_shape(bool protect, const GroupKernel &k, const Mx4Args &g, int *rows, int *columns)
{
    *rows = k.kind == GROUP_KERNEL_BIG ? 256 : k.kind == GROUP_KERNEL_FEW ? 16 : 64;
    *columns = k.kind == GROUP_KERNEL_BIG ? 256 : k.kind == GROUP_KERNEL_FEW ? mx4_few_columns(protect, g) : k.tiles == TILE_64_128 ? 128 : 64;
}

bool mx4_plan(bool protect, Mx4Args &g, GroupKernel *k)
{
    long n_pass = 0;
    if (protect) {
        g.pass_win = (int)ceil_div(g.K, PASS_BYTES);
        g.pass_inv = map_inverse(g.pass_win);
        // at most 64 items to a group of average size, of up to 512 rows (7155 x 334 x 768, one group, protected: items of 32 rows 19.4 us, so 15.2)
        g.pass_log2 = 0;
        while (g.pass_log2 < 4 && ceil_div(g.M, g.groups) > 64L * 4 * PASS_ROWS << g.pass_log2) ++g.pass_log2;
        n_pass = ceil_div(row_tiles(g.M, g.groups, 4 * PASS_ROWS << g.pass_log2) * g.pass_win, 8) * 8;
        if (n_pass > MAX_GRID_X) return false;
        g.n_pass = (int)n_pass;
    }
    const Mx4Problem p = {ceil_div(g.M, g.groups), g.N, g.groups, (int)ceil_div(g.K, SLAB_BYTES), g.K * (1.0 + 1.0 / 16), protect};
    *k = {GROUP_KERNEL_TILE, TILE_64};
    double us = mx4_tile_us(p, 64);
    if (mx4_tile_us(p, 128) < us) { k->tiles = TILE_64_128; us = mx4_tile_us(p, 128); }
    // whole slabs, three at least; 32-bit offsets inside a tile
    constexpr long ROW = 1L << 22;
    if (g.K % SLAB_BYTES == 0 && g.K >= 3 * SLAB_BYTES && g.groups <= 256 && g.lda < ROW && g.ldb < ROW && g.ld_sa < ROW && g.ld_sb < ROW && 1.1 * mx4_big_us(p) < us) {
        k->kind = GROUP_KERNEL_BIG;
        us = 1.1 * mx4_big_us(p);
    }
    if (mx4_few_fits(protect, g) && mx4_few_us(p) < us) k->kind = GROUP_KERNEL_FEW;
    if (k->kind == GROUP_KERNEL_BIG) return row_tiles(g.M, g.groups, 128) * ceil_div(g.N, 256) < 1L << 31;      // (a list that its workgroups walk)
    int rows, columns;
    mx4_tile_shape(protect, *k, g, &rows, &columns);
    const long wgs = k->kind == GROUP_KERNEL_FEW ? mx4_few_workgroups(protect, g) : ceil_div(row_tiles(g.M, g.groups, rows) * ceil_div(g.N, columns), 8) * 8;
    return n_pass + wgs <= MAX_GRID_X;
}

}  // namespace abft
