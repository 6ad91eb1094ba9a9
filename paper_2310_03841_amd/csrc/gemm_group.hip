// Which kernel a product over groups of rows takes.
#include "gemm_group.h"
#include "gemm_group_big.h"

namespace abft {

// ---- The kernel of a problem is the one of the least estimated time, of groups of average rows (the host does not know them one by one).  us.
// Against the best of the kernels, each forced, it takes on average (random problems, 1 to 64 groups, sizes 64 to 4096, uneven rows): products 1.025 (89), those the
// fast kernel's tiles can do 1.036 (89), of up to 48 rows to a group 1.033 (89), gradients 1.044 (87); calls of 5 us, which the host bounds, among them.
// Both sides (tiles of 64 x 64 / of 64 x 128 / of the fast kernel / few rows): bf16 12608 x 1856 x 256 in 6 groups 37.1 / 33.7 / 22.3 / -; int8 888 x
// 208 x 3968 in 6, protected, 16.8 / 20.6 / 35.9 / -; bf16 86 x 320 x 608 in 2 5.5 / 6.9 / - / 4.6; int8 975 x 2816 x 576 in 39 18.5 / 18.5 / - / 26.9.
// All rows in one group of many take no longer than an even split (120 problems), but up to 4 times as long as a call that knows of the one group (int8 1024 rows
// in 64 groups, 4096 x 1024, protected: even 89.1, all in one 80.9, by few rows; the one known 20.6, by tiles).
struct GroupProblem { int rows, N, K, groups, es; bool protect, depth; };

static int slabs_of(const GroupProblem &p) { return (int)std::max(1L, ceil_div((long)p.K * p.es, SLAB_BYTES)); }

// Tiles by four waves: rounds of 256 compute units, each a slab at a time (alone on a compute unit a tile waits for its loads) and an end, where C is
// stored; or reading the matrices, if that is longer.  Protected, the end has sums, and the check kernel reads the matrices again.
static double tile_us(const GroupProblem &p, int tiles)
{
    const int bn = tiles == TILE_64_128 ? 128 : 64;
    const double slab = bn == 128 ? 0.30 : 0.22, alone = bn == 128 ? 0.39 : 0.25, end = (bn == 128 ? 1.6 : 0.8) * (p.protect ? 1.8 : 1.0);
    const long n = ceil_div(ceil_div(p.rows, 64) * ceil_div(p.N, bn) * p.groups, 256);
    const double matrices = p.depth ? 0.0 : (double)p.groups * p.N * p.K * p.es;
    return std::max(n > 1 ? n * (slabs_of(p) * slab + end) : slabs_of(p) * alone + end, matrices / 5e6) + (p.protect ? matrices / 6e6 : 0.0);
}

// Tiles of the fast kernel, one to a compute unit: a round for those of 256 rows, 0.57 of one (protected 0.66) for those of 128; the last round is half empty.
// Tiles that hang over the right edge inside a wave's 64 columns store element by element, 20 us more.
static double big_us(const GroupProblem &p)
{
    const double half = p.protect ? 0.66 : 0.57;
    const long tall = ((p.rows >> 8) + ((p.rows & 255) > 128)) * ceil_div(p.N, 256) * p.groups;
    const long small = ((((p.rows & 255) + 127) >> 7) & 1) * ceil_div(p.N, 256) * p.groups;
    const double rounds = ((double)tall + half * small) / 256;
    const double matrices = p.depth ? 0.0 : (double)p.groups * p.N * p.K * p.es;
    const double least = tall > 128 ? 1.0 : half, n = rounds < least ? least : rounds + 0.3;
    return n * ((p.protect ? 9.0 : 5.0) + (p.N % 64 ? 20.0 / ceil_div(p.N, 256) : 0.0) + 1.5 * std::max(3, slabs_of(p))) + (p.protect ? matrices / 6e6 : 0.0);
}

// Sixteen rows and 32 columns to a workgroup, which reads both over all of K: the L2 caches, or the matrices from memory, and its start and end.  Protected,
// the sums of its rows of A, and, floating point, the vector instructions of the columns' check: 3.2 TB/s of the matrices.
static double few_us(const GroupProblem &p)
{
    const double tiles = (double)p.groups * (ceil_div(p.rows, 16) + (p.groups > 1 && p.rows > 4 ? 0.3 : 0.0)) * ceil_div(p.N, 32), row = (double)p.K * p.es;
    const bool slow = p.protect && p.es == 2;
    const double read = std::max(tiles * 48 * row / 8e6, slow ? tiles * 32 * row / 3.2e6 : 0.0);
    return (slow ? 3.0 : p.protect ? 1.0 : 0.5) + tiles * (slow ? 1e-3 : 2e-3) + std::max(read, (double)p.groups * p.N * row / 5e6);
}

static GroupKernel group_kernel(int dt, bool transB, bool protect, const GroupArgs &g)
{
    const int es = elem_size(dt), ke = SLAB_BYTES / es;
    const GroupProblem p = {(int)ceil_div(g.M, g.groups), g.N, g.K, g.groups, es, protect, false};
    GroupKernel best = {GROUP_KERNEL_TILE, TILE_64};
    double us = tile_us(p, TILE_64);
    if (tile_us(p, TILE_64_128) < us) { best.tiles = TILE_64_128; us = tile_us(p, TILE_64_128); }
    else if (ceil_div(p.rows, 64) * ceil_div(p.N, 64) * p.groups <= 256) best.tiles = TILE_64_4;
    constexpr long ROW = 1L << 23, ALL = 1L << 31;               // 32-bit offsets: of a row inside a tile; of all rows of k
    if (g.K % ke == 0 && g.K >= 3 * ke && g.groups <= 256 && g.lda * es < ROW && (transB ? g.ldb * es < ROW : es == 2 && g.K * g.ldb * es < ALL) && big_us(p) < us) {
        best.kind = GROUP_KERNEL_BIG;
        us = big_us(p);
    }
    if (transB && group_few_fits(dt, protect, g) && few_us(p) < us) best.kind = GROUP_KERNEL_FEW;
    return best;
}

void group_tile_shape(const GroupKernel &k, const GroupArgs &g, int *rows, int *columns)
{
    *rows = k.kind == GROUP_KERNEL_BIG ? 256 : k.kind == GROUP_KERNEL_FEW ? 16 : 64;
    *columns = k.kind == GROUP_KERNEL_BIG ? 256 : k.kind == GROUP_KERNEL_FEW ? group_few_columns(g) : k.tiles == TILE_64_128 ? 128 : 64;
}

// Workgroups of a kernel's launch that take tiles (launch_one, launch_few_one), or tiles of the list that a launch of one to a compute unit walks; tall: rows of
// tiles by their height.
template <typename F> static bool tiles_fit(const GroupKernel &k, const GroupArgs &g, long n_pass, const F &tall)
{
    if (k.kind == GROUP_KERNEL_BIG) return tall(128) * ceil_div(g.N, 256) < 1L << 31;
    int rows, columns;
    group_tile_shape(k, g, &rows, &columns);
    const long wgs = k.kind == GROUP_KERNEL_FEW ? group_few_workgroups(g) : ceil_div(tall(rows) * ceil_div(g.N, columns), 8) * 8;
    return n_pass + wgs <= MAX_GRID_X;
}

bool group_plan(int dt, bool transB, bool protect, GroupArgs &g, GroupKernel *k)
{
    long n_pass = 0;
    if (protect) {
        g.pass_win = (int)ceil_div((long)g.K * elem_size(dt), PASS_BYTES);
        g.pass_inv = map_inverse(g.pass_win);
        n_pass = ceil_div(row_tiles(g.M, g.groups, 4 * PASS_ROWS) * g.pass_win, 8) * 8;
        if (n_pass > MAX_GRID_X) return false;
        g.n_pass = (int)n_pass;
    }
    *k = group_kernel(dt, transB, protect, g);
    return tiles_fit(*k, g, n_pass, [&](int bm) { return row_tiles(g.M, g.groups, bm); });
}

hipError_t launch_group(int dt, int ot, bool protect, bool transB, const GroupKernel &k, GroupArgs &g, const uint32_t *b_max, const Verdict *v, hipStream_t st)
{
    switch (k.kind) {
    case GROUP_KERNEL_FEW: {
        const float tau = !v ? 0.f : v->tau_override_cols > 0.f ? v->tau_override_cols : v->tau_override;
        return launch_group_few(dt, ot, protect, g, b_max, tau, st);
    }
    case GROUP_KERNEL_BIG:
        if (dt != DT_I8) g.cc_acc = g.rc_acc = nullptr;          // these tiles add to the sums themselves
        switch (dt) {
        case DT_I8:   return launch_group_big_i8(ot, protect, g, st);
        case DT_BF16: return launch_group_big_bf16(protect, transB, g, st);
        default:      return launch_group_big_f16(protect, transB, g, st);
        }
    default:
        switch (dt) {
        case DT_I8:   return launch_group_rows_i8(ot, k.tiles, protect, transB, g, st);
        case DT_BF16: return launch_group_rows_bf16(k.tiles, protect, transB, g, st);
        default:      return launch_group_rows_f16(k.tiles, protect, transB, g, st);
        }
    }
}

bool group_plan_wgrad(const GroupArgs &g, GroupKernel *k)
{
    const GroupProblem p = {g.K, g.N, (int)ceil_div(g.M, g.groups), g.groups, 2, false, true};
    constexpr long ALL = 1L << 31;
    // (a group's depth may be nearly all rows; of a slab more than there are, three at least, is asked for)
    const long most = ((long)g.M + 4 * 64) * 2;
    const double wide = tile_us(p, TILE_64_128), square = tile_us(p, TILE_64);
    k->kind = most * g.lda < ALL && most * g.ldb < ALL && g.groups <= 4096 && big_us(p) < std::min(wide, square) ? GROUP_KERNEL_BIG : GROUP_KERNEL_TILE;
    k->tiles = wide < square ? TILE_64_128 : ceil_div(p.rows, 64) * ceil_div(p.N, 64) * p.groups <= 256 ? TILE_64_4 : TILE_64;
    return tiles_fit(*k, g, 0, [&](int bm) { return ceil_div(g.K, bm) * g.groups; });
}

hipError_t launch_group_wgrad(int dt, const GroupKernel &k, GroupArgs &g, hipStream_t st)
{
    if (k.kind == GROUP_KERNEL_BIG) return launch_group_big_wgrad(dt, g, st);
    return dt == DT_BF16 ? launch_group_depth_bf16(k.tiles, g, st) : launch_group_depth_f16(k.tiles, g, st);
}

}  // namespace abft
