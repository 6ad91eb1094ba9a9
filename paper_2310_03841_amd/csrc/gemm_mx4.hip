// Products over groups of rows of 4-bit operands: tiles by four waves, and which kernel a call takes.
#include "gemm_group.h"
#include "gemm_mx4.h"

namespace abft {

enum { MX4_64, MX4_64_128, MX4_128 };

template <int OT> static hipError_t launch_of(int tiles, bool protect, Mx4Args &g, hipStream_t st)
{
    switch (tiles) {
    case MX4_64:     return protect ? launch_one<DT_MX4, OT, 64, 64, 3, true, GROUP_ROWS, true>(g, st) : launch_one<DT_MX4, OT, 64, 64, 3, false, GROUP_ROWS, true>(g, st);
    case MX4_64_128: return protect ? launch_one<DT_MX4, OT, 64, 128, 3, true, GROUP_ROWS, true>(g, st) : launch_one<DT_MX4, OT, 64, 128, 3, false, GROUP_ROWS, true>(g, st);
    default:         return protect ? launch_one<DT_MX4, OT, 128, 128, 3, true, GROUP_ROWS, true>(g, st) : launch_one<DT_MX4, OT, 128, 128, 3, false, GROUP_ROWS, true>(g, st);
    }
}
hipError_t launch_mx4_rows(int ot, int tiles, bool protect, Mx4Args &g, hipStream_t st)
{
    return ot == DT_BF16 ? launch_of<DT_BF16>(tiles, protect, g, st) : launch_of<DT_F16>(tiles, protect, g, st);
}

bool mx4_plan(bool protect, Mx4Args &g, GroupKernel *k)
{
    long n_pass = 0;
    if (protect) {
        g.pass_win = (int)ceil_div(g.K, PASS_BYTES);
        g.pass_inv = map_inverse(g.pass_win);
        n_pass = ceil_div(row_tiles(g.M, g.groups, 4 * PASS_ROWS) * g.pass_win, 8) * 8;
        if (n_pass > MAX_GRID_X) return false;
        g.n_pass = (int)n_pass;
    }
    const long rows = ceil_div(g.M, g.groups);
    k->kind = GROUP_KERNEL_TILE;
    k->tiles = MX4_64;
    if (ceil_div(rows, 128) * ceil_div(g.N, 128) * g.groups >= 256) k->tiles = MX4_128;
    else if (ceil_div(rows, 64) * ceil_div(g.N, 128) * g.groups >= 256) k->tiles = MX4_64_128;
    if (rows <= 16 && mx4_few_fits(protect, g)) k->kind = GROUP_KERNEL_FEW;
    const int bm = k->tiles == MX4_128 ? 128 : 64, bn = k->tiles == MX4_64 ? 64 : 128;
    const long wgs = k->kind == GROUP_KERNEL_FEW ? mx4_few_workgroups(g) : ceil_div(row_tiles(g.M, g.groups, bm) * ceil_div(g.N, bn), 8) * 8;
    return n_pass + wgs <= MAX_GRID_X;
}

}  // namespace abft
