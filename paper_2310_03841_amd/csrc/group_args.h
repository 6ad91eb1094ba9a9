// Products over groups of rows: what their kernels share.  The rows of A and C are sorted by group; group e has the rows
// offsets[e] .. offsets[e + 1] and a matrix B of its own.  The offsets lie in device memory, so the host knows only how many rows and
// groups there are; it launches as many workgroups as any split of the rows needs, and each finds its tile.
#pragma once
#include "abft_device.h"
#include "gemm_args.h"

namespace abft {

struct GroupArgs {
    const uint8_t *A, *B;
    uint8_t *C;
    const int *offsets;                   // [groups + 1]; null: one group of all rows
    int M, N, K, groups;                  // M: rows over all groups (of a gradient of weights: the depth)
    long lda, ldb, ldc, sB;               // elements
    int tiles_n;
    uint32_t group_inv;                   // map_inverse(tiles_n)
    int inj_b, inj_row, inj_col, inj_bit; // armed accumulator flip (inj_b < 0: none); the row counts from its group's first
    const float *row_scale, *col_scale;   // [M], [groups][N], or null
    const float *bias;                    // [N], or null; behind the scales
    // protected: sums start at zero and are added to with atomics
    uint32_t *cc_obs, *rc_obs;            // observed sums of C  [groups][N], [M]: integers
    double *cc_acc, *rc_acc;              // floating point: the same in doubles, whose rounding hides the order of additions
    uint32_t *rc_pred;                    // A b of each row's group  [M]
    uint32_t *a_sum, *a_max;              // e^T A and max|A| of a group's rows  [groups][K], [groups]
    const uint32_t *b_sum;                // B e of each group  [groups][K]
    uint32_t *counts;                     // cleared for the check kernel
    int deep_first;                       // tiles of a gradient go by the depth of their groups (big_deep_first)
    int n_pass, pass_win;                 // workgroups that pass over A, ahead of those that take tiles; windows along K
    uint32_t pass_inv;                    // map_inverse(pass_win)
};

// Of 4-bit operands: K, lda, ldb and sB count bytes, of two elements each, and K whole blocks of 16; sums along K have 2 K terms.
struct Mx4Args : GroupArgs {
    const uint8_t *sa, *sb;               // powers of two of the blocks, with a bias of 127: rows of A, of B
    long ld_sa, ld_sb, stride_sb;         // bytes
    int pass_log2;                        // rows to an item of the pass over A: 2^pass_log2 times those of one trip
};
template <int DT> struct GroupArgsOf { typedef GroupArgs type; };
template <> struct GroupArgsOf<DT_MX4> { typedef Mx4Args type; };

// The rows of group e: whatever the offsets hold, inside [0, M].
__device__ __forceinline__ void group_rows(const int *offsets, int M, int e, int *first, int *rows)
{
    if (!offsets) { *first = 0; *rows = M; return; }
    int a = offsets[e], b = offsets[e + 1];
    a = a < 0 ? 0 : a > M ? M : a;
    b = b < a ? a : b > M ? M : b;
    *first = a;
    *rows = b - a;
}

// The group that row r belongs to, -1: none.  By halving: of the groups that start at or ahead of r, the last.
__device__ __forceinline__ int group_of(const int *offsets, int M, int groups, int r, int *end)
{
    if (!offsets) { *end = M; return 0; }
    int lo = 0, hi = groups;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (offsets[mid] <= r) lo = mid;
        else hi = mid;
    }
    int first, rows;
    group_rows(offsets, M, lo, &first, &rows);
    *end = first + rows;
    return r >= first && r < first + rows ? lo : -1;
}

// Sum over the lanes up to and with this one.
__device__ __forceinline__ int wave_prefix(int v)
{
    v += dpp_mov<0x111>(v);                                      // row_shr:1, 2, 4, 8 inside 16 lanes
    v += dpp_mov<0x112>(v);
    v += dpp_mov<0x114>(v);
    v += dpp_mov<0x118>(v);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);     // row_bcast:15 into rows 1 and 3
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);     // row_bcast:31 into rows 2 and 3
    return v;
}

// The rows of a lane's group, of up to 64: read once and kept, since a trip to memory ahead of every tile is 1 us of its 15 to 30.
struct GroupLane { int first, rows; };
__device__ __forceinline__ GroupLane group_lane(const GroupArgs &g, int e)
{
    GroupLane l = {0, 0};
    if (e < g.groups) group_rows(g.offsets, g.M, e, &l.first, &l.rows);
    return l;
}

// The group that item L of a list belongs to, and its place among that group's; of a group of so many rows there are of(rows) items.
template <typename OF>
__device__ __forceinline__ bool find_group(const GroupArgs &g, GroupLane mine, const OF &of, int *L, int *e, int *first, int *rows)
{
    const int lane = threadIdx.x & 63;
    int base = 0;
    for (int e0 = 0; e0 < g.groups; e0 += 64) {
        if (g.groups > 64) mine = group_lane(g, e0 + lane);
        const int n = of(mine.rows), upto = base + wave_prefix(n);
        const uint64_t behind = __ballot(upto > *L);
        if (behind) {
            const int l = __builtin_ctzll(behind);
            *e = e0 + l;
            *L -= __builtin_amdgcn_readlane(upto - n, l);
            *first = __builtin_amdgcn_readlane(mine.first, l);
            *rows = __builtin_amdgcn_readlane(mine.rows, l);
            return true;
        }
        base = __builtin_amdgcn_readlane(upto, 63);
    }
    return false;
}

struct GroupTile { int e, tm, tn, first, rows; };

// The tile of workgroup `bid` of those that take tiles, of BM rows each: false, there is none for it.  Every wave finds it by itself, 64 groups at
// a time.  Consecutive tiles of an XCD are a group's, in the order of map_tile, so what shares rows of A or B meets in one L2.
// tiles_n, inv: tiles along the other direction, map_inverse of them.
// BM: a power of two, times 2^log2.
template <int BM> __device__ __forceinline__ bool find_tile(const GroupArgs &g, int tiles_n, uint32_t inv, int bid, GroupTile *t, int log2 = 0)
{
    static_assert((BM & (BM - 1)) == 0, "shifts for quotients");
    const int lane = threadIdx.x & 63;
    const int shift = __builtin_ctz(BM) + log2;
    auto rows_of = [&](int rows) __attribute__((always_inline)) { return (int)(((uint32_t)rows + (1u << shift) - 1u) >> shift); };
    auto tiles_of = [&](int rows) __attribute__((always_inline)) { return rows_of(rows) * tiles_n; };
    GroupLane mine = {0, 0};
    int total = 0;
    if (g.groups == 1) {
        group_rows(g.offsets, g.M, 0, &t->first, &t->rows);
        t->e = 0;
        total = tiles_of(t->rows);
    } else {
        for (int e0 = 0; e0 < g.groups; e0 += 64) {
            mine = group_lane(g, e0 + lane);
            total += wave_sum(tiles_of(mine.rows));
        }
        total = __builtin_amdgcn_readfirstlane(total);
    }
    const int q = total >> 3, r = total & 7, xcd = bid & 7, i = bid >> 3;
    if (i >= q + (xcd < r ? 1 : 0)) return false;                // more workgroups than tiles
    int L = xcd * q + (xcd < r ? xcd : r) + i;
    if (g.groups > 1 && !find_group(g, mine, tiles_of, &L, &t->e, &t->first, &t->rows)) return false;
    tile_at(L, rows_of(t->rows), tiles_n, inv, &t->tm, &t->tn);
    return true;
}

// The kernel that a product takes: tiles by four waves (gemm_group.h, of the shape `tiles`), of the fast kernel (gemm_group_big.h), or few rows
// (gemm_group_few.hip), whose kernel checks the columns itself: cc_obs then holds a mark for each that disagrees.
enum { GROUP_KERNEL_TILE, GROUP_KERNEL_BIG, GROUP_KERNEL_FEW };
struct GroupKernel { int kind, tiles; };
// Of a product, and of a gradient of weights; what g says of the pass over A.  False: more workgroups, or tiles in its list, than a launch or an int counts.
// Asked once to a call, ahead of all that changes anything.
bool group_plan(int dt, bool transB, bool protect, GroupArgs &g, GroupKernel *k);
bool group_plan_wgrad(const GroupArgs &g, GroupKernel *k);
// Rows and columns of C that a workgroup of a product's kernel takes at a time.
void group_tile_shape(const GroupKernel &k, const GroupArgs &g, int *rows, int *columns);
// Whether the kernel of few rows has room for what it keeps; its columns to a workgroup; workgroups with tiles.
bool group_few_fits(int dt, bool protect, const GroupArgs &g);
int group_few_columns(const GroupArgs &g);
long group_few_workgroups(const GroupArgs &g);
// Its shares of the observed sums of rows, for every sixteen columns one after the other, [M] words each: they take the place of the sums in doubles (2 (groups N +
// M) words), of which it keeps none.
inline uint32_t *group_few_shares(const GroupArgs &g) { return reinterpret_cast<uint32_t *>(g.cc_acc); }
hipError_t launch_group_few(int dt, int ot, bool protect, GroupArgs &g, const uint32_t *b_max, float tau_cols, hipStream_t st);

}  // namespace abft
