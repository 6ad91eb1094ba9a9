// Products over groups of rows that fill the chip: the tiles of the fast GEMM kernel (gemm_fast_tile.h) over the groups of group_args.h, and over
// the depths of the groups for the gradient of their matrices.
//
// A group's rows are covered by tiles of 256, the last 128 of them, where no more are left over, by one of 128.  One workgroup to a compute unit walks
// the list with the grid's stride.  What would be a last round of few tiles of 256 is dealt out as twice as many of 128 rows where that ends sooner (a tile of
// 128 rows takes 0.57 of the time of one of 256, protected 0.66).  Tiles of 128 rows come first, as in the fast kernel: the compute units that start
// with one are ahead of the others from then on, so that not all store C at once, and they are the first with what is left in the last round (all tiles
// of 256 first / so, one group, unprotected: bf16 12608 x 3072 x 768 61.3 / 54.0 us, int8 54.8 / 48.3).  Protected, the
// pass over A comes last, 64 rows and a window to an item, by the compute units that have no tile in the last round, unless those are few.
#pragma once
#include "gemm_fast_tile.h"
#include "group_args.h"
#include "group_passes.h"

namespace abft {

enum { BIG_ROWS, BIG_DEPTH };

// A gradient's tiles take as long as their group is deep.  Up to 64 groups are put in the order of their depth, what is cut in halves the least deep, and
// the rounds are dealt out one way and the other, so that every compute unit has about as much to do.  Worth it from two rounds on, of groups of 512 rows on
// average: with fewer the stores of C count for more, and the tiles of a round are no longer neighbours of those of the one behind it.  (bf16 2048 x 1024, group
// by group / so, us: 13 groups of 64 rows on average 20.0 / 22.6, of 512 37.9 / 37.8, of 1024 74.6 / 62.6; 34 groups of 256 58.8 / 62.2, of 512 87.3 / 85.9;
// 6 groups of 512, one round, 21.7 / 22.0; 16 groups of 3072 x 768 and 0 to 1377 rows 83.5 / 70.)
inline bool big_deep_first(const GroupArgs &g, int tiles_n, int cus)
{
    return g.groups > 1 && g.groups <= 64 && g.M / g.groups >= 512 && (g.K + 255L) / 256 * tiles_n * g.groups > cus;
}

// The arguments of one tile, formed where they are used: behind the main loop they are read again rather than held across it.
template <int OT, int GROUP> struct GroupSource {
    static constexpr bool LAYER_BIAS = false;            // (a bias of scaled products is outside the checked sums)
    int e, first, rows;
    template <bool AGAIN> __device__ __forceinline__ GemmArgs get(const GemmArgs &) const
    {
        const GroupArgs &a = kernel_args<GroupArgs>();
        GemmArgs g = {};
        g.C = a.C + (GROUP == BIG_DEPTH ? (long)e * a.sB : (long)first * a.ldc) * Traits<OT>::OS;
        g.M = GROUP == BIG_DEPTH ? a.K : rows;
        g.N = a.N;
        g.ldc = a.ldc;
        g.inj_b = a.inj_b == e ? 0 : -1;
        g.inj_row = a.inj_row; g.inj_col = a.inj_col; g.inj_bit = a.inj_bit;
        g.cc_obs = a.cc_obs + (long)e * a.N;
        g.rc_obs = a.rc_obs + first;
        g.a_given = 1;                                   // the pass over A is another kernel's
        return g;
    }
    __device__ __forceinline__ EpiScale scales(int m0, int n0, int t, int M, int N) const
    {
        const GroupArgs &a = kernel_args<GroupArgs>();
        const int r = first + (m0 + t < M ? m0 + t : M - 1), c = n0 + t < N ? n0 + t : N - 1;
        EpiScale s = {1.f, 1.f, 0.f};
        if (a.row_scale) s.row = a.row_scale[r];
        if (a.col_scale) s.col = a.col_scale[(long)e * N + c];
        if (a.bias) s.bias = a.bias[c];
        return s;
    }
};

struct BigTile { int e, first, rows, m0, tn; bool tall; };

// The place of a lane's group among up to 64 by their depth, the deepest first.
__device__ __forceinline__ int depth_rank(const GroupArgs &g)
{
    const int lane = threadIdx.x & 63, groups = g.groups;
    // (the order of groups deeper than 2^24 is of no account)
    const int key = lane < groups ? min(group_lane(g, lane).rows, (1 << 24) - 1) * 64 + 63 - lane : -1;
    int rank = 0;
#pragma unroll 8
    for (int e = 0; e < groups; ++e) rank += __builtin_amdgcn_readlane(key, e) > key ? 1 : 0;
    return lane < groups ? rank : 64;
}

// Tile t of the list: false, there is none, and *tiles are all.
template <int GROUP, bool PROT> __device__ __forceinline__ bool big_tile(const GroupArgs &g, const GroupLane &kept, int rank, int t, int wgs, BigTile *o, int *tiles)
{
    const int lane = threadIdx.x & 63, tiles_n = g.tiles_n;
    // rows of tiles of 256, of 128, of a product of so many rows
    auto tall_of = [&](int rows) __attribute__((always_inline)) { return (rows >> 8) + ((rows & 255) > 128); };
    auto small_of = [&](int rows) __attribute__((always_inline)) { return ((rows & 255) + 127) >> 7 & 1; };
    GroupLane mine = kept;
    int talls, smalls;                                           // rows of tiles of all groups
    if constexpr (GROUP == BIG_DEPTH) {
        talls = tall_of(g.K) * g.groups;
        smalls = small_of(g.K) * g.groups;
    } else {
        talls = smalls = 0;
        for (int e0 = 0; e0 < g.groups; e0 += 64) {
            if (g.groups > 64) mine = group_lane(g, e0 + lane);
            talls += wave_sum(tall_of(mine.rows));
            smalls += wave_sum(small_of(mine.rows));
        }
        talls = __builtin_amdgcn_readfirstlane(talls);
        smalls = __builtin_amdgcn_readfirstlane(smalls);
    }
    const int nt = talls * tiles_n, ns = smalls * tiles_n, over = nt % wgs;
    constexpr int HALF = PROT ? 66 : 57;                         // of 100
    auto rounds = [&](int n) __attribute__((always_inline)) { return (n + wgs - 1) / wgs; };
    const bool split = over > 0 && HALF * rounds(2 * over + ns) < 100 + HALF * rounds(max(over + ns - wgs, 0));
    const int whole = split ? nt - over : nt, halves = split ? 2 * over : 0;
    // as map_tile: what runs on one XCD at a time lies together
    auto deal = [&](int i, int n) __attribute__((always_inline)) {
        const int q = n >> 3, r = n & 7, xcd = i & 7;
        return xcd * q + (xcd < r ? xcd : r) + (i >> 3);
    };
    int L, half = 0;
    bool left_over = false;
    o->tall = false;
    *tiles = halves + ns + whole;
    if (GROUP == BIG_DEPTH && g.deep_first) {
        // by falling depth, a round at a time, each the other way round than the one ahead of it, and the last round first
        const int k = t / wgs, last = rounds(*tiles) - 1, slot = deal(t - k * wgs, wgs);
        auto place = [&](int r) __attribute__((always_inline)) { return r * wgs + (r & 1 ? wgs - 1 - slot : slot); };
        const int r = last - k - (place(last) < *tiles ? 0 : 1);
        if (r < 0) return false;
        L = place(r);
        if (L < whole) {
            o->tall = true;
        } else if ((L -= whole) < ns) {
            left_over = true;
        } else {
            half = (L -= ns) & 1;
            L = whole + (L >> 1);
        }
    } else if (t < halves) {
        const int h = deal(t, halves);
        L = whole + (h >> 1);
        half = h & 1;
    } else if ((t -= halves) < ns) {
        L = deal(t, ns);
        left_over = true;
    } else if ((t -= ns) < whole) {
        L = deal(t, whole);
        o->tall = true;
    } else {
        return false;
    }
    if constexpr (GROUP == BIG_DEPTH) {
        const int per = (left_over ? small_of(g.K) : tall_of(g.K)) * tiles_n, nth = L / per;
        L -= nth * per;
        o->e = g.deep_first ? __builtin_ctzll(__ballot(rank == nth)) : nth;
        group_rows(g.offsets, g.M, o->e, &o->first, &o->rows);
    } else {
        const bool found = find_group(g, kept, [&](int rows) { return (left_over ? small_of(rows) : tall_of(rows)) * tiles_n; }, &L, &o->e, &o->first, &o->rows);
        if (!found) return false;
    }
    const int height = GROUP == BIG_DEPTH ? g.K : o->rows;
    int tm = 0, tn = 0;
    tile_at(L, tall_of(height), tiles_n, g.group_inv, &tm, &tn);             // (of no use to a tile of left-over rows, whose column L is)
    o->m0 = left_over ? height & ~255 : tm * 256 + half * 128;
    o->tn = left_over ? L : tn;
    return true;
}

template <int DT, int OT, bool PROT, int GROUP, bool BT>
__global__ __launch_bounds__(64 * FAST_WAVES) void gemm_group_big_kernel(GroupArgs)
{
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    constexpr bool DEPTH = GROUP == BIG_DEPTH;
    constexpr int MODE = PROT ? FAST_BESIDE : FAST_PLAIN, ES = Traits<DT>::ES;
    fetch_args<GroupArgs>();
    GroupLane kept = {0, 0};
    int rank = 0;
    if constexpr (!DEPTH) kept = group_lane(kernel_args<GroupArgs>(), threadIdx.x & 63);
    else if (kernel_args<GroupArgs>().deep_first) rank = depth_rank(kernel_args<GroupArgs>());
    int tiles;
    for (int t = blockIdx.x;; t += gridDim.x) {
        const GroupArgs &a = kernel_args<GroupArgs>();
        if (PROT && t == 0 && threadIdx.x < 5) a.counts[threadIdx.x] = 0u;       // completed by the check kernel
        BigTile b;
        if (!big_tile<GROUP, PROT>(a, kept, rank, t, (int)gridDim.x, &b, &tiles)) break;
        // the epilogue's last reads of LDS precede the next tile's first writes
        if (t != (int)blockIdx.x) asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        GemmArgs g = {};
        g.A = a.A + (long)b.first * a.lda * ES;
        g.B = a.B + (DEPTH ? (long)b.first * a.ldb : (long)b.e * a.sB) * ES;
        g.M = DEPTH ? a.K : b.rows;
        g.N = a.N;
        g.K = DEPTH ? b.rows : a.K;
        g.lda = a.lda; g.ldb = a.ldb;
        const GroupSource<OT, GROUP> source = {b.e, b.first, b.rows};
        if (b.tall) fast_tile<DT, OT, 256, MODE, STO_NO, DEPTH, BT>(g, source, smem, b.m0, b.tn * 256, 0, b.tn);
        else fast_tile<DT, OT, 128, MODE, STO_NO, DEPTH, BT>(g, source, smem, b.m0, b.tn * 256, 0, b.tn);
    }
    if constexpr (PROT) {
        constexpr int ROWS = FAST_WAVES * PASS_ROWS;
        const GroupArgs &a = kernel_args<GroupArgs>();
        int passes = 0;
        GroupLane mine = kept;
        auto passes_of = [&](int rows) __attribute__((always_inline)) { return (rows + ROWS - 1) / ROWS * a.pass_win; };
        for (int e0 = 0; e0 < a.groups; e0 += 64) {
            if (a.groups > 64) mine = group_lane(a, e0 + (threadIdx.x & 63));
            passes += wave_sum(passes_of(mine.rows));
        }
        passes = __builtin_amdgcn_readfirstlane(passes);
        int busy = tiles % (int)gridDim.x, free = (int)gridDim.x - busy;
        if (passes > 4 * free) { busy = 0; free = (int)gridDim.x; }
        for (int p = (int)blockIdx.x - busy; p >= 0 && p < passes; p += free) {
            BigTile b;
            int L = p;
            if (!find_group(a, kept, passes_of, &L, &b.e, &b.first, &b.rows)) break;
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
            const int row = L / a.pass_win;
            group_pass<DT, FAST_WAVES>(a, b.e, b.first, b.rows, row * ROWS, L - row * a.pass_win, smem);
        }
    }
}

template <int DT, int OT, bool PROT, int GROUP, bool BT> static hipError_t launch_big_one(GroupArgs &g, hipStream_t st)
{
    hipError_t e;
    const int cus = device_cu_count(&e);
    if (e != hipSuccess) return e;
    constexpr int smem = fast_lds_bytes<PROT ? FAST_BESIDE : FAST_PLAIN>();
    auto kern = gemm_group_big_kernel<DT, OT, PROT, GROUP, BT>;
    e = ensure_max_lds(reinterpret_cast<const void *>(kern), smem);
    if (e != hipSuccess) return e;
    g.tiles_n = (g.N + 255) / 256;
    g.group_inv = map_inverse(g.tiles_n);
    g.deep_first = GROUP == BIG_DEPTH && big_deep_first(g, g.tiles_n, cus);
    hipLaunchKernelGGL(kern, dim3((unsigned)cus), dim3(64 * FAST_WAVES), smem, st, g);
    return hipGetLastError();
}

// Each in a file of its own, for the time it takes to compile them.
hipError_t launch_group_big_i8(int ot, bool protect, GroupArgs &g, hipStream_t st);
hipError_t launch_group_big_bf16(bool protect, bool transB, GroupArgs &g, hipStream_t st);
hipError_t launch_group_big_f16(bool protect, bool transB, GroupArgs &g, hipStream_t st);
hipError_t launch_group_big_wgrad(int dt, GroupArgs &g, hipStream_t st);

}  // namespace abft
