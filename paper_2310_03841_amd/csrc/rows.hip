// Rows of tokens to their experts and back: entries (a token's choice each) sorted by group, rows gathered in that order, the experts' rows combined, and the
// gradient of that.
#include "abft_device.h"
#include "block_out.h"
#include "route_args.h"

namespace abft {

// ---------------------------------------------------------------- entries by group
// A stable counting sort.  A wave takes 64 entries at a time; a lane's rank among the equal ones of its wave comes from ballots over the bits of
// the group's number, so that nothing is counted with atomics and the order is the entries' own.  Of more entries than one workgroup's, a first kernel counts
// each workgroup's groups, and every workgroup adds up those ahead of it.
// Bound by latency: one workgroup for a call's few entries, of no more waves than they and the groups need (64 entries, 32 groups: sixteen waves 4.1 us, one 2.2).  50432 entries, 64 groups:
// 4096 of them to a workgroup and one thread to a group's counts in all workgroups 4.6 + 6.2 us; 1024, and the threads sharing out the counts, 3.4 + 4.8 (behind other kernels 4.6 + 4.9).
constexpr int ROWS_MOST = 1024;                              // threads

struct GroupRowsArgs {
    const int *group;
    int n, groups, bits, blocks, iters;   // iters: times that a workgroup takes its threads' entries
    int *offsets, *order, *place;
    uint32_t *hist;                       // [blocks][groups]
};

// Lanes of the wave that are in the same group as this one.
__device__ __forceinline__ uint64_t same_group(int e, bool in, int bits)
{
    uint64_t m = __ballot(in);
    for (int b = 0; b < bits; ++b) {
        const bool set = e >> b & 1;
        const uint64_t v = __ballot(set);
        m &= set ? v : ~v;
    }
    return m;
}

// Entries i0 .. of a wave, TRIPS times 64 of them.  cnt: [waves][groups], zero.  Each trip's group, -1 for none, and its rank in the wave.
template <int TRIPS> __device__ __forceinline__ void count_groups(const GroupRowsArgs &a, int *cnt, long i0, int (&e)[TRIPS], int (&rank)[TRIPS])
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int j = 0; j < TRIPS; ++j) e[j] = i0 + 64 * j + lane < a.n ? a.group[i0 + 64 * j + lane] : -1;
    int *const mine = cnt + wave * a.groups;
#pragma unroll
    for (int j = 0; j < TRIPS; ++j) {
        const bool in = e[j] >= 0 && e[j] < a.groups;
        if (!in) e[j] = -1;
        rank[j] = 0;
        if (i0 + 64 * j >= a.n) continue;                        // (the wave together)
        const uint64_t m = same_group(e[j], in, a.bits);
        const int ahead = __popcll(m & ((1ull << lane) - 1)), all = __popcll(m);
        const int base = in ? mine[e[j]] : 0;
        rank[j] = base + ahead;
        __builtin_amdgcn_wave_barrier();
        if (in && ahead == all - 1) mine[e[j]] = base + all;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
}

__global__ __launch_bounds__(ROWS_MOST) void group_hist_kernel(GroupRowsArgs a)
{
    extern __shared__ int rows_lds[];
    constexpr int THREADS = ROWS_MOST, WAVES = THREADS / 64;
    for (int i = threadIdx.x; i < WAVES * a.groups; i += THREADS) rows_lds[i] = 0;
    __syncthreads();
    for (int it = 0; it < a.iters; ++it) {
        int e[1], rank[1];
        count_groups<1>(a, rows_lds, ((long)blockIdx.x * a.iters + it) * THREADS + (threadIdx.x & ~63), e, rank);
    }
    __syncthreads();
    for (int g = threadIdx.x; g < a.groups; g += THREADS) {
        int s = 0;
        for (int w = 0; w < WAVES; ++w) s += rows_lds[w * a.groups + g];
        a.hist[(long)blockIdx.x * a.groups + g] = (uint32_t)s;
    }
}

// At least as many threads as groups.
template <int TRIPS> __global__ __launch_bounds__(ROWS_MOST) void group_place_kernel(GroupRowsArgs a)
{
    extern __shared__ int rows_lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, threads = blockDim.x, waves = threads >> 6;
    int *const cnt = rows_lds, *const sums = cnt + waves * a.groups, *const totals = sums + 16;        // totals: [2][groups]
    for (int i = tid; i < (waves + 2) * a.groups + 16; i += threads) cnt[i] = 0;
    __syncthreads();
    const long block0 = (long)blockIdx.x * a.iters * threads * TRIPS;
    int e[TRIPS], rank[TRIPS];
    count_groups<TRIPS>(a, cnt, block0 + wave * 64 * TRIPS, e, rank);
    // entries of each group in all workgroups, and in those ahead: the threads share out the workgroups
    if (a.blocks > 1) {
        const int parts = threads / a.groups, part = tid / a.groups, g = tid - part * a.groups;
        if (part < parts) {
            int total = 0, before = 0;
#pragma unroll 4
            for (int b = part; b < a.blocks; b += parts) {
                const int h = (int)a.hist[(long)b * a.groups + g];
                total += h;
                before += b < (int)blockIdx.x ? h : 0;
            }
            atomicAdd(totals + g, total);                        // (in LDS, of integers: in any order)
            atomicAdd(totals + a.groups + g, before);
        }
    }
    __syncthreads();
    int total = 0, before = 0;
    if (tid < a.groups) {
        if (a.blocks == 1) {
            for (int w = 0; w < waves; ++w) total += cnt[w * a.groups + tid];
        } else {
            total = totals[tid];
            before = totals[a.groups + tid];
        }
    }
    int upto = total;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int v = __shfl_up(upto, d);
        if (lane >= d) upto += v;
    }
    if (lane == 63) sums[wave] = upto;
    __syncthreads();
    int ahead = 0, all = 0;
    for (int w = 0; w < waves; ++w) {
        const int s = sums[w];
        ahead += w < wave ? s : 0;
        all += s;
    }
    int at = ahead + upto - total;                               // the group's next row
    if (blockIdx.x == 0 && tid < a.groups) {
        a.offsets[tid] = at;
        if (tid == a.groups - 1) a.offsets[a.groups] = all;
    }
    at += before;
    for (int it = 0;;) {
        if (tid < a.groups)
            for (int w = 0; w < waves; ++w) {
                const int c = cnt[w * a.groups + tid];
                cnt[w * a.groups + tid] = at;
                at += c;
            }
        __syncthreads();
        const long i0 = block0 + (long)it * threads * TRIPS + wave * 64 * TRIPS + lane;
#pragma unroll
        for (int j = 0; j < TRIPS; ++j) {
            const long i = i0 + 64 * j;
            if (i >= a.n) break;
            const int r = e[j] >= 0 ? cnt[wave * a.groups + e[j]] + rank[j] : -1;
            a.place[i] = r;
            if (r >= 0) a.order[r] = (int)i;
            if (i >= all) a.order[i] = -1;                       // rows behind the last group
        }
        if (++it == a.iters) break;
        __syncthreads();
        for (int i = tid; i < waves * a.groups; i += threads) cnt[i] = 0;
        __syncthreads();
        count_groups<TRIPS>(a, cnt, i0 - lane + threads * TRIPS, e, rank);
        __syncthreads();
    }
}

// One workgroup for up to 2048 entries, of 64 threads or as many as there are groups, and four entries to a thread.  Of more entries, 1024 threads with one each, and up to 512
// workgroups, which go through theirs one thousand at a time: each of them reads the counts of all.
constexpr int ROWS_ONE = 2048, ROWS_BLOCKS = 512;
static int rows_iters(long n) { return n <= ROWS_ONE ? 1 : (int)((n + (long)ROWS_MOST * ROWS_BLOCKS - 1) / ((long)ROWS_MOST * ROWS_BLOCKS)); }
static int rows_blocks(long n) { return n <= ROWS_ONE ? 1 : (int)((n + (long)ROWS_MOST * rows_iters(n) - 1) / ((long)ROWS_MOST * rows_iters(n))); }
size_t group_rows_words(long n, int groups) { return n <= ROWS_ONE ? 0 : (size_t)(n < (long)ROWS_MOST * ROWS_BLOCKS ? rows_blocks(n) : ROWS_BLOCKS) * groups; }

hipError_t launch_group_rows(const int *group, int n, int groups, int *offsets, int *order, int *place, uint32_t *hist, hipStream_t st)
{
    int bits = 0;
    while ((1 << bits) < groups) ++bits;
    const GroupRowsArgs a = {group, n, groups, bits, rows_blocks(n), rows_iters(n), offsets, order, place, hist};
    const int least = (groups + 63) / 64 * 64, whole = (n + 255) / 256 * 64;
    const int threads = n > ROWS_ONE ? ROWS_MOST : least > whole ? least : whole;
    const int lds = ((threads / 64 + 2) * groups + 16) * 4;
    constexpr int MOST = ((ROWS_MOST / 64 + 2) * GROUP_ROWS_MAX + 16) * 4;
    auto place_kernel = n > ROWS_ONE ? group_place_kernel<1> : group_place_kernel<4>;
    hipError_t e = hipSuccess;
    if (lds > 64 * 1024) {
        e = ensure_max_lds(reinterpret_cast<const void *>(place_kernel), MOST);
        if (e == hipSuccess) e = ensure_max_lds(reinterpret_cast<const void *>(group_hist_kernel), MOST);
        if (e != hipSuccess) return e;
    }
    if (n > ROWS_ONE) {
        hipLaunchKernelGGL(group_hist_kernel, dim3((unsigned)a.blocks), dim3((unsigned)threads), lds, st, a);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    hipLaunchKernelGGL(place_kernel, dim3((unsigned)a.blocks), dim3((unsigned)threads), lds, st, a);
    return hipGetLastError();
}

// ---------------------------------------------------------------- rows in the order of their groups
struct GatherArgs {
    const uint8_t *X;
    uint8_t *Y;
    const int *order;
    int tokens, rows, topk, bytes;        // bytes of a row that are copied
    long ldx, ldy;
};

// Rows of more bytes than this go past the caches.  (On their way / so, us, 1024 columns of bf16: 12608 tokens to 4 experts each, 103 MB, 38.8 / 37.3, with the product of 768
// columns that reads them 131.5 / 125.3, of 128 75.7 / 73.5; 3152 tokens, 26 MB, 15.4 / 15.2, with the product 49.3 / 51.5.)  Rows of up to 512 bytes do not: 128 columns, 100000 tokens to 4 experts
// each, 30.4 / 29.6, with a product of 256 columns 152 / 169; 64 columns, 200000 tokens, 30.5 / 29.8 and 238 / 255.  (From 256 columns on they gain: 60000 tokens 35.9 / 35.0 and 97.8 / 92.8.)
constexpr long FAR_BYTES = 64L << 20;

// Bound by memory: 103 MB written and, for four copies on eight L2s, 93 read of 26 that there are, 6.6 TB/s in 29.7 us (4.3 of the 129 that have to move).  (Tokens dealt out to the XCDs, so that their copies meet in one L2: 48 us of the kernel
// alone for 29.)
// Chunk c of a row of so many bytes
template <bool FAR> __device__ __forceinline__ void put_bytes(uint8_t *dst, const i32x4 &v, int c, int bytes)
{
    const int n = bytes - c * 16;
    i32x4 *const at = reinterpret_cast<i32x4 *>(dst + (long)c * 16);
    if (n >= 16 && FAR) __builtin_nontemporal_store(v, at);
    else if (n >= 16) *at = v;
    else for (int b = 0; b < n; ++b) dst[(long)c * 16 + b] = (uint8_t)((uint32_t)v[b >> 2] >> (8 * (b & 3)));
}

// 16 bytes of a row to a lane, LPR lanes to a row, NC such pieces of a lane on their way.
template <int LPR, int NC, bool FAR> __device__ __forceinline__ void copy_row(const uint8_t *src, uint8_t *dst, int bytes, int l)
{
    const int nch = (bytes + 15) / 16;
    for (int c0 = 0; c0 < nch; c0 += LPR * NC) {
        i32x4 v[NC];
#pragma unroll
        for (int i = 0; i < NC; ++i) v[i] = *reinterpret_cast<const i32x4 *>(src + (long)min(c0 + LPR * i + l, nch - 1) * 16);
#pragma unroll
        for (int i = 0; i < NC; ++i) put_bytes<FAR>(dst, v[i], c0 + LPR * i + l, bytes);
    }
}

template <int LPR, int NC, bool FAR> __global__ __launch_bounds__(256) void gather_rows_kernel(GatherArgs a)
{
    fetch_args<GatherArgs>();
    const long r = flat_block() * (256 / LPR) + threadIdx.x / LPR;
    if (r >= a.rows) return;
    const int i = a.order[r], t = i / a.topk;
    if (i >= 0 && t < a.tokens) copy_row<LPR, NC, FAR>(a.X + t * a.ldx, a.Y + r * a.ldy, a.bytes, threadIdx.x % LPR);
}

template <int LPR, int NC, bool FAR> static hipError_t launch_gather_one(const GatherArgs &a, hipStream_t st)
{
    hipLaunchKernelGGL((gather_rows_kernel<LPR, NC, FAR>), flat_grid(((long)a.rows + 256 / LPR - 1) / (256 / LPR)), dim3(256), 0, st, a);
    return hipGetLastError();
}
hipError_t launch_gather_rows(int es, const void *X, int tokens, int cols, long ldx, const int *order, int rows, int topk, void *Y, long ldy, hipStream_t st)
{
    const GatherArgs a = {(const uint8_t *)X, (uint8_t *)Y, order, tokens, rows, topk, cols * es, ldx, ldy};
    const int nch = (a.bytes + 15) / 16;
    if ((long)rows * a.bytes > FAR_BYTES && nch > 32) return nch <= 64 ? launch_gather_one<64, 1, true>(a, st) : nch <= 128 ? launch_gather_one<64, 2, true>(a, st) : launch_gather_one<64, 4, true>(a, st);
    if (nch <= 8)   return launch_gather_one<8, 1, false>(a, st);
    if (nch <= 16)  return launch_gather_one<16, 1, false>(a, st);
    if (nch <= 32)  return launch_gather_one<32, 1, false>(a, st);
    if (nch <= 64)  return launch_gather_one<64, 1, false>(a, st);
    if (nch <= 128) return launch_gather_one<64, 2, false>(a, st);
    return launch_gather_one<64, 4, false>(a, st);
}

// ---------------------------------------------------------------- and back to their tokens
// 16 bytes of a row to a lane.  Sums in fp32, in the order of a token's choices, the base first.
// Bound by memory: rows of 2 KB in any order.  12608 tokens of 1001 fp16 columns, two choices and a base: 25.5 us for 101 MB, 4.0 TB/s (a token to half a wave, four chunks to a lane,
// 26.3); the gradient 23.5 us for 126 MB, 5.4 TB/s.  Stores past the caches would take both in turn from 48.9 to 41.4, and cost a product that reads what they wrote more than that: 12608 tokens, 1024
// columns of bf16, two choices, with a product of 768 columns behind it: combine 41.0 / 42.8, gradient 65.9 / 71.1; four choices 49.4 / 50.4 and 118.7 / 125.8.
__device__ __forceinline__ void put_chunk(uint8_t *dst, const uint32_t (&o)[4], int n)        // n: elements of the chunk inside the row
{
    if (n >= 8) *reinterpret_cast<i32x4 *>(dst) = i32x4{(int)o[0], (int)o[1], (int)o[2], (int)o[3]};
    else for (int e = 0; e < n; ++e) reinterpret_cast<uint16_t *>(dst)[e] = (uint16_t)(o[e >> 1] >> (16 * (e & 1)));
}

// A slice of a token's row, NC chunks to each of LPR lanes, or the whole row; the rows of U choices are on their way together.
template <int DT, int LPR, int NC> __global__ __launch_bounds__(256) void combine_rows_kernel(CombineArgs a)
{
    using T = Traits<DT>;
    constexpr int U = NC == 1 ? 4 : 2;
    fetch_args<CombineArgs>();
    const int nch = (a.cols + 7) / 8, c0 = (int)blockIdx.z * 64 * NC + threadIdx.x % LPR;
    const long t = flat_block() * (256 / LPR) + threadIdx.x / LPR;
    if (t >= a.tokens) return;
    const int *place = a.place + t * a.topk;
    const float *weight = a.weight + (a.weight ? t * a.topk : 0);
    float s[NC][8];
    i32x4 b[NC];
#pragma unroll
    for (int q = 0; q < NC; ++q) {
        b[q] = i32x4{0, 0, 0, 0};
        if (a.base) b[q] = *reinterpret_cast<const i32x4 *>(a.base + t * a.ldb + (long)min(c0 + LPR * q, nch - 1) * 16);
    }
    for (int j0 = 0; j0 < a.topk; j0 += U) {
        int r[U];
        float w[U];
        i32x4 v[U][NC];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int j = min(j0 + u, a.topk - 1);
            r[u] = place[j];
            w[u] = a.weight ? weight[j] : 1.f;
            if (j0 + u >= a.topk || r[u] >= a.rows) r[u] = -1;
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int q = 0; q < NC; ++q)
                if (r[u] >= 0) v[u][q] = *reinterpret_cast<const i32x4 *>(a.Y + r[u] * a.ldy + (long)min(c0 + LPR * q, nch - 1) * 16);
        if (j0 == 0) {
#pragma unroll
            for (int q = 0; q < NC; ++q)
#pragma unroll
                for (int e = 0; e < 8; ++e) s[q][e] = (float)T::elem(b[q], e);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (r[u] >= 0) {
#pragma unroll
                for (int q = 0; q < NC; ++q)
#pragma unroll
                    for (int e = 0; e < 8; ++e) s[q][e] = __builtin_fmaf(w[u], (float)T::elem(v[u][q], e), s[q][e]);
            }
    }
#pragma unroll
    for (int q = 0; q < NC; ++q) {
        const int c = c0 + LPR * q;
        uint32_t o[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = pack2<DT>(s[q][2 * e], s[q][2 * e + 1]);
        put_chunk(a.out + t * a.ldo + (long)c * 16, o, a.cols - c * 8);
    }
}

// The gradient, LPR lanes to a token, which keep NC chunks of dout each: dY[row] = w dout, dweight = dout . Y[row], summed in fp32 by a lane's chunks, then over the
// lanes.  LONG: rows of more chunks, dout read again with every choice.
template <int DT, int LPR, int NC, bool LONG> __global__ __launch_bounds__(256) void combine_grad_kernel(CombineArgs a)
{
    using T = Traits<DT>;
    fetch_args<CombineArgs>();
    const int l = threadIdx.x % LPR, nch = (a.cols + 7) / 8;
    const long t = flat_block() * (256 / LPR) + threadIdx.x / LPR;
    if (t >= a.tokens) return;
    i32x4 d[NC], y[NC];
    auto load = [&](i32x4 (&v)[NC], const uint8_t *row, int c0) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < NC; ++i) v[i] = *reinterpret_cast<const i32x4 *>(row + (long)min(c0 + LPR * i + l, nch - 1) * 16);
    };
    auto cut = [&](i32x4 (&v)[NC], int c0) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            const int c = c0 + LPR * i + l;
            if (c >= nch - 1) v[i] = mask_chunk(v[i], c < nch ? 2 * (a.cols - c * 8) : 0);
        }
    };
    const uint8_t *dout = a.dout + t * a.ldo;
    if (!LONG) load(d, dout, 0);
    bool whole = true;                                           // what lies behind the row is still in d
    for (int j = 0; j < a.topk; ++j) {
        const int r = a.place[t * a.topk + j];
        const bool in = r >= 0 && r < a.rows;
        float dot = 0.f;
        if (in) {
            const float w = a.weight ? a.weight[t * a.topk + j] : 1.f;
            for (int c0 = 0; c0 < (LONG ? nch : 1); c0 += LPR * NC) {
                if (LONG) load(d, dout, c0);
                if (a.dweight) load(y, a.Y + r * a.ldy, c0);
                if (LONG || whole) cut(d, c0);
                whole = false;
                if (a.dweight) cut(y, c0);
#pragma unroll
                for (int i = 0; i < NC; ++i) {
                    const int c = c0 + LPR * i + l;
                    uint32_t o[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float x0 = (float)T::elem(d[i], 2 * e), x1 = (float)T::elem(d[i], 2 * e + 1);
                        if (a.dweight) dot = __builtin_fmaf(x1, (float)T::elem(y[i], 2 * e + 1), __builtin_fmaf(x0, (float)T::elem(y[i], 2 * e), dot));
                        o[e] = pack2<DT>(w * x0, w * x1);
                    }
                    if (a.dY) put_chunk(a.dY + r * a.lddy + (long)c * 16, o, a.cols - c * 8);
                }
            }
        }
        if (a.dweight) {
            dot = seg_sum(dot, LPR);
            if (l == 0) a.dweight[t * a.topk + j] = in ? dot : 0.f;
        }
    }
}

// A slice to a z of the grid.
template <int DT, int LPR, int NC> static hipError_t launch_combine_one(const CombineArgs &a, hipStream_t st)
{
    dim3 grid = flat_grid(((long)a.tokens + 256 / LPR - 1) / (256 / LPR));
    grid.z = LPR == 64 ? (unsigned)(((a.cols + 7) / 8 + 64 * NC - 1) / (64 * NC)) : 1u;
    hipLaunchKernelGGL((combine_rows_kernel<DT, LPR, NC>), grid, dim3(256), 0, st, a);
    return hipGetLastError();
}
template <int DT, int LPR, int NC, bool LONG> static hipError_t launch_grad_one(const CombineArgs &a, hipStream_t st)
{
    hipLaunchKernelGGL((combine_grad_kernel<DT, LPR, NC, LONG>), flat_grid(((long)a.tokens + 256 / LPR - 1) / (256 / LPR)), dim3(256), 0, st, a);
    return hipGetLastError();
}
template <int DT> static hipError_t launch_combine_type(bool grad, const CombineArgs &a, hipStream_t st)
{
    const int nch = (a.cols + 7) / 8;
    if (!grad) {
        if (nch <= 8)  return launch_combine_one<DT, 8, 1>(a, st);
        if (nch <= 16) return launch_combine_one<DT, 16, 1>(a, st);
        if (nch <= 32) return launch_combine_one<DT, 32, 1>(a, st);
        // two chunks to a lane once there are waves enough: one / two, us, 1024 columns, 1024 tokens of 8 choices 4.9 / 5.5, 2048 7.4 / 7.7, 12608 of 2 13.4 / 12.7; 4096 columns, 2048 tokens of 2
        // 9.3 / 9.0, 4096 16.2 / 16.5
        if (nch <= 64 || a.tokens < 2048) return launch_combine_one<DT, 64, 1>(a, st);
        return launch_combine_one<DT, 64, 2>(a, st);
    }
    if (nch <= 8)   return launch_grad_one<DT, 8, 1, false>(a, st);
    if (nch <= 16)  return launch_grad_one<DT, 16, 1, false>(a, st);
    if (nch <= 32)  return launch_grad_one<DT, 32, 1, false>(a, st);
    if (nch <= 64)  return launch_grad_one<DT, 64, 1, false>(a, st);
    if (nch <= 128) return launch_grad_one<DT, 64, 2, false>(a, st);
    if (nch <= 256) return launch_grad_one<DT, 64, 4, false>(a, st);
    if (nch <= 512) return launch_grad_one<DT, 64, 8, false>(a, st);
    return launch_grad_one<DT, 64, 4, true>(a, st);
}
hipError_t launch_combine_rows(int dt, bool grad, const CombineArgs &a, hipStream_t st)
{
    return dt == DT_BF16 ? launch_combine_type<DT_BF16>(grad, a, st) : launch_combine_type<DT_F16>(grad, a, st);
}

}  // namespace abft
