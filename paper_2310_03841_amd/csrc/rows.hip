// Rows of tokens to their experts and back: entries (a token's choice each) sorted by group, rows gathered in that order, the experts' rows combined, and the
// gradient of that.
#include "abft_device.h"
#include "block_out.h"
#include "route_args.h"

namespace abft {

// ---------------------------------------------------------------- entries by group
// A stable counting sort.  A workgroup has SEG entries, a wave 256 of them; a lane's rank among the equal ones of its wave comes from ballots over the bits of
// the group's number, so that nothing is counted with atomics and the order is the entries' own.  Of more entries than one workgroup's, a first kernel counts
// each workgroup's groups, and every workgroup adds up those ahead of it.
constexpr int ROWS_WAVES = 16, ROWS_TRIPS = 4, ROWS_SEG = ROWS_WAVES * 64 * ROWS_TRIPS;

struct GroupRowsArgs {
    const int *group;
    int n, groups, bits, blocks;
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

// cnt: [ROWS_WAVES][groups], zero.  Each trip's group and its rank in the wave.
__device__ __forceinline__ void count_groups(const GroupRowsArgs &a, int *cnt, int (&e)[ROWS_TRIPS], int (&rank)[ROWS_TRIPS])
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const long i0 = (long)blockIdx.x * ROWS_SEG + wave * 64 * ROWS_TRIPS + lane;
#pragma unroll
    for (int j = 0; j < ROWS_TRIPS; ++j) e[j] = i0 + 64 * j < a.n ? a.group[i0 + 64 * j] : -1;
    int *const mine = cnt + wave * a.groups;
#pragma unroll
    for (int j = 0; j < ROWS_TRIPS; ++j) {
        const bool in = e[j] >= 0 && e[j] < a.groups;
        if (!in) e[j] = -1;
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

__global__ __launch_bounds__(64 * ROWS_WAVES) void group_hist_kernel(GroupRowsArgs a)
{
    extern __shared__ int rows_lds[];
    for (int i = threadIdx.x; i < ROWS_WAVES * a.groups; i += 64 * ROWS_WAVES) rows_lds[i] = 0;
    __syncthreads();
    int e[ROWS_TRIPS], rank[ROWS_TRIPS];
    count_groups(a, rows_lds, e, rank);
    __syncthreads();
    for (int g = threadIdx.x; g < a.groups; g += 64 * ROWS_WAVES) {
        int s = 0;
        for (int w = 0; w < ROWS_WAVES; ++w) s += rows_lds[w * a.groups + g];
        a.hist[(long)blockIdx.x * a.groups + g] = (uint32_t)s;
    }
}

__global__ __launch_bounds__(64 * ROWS_WAVES) void group_place_kernel(GroupRowsArgs a)
{
    extern __shared__ int rows_lds[];
    int *const cnt = rows_lds, *const sums = cnt + ROWS_WAVES * a.groups;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    for (int i = tid; i < ROWS_WAVES * a.groups; i += 64 * ROWS_WAVES) cnt[i] = 0;
    __syncthreads();
    int e[ROWS_TRIPS], rank[ROWS_TRIPS];
    count_groups(a, cnt, e, rank);
    __syncthreads();
    // a thread to a group: its entries in all workgroups, in those ahead, in the waves ahead
    int total = 0, before = 0;
    if (tid < a.groups) {
        if (a.blocks == 1) {
            for (int w = 0; w < ROWS_WAVES; ++w) total += cnt[w * a.groups + tid];
        } else {
#pragma unroll 8
            for (int b = 0; b < a.blocks; ++b) {
                const int h = (int)a.hist[(long)b * a.groups + tid];
                total += h;
                before += b < (int)blockIdx.x ? h : 0;
            }
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
#pragma unroll
    for (int w = 0; w < ROWS_WAVES; ++w) {
        const int s = sums[w];
        ahead += w < wave ? s : 0;
        all += s;
    }
    if (tid < a.groups) {
        const int first = ahead + upto - total;
        if (blockIdx.x == 0) {
            a.offsets[tid] = first;
            if (tid == a.groups - 1) a.offsets[a.groups] = all;
        }
        int at = first + before;
        for (int w = 0; w < ROWS_WAVES; ++w) {
            const int c = cnt[w * a.groups + tid];
            cnt[w * a.groups + tid] = at;
            at += c;
        }
    }
    __syncthreads();
    const long i0 = (long)blockIdx.x * ROWS_SEG + wave * 64 * ROWS_TRIPS + lane;
#pragma unroll
    for (int j = 0; j < ROWS_TRIPS; ++j) {
        const long i = i0 + 64 * j;
        if (i >= a.n) break;
        const int r = e[j] >= 0 ? cnt[wave * a.groups + e[j]] + rank[j] : -1;
        a.place[i] = r;
        if (r >= 0) a.order[r] = (int)i;
        if (i >= all) a.order[i] = -1;                           // rows behind the last group
    }
}

static int rows_blocks(long n) { return (int)((n + ROWS_SEG - 1) / ROWS_SEG); }
size_t group_rows_words(long n, int groups) { return rows_blocks(n) > 1 ? (size_t)rows_blocks(n) * groups : 0; }

hipError_t launch_group_rows(const int *group, int n, int groups, int *offsets, int *order, int *place, uint32_t *hist, hipStream_t st)
{
    int bits = 0;
    while ((1 << bits) < groups) ++bits;
    const GroupRowsArgs a = {group, n, groups, bits, rows_blocks(n), offsets, order, place, hist};
    const int lds = (ROWS_WAVES * groups + ROWS_WAVES) * 4, most = (ROWS_WAVES * GROUP_ROWS_MAX + ROWS_WAVES) * 4;
    hipError_t e = ensure_max_lds(reinterpret_cast<const void *>(group_place_kernel), most);
    if (e != hipSuccess) return e;
    if (a.blocks > 1) {
        e = ensure_max_lds(reinterpret_cast<const void *>(group_hist_kernel), most);
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL(group_hist_kernel, dim3((unsigned)a.blocks), dim3(64 * ROWS_WAVES), lds, st, a);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(group_place_kernel, dim3((unsigned)a.blocks), dim3(64 * ROWS_WAVES), lds, st, a);
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

__global__ __launch_bounds__(256) void gather_rows_kernel(GatherArgs a)
{
    fetch_args<GatherArgs>();
    const int lane = threadIdx.x & 63, nch = (a.bytes + 15) / 16;
    for (long r = (long)blockIdx.x * 4 + (threadIdx.x >> 6); r < a.rows; r += (long)gridDim.x * 4) {
        const int i = a.order[r], t = i / a.topk;
        if (i < 0 || t >= a.tokens) continue;
        const uint8_t *src = a.X + t * a.ldx;
        uint8_t *dst = a.Y + r * a.ldy;
        for (int c = lane; c < nch; c += 64) {
            const i32x4 v = *reinterpret_cast<const i32x4 *>(src + (long)c * 16);
            const int n = a.bytes - c * 16;
            if (n >= 16) *reinterpret_cast<i32x4 *>(dst + (long)c * 16) = v;
            else for (int b = 0; b < n; ++b) dst[(long)c * 16 + b] = (uint8_t)((uint32_t)v[b >> 2] >> (8 * (b & 3)));
        }
    }
}

hipError_t launch_gather_rows(int es, const void *X, int tokens, int cols, long ldx, const int *order, int rows, int topk, void *Y, long ldy, hipStream_t st)
{
    const GatherArgs a = {(const uint8_t *)X, (uint8_t *)Y, order, tokens, rows, topk, cols * es, ldx, ldy};
    const long wgs = ((long)rows + 3) / 4;
    hipLaunchKernelGGL(gather_rows_kernel, dim3((unsigned)(wgs < MAX_GRID_X ? wgs : MAX_GRID_X)), dim3(256), 0, st, a);
    return hipGetLastError();
}

// ---------------------------------------------------------------- and back to their tokens
// 16 bytes of a row to a lane.  Sums in fp32, in the order of a token's choices, the base first.
__device__ __forceinline__ void put_chunk(uint8_t *dst, const uint32_t (&o)[4], int n)        // n: elements of the chunk inside the row
{
    if (n >= 8) *reinterpret_cast<i32x4 *>(dst) = i32x4{(int)o[0], (int)o[1], (int)o[2], (int)o[3]};
    else for (int e = 0; e < n; ++e) reinterpret_cast<uint16_t *>(dst)[e] = (uint16_t)(o[e >> 1] >> (16 * (e & 1)));
}

template <int DT> __global__ __launch_bounds__(256) void combine_rows_kernel(CombineArgs a)
{
    using T = Traits<DT>;
    fetch_args<CombineArgs>();
    const int lane = threadIdx.x & 63, nch = (a.cols + 7) / 8, slices = (nch + 63) / 64;
    const long items = (long)a.tokens * slices;
    for (long it = (long)blockIdx.x * 4 + (threadIdx.x >> 6); it < items; it += (long)gridDim.x * 4) {
        const int t = (int)(it / slices), c = (int)(it - (long)t * slices) * 64 + lane;
        if (c >= nch) continue;
        float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (a.base) {
            const i32x4 v = *reinterpret_cast<const i32x4 *>(a.base + t * a.ldb + (long)c * 16);
#pragma unroll
            for (int e = 0; e < 8; ++e) s[e] = (float)T::elem(v, e);
        }
        for (int j = 0; j < a.topk; ++j) {
            const int r = a.place[(long)t * a.topk + j];
            if (r < 0 || r >= a.rows) continue;
            const float w = a.weight ? a.weight[(long)t * a.topk + j] : 1.f;
            const i32x4 v = *reinterpret_cast<const i32x4 *>(a.Y + r * a.ldy + (long)c * 16);
#pragma unroll
            for (int e = 0; e < 8; ++e) s[e] = __builtin_fmaf(w, (float)T::elem(v, e), s[e]);
        }
        uint32_t o[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = pack2<DT>(s[2 * e], s[2 * e + 1]);
        put_chunk(a.out + t * a.ldo + (long)c * 16, o, a.cols - c * 8);
    }
}

// The gradient, a wave to a token: dY[row] = w dout, dweight = dout . Y[row], summed in fp32 by a lane's chunks, then over the lanes.
template <int DT> __global__ __launch_bounds__(256) void combine_grad_kernel(CombineArgs a)
{
    using T = Traits<DT>;
    fetch_args<CombineArgs>();
    const int lane = threadIdx.x & 63, nch = (a.cols + 7) / 8;
    for (long t = (long)blockIdx.x * 4 + (threadIdx.x >> 6); t < a.tokens; t += (long)gridDim.x * 4) {
        for (int j = 0; j < a.topk; ++j) {
            const int r = a.place[t * a.topk + j];
            const bool in = r >= 0 && r < a.rows;
            float dot = 0.f;
            if (in) {
                const float w = a.weight ? a.weight[t * a.topk + j] : 1.f;
                for (int c = lane; c < nch; c += 64) {
                    const int n = a.cols - c * 8;
                    const i32x4 d = mask_chunk(*reinterpret_cast<const i32x4 *>(a.dout + t * a.ldo + (long)c * 16), 2 * n);
                    float x[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = (float)T::elem(d, e);
                    if (a.dweight) {
                        const i32x4 y = mask_chunk(*reinterpret_cast<const i32x4 *>(a.Y + r * a.ldy + (long)c * 16), 2 * n);
#pragma unroll
                        for (int e = 0; e < 8; ++e) dot = __builtin_fmaf(x[e], (float)T::elem(y, e), dot);
                    }
                    uint32_t o[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[e] = pack2<DT>(w * x[2 * e], w * x[2 * e + 1]);
                    if (a.dY) put_chunk(a.dY + r * a.lddy + (long)c * 16, o, n);
                }
            }
            if (a.dweight) {
                dot = wave_sum(dot);
                if (lane == 0) a.dweight[t * a.topk + j] = in ? dot : 0.f;
            }
        }
    }
}

hipError_t launch_combine_rows(int dt, bool grad, const CombineArgs &a, hipStream_t st)
{
    const long slices = ((a.cols + 7) / 8 + 63) / 64, items = grad ? a.tokens : a.tokens * slices, wgs = (items + 3) / 4;
    const dim3 grid((unsigned)(wgs < MAX_GRID_X ? wgs : MAX_GRID_X));
    if (grad) {
        if (dt == DT_BF16) hipLaunchKernelGGL(combine_grad_kernel<DT_BF16>, grid, dim3(256), 0, st, a);
        else               hipLaunchKernelGGL(combine_grad_kernel<DT_F16>, grid, dim3(256), 0, st, a);
    } else {
        if (dt == DT_BF16) hipLaunchKernelGGL(combine_rows_kernel<DT_BF16>, grid, dim3(256), 0, st, a);
        else               hipLaunchKernelGGL(combine_rows_kernel<DT_F16>, grid, dim3(256), 0, st, a);
    }
    return hipGetLastError();
}

}  // namespace abft
