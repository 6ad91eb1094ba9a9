// Behind a protected product over groups (gemm_group.hip), which has left e^T A and max|A| of each group, the row predictions and the observed
// sums: the column prediction of each group, a B from one read of its matrix, the comparisons, flags and counts (Sec. III-B.1, item (2)).
#include <type_traits>

#include "abft_device.h"
#include "check_dots.h"
#include "gemm_mx4.h"
#include "group_args.h"
#include "mx4_device.h"

namespace abft {

struct GroupCheckArgs {
    const uint8_t *B;
    const int *offsets;
    int M, N, K, groups;
    long ldb, sB;
    const uint32_t *a_sum, *a_max, *b_max;
    uint32_t *cc_obs, *rc_obs, *cc_pred;
    const uint32_t *rc_pred;
    const double *cc_acc, *rc_acc;
    const uint32_t *shares;               // COLS_MARKED: of the observed sums of rows, [(N + 15) / 16][M]
    float tau_k, tau_override, tau_override_cols;      // 1e-3 K
    uint8_t *row_flag, *col_flag;
    uint32_t *counts;
    int row_units, col_units;             // of 256 rows each, COLS_MARKED: four; per group
    uint32_t *zero_ptr, *zero2_ptr;       // regions for calls to come, which every workgroup helps to clear
    size_t zero_words, zero2_words;
};

// 4-bit operands: ldb, sB and K in bytes, as Mx4Args has them
struct Mx4CheckArgs : GroupCheckArgs {
    const uint8_t *sb;
    long ld_sb, stride_sb;
};
template <int DT> struct GroupCheckArgsOf { typedef GroupCheckArgs type; };
template <> struct GroupCheckArgsOf<DT_MX4> { typedef Mx4CheckArgs type; };

// Dots of RW rows of 4-bit B with a vector of 2 K terms, by vector instructions: a block of a row to a lane, and the vector's 32 terms of it in registers, 64 blocks at a time.
template <int RW> __device__ __forceinline__ void mx4_row_dots(const uint8_t *X, long ld, const uint8_t *S, long lds, int row0, int rows, int K, const uint32_t *vec, float (&dot)[RW])
{
    const int lane = threadIdx.x & 63, nb = K / 16;
#pragma unroll
    for (int j = 0; j < RW; ++j) dot[j] = 0.f;
    for (int b0 = 0; b0 < nb; b0 += 64) {
        const int at = min(b0 + lane, nb - 1);
        i32x4 v[RW];
        uint32_t s[RW];
#pragma unroll
        for (int j = 0; j < RW; ++j) {
            const long r = min(row0 + j, rows - 1);
            v[j] = *reinterpret_cast<const i32x4 *>(X + r * ld + at * 16);
            s[j] = S[r * lds + at];
        }
        float a[32];
#pragma unroll
        for (int q4 = 0; q4 < 8; ++q4) {
            const i32x4_word w = *reinterpret_cast<const i32x4_word *>(vec + at * 32 + 4 * q4);
#pragma unroll
            for (int i = 0; i < 4; ++i) a[4 * q4 + i] = b0 + lane < nb ? __uint_as_float((uint32_t)w[i]) : 0.f;
        }
#pragma unroll
        for (int j = 0; j < RW; ++j) {
            float x[32];
            mx4_values(v[j], mx4_unit(s[j]), x);
#pragma unroll
            for (int q = 0; q < 32; ++q) dot[j] = __builtin_fmaf(x[q], a[q], dot[j]);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
#pragma unroll
    for (int j = 0; j < RW; ++j) dot[j] = wave_sum(dot[j]);
}

// The same of sixteen rows, by MFMAs, of up to 32 blocks: the vector in terms of 8 bits in LDS, for all four waves, and every load of B ahead of them.  p[i]: the dot of row
// row0 + 4 (lane / 16) + i.  (By vector instructions / so, us: 16 groups of 4096 x 1024, the kernel 11.0 / 9.5; the protected call of 3000 x 1000 x 96 in 4 12.4 / 11.2; in windows of 32 blocks, where rows are
// deeper and workgroups few, that of 6000 x 1024 x 4096 in 8 39.5 / 46.4.)
constexpr int DOTS_BLOCKS = 32, DOTS_ROWS = 16;
__device__ __forceinline__ void mx4_tile_dots(const uint8_t *X, long ld, const uint8_t *S, long lds, int row0, int rows, int K, const uint32_t *vec, uint8_t *smem, float (&p)[4])
{
    static_assert(DOTS_BLOCKS * 8 == 256, "four terms of the vector to a thread");
    const int tid = threadIdx.x, lane = tid & 63, piece = lane >> 4, nb = K / 16;
    const long r = min(row0 + (lane & 15), rows - 1);
    const uint8_t *const src = X + r * ld, *const sc = S + r * lds;
    uint8_t *const terms = smem, *const powers = smem + DOTS_BLOCKS * TERMS * 32;
    const i32x4_word a = *reinterpret_cast<const i32x4_word *>(vec + min(tid, nb * 8 - 1) * 4);
    i32x4 b[DOTS_BLOCKS / 4];
    uint2 s[DOTS_BLOCKS / 8];
#pragma unroll
    for (int u = 0; u < DOTS_BLOCKS / 4; ++u) {
        if (4 * u >= nb) break;
        const int over = 4 * u + 4 <= nb ? 0 : max(4 * u + piece - (nb - 1), 0);             // (of the last four blocks alone)
        b[u] = *reinterpret_cast<const i32x4 *>(src + (4 * u + piece - over) * 16);
    }
    // (rows of powers of two are whole 16 bytes)
#pragma unroll
    for (int u = 0; u < DOTS_BLOCKS / 8; ++u) {
        if (8 * u >= nb) break;
        s[u] = *reinterpret_cast<const uint2 *>(sc + 8 * u);
    }
    f32x4 v;
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q] = __uint_as_float((uint32_t)a[q]);
    if (tid < nb * 8) mx4_put_terms(v, tid & 7, terms + (tid >> 3) * TERMS * 32, powers + (tid >> 3) * 8);
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");         // (over LDS alone: B may still be on its way)
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int u = 0; u < DOTS_BLOCKS / 4; ++u) {
        if (4 * u >= nb) break;
        // past the last block nothing is multiplied, whatever it holds
        const bool in = 4 * u + piece < nb;
        const i32x4 bv = in ? b[u] : i32x4{0, 0, 0, 0};
        const uint32_t bsv = in ? ((u & 1 ? s[u >> 1].y : s[u >> 1].x) >> (8 * piece)) & 0xFFu : 0u;
        i32x8 ev;
        uint32_t esv;
        mx4_get_terms(terms, powers, 4 * u, nb, lane, ev, esv);
        acc = mfma16_mx4_f8(bv, ev, acc, bsv, esv);
        __builtin_amdgcn_sched_barrier(0);                       // (terms of one step at a time in registers)
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = row16_sum(acc[i]);        // (of the terms)
}

constexpr int GCHK_KN_LANES = 4;          // chunk columns of a unit over a B stored K x N (64 lanes run along k)

// What is left to do of the columns: their predictions from B stored N x K or K x N, or nothing but to write down what the product's kernel marked.
enum { COLS_NK, COLS_KN, COLS_MARKED };

// RW: rows of B to a wave (4 bits: sixteen are a tile of MFMAs)
template <int DT, int RW, int COLS>
__global__ __launch_bounds__(256) void group_check_kernel(typename GroupCheckArgsOf<DT>::type f)
{
    using T = Traits<DT>;
    typedef typename T::acc_t acc_t;
    constexpr bool MX4 = DT == DT_MX4;
    static_assert(!MX4 || COLS == COLS_NK, "4-bit B is stored N x K");
    constexpr int ES = T::ES, CE = 16 / ES;
    __shared__ acc_t part[4][GCHK_KN_LANES * CE];
    fetch_args<typename GroupCheckArgsOf<DT>::type>();
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    for (size_t i = (size_t)blockIdx.x * 256 + tid; i < f.zero_words; i += (size_t)gridDim.x * 256) f.zero_ptr[i] = 0u;
    for (size_t i = (size_t)blockIdx.x * 256 + tid; i < f.zero2_words; i += (size_t)gridDim.x * 256) f.zero2_ptr[i] = 0u;
    auto tolerance = [&](int e) __attribute__((always_inline)) {
        if (T::IS_INT) return 0.f;
        return f.tau_override > 0.f ? f.tau_override : f.tau_k * __uint_as_float(f.a_max[e]) * __uint_as_float(f.b_max[e]);
    };
    auto tolerance_cols = [&](int e) __attribute__((always_inline)) { return f.tau_override_cols > 0.f ? f.tau_override_cols : tolerance(e); };
    auto observed = [&](uint32_t *sum, const double *acc, long o) __attribute__((always_inline)) {
        if (T::IS_INT || !acc) return sum[o];
        const uint32_t w = __float_as_uint((float)acc[o]);
        sum[o] = w;
        return w;
    };
    int u = blockIdx.x;
    if (COLS == COLS_MARKED && u < f.row_units) {
        // a wave to a row: its shares, in doubles where they round
        const int r = u * 4 + wave, n = (f.N + 15) / 16;
        if (r >= f.M) return;
        int end;
        const int e = group_of(f.offsets, f.M, f.groups, r, &end);
        bool fl = false;
        if (e >= 0) {
            typename std::conditional<T::IS_INT, int, double>::type s = 0;
            for (int i = lane; i < n; i += 64) s += from_word<acc_t>(f.shares[(long)i * f.M + r]);
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) s += __shfl_xor(s, d);
            const uint32_t obs = as_word((acc_t)s);
            if (lane == 0) f.rc_obs[r] = obs;
            fl = mismatch<T::IS_INT>(obs, f.rc_pred[r], tolerance(e));
        }
        if (lane == 0) {
            f.row_flag[r] = fl ? 1 : 0;
            if (fl) report_flags(f.counts, 0, 1u);
        }
        return;
    }
    if (u < f.row_units) {
        const int r = u * 256 + tid;
        bool fl = false;
        if (r < f.M) {
            int end;
            const int e = group_of(f.offsets, f.M, f.groups, r, &end);
            if (e >= 0) fl = mismatch<T::IS_INT>(observed(f.rc_obs, f.rc_acc, r), f.rc_pred[r], tolerance(e));
            f.row_flag[r] = fl ? 1 : 0;
        }
        const unsigned nf = __popcll(__ballot(fl));
        if (nf && lane == 0) report_flags(f.counts, 0, nf);
        return;
    }
    u -= f.row_units;
    if constexpr (COLS == COLS_MARKED) {
        const int o = u * 256 + tid;                             // over all groups
        const bool fl = o < f.N * f.groups && f.cc_obs[o] != 0u;
        if (o < f.N * f.groups) f.col_flag[o] = fl ? 1 : 0;
        const unsigned nf = __popcll(__ballot(fl));
        if (nf && lane == 0) report_flags(f.counts, 1, nf);
        return;
    }
    const int e = u / f.col_units, unit = u - e * f.col_units;
    const int N = f.N, K = f.K;
    int first, rows;
    group_rows(f.offsets, f.M, e, &first, &rows);
    const uint8_t *Bb = f.B + (long)e * f.sB * ES;
    const uint32_t *asum = f.a_sum + (long)e * K * (MX4 ? 2 : 1);
    bool mine_ok = false;
    int n = 0;
    acc_t pred = T::zero();
    if constexpr (COLS == COLS_NK) {
        const int row0 = (unit * 4 + wave) * RW;
        if constexpr (MX4 && RW == DOTS_ROWS) {
            __shared__ __attribute__((aligned(16))) uint8_t smem[DOTS_BLOCKS * TERM_BYTES];
            const int i = lane & 15;
            n = row0 + 4 * (lane >> 4) + i;
            mine_ok = i < 4 && n < N;
            // (a group without rows: nothing of its matrix is read)
            if (rows > 0) {
                float dot[4];
                mx4_tile_dots(Bb, f.ldb, f.sb + (long)e * f.stride_sb, f.ld_sb, row0, N, K, asum, smem, dot);
#pragma unroll
                for (int j = 0; j < 4; ++j) pred = i == j ? dot[j] : pred;
            }
        } else {
            n = row0 + lane;
            mine_ok = lane < RW && n < N;
            if (rows > 0 && row0 < N) {
                acc_t dot[RW];
                if constexpr (MX4) mx4_row_dots<RW>(Bb, f.ldb, f.sb + (long)e * f.stride_sb, f.ld_sb, row0, N, K, asum, dot);
                else row_dots<DT, RW>(Bb, f.ldb, row0, N, K, asum, false, dot);
#pragma unroll
                for (int j = 0; j < RW; ++j) pred = lane == j ? dot[j] : pred;
            }
        }
    } else {
        const int cx = tid % GCHK_KN_LANES, ky = tid / GCHK_KN_LANES;
        const int col0 = unit * GCHK_KN_LANES * CE, nst = col0 + cx * CE;
        n = col0 + tid;
        mine_ok = tid < GCHK_KN_LANES * CE && n < N;
        if (rows > 0) {
            acc_t colp[CE];
#pragma unroll
            for (int q = 0; q < CE; ++q) colp[q] = T::zero();
            constexpr int U = 8;
            for (int k0 = ky; k0 < K; k0 += 64 * U) {
                i32x4 v[U];
                acc_t ak[U];
#pragma unroll
                for (int j = 0; j < U; ++j) {
                    const int k = min(k0 + 64 * j, K - 1);
                    v[j] = *reinterpret_cast<const i32x4 *>(Bb + ((long)k * f.ldb + (nst < N ? nst : 0)) * ES);
                    ak[j] = from_word<acc_t>(asum[k]);
                }
#pragma unroll
                for (int j = 0; j < U; ++j)
                    if (k0 + 64 * j < K) {
#pragma unroll
                        for (int q = 0; q < CE; ++q) colp[q] = add_t(colp[q], mul_t(T::elem(v[j], q), ak[j]));
                    }
            }
#pragma unroll
            for (int q = 0; q < CE; ++q) {
                acc_t t = colp[q];
                t = add_t(t, dpp_get<0x124>(t));                 // row_ror:4 inside 16 lanes
                t = add_t(t, dpp_get<0x128>(t));                 // row_ror:8
                t = add_xor16(t);
                t = add_xor32(t);
                if (lane < GCHK_KN_LANES) part[wave][cx * CE + q] = t;
            }
        }
        __syncthreads();
        if (rows > 0 && mine_ok) pred = add_t(add_t(part[0][tid], part[1][tid]), add_t(part[2][tid], part[3][tid]));
    }
    bool fl = false;
    if (mine_ok) {
        const long o = (long)e * N + n;
        f.cc_pred[o] = as_word(pred);
        const uint32_t obs = observed(f.cc_obs, f.cc_acc, o);
        fl = rows > 0 && mismatch<T::IS_INT>(obs, as_word(pred), tolerance_cols(e));
        f.col_flag[o] = fl ? 1 : 0;
    }
    const unsigned nf = __popcll(__ballot(fl));
    if (nf && lane == 0) report_flags(f.counts, 1, nf);
}

constexpr int GCHK_ROWS = 4;              // rows of B to a wave

// What all launches fill in alike.
static void check_args(GroupCheckArgs &f, const GroupArgs &g, float k, const Workspace &w, const Verdict &v, const OneLaunch &end)
{
    f.B = g.B; f.offsets = g.offsets;
    f.M = g.M; f.N = g.N; f.K = g.K; f.groups = g.groups; f.ldb = g.ldb; f.sB = g.sB;
    f.a_sum = g.a_sum; f.a_max = g.a_max; f.b_max = w.b_max;
    f.cc_obs = g.cc_obs; f.rc_obs = g.rc_obs; f.cc_pred = w.cc_pred; f.rc_pred = g.rc_pred;
    f.cc_acc = g.cc_acc; f.rc_acc = g.rc_acc; f.shares = group_few_shares(g);
    f.tau_k = 1e-3f * k; f.tau_override = v.tau_override; f.tau_override_cols = v.tau_override_cols;
    f.row_flag = v.row_flag; f.col_flag = v.col_flag; f.counts = v.counts;
    f.zero_ptr = end.zero_ptr; f.zero_words = end.zero_ptr ? end.zero_words : 0;
    f.zero2_ptr = end.zero2_ptr; f.zero2_words = end.zero2_ptr ? end.zero2_words : 0;
}

// Workgroups of a launch, at most 2^22 with rows (marked: of at most 2^21 rows) and 2^23 + 2^16 with columns, for up to 2^30 rows and 2^27 columns over all
// groups.  per: columns to a workgroup.
static dim3 check_grid(GroupCheckArgs &f, bool marked, int per)
{
    f.row_units = marked ? (f.M + 3) / 4 : (f.M + 255) / 256;
    f.col_units = (f.N + per - 1) / per;
    const long cols = (long)f.N * f.groups;
    return dim3((unsigned)(f.row_units + (marked ? (cols + 255) / 256 : (long)f.col_units * f.groups)));
}

hipError_t launch_group_check(int dt, const GroupKernel &k, const GroupArgs &g, bool transB, const Workspace &w, const Verdict &v, const OneLaunch &end, hipStream_t st)
{
    constexpr int RW = GCHK_ROWS;
    GroupCheckArgs f;
    check_args(f, g, (float)g.K, w, v, end);
    const bool marked = k.kind == GROUP_KERNEL_FEW;
    const dim3 grid = check_grid(f, marked, transB ? 4 * RW : GCHK_KN_LANES * (16 / elem_size(dt)));
#define GROUP_CHECK(DT) \
    if (marked)      hipLaunchKernelGGL((group_check_kernel<DT, RW, COLS_MARKED>), grid, dim3(256), 0, st, f); \
    else if (transB) hipLaunchKernelGGL((group_check_kernel<DT, RW, COLS_NK>), grid, dim3(256), 0, st, f); \
    else             hipLaunchKernelGGL((group_check_kernel<DT, RW, COLS_KN>), grid, dim3(256), 0, st, f)
    switch (dt) {
    case DT_I8:   GROUP_CHECK(DT_I8); break;
    case DT_BF16: GROUP_CHECK(DT_BF16); break;
    case DT_F16:  GROUP_CHECK(DT_F16); break;
    default: return hipErrorInvalidValue;
    }
#undef GROUP_CHECK
    return hipGetLastError();
}

hipError_t launch_mx4_check(const GroupKernel &k, const Mx4Args &g, int K, const Workspace &w, const Verdict &v, const OneLaunch &end, hipStream_t st)
{
    constexpr int DEEP = 8;                                      // rows to a wave where they are of more blocks than a tile's
    Mx4CheckArgs f;
    check_args(f, g, (float)K, w, v, end);
    f.sb = g.sb; f.ld_sb = g.ld_sb; f.stride_sb = g.stride_sb;
    const bool marked = k.kind == GROUP_KERNEL_FEW, deep = g.K / 16 > DOTS_BLOCKS;
    const dim3 grid = check_grid(f, marked, 4 * (deep ? DEEP : DOTS_ROWS));
    // (marked: fp32 sums and nothing of the operands)
    if (marked)    hipLaunchKernelGGL((group_check_kernel<DT_BF16, GCHK_ROWS, COLS_MARKED>), grid, dim3(256), 0, st, (const GroupCheckArgs &)f);
    else if (deep) hipLaunchKernelGGL((group_check_kernel<DT_MX4, DEEP, COLS_NK>), grid, dim3(256), 0, st, f);
    else           hipLaunchKernelGGL((group_check_kernel<DT_MX4, DOTS_ROWS, COLS_NK>), grid, dim3(256), 0, st, f);
    return hipGetLastError();
}

// ---- b = B e and max|B| of each group: a workgroup to 64 bytes (four blocks) of every row, sixteen rows of them to a wave at a time.  In a fixed order.  (16 waves, for what they have
// on their way together: 32 groups of 4096 x 1024 50 us with four.)
// zero: words that every workgroup helps to clear.
struct Mx4EncodeArgs {
    const uint8_t *B, *sb;
    int N, K;                             // K: bytes
    long ldb, sB, ld_sb, stride_sb;
    uint32_t *b_sum, *b_max;
    uint32_t *zero;
    size_t zero_words;
};
constexpr int ENCODE_WAVES = 16;
__global__ __launch_bounds__(64 * ENCODE_WAVES) void mx4_encode_kernel(Mx4EncodeArgs a)
{
    constexpr int W = ENCODE_WAVES, THREADS = 64 * W;
    __shared__ float part[W][4 * 32], tops[W];
    fetch_args<Mx4EncodeArgs>();
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const unsigned column = blockIdx.z * gridDim.x + blockIdx.x;         // four blocks of K each
    const size_t wg = ((size_t)blockIdx.z * gridDim.y + blockIdx.y) * gridDim.x + blockIdx.x, wgs = (size_t)gridDim.x * gridDim.y * gridDim.z;
    for (size_t i = wg * THREADS + tid; i < a.zero_words; i += wgs * THREADS) a.zero[i] = 0u;
    const int e = blockIdx.y, nb = a.K / 16, block = column * 4 + (tid & 3), at = min(block, nb - 1);
    const uint8_t *src = a.B + (long)e * a.sB + at * 16, *sc = a.sb + (long)e * a.stride_sb + at;
    float sum[32], top = 0.f;
#pragma unroll
    for (int q = 0; q < 32; ++q) sum[q] = 0.f;
    constexpr int U = 4;
    for (int r0 = tid >> 2; r0 < a.N; r0 += 16 * W * U) {
        i32x4 v[U];
        uint32_t s[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const long r = min(r0 + 16 * W * u, a.N - 1);
            v[u] = *reinterpret_cast<const i32x4 *>(src + r * a.ldb);
            s[u] = sc[r * a.ld_sb];
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (r0 + 16 * W * u >= a.N) break;
            float x[32];
            mx4_values(v[u], mx4_unit(s[u]), x);
#pragma unroll
            for (int q = 0; q < 32; ++q) {
                sum[q] += x[q];
                top = fmaxf(top, fabsf(x[q]));
            }
        }
    }
#pragma unroll
    for (int q = 0; q < 32; ++q) {
        float t = sum[q];
        t += dpp_get<0x124>(t);                                  // row_ror:4 inside 16 lanes
        t += dpp_get<0x128>(t);                                  // row_ror:8
        t = add_xor32(add_xor16(t));
        if (lane < 4) part[wave][lane * 32 + q] = t;
    }
    top = wave_max(block < nb ? top : 0.f);
    if (lane == 0) tops[wave] = top;
    __syncthreads();
    if (tid < 128 && column * 4 + (tid >> 5) < (unsigned)nb) {
        float t = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) t += part[w][tid];
        a.b_sum[(long)e * 2 * a.K + (long)column * 128 + tid] = __float_as_uint(t);
    }
    if (tid == 0) {
        float m = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) m = fmaxf(m, tops[w]);
        if (m > 0.f) atomicMax(a.b_max + e, __float_as_uint(m));
    }
}

hipError_t launch_mx4_encode(const Mx4Args &g, const Workspace &w, uint32_t *zero, size_t zero_words, hipStream_t st)
{
    const Mx4EncodeArgs a = {g.B, g.sb, g.N, g.K, g.ldb, g.sB, g.ld_sb, g.stride_sb, w.b_sum, w.b_max, zero, zero_words};
    // (up to 2^22 workgroups of 2^10 threads along K, which is more than one direction of a launch has)
    constexpr unsigned X = 1u << 21;
    const unsigned wgs = (unsigned)((g.K / 16 + 3) / 4);
    hipLaunchKernelGGL(mx4_encode_kernel, dim3(wgs < X ? wgs : X, (unsigned)g.groups, (wgs + X - 1) / X), dim3(64 * ENCODE_WAVES), 0, st, a);
    return hipGetLastError();
}

}  // namespace abft
