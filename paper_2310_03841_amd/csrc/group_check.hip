// Behind a protected product over groups (gemm_group.hip), which has left e^T A and max|A| of each group, the row predictions and the observed
// sums: the column prediction of each group, a B from one read of its matrix, the comparisons, flags and counts (Sec. III-B.1, item (2)).
#include <type_traits>

#include "abft_device.h"
#include "check_dots.h"
#include "group_args.h"

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
    float tau_override, tau_override_cols;
    uint8_t *row_flag, *col_flag;
    uint32_t *counts;
    int row_units, col_units;             // of 256 rows each, COLS_MARKED: four; per group
    uint32_t *zero_ptr, *zero2_ptr;       // regions for calls to come, which every workgroup helps to clear
    size_t zero_words, zero2_words;
};

constexpr int GCHK_KN_LANES = 4;          // chunk columns of a unit over a B stored K x N (64 lanes run along k)

// What is left to do of the columns: their predictions from B stored N x K or K x N, or nothing but to write down what the product's kernel marked.
enum { COLS_NK, COLS_KN, COLS_MARKED };

template <int DT, int RW, int COLS>
__global__ __launch_bounds__(256) void group_check_kernel(GroupCheckArgs f)
{
    using T = Traits<DT>;
    typedef typename T::acc_t acc_t;
    constexpr int ES = T::ES, CE = 16 / ES;
    __shared__ acc_t part[4][GCHK_KN_LANES * CE];
    fetch_args<GroupCheckArgs>();
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    for (size_t i = (size_t)blockIdx.x * 256 + tid; i < f.zero_words; i += (size_t)gridDim.x * 256) f.zero_ptr[i] = 0u;
    for (size_t i = (size_t)blockIdx.x * 256 + tid; i < f.zero2_words; i += (size_t)gridDim.x * 256) f.zero2_ptr[i] = 0u;
    auto tolerance = [&](int e) __attribute__((always_inline)) {
        if (T::IS_INT) return 0.f;
        return f.tau_override > 0.f ? f.tau_override : (1e-3f * (float)f.K) * __uint_as_float(f.a_max[e]) * __uint_as_float(f.b_max[e]);
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
    const uint32_t *asum = f.a_sum + (long)e * K;
    bool mine_ok = false;
    int n = 0;
    acc_t pred = T::zero();
    if constexpr (COLS == COLS_NK) {
        const int row0 = (unit * 4 + wave) * RW;
        n = row0 + lane;
        mine_ok = lane < RW && n < N;
        // (a group without rows: nothing of its matrix is read)
        if (rows > 0 && row0 < N) {
            acc_t dot[RW];
            row_dots<DT, RW>(Bb, f.ldb, row0, N, K, asum, false, dot);
#pragma unroll
            for (int j = 0; j < RW; ++j) pred = lane == j ? dot[j] : pred;
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

hipError_t launch_group_check(int dt, const GroupKernel &k, const GroupArgs &g, bool transB, const Workspace &w, const Verdict &v, const OneLaunch &end, hipStream_t st)
{
    constexpr int RW = 4;
    GroupCheckArgs f;
    f.B = g.B; f.offsets = g.offsets;
    f.M = g.M; f.N = g.N; f.K = g.K; f.groups = g.groups; f.ldb = g.ldb; f.sB = g.sB;
    f.a_sum = g.a_sum; f.a_max = g.a_max; f.b_max = w.b_max;
    f.cc_obs = g.cc_obs; f.rc_obs = g.rc_obs; f.cc_pred = w.cc_pred; f.rc_pred = g.rc_pred;
    f.cc_acc = g.cc_acc; f.rc_acc = g.rc_acc; f.shares = group_few_shares(g);
    f.tau_override = v.tau_override; f.tau_override_cols = v.tau_override_cols;
    f.row_flag = v.row_flag; f.col_flag = v.col_flag; f.counts = v.counts;
    f.zero_ptr = end.zero_ptr; f.zero_words = end.zero_ptr ? end.zero_words : 0;
    f.zero2_ptr = end.zero2_ptr; f.zero2_words = end.zero2_ptr ? end.zero2_words : 0;
    const bool marked = k.kind == GROUP_KERNEL_FEW;
    const int per = transB ? 4 * RW : GCHK_KN_LANES * (16 / elem_size(dt));
    f.row_units = marked ? (g.M + 3) / 4 : (g.M + 255) / 256;
    f.col_units = (g.N + per - 1) / per;
    // at most 2^22 units of rows (marked: of at most 2^21 rows) and 2^23 + 2^16 of columns, for up to 2^30 rows and 2^27 columns over all groups
    const long cols = (long)g.N * g.groups, units = f.row_units + (marked ? (cols + 255) / 256 : (long)f.col_units * g.groups);
    const dim3 grid((unsigned)units);
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

}  // namespace abft
