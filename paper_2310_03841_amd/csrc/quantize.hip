// Rows (tokens) of a 16-bit type to int8 with a scale each: scale = max|x| / 127, q = 127 x / max|x| rounded to nearest even.
//
// x times 127 / max|x|, the factor rounded to fp32 and the product where it becomes an integer, is off by at most 2^-24 of itself ahead of that.  A quotient of
// [2^j, 2^(j+1)) that is not a tie lies at least 2^(j-20) away from one, as x has at most 8 - j binary places fewer than max|x| and both have
// 11 bits: it goes the right way.  Where the nearest integer is almost a half away a tie may be meant, and a division decides, of 127 x (18 significant
// bits: exact) by max|x| with one rounding, which moves it by 2^(j-24) at most and keeps ties; so it does in rows of very large or very small
// values, which are multiplied by a power of two for it.  The result is the one of exact arithmetic.
//
// Bound by memory: two bytes read and one written per element.  A wave takes a row, 16 bytes of it to a lane and load, and keeps it in
// registers between its maximum and its quotients.  (A division to every element, some 14 instructions: bf16 12608 x 3072 33.9 us,
// 25.2 so.  Stores that bypass the caches: 28.1 -> 25.8 on the card for the kernel alone, but the product that reads Q behind it waits for it: both
// together 50432 x 768 by 768 64.5 -> 70, 4096 x 1024 by 1024 17.5 -> 18.2.)
#include "abft_device.h"
#include "group_args.h"

namespace abft {

struct QuantArgs {
    const uint8_t *X;
    uint8_t *Q;
    float *scale;
    int rows, cols;
    long ldx, ldq;                        // elements
};

// NC: chunks of 16 bytes of a row that a lane keeps; a row has at most 64 NC of them, or (LONG) more, and then is read twice.
template <int DT, int NC, bool LONG>
__global__ __launch_bounds__(256) void quantize_kernel(QuantArgs a)
{
    using T = Traits<DT>;
    fetch_args<QuantArgs>();
    constexpr uint32_t INF_BITS = DT == DT_BF16 ? 0x7F80u : 0x7C00u;
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
    const int lane = threadIdx.x & 63;
    const int nch = (a.cols + 7) / 8;
    for (long r = (long)blockIdx.x * 4 + (threadIdx.x >> 6); r < a.rows; r += (long)gridDim.x * 4) {
        const uint8_t *src = a.X + r * a.ldx * 2;
        uint8_t *dst = a.Q + r * a.ldq;
        i32x4 x[NC];
        u16x2 m2 = {0, 0};
        auto load = [&](int c0) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < NC; ++i) {
                const int c = c0 + 64 * i + lane;
                x[i] = *reinterpret_cast<const i32x4 *>(src + (long)(c < nch ? c : nch - 1) * 16);
            }
#pragma unroll
            for (int i = 0; i < NC; ++i) {
                const int c = c0 + 64 * i + lane;
                if (c >= nch - 1) x[i] = mask_chunk(x[i], c < nch ? (a.cols - c * 8) * 2 : 0);
            }
        };
        auto largest = [&]() __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < NC; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) m2 = __builtin_elementwise_max(m2, __builtin_bit_cast(u16x2, x[i][e] & 0x7FFF7FFF));
        };
        if constexpr (LONG) {
            for (int c0 = 0; c0 < nch; c0 += 64 * NC) {
                load(c0);
                largest();
            }
        } else {
            load(0);
            largest();
        }
        const uint32_t top = wave_max_u32(m2[0] > m2[1] ? m2[0] : m2[1]);
        // a row with an Inf or a NaN has no scale: NaN, so that nothing made of it looks sound, and zeros
        const bool sound = top < INF_BITS;
        const float amax = DT == DT_BF16 ? bf16_bits_to_f32(top) : f16_bits_to_f32(top);
        if (lane == 0) a.scale[r] = sound ? __fdiv_rn(amax, 127.f) : __builtin_nanf("");
        const bool any = sound && top != 0u;
        const float power = DT == DT_F16 ? 1.f : amax >= 0x1p64f ? 0x1p-64f : amax < 0x1p-64f ? 0x1p64f : 1.f;
        constexpr float MAGIC = 0x1.8p23f;
        const float unit = 127.f * power, over = amax * power, factor = any ? __fdiv_rn(127.f, over) : 0.f;
        auto put = [&](int c0) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < NC; ++i) {
                const int c = c0 + 64 * i + lane;
                // an integer in the low bits of 1.5 2^23 and it
                float r[8], far = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float v = (float)T::elem(x[i], e);
                    r[e] = __builtin_fmaf(v, factor, MAGIC);
                    far = fmaxf(far, fabsf(__builtin_fmaf(v, factor, MAGIC - r[e])));
                }
                if (__builtin_expect(__any(far > 0.5f - 0x1p-14f) || power != 1.f, 0)) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) r[e] = MAGIC + __builtin_rintf(__fdiv_rn(unit * (float)T::elem(x[i], e), over));
                }
                uint32_t w[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    auto bits = [&](int e) __attribute__((always_inline)) { return __float_as_uint(r[4 * h + e]); };
                    const uint32_t lo = __builtin_amdgcn_perm(bits(1), bits(0), 0x0C0C0400u), hi = __builtin_amdgcn_perm(bits(3), bits(2), 0x0C0C0400u);
                    w[h] = any ? __builtin_amdgcn_perm(hi, lo, 0x05040100u) : 0u;
                }
                const int n = a.cols - c * 8;                    // elements of the chunk inside the row
                if (n >= 8) {
                    *reinterpret_cast<uint2 *>(dst + (long)c * 8) = make_uint2(w[0], w[1]);
                } else {
                    for (int e = 0; e < n; ++e) dst[(long)c * 8 + e] = (uint8_t)(w[e >> 2] >> (8 * (e & 3)));
                }
            }
        };
        if constexpr (LONG) {
            for (int c0 = 0; c0 < nch; c0 += 64 * NC) {
                load(c0);
                put(c0);
            }
        } else {
            put(0);
        }
    }
}

template <int DT> static hipError_t launch_quantize_type(const QuantArgs &a, hipStream_t st)
{
    const int nch = (a.cols + 7) / 8;
    const long wgs = ((long)a.rows + 3) / 4;
    const dim3 grid((unsigned)(wgs < MAX_GRID_X ? wgs : MAX_GRID_X));
    if (nch <= 64)       hipLaunchKernelGGL((quantize_kernel<DT, 1, false>), grid, dim3(256), 0, st, a);
    else if (nch <= 128) hipLaunchKernelGGL((quantize_kernel<DT, 2, false>), grid, dim3(256), 0, st, a);
    else if (nch <= 192) hipLaunchKernelGGL((quantize_kernel<DT, 3, false>), grid, dim3(256), 0, st, a);
    else if (nch <= 256) hipLaunchKernelGGL((quantize_kernel<DT, 4, false>), grid, dim3(256), 0, st, a);
    else if (nch <= 384) hipLaunchKernelGGL((quantize_kernel<DT, 6, false>), grid, dim3(256), 0, st, a);
    else if (nch <= 512) hipLaunchKernelGGL((quantize_kernel<DT, 8, false>), grid, dim3(256), 0, st, a);
    else                 hipLaunchKernelGGL((quantize_kernel<DT, 8, true>), grid, dim3(256), 0, st, a);
    return hipGetLastError();
}

hipError_t launch_quantize_rows(int dt, const void *X, int rows, int cols, long ldx, void *Q, long ldq, float *scale, hipStream_t st)
{
    const QuantArgs a = {(const uint8_t *)X, (uint8_t *)Q, scale, rows, cols, ldx, ldq};
    return dt == DT_BF16 ? launch_quantize_type<DT_BF16>(a, st) : launch_quantize_type<DT_F16>(a, st);
}

}  // namespace abft
