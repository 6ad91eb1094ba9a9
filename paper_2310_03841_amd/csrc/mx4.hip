// Rows of a 16-bit type to 4-bit floating point in blocks of 32 with a power of two each, and back.
//
// A block's power of two is 2^e, e the exponent of its largest magnitude less 2, that of the largest element 6 = 1.5 2^2 (not below -127); x 2^-e goes to
// the nearest element, ties to the even code, and what lies above 6 (up to 8) to 6.  x 2^-e is exact, so one rounding is all there is.
//
// Bound by memory: two bytes read and about half a byte written per element, and the other way round.  Four lanes to a block, 16 bytes of the 16-bit row each.
#include "abft_device.h"
#include "mx4_device.h"

namespace abft {

struct Mx4RowArgs {
    const uint8_t *X;
    uint8_t *Q, *S;
    const int *order;                     // row r of Q is row order[r] / topk of X; none: left as it is.  Null: row r
    int tokens, rows, cols, topk;
    long ldx, ldq, lds;                   // bytes
};

// The row of X that becomes row r, -1: none.
__device__ __forceinline__ int source_row(const int *order, int tokens, int topk, int r)
{
    if (!order) return r;
    const int i = order[r];
    const int t = i / topk;
    return i >= 0 && t < tokens ? t : -1;
}

template <int DT> __global__ __launch_bounds__(256) void mx4_quantize_kernel(Mx4RowArgs a)
{
    using T = Traits<DT>;
    fetch_args<Mx4RowArgs>();
    const int lane = threadIdx.x & 63;
    const int nq = (a.cols + 31) / 32 * 4, nch = (a.cols + 7) / 8;               // quarters of blocks, chunks of 16 bytes
    for (long r = (long)blockIdx.x * 4 + (threadIdx.x >> 6); r < a.rows; r += (long)gridDim.x * 4) {
        const int t = source_row(a.order, a.tokens, a.topk, (int)r);
        if (t < 0) continue;
        const uint8_t *src = a.X + t * a.ldx;
        for (int c0 = 0; c0 < nq; c0 += 64) {
            const int c = c0 + lane;
            i32x4 x = *reinterpret_cast<const i32x4 *>(src + (long)(c < nch ? c : nch - 1) * 16);
            if (c >= nch - 1) x = mask_chunk(x, c < nch ? (a.cols - c * 8) * 2 : 0);
            float v[8], top = 0.f;
            uint32_t bits = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                v[e] = (float)T::elem(x, e);
                const uint32_t m = __float_as_uint(v[e]) & 0x7FFFFFFFu;
                bits = m > bits ? m : bits;
            }
            auto up = [&](uint32_t w) __attribute__((always_inline)) { bits = w > bits ? w : bits; };
            up((uint32_t)dpp_mov<0xB1>((int)bits));                              // lane ^ 1
            up((uint32_t)dpp_mov<0x4E>((int)bits));                              // lane ^ 2
            (void)top;
            // (Inf and NaN have the largest exponent: 255, a block of NaN)
            const int field = (int)(bits >> 23), s = field == 255 ? 255 : field > 2 ? field - 2 : 0;
            uint32_t w = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float m = fabsf(__builtin_ldexpf(v[e], 127 - s));
                const uint32_t code = (m > 0.25f) + (m >= 0.75f) + (m > 1.25f) + (m >= 1.75f) + (m > 2.5f) + (m >= 3.5f) + (m > 5.f);
                w |= (code | (__float_as_uint(v[e]) >> 31 << 3)) << (4 * e);
            }
            if (s == 255) w = 0;
            if (c < nq) {
                *reinterpret_cast<uint32_t *>(a.Q + r * a.ldq + (long)c * 4) = w;
                if ((lane & 3) == 0) a.S[r * a.lds + (c >> 2)] = (uint8_t)s;
            }
        }
    }
}

template <int DT> __global__ __launch_bounds__(256) void mx4_dequantize_kernel(Mx4RowArgs a)
{
    fetch_args<Mx4RowArgs>();
    const int lane = threadIdx.x & 63, nch = (a.cols + 7) / 8;
    for (long r = (long)blockIdx.x * 4 + (threadIdx.x >> 6); r < a.rows; r += (long)gridDim.x * 4) {
        const uint8_t *src = a.Q + r * a.ldq, *sc = a.S + r * a.lds;
        uint8_t *dst = const_cast<uint8_t *>(a.X) + r * a.ldx;
        for (int c = lane; c < nch; c += 64) {
            const uint32_t w = *reinterpret_cast<const uint32_t *>(src + (long)c * 4), s = sc[c >> 2];
            uint32_t o[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float v[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint32_t code = w >> (8 * e + 4 * h) & 15u, mag = code & 7u;
                    const float m = mag < 2 ? 0.5f * (float)mag : __uint_as_float((126u + (mag >> 1)) << 23 | (mag & 1u) << 22);
                    const float x = s == 255u ? __builtin_nanf("") : __builtin_ldexpf(m, (int)s - 127);
                    v[h] = code & 8u ? -x : x;
                }
                o[e] = DT == DT_BF16 ? f32_to_bf16_bits(v[0]) | f32_to_bf16_bits(v[1]) << 16 : f32_to_f16_bits(v[0]) | f32_to_f16_bits(v[1]) << 16;
            }
            const int n = a.cols - c * 8;                        // elements of the chunk inside the row
            if (n >= 8) *reinterpret_cast<i32x4 *>(dst + (long)c * 16) = i32x4{(int)o[0], (int)o[1], (int)o[2], (int)o[3]};
            else for (int e = 0; e < n; ++e) reinterpret_cast<uint16_t *>(dst + (long)c * 16)[e] = (uint16_t)(o[e >> 1] >> (16 * (e & 1)));
        }
    }
}

static dim3 row_grid(int rows)
{
    const long wgs = ((long)rows + 3) / 4;
    return dim3((unsigned)(wgs < MAX_GRID_X ? wgs : MAX_GRID_X));
}

hipError_t launch_quantize_mx4(int dt, const void *X, int tokens, int cols, long ldx, const int *order, int rows, int topk, void *Q, long ldq, void *S, long lds, hipStream_t st)
{
    const Mx4RowArgs a = {(const uint8_t *)X, (uint8_t *)Q, (uint8_t *)S, order, tokens, rows, cols, topk, ldx, ldq, lds};
    if (dt == DT_BF16) hipLaunchKernelGGL(mx4_quantize_kernel<DT_BF16>, row_grid(rows), dim3(256), 0, st, a);
    else               hipLaunchKernelGGL(mx4_quantize_kernel<DT_F16>, row_grid(rows), dim3(256), 0, st, a);
    return hipGetLastError();
}

hipError_t launch_dequantize_mx4(int dt, const void *Q, long ldq, const void *S, long lds, int rows, int cols, void *X, long ldx, hipStream_t st)
{
    const Mx4RowArgs a = {(const uint8_t *)X, (uint8_t *)const_cast<void *>(Q), (uint8_t *)const_cast<void *>(S), nullptr, rows, rows, cols, 1, ldx, ldq, lds};
    if (dt == DT_BF16) hipLaunchKernelGGL(mx4_dequantize_kernel<DT_BF16>, row_grid(rows), dim3(256), 0, st, a);
    else               hipLaunchKernelGGL(mx4_dequantize_kernel<DT_F16>, row_grid(rows), dim3(256), 0, st, a);
    return hipGetLastError();
}

}  // namespace abft
