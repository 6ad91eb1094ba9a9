// Rows of a 16-bit type to 4-bit floating point in blocks of 32 with a power of two each, and back.
//
// A block's power of two is 2^e, e the exponent of its largest magnitude less 2, that of the largest element 6 = 1.5 2^2 (not below -127); x 2^-e goes to
// the nearest element, ties to the even code, and what lies above 6 (up to 8) to 6.  x 2^-e is exact, so one rounding is all there is.
//
// Bound by memory: two bytes read and about half a byte written per element, and the other way round.  Four lanes to a block, 16 bytes of the 16-bit row each, all of a row's loads
// ahead.  12608 rows of 4096 bf16, gathered from 6304 tokens: 28 us (52 MB read, most of it twice, 27 written), and back 22 us (131 MB, 6.0 TB/s); both in turn
// 50 us, with elements found by comparisons and fewer loads on their way 75.  Stores past the caches gain nothing.
#include "abft_device.h"
#include "gemm_epilogue.h"
#include "mx4_device.h"
#include "route_args.h"

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

// Sixteen bytes of the 16-bit row to 4 bytes of codes, by the conversions of gfx950: one rounding to nearest even of x / unit, magnitudes above 6 to 6, the sign kept.
template <int DT> __device__ __forceinline__ uint32_t to_codes(const i32x4 &x, float unit)
{
    uint32_t w = 0;
    // (as words of their own: the built-in cast of a vector's element takes the first one)
    const int x0 = x[0], x1 = x[1], x2 = x[2], x3 = x[3];
    if constexpr (DT == DT_BF16) {
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2_t, x0), unit, 0);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2_t, x1), unit, 1);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2_t, x2), unit, 2);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2_t, x3), unit, 3);
    } else {
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(w, __builtin_bit_cast(f16x2_t, x0), unit, 0);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(w, __builtin_bit_cast(f16x2_t, x1), unit, 1);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(w, __builtin_bit_cast(f16x2_t, x2), unit, 2);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(w, __builtin_bit_cast(f16x2_t, x3), unit, 3);
    }
    return w;
}
// And back, rounded once.
template <int DT> __device__ __forceinline__ i32x4 from_codes(uint32_t w, float unit)
{
    i32x4 o;
    if constexpr (DT == DT_BF16) {
        o[0] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, unit, 0));
        o[1] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, unit, 1));
        o[2] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, unit, 2));
        o[3] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, unit, 3));
    } else {
        o[0] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, unit, 0));
        o[1] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, unit, 1));
        o[2] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, unit, 2));
        o[3] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, unit, 3));
    }
    return o;
}

// LPR: lanes to a row; NC: chunks of 16 bytes (quarters of a block) that a lane has on their way
template <int DT, int LPR, int NC> __global__ __launch_bounds__(256) void mx4_quantize_kernel(Mx4RowArgs a)
{
    fetch_args<Mx4RowArgs>();
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
    constexpr int EXP = DT == DT_BF16 ? 7 : 10, TOP = DT == DT_BF16 ? 255 : 31;      // place of the exponent, that of Inf and NaN
    const int l = threadIdx.x % LPR;
    const int nq = (a.cols + 31) / 32 * 4, nch = (a.cols + 7) / 8;               // quarters of blocks, chunks of the row
    const long r = flat_block() * (256 / LPR) + threadIdx.x / LPR;
    const int t = r < a.rows ? source_row(a.order, a.tokens, a.topk, (int)r) : -1;
    if (t < 0) return;                                           // (all lanes of a row together)
    const uint8_t *src = a.X + t * a.ldx;
    for (int c0 = 0; c0 < nq; c0 += LPR * NC) {
        i32x4 x[NC];
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            const int c = c0 + LPR * i + l;
            x[i] = *reinterpret_cast<const i32x4 *>(src + (long)(c < nch ? c : nch - 1) * 16);
        }
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            const int c = c0 + LPR * i + l;
            if (c >= nch - 1) x[i] = mask_chunk(x[i], c < nch ? (a.cols - c * 8) * 2 : 0);
            u16x2 m2 = {0, 0};
#pragma unroll
            for (int e = 0; e < 4; ++e) m2 = __builtin_elementwise_max(m2, __builtin_bit_cast(u16x2, x[i][e] & 0x7FFF7FFF));
            uint32_t top = m2[0] > m2[1] ? m2[0] : m2[1];
            auto up = [&](uint32_t w) __attribute__((always_inline)) { top = w > top ? w : top; };
            up((uint32_t)dpp_mov<0xB1>((int)top));                               // lane ^ 1
            up((uint32_t)dpp_mov<0x4E>((int)top));                               // lane ^ 2
            // the exponent of the largest as fp32 has it (an fp16 number that is not normal becomes one), less two
            const bool sound = (int)(top >> EXP) < TOP;
            const int field = (int)(__float_as_uint(DT == DT_BF16 ? bf16_bits_to_f32(top) : f16_bits_to_f32(top)) >> 23);
            const uint32_t s = !sound ? 255u : field > 2 ? (uint32_t)(field - 2) : 0u;
            const uint32_t w = sound ? to_codes<DT>(x[i], mx4_unit(s)) : 0u;
            if (c < nq) {
                *reinterpret_cast<uint32_t *>(a.Q + r * a.ldq + (long)c * 4) = w;
                if ((l & 3) == 0) a.S[r * a.lds + (c >> 2)] = (uint8_t)s;
            }
        }
    }
}

template <int DT, int LPR, int NC> __global__ __launch_bounds__(256) void mx4_dequantize_kernel(Mx4RowArgs a)
{
    fetch_args<Mx4RowArgs>();
    const int l = threadIdx.x % LPR, nch = (a.cols + 7) / 8;
    const long r = flat_block() * (256 / LPR) + threadIdx.x / LPR;
    if (r >= a.rows) return;
    const uint8_t *src = a.Q + r * a.ldq, *sc = a.S + r * a.lds;
    uint8_t *dst = const_cast<uint8_t *>(a.X) + r * a.ldx;
    for (int c0 = 0; c0 < nch; c0 += LPR * NC) {
        uint32_t w[NC], s[NC];
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            const int c = min(c0 + LPR * i + l, nch - 1);
            w[i] = *reinterpret_cast<const uint32_t *>(src + (long)c * 4);
            s[i] = sc[c >> 2];
        }
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            const int c = c0 + LPR * i + l, n = a.cols - c * 8;                  // elements of the chunk inside the row
            i32x4 o = from_codes<DT>(w[i], mx4_unit(s[i]));
            if (s[i] == 255u) o = DT == DT_BF16 ? i32x4{0x7FC07FC0, 0x7FC07FC0, 0x7FC07FC0, 0x7FC07FC0} : i32x4{0x7E007E00, 0x7E007E00, 0x7E007E00, 0x7E007E00};
            if (n >= 8) *reinterpret_cast<i32x4 *>(dst + (long)c * 16) = o;
            else for (int e = 0; e < n; ++e) reinterpret_cast<uint16_t *>(dst + (long)c * 16)[e] = (uint16_t)((uint32_t)o[e >> 1] >> (16 * (e & 1)));
        }
    }
}

// Lanes for a row's chunks, several rows to a wave where those are few, and up to eight chunks of a lane on their way.
template <template <int, int> class LAUNCH> static hipError_t launch_rows4(const Mx4RowArgs &a, hipStream_t st)
{
    const int nq = (a.cols + 31) / 32 * 4;
    if (nq <= 8)   return LAUNCH<8, 1>::go(a, st);
    if (nq <= 16)  return LAUNCH<16, 1>::go(a, st);
    if (nq <= 32)  return LAUNCH<32, 1>::go(a, st);
    if (nq <= 64)  return LAUNCH<64, 1>::go(a, st);
    if (nq <= 128) return LAUNCH<64, 2>::go(a, st);
    if (nq <= 256) return LAUNCH<64, 4>::go(a, st);
    return LAUNCH<64, 8>::go(a, st);
}
template <int DT> struct Quantize {
    template <int LPR, int NC> struct Launch {
        static hipError_t go(const Mx4RowArgs &a, hipStream_t st)
        {
            hipLaunchKernelGGL((mx4_quantize_kernel<DT, LPR, NC>), flat_grid(((long)a.rows + 256 / LPR - 1) / (256 / LPR)), dim3(256), 0, st, a);
            return hipGetLastError();
        }
    };
};
template <int DT> struct Dequantize {
    template <int LPR, int NC> struct Launch {
        static hipError_t go(const Mx4RowArgs &a, hipStream_t st)
        {
            hipLaunchKernelGGL((mx4_dequantize_kernel<DT, LPR, NC>), flat_grid(((long)a.rows + 256 / LPR - 1) / (256 / LPR)), dim3(256), 0, st, a);
            return hipGetLastError();
        }
    };
};

hipError_t launch_quantize_mx4(int dt, const void *X, int tokens, int cols, long ldx, const int *order, int rows, int topk, void *Q, long ldq, void *S, long lds, hipStream_t st)
{
    const Mx4RowArgs a = {(const uint8_t *)X, (uint8_t *)Q, (uint8_t *)S, order, tokens, rows, cols, topk, ldx, ldq, lds};
    return dt == DT_BF16 ? launch_rows4<Quantize<DT_BF16>::Launch>(a, st) : launch_rows4<Quantize<DT_F16>::Launch>(a, st);
}

hipError_t launch_dequantize_mx4(int dt, const void *Q, long ldq, const void *S, long lds, int rows, int cols, void *X, long ldx, hipStream_t st)
{
    const Mx4RowArgs a = {(const uint8_t *)X, (uint8_t *)const_cast<void *>(Q), (uint8_t *)const_cast<void *>(S), nullptr, rows, rows, cols, 1, ldx, ldq, lds};
    return dt == DT_BF16 ? launch_rows4<Dequantize<DT_BF16>::Launch>(a, st) : launch_rows4<Dequantize<DT_F16>::Launch>(a, st);
}

}  // namespace abft
