// 4-bit floating point in blocks of 32 that share a power of two: what its kernels share.
//
// An element is a sign, two bits of exponent and one of mantissa: 0, 1/2, 1, 3/2, 2, 3, 4, 6.  Two lie in a byte, the first in its low half.  A block's power of two
// is a byte, the exponent plus 127; 255 makes the block NaN.  Sixteen bytes are a block: what a lane of an MFMA takes, and its power of two is the lane's
// scale.
#pragma once
#include "abft_device.h"

namespace abft {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef short s16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

template <> struct Traits<DT_MX4> {
    typedef float acc_t;
    typedef f32x16 accv_t;
    static constexpr int ES = 1;       // a byte of two elements
    static constexpr bool IS_INT = false;
    __device__ static __forceinline__ acc_t zero() { return 0.f; }
};

__device__ __forceinline__ i32x8 mx4_operand(const i32x4 &v) { return __builtin_shufflevector(v, v, 0, 1, 2, 3, -1, -1, -1, -1); }

// BYTE: of the scale words, whose others are not looked at
template <int BYTE> __device__ __forceinline__ f32x16 mfma_mx4(const i32x4 &a, const i32x4 &b, const f32x16 &c, uint32_t sa, uint32_t sb)
{
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(mx4_operand(a), mx4_operand(b), c, 4, 4, BYTE, (int)sa, BYTE, (int)sb);
}
template <int BYTE> __device__ __forceinline__ f32x4 mfma16_mx4(const i32x4 &a, const i32x4 &b, const f32x4 &c, uint32_t sa, uint32_t sb)
{
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(mx4_operand(a), mx4_operand(b), c, 4, 4, BYTE, (int)sa, BYTE, (int)sb);
}

// b: of 8 bits (e4m3); a lane's first sixteen are those of half a block and its others of the block two on (lane 16 q + i: half q % 2 of block q / 2), its power of two that of
// block q all the same
__device__ __forceinline__ f32x4 mfma16_mx4_f8(const i32x4 &a, const i32x8 &b, const f32x4 &c, uint32_t sa, uint32_t sb)
{
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(mx4_operand(a), b, c, 4, 0, 0, (int)sa, 0, (int)sb);
}

// 2^(s - 127) as the conversions take it (they look at its exponent alone).
__device__ __forceinline__ float mx4_unit(uint32_t s) { return __uint_as_float(s << 23); }

// Four fp32 values of a block's 32, the others in the seven lanes beside this one (part: which of the eight), as terms of 8 bits (e4m3): each term has a power of two for the block, 2^-5 of
// the one before it.  The first takes the block's largest value, below 2^8 of its power, to within 2^3 of that, and each the rest of the one before in the same way: what is
// left behind is below 2^-25 of the largest.  A block with an Inf or a NaN is NaN.  terms: TERMS times 32 bytes; powers: TERMS bytes of eight.
constexpr int TERMS = 5, TERM_BYTES = TERMS * 32 + 8;        // LDS for a block
__device__ __forceinline__ void mx4_put_terms(f32x4 v, int part, uint8_t *terms, uint8_t *powers)
{
    uint32_t most = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) most = max(most, __float_as_uint(v[j]) & 0x7FFFFFFFu);
    most = max(most, (uint32_t)dpp_mov<0xB1>((int)most));            // lane ^ 1
    most = max(most, (uint32_t)dpp_mov<0x4E>((int)most));            // lane ^ 2
    most = max(most, (uint32_t)dpp_mov<0x141>((int)most));           // i <-> 7 - i inside 8 lanes
    const int field = (int)(most >> 23);
#pragma unroll
    for (int p = 0; p < TERMS; ++p) {
        const uint32_t power = field == 255 ? 255u : (uint32_t)max(field - 7 - 5 * p, 0);
        const float unit = mx4_unit(power);
        s16x2 o = {0, 0};
        o = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(o, v[0], v[1], unit, false);
        o = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(o, v[2], v[3], unit, true);
        const int word = __builtin_bit_cast(int, o);
        *reinterpret_cast<int *>(terms + p * 32 + part * 4) = word;
        if (part == p) powers[p] = (uint8_t)power;
        const f32x2 lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(word, unit, false), hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(word, unit, true);
        v -= f32x4{lo[0], lo[1], hi[0], hi[1]};
    }
}
// Those of blocks c0 .. c0 + 3 of nb (zeros behind them) as an operand of mfma16_mx4_f8, a term to a row.
__device__ __forceinline__ void mx4_get_terms(const uint8_t *terms, const uint8_t *powers, int c0, int nb, int lane, i32x8 &v, uint32_t &power)
{
    const int term = lane & 15, piece = lane >> 4;
    v = i32x8{0, 0, 0, 0, 0, 0, 0, 0};
    power = 0;
    if (term < TERMS) {
        const int c = c0 + (piece >> 1);
        const uint8_t *at = terms + (c * TERMS + term) * 32 + (piece & 1) * 16;
        i32x4 lo = {0, 0, 0, 0}, hi = {0, 0, 0, 0};
        if (c < nb) lo = *reinterpret_cast<const i32x4 *>(at);
        if (c + 2 < nb) hi = *reinterpret_cast<const i32x4 *>(at + 2 * TERMS * 32);
        v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        if (c0 + piece < nb) power = powers[(c0 + piece) * 8 + term];
    }
}

// The 32 values of a block.
__device__ __forceinline__ void mx4_values(const i32x4 &v, float unit, float (&x)[32])
{
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const f32x2 p0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4((uint32_t)v[w], unit, 0), p1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4((uint32_t)v[w], unit, 1);
        const f32x2 p2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4((uint32_t)v[w], unit, 2), p3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4((uint32_t)v[w], unit, 3);
        x[8 * w] = p0[0]; x[8 * w + 1] = p0[1]; x[8 * w + 2] = p1[0]; x[8 * w + 3] = p1[1];
        x[8 * w + 4] = p2[0]; x[8 * w + 5] = p2[1]; x[8 * w + 6] = p3[0]; x[8 * w + 7] = p3[1];
    }
}

}  // namespace abft
