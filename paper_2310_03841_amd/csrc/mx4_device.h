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
