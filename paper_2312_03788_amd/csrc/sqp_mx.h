// Microscaled numbers: blocks of 32 values along a row with one power-of-two scale in a byte (the exponent plus 127),
// elements e2m1 (two to a byte, the first in the low half) or e4m3.
#pragma once
#include "sqp_rows.h"

constexpr int SQP_MX_BLOCK = 32;

#ifdef __HIPCC__
// The scale's byte for a block whose largest magnitude has these bits: the least power of two with which that magnitude rounds to a
// value of the type.  Of e2m1 (6 = 1.5 x 2^2 is the largest) magnitudes from 1.75 x 2^x on would round to 8 with the scale 2^(x - 2); of e4m3
// (448 = 1.75 x 2^8) those beyond 1.8125 x 2^x, which is the middle of 448 and 480 and goes to 448, the even one.  So an addition
// to the mantissa's bits carries exactly where the next scale is due.  Below 2^-100: byte 0 (and codes 0); infinities and NaN: 255.
template <int TYPE>
__device__ __forceinline__ uint32_t sqp_mx_byte(uint32_t amax_bits)
{
    const uint32_t e = TYPE == SQP_E2M1 ? ((amax_bits + 0x200000u) >> 23) - 2u : ((amax_bits + 0x17ffffu) >> 23) - 8u;
    return amax_bits >= 0x7f800000u ? 255u : amax_bits < 0x0d800000u ? 0u : e;
}

// Eight values of a block with this scale byte to codes: one word (e2m1) or two.  Dividing by a power of two is exact, so a code is one
// rounding (to nearest, even) away from its value.
__device__ __forceinline__ uint32_t sqp_mx_e2m1_codes8(const float *f, uint32_t byte)
{
    const float scale = __builtin_bit_cast(float, byte << 23);
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[0], f[1], scale, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[2], f[3], scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[4], f[5], scale, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[6], f[7], scale, 3);
    return byte == 0u || byte == 255u ? 0u : w;
}

__device__ __forceinline__ uint2 sqp_mx_e4m3_codes8(const float *f, uint32_t byte)
{
    const float inverse = __builtin_bit_cast(float, (254u - byte) << 23);
    const uint2 w = sqp_codes8<SQP_E4M3>(f, inverse);
    return byte == 0u || byte == 255u ? make_uint2(0, 0) : w;
}

// The largest of four neighbouring lanes, which hold a block's 32 values together.
__device__ __forceinline__ uint32_t sqp_quad_max(uint32_t x)
{
    x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0xb1, 0xf, 0xf, true));         // lanes 1, 0, 3, 2
    return max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x4e, 0xf, 0xf, true));      // lanes 2, 3, 0, 1
}

// Eight e2m1 codes of a word as values times the scale, fp32 (exact; a scale of NaN makes NaN of them).
__device__ __forceinline__ void sqp_mx_e2m1_values8(uint32_t w, float scale, float *f)
{
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 1);
    const f32x2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 3);
    f[0] = a.x; f[1] = a.y; f[2] = b.x; f[3] = b.y; f[4] = c.x; f[5] = c.y; f[6] = d.x; f[7] = d.y;
}
#endif
