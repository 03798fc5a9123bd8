// Rows of fp16 values in fp32 and back, 8-bit codes with one scale per row: shared by the kernels around the residual stream
// and the key / value cache.
#pragma once
#include "sqp_common.h"

// Codes of a type: element size, and the largest magnitude a code stands for.
template <int TYPE> struct SqpCode;
template <> struct SqpCode<SQP_FP16> { static constexpr int BYTES = 2; };
template <> struct SqpCode<SQP_INT8> { static constexpr int BYTES = 1; static constexpr float MAX = 127.0f; };
template <> struct SqpCode<SQP_E4M3> { static constexpr int BYTES = 1; static constexpr float MAX = 448.0f; };

__device__ __forceinline__ void sqp_widen8(const uint4 v, float *f)
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const h16x2 p = __builtin_bit_cast(h16x2, w[i]);
        f[2 * i] = (float)p.x;
        f[2 * i + 1] = (float)p.y;
    }
}

__device__ __forceinline__ uint32_t sqp_half2(float a, float b)
{
    h16x2 r;
    r.x = (h16)a;
    r.y = (h16)b;
    return __builtin_bit_cast(uint32_t, r);
}

__device__ __forceinline__ uint4 sqp_narrow8(const float *f)
{
    return make_uint4(sqp_half2(f[0], f[1]), sqp_half2(f[2], f[3]), sqp_half2(f[4], f[5]), sqp_half2(f[6], f[7]));
}

// Magnitudes are compared as the bits of |x|: the order of the numbers, and NaN above infinity above every number, so that
// a row that holds one of those is known by its maximum.
__device__ __forceinline__ uint32_t sqp_abs_bits(float x) { return __builtin_bit_cast(uint32_t, x) & 0x7fffffffu; }

// Step between codes (the scale) and its inverse for a row whose largest magnitude has these bits.  Rows below 2^-100 are
// stored as zeros (the inverse of their step would overflow); a row with an infinity or NaN gets the scale NaN, so that all
// of it reads back as NaN.
template <int TYPE>
__device__ __forceinline__ void sqp_row_step(uint32_t amax_bits, float &step, float &inverse)
{
    const float a = __builtin_bit_cast(float, amax_bits);
    if (amax_bits >= 0x7f800000u) {
        step = __builtin_bit_cast(float, 0x7fc00000u);
        inverse = 0.0f;
    } else {
        const bool some = a >= 0x1p-100f;
        step = some ? a / SqpCode<TYPE>::MAX : 0.0f;
        inverse = some ? SqpCode<TYPE>::MAX / a : 0.0f;
    }
}

// Eight values to eight codes: the product with the inverse step is within 2^-22 of the code range, so that rounding to
// nearest even ends inside it without a clamp.
template <int TYPE>
__device__ __forceinline__ uint2 sqp_codes8(const float *f, float inverse)
{
    uint32_t w[2];
#pragma unroll
    for (int i = 0; i < 2; i++) {
        const float a = f[4 * i] * inverse, b = f[4 * i + 1] * inverse, c = f[4 * i + 2] * inverse, d = f[4 * i + 3] * inverse;
        if constexpr (TYPE == SQP_E4M3) {
            int v = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
            v = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, v, true);
            w[i] = (uint32_t)v;
        } else {
            const int ia = (int)rintf(a), ib = (int)rintf(b), ic = (int)rintf(c), id = (int)rintf(d);
            w[i] = (uint32_t)(ia & 255) | (uint32_t)(ib & 255) << 8 | (uint32_t)(ic & 255) << 16 | (uint32_t)id << 24;
        }
    }
    return make_uint2(w[0], w[1]);
}

// Four codes of a word as two pairs of fp16 values (every code of either type is an fp16 number, so this is exact).
template <int TYPE>
__device__ __forceinline__ void sqp_halves4(uint32_t w, h16x2 &lo, h16x2 &hi)
{
    if constexpr (TYPE == SQP_E4M3) {
        lo = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)w, 1.0f, false);
        hi = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)w, 1.0f, true);
    } else {
        // 0x6400 | (b ^ 0x80) is the fp16 number 1024 + 128 + b
        const h16x2 off = {(h16)1152.0f, (h16)1152.0f};
        lo = __builtin_bit_cast(h16x2, __builtin_amdgcn_perm(0u, w, 0x0c010c00u) ^ 0x64806480u) - off;
        hi = __builtin_bit_cast(h16x2, __builtin_amdgcn_perm(0u, w, 0x0c030c02u) ^ 0x64806480u) - off;
    }
}
