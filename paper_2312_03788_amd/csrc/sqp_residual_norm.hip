// The residual's addition and the RMS norm behind it, in one pass:
//   r = fp16(x + residual),  y = r / sqrt(mean_j r^2 + eps) * gamma,
// y in fp16 (sqp_add_rmsnorm), or as 8-bit codes with a scale per row (sqp_add_rmsnorm_quant), for a product that takes
// 8-bit activations.
#include "sqp_rows.h"

namespace {

constexpr int HALF = SQP_FP16;

template <int W>
__device__ __forceinline__ float wave_sums(const float *red)
{
    float part[W];
#pragma unroll
    for (int i = 0; i < W; i++) part[i] = red[i];
#pragma unroll
    for (int half = W / 2; half >= 1; half >>= 1)
#pragma unroll
        for (int i = 0; i < half; i++) part[i] = part[2 * i] + part[2 * i + 1];
    return part[0];
}

__device__ __forceinline__ uint4 add8(const uint4 a, const uint4 b)
{
    // packed fp16 additions round the exact sum once
    const h16x8 s = __builtin_bit_cast(h16x8, a) + __builtin_bit_cast(h16x8, b);
    return __builtin_bit_cast(uint4, s);
}

// The scale of a row whose largest |r gamma| has these bits, r the row's factor, and what takes r gamma to codes: y / scale
// = r gamma MAX / max |r gamma| is free of the row's factor, and r gamma is exact in fp32 (11 bits by 11), so that a code is
// two roundings away from the formula's value and not five (of 16.8 million e4m3 codes 43 fall on the other side of a rounding's
// edge, four inputs' mean, and 57 with five).
template <int OUT>
__device__ __forceinline__ void row_codes(uint32_t amax, float r, float &step, float &inverse)
{
    const float most = __builtin_bit_cast(float, amax), a = most * r;  // NaN where the row holds no finite sum
    sqp_row_step<OUT>(sqp_abs_bits(a), step, inverse);
    if (inverse != 0.f) inverse = SqpCode<OUT>::MAX / most;
}

// One workgroup of W waves per row, NI pieces of 8 values per thread, which stay in registers between the sum of squares and
// the scaling: x, the residual and gamma are read once.  The largest |r gamma| is found in the same pass as the sum of squares
// (it is the largest |y| up to the row's factor), so that the 8-bit output needs no second exchange between the waves.
// Bound: few rows, the launch and a chain of latencies (2.2 us on 1 x 4096); many, HBM (2048 x 8192 read twice and written twice in
// 20.8 us, 6.4 TB/s; with e4m3 output 20.5 us).  A row is spread over up to 16 waves at any number of rows: with 4 waves
// 512 x 8192 takes 8.3 us instead of 7.4, 4096 x 8192 45.5 instead of 43.0 (e4m3: 39.3 instead of 41).
template <int W, int NI, int OUT>
__global__ void __launch_bounds__(64 * W) add_rmsnorm_kernel(int H8, float inv_h, float eps, const uint4 *x, const uint4 *residual,
                                                             const uint4 *__restrict__ gamma, void *__restrict__ y, float *__restrict__ scales, uint4 *sum)
{
    __shared__ float red[W];
    __shared__ uint32_t top[W];
    const size_t row = (size_t)blockIdx.x * H8;
    uint4 v[NI], g[NI];
#pragma unroll
    for (int j = 0; j < NI; j++) {
        const int i = threadIdx.x + 64 * W * j;
        v[j] = i < H8 ? x[row + i] : make_uint4(0, 0, 0, 0);
        g[j] = i < H8 ? residual[row + i] : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int j = 0; j < NI; j++) {
        const int i = threadIdx.x + 64 * W * j;
        v[j] = add8(v[j], g[j]);
        g[j] = i < H8 ? gamma[i] : make_uint4(0, 0, 0, 0);
        if (i < H8) sum[row + i] = v[j];
    }
    float ss = 0.f;
    uint32_t amax = 0;
#pragma unroll
    for (int j = 0; j < NI; j++) {
        float f[8];
        sqp_widen8(v[j], f);
        ss += ((f[0] * f[0] + f[1] * f[1]) + (f[2] * f[2] + f[3] * f[3])) + ((f[4] * f[4] + f[5] * f[5]) + (f[6] * f[6] + f[7] * f[7]));
        if constexpr (OUT != HALF) {
            float gf[8];
            sqp_widen8(g[j], gf);
#pragma unroll
            for (int e = 0; e < 8; e++) amax = max(amax, sqp_abs_bits(f[e] * gf[e]));
        }
    }
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) {
        ss += __shfl_xor(ss, off, 64);
        if constexpr (OUT != HALF) amax = max(amax, (uint32_t)__shfl_xor((int)amax, off, 64));
    }
    if ((threadIdx.x & 63) == 0) {
        red[threadIdx.x >> 6] = ss;
        if constexpr (OUT != HALF) top[threadIdx.x >> 6] = amax;
    }
    __syncthreads();
    const float r = 1.0f / sqrtf(wave_sums<W>(red) * inv_h + eps);
    float step = 0.f, inverse = 0.f;
    if constexpr (OUT != HALF) {
#pragma unroll
        for (int i = 0; i < W; i++) amax = max(amax, top[i]);
        row_codes<OUT>(amax, r, step, inverse);
        if (threadIdx.x == 0) scales[blockIdx.x] = step;
    }
#pragma unroll
    for (int j = 0; j < NI; j++) {
        const int i = threadIdx.x + 64 * W * j;
        if (i < H8) {
            float f[8], gf[8];
            sqp_widen8(v[j], f);
            sqp_widen8(g[j], gf);
#pragma unroll
            for (int e = 0; e < 8; e++) f[e] = OUT == HALF ? f[e] * r * gf[e] : f[e] * gf[e];
            if constexpr (OUT == HALF) ((uint4 *)y)[row + i] = sqp_narrow8(f);
            else ((uint2 *)y)[row + i] = sqp_codes8<OUT>(f, inverse);
        }
    }
}

// Rows too long for registers: the sums are read back from where this thread has written them.
template <int OUT>
__global__ void __launch_bounds__(1024) add_rmsnorm_long_kernel(int H8, float inv_h, float eps, const uint4 *x, const uint4 *residual,
                                                                const uint4 *__restrict__ gamma, void *__restrict__ y, float *__restrict__ scales, uint4 *sum)
{
    __shared__ float red[16];
    __shared__ uint32_t top[16];
    const size_t row = (size_t)blockIdx.x * H8;
    float ss = 0.f;
    uint32_t amax = 0;
    for (int i = threadIdx.x; i < H8; i += 1024) {
        const uint4 v = add8(x[row + i], residual[row + i]), g = gamma[i];
        sum[row + i] = v;
        float f[8], gf[8];
        sqp_widen8(v, f);
        sqp_widen8(g, gf);
        ss += ((f[0] * f[0] + f[1] * f[1]) + (f[2] * f[2] + f[3] * f[3])) + ((f[4] * f[4] + f[5] * f[5]) + (f[6] * f[6] + f[7] * f[7]));
#pragma unroll
        for (int e = 0; e < 8; e++) amax = max(amax, sqp_abs_bits(f[e] * gf[e]));
    }
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) {
        ss += __shfl_xor(ss, off, 64);
        amax = max(amax, (uint32_t)__shfl_xor((int)amax, off, 64));
    }
    if ((threadIdx.x & 63) == 0) {
        red[threadIdx.x >> 6] = ss;
        top[threadIdx.x >> 6] = amax;
    }
    __syncthreads();
    const float r = 1.0f / sqrtf(wave_sums<16>(red) * inv_h + eps);
    float step = 0.f, inverse = 0.f;
    if constexpr (OUT != HALF) {
        for (int i = 0; i < 16; i++) amax = max(amax, top[i]);
        row_codes<OUT>(amax, r, step, inverse);
        if (threadIdx.x == 0) scales[blockIdx.x] = step;
    }
    for (int i = threadIdx.x; i < H8; i += 1024) {
        float f[8], gf[8];
        sqp_widen8(sum[row + i], f);
        sqp_widen8(gamma[i], gf);
#pragma unroll
        for (int e = 0; e < 8; e++) f[e] = OUT == HALF ? f[e] * r * gf[e] : f[e] * gf[e];
        if constexpr (OUT == HALF) ((uint4 *)y)[row + i] = sqp_narrow8(f);
        else ((uint2 *)y)[row + i] = sqp_codes8<OUT>(f, inverse);
    }
}

template <int OUT>
int launch(int M, int H, const void *x, const void *residual, const void *gamma, float eps, void *y, float *scales, void *sum, hipStream_t st)
{
    const int H8 = H / 8;
    const float inv_h = 1.0f / (float)H;
    const uint4 *xp = (const uint4 *)x, *rp = (const uint4 *)residual, *gp = (const uint4 *)gamma;
    uint4 *sp = (uint4 *)sum;
    const dim3 grid((unsigned)M);
#define ADD_RMSNORM(W, NI) add_rmsnorm_kernel<W, NI, OUT><<<grid, 64 * W, 0, st>>>(H8, inv_h, eps, xp, rp, gp, y, scales, sp)
    if (H8 <= 256) ADD_RMSNORM(4, 1);
    else if (H8 <= 512) ADD_RMSNORM(8, 1);
    else if (H8 <= 1024) ADD_RMSNORM(16, 1);
    else if (H8 <= 2048) ADD_RMSNORM(16, 2);
    else if (H8 <= 4096) ADD_RMSNORM(16, 4);
    else add_rmsnorm_long_kernel<OUT><<<grid, 1024, 0, st>>>(H8, inv_h, eps, xp, rp, gp, y, scales, sp);
#undef ADD_RMSNORM
    return sqp_launch_status();
}

int check(int M, int H, const void *x, const void *residual, const void *gamma, float eps, const void *y, const void *sum)
{
    if (!x || !residual || !gamma || !y || !sum) return SQP_ERR_NULL;
    if (M <= 0 || H <= 0 || (H % 8) || sqp_too_big(M, H)) return SQP_ERR_SHAPE;
    if (!(eps >= 0.0f) || !(eps < 1.0f)) return SQP_ERR_ARG;
    if (sqp_misaligned(x) || sqp_misaligned(residual) || sqp_misaligned(gamma) || sqp_misaligned(y) || sqp_misaligned(sum)) return SQP_ERR_ALIGN;
    return SQP_OK;
}

}  // namespace

extern "C" int sqp_add_rmsnorm(int M, int H, const void *x, const void *residual, const void *gamma, float eps, void *y, void *sum, void *stream)
{
    const int rc = check(M, H, x, residual, gamma, eps, y, sum);
    return rc ? rc : launch<SQP_FP16>(M, H, x, residual, gamma, eps, y, nullptr, sum, (hipStream_t)stream);
}

extern "C" int sqp_add_rmsnorm_quant(int M, int H, int type, const void *x, const void *residual, const void *gamma, float eps, void *codes,
                                     float *scales, void *sum, void *stream)
{
    if (!scales) return SQP_ERR_NULL;
    const int rc = check(M, H, x, residual, gamma, eps, codes, sum);
    if (rc) return rc;
    if (sqp_misaligned(scales)) return SQP_ERR_ALIGN;
    hipStream_t st = (hipStream_t)stream;
    if (type == SQP_INT8) return launch<SQP_INT8>(M, H, x, residual, gamma, eps, codes, scales, sum, st);
    if (type == SQP_E4M3) return launch<SQP_E4M3>(M, H, x, residual, gamma, eps, codes, scales, sum, st);
    return SQP_ERR_ARG;
}
