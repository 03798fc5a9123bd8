// Blocks of 32 with a power-of-two scale: rows of activations into blocks and back, a weight [K][N] into the blocks of its columns, and
// the residual's addition with the RMS norm behind it, its output in blocks.  All are single streaming passes.
#include "sqp_mx.h"

namespace {

// A thread takes eight values, four neighbouring lanes a block: 16-byte loads, whole lines of codes.  K is a multiple of 32, so
// blocks follow each other through the whole tensor and the rows do not matter.  Bound: HBM; 2048 x 8192 into e4m3 10.3 us, 51 MB, 4.9 TB/s (called
// in a row; 1001 x 5120 4.8), back from e2m1 10240 x 8192 35 us, 212 MB, 6.1 TB/s.
template <int TYPE>
__global__ void __launch_bounds__(256) mx_quantize_kernel(long pieces, const uint4 *__restrict__ x, void *__restrict__ codes, uint8_t *__restrict__ scales)
{
    const long i = (long)blockIdx.x * 256 + threadIdx.x;
    if (i >= pieces) return;  // (a whole block of lanes)
    float f[8];
    sqp_widen8(x[i], f);
    uint32_t amax = 0;
#pragma unroll
    for (int j = 0; j < 8; j++) amax = max(amax, sqp_abs_bits(f[j]));
    const uint32_t byte = sqp_mx_byte<TYPE>(sqp_quad_max(amax));
    if constexpr (TYPE == SQP_E2M1) ((uint32_t *)codes)[i] = sqp_mx_e2m1_codes8(f, byte);
    else ((uint2 *)codes)[i] = sqp_mx_e4m3_codes8(f, byte);
    if ((i & 3) == 0) scales[i >> 2] = (uint8_t)byte;
}

template <int TYPE>
__global__ void __launch_bounds__(256) mx_dequantize_kernel(long pieces, const void *__restrict__ codes, const uint8_t *__restrict__ scales, uint4 *__restrict__ x)
{
    const long i = (long)blockIdx.x * 256 + threadIdx.x;
    if (i >= pieces) return;
    const uint32_t byte = scales[i >> 2];
    float f[8];
    if constexpr (TYPE == SQP_E2M1) {
        sqp_mx_e2m1_values8(((const uint32_t *)codes)[i], __builtin_bit_cast(float, byte << 23), f);
    } else {
        const uint2 c = ((const uint2 *)codes)[i];
        const uint32_t w[2] = {c.x, c.y};
        // (a byte of 0 stands for 2^-127, which is no normal number)
        const float scale = __builtin_bit_cast(float, byte == 255u ? 0x7fc00000u : byte == 0u ? 0x00400000u : byte << 23);
#pragma unroll
        for (int j = 0; j < 2; j++) {
            h16x2 lo, hi;
            sqp_halves4<SQP_E4M3>(w[j], lo, hi);
            f[4 * j] = (float)lo.x * scale;
            f[4 * j + 1] = (float)lo.y * scale;
            f[4 * j + 2] = (float)hi.x * scale;
            f[4 * j + 3] = (float)hi.y * scale;
        }
    }
    x[i] = sqp_narrow8(f);
}

// A weight w [K][N] into blocks along K, one row of codes per column: codes [N][K / 2], scales [N][K / 32].  A workgroup takes 128
// columns by 256 k; a thread four columns by a block (32 loads of 8 bytes: 256 bytes of a row over 32 lanes), and the codes change
// places through shared memory, so that 128 bytes of a column leave together.  10240 x 8192: 42 us, 212 MB, 5.0 TB/s (64 columns, 4 bytes
// per load: 49).
__global__ void __launch_bounds__(256) mx_quantize_weight_kernel(int N, int K, const h16 *__restrict__ w, uint4 *__restrict__ codes, uint8_t *__restrict__ scales)
{
    constexpr int COLS = 128;
    __shared__ uint4 s_codes[COLS][9];
    __shared__ uint8_t s_scales[COLS][8];
    const int quad = threadIdx.x & 31, kb = threadIdx.x >> 5, blocks = K / SQP_MX_BLOCK;
    const int n0 = blockIdx.x * COLS, kb0 = blockIdx.y * 8, n = n0 + 4 * quad;
    if (n < N && kb0 + kb < blocks) {
        const h16 *p = w + (size_t)(kb0 + kb) * SQP_MX_BLOCK * N + n;
        typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
        u32x2 v[32];
#pragma unroll
        for (int j = 0; j < 32; j++) v[j] = __builtin_nontemporal_load((const u32x2 *)(p + (size_t)j * N));
#pragma unroll
        for (int c = 0; c < 4; c++) {
            float f[32];
            uint32_t amax = 0;
#pragma unroll
            for (int j = 0; j < 32; j++) {
                const uint32_t word = c >> 1 ? v[j].y : v[j].x;
                const h16x2 both = __builtin_bit_cast(h16x2, word);
                f[j] = c & 1 ? (float)both.y : (float)both.x;
                amax = max(amax, sqp_abs_bits(f[j]));
            }
            const uint32_t byte = sqp_mx_byte<SQP_E2M1>(amax);
            s_codes[4 * quad + c][kb] = make_uint4(sqp_mx_e2m1_codes8(f, byte), sqp_mx_e2m1_codes8(f + 8, byte), sqp_mx_e2m1_codes8(f + 16, byte),
                                                   sqp_mx_e2m1_codes8(f + 24, byte));
            s_scales[4 * quad + c][kb] = (uint8_t)byte;
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < COLS / 32; i++) {
        const int unit = threadIdx.x + 256 * i, col = unit >> 3, b = unit & 7;
        if (n0 + col < N && kb0 + b < blocks) {
            codes[(size_t)(n0 + col) * blocks + kb0 + b] = s_codes[col][b];
            scales[(size_t)(n0 + col) * blocks + kb0 + b] = s_scales[col][b];
        }
    }
}

// ---------------------------------------------------------------- residual, norm, blocks

// z = r gamma / sqrt(mean r^2 + eps) is taken in 64 bits: a 32-bit z would put one in some millions of values on the other side of a border
// between two codes, and two codes are up to a half of the value apart; at 2^-45 it is one in 2^40.  Of the double only what decides is kept: its 20 leading
// mantissa bits, and whether anything is behind them, as the lowest bit of a float (all borders have four mantissa bits at most).
__device__ __forceinline__ float mx_sticky(double z)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, z);
    const uint32_t hi = (uint32_t)(b >> 32), lo = (uint32_t)b, size = hi & 0x7fffffffu;
    uint32_t f = ((size - (896u << 20)) << 3) | (lo != 0u ? 1u : 0u);
    f = size >= 0x7ff00000u ? 0x7fc00000u : size < (897u << 20) ? 0u : f;  // (below 2^-126: zero in any block)
    return __builtin_bit_cast(float, f | (hi & 0x80000000u));
}

__device__ __forceinline__ uint4 mx_add8(const uint4 a, const uint4 b)
{
    // packed fp16 additions round the exact sum once
    return __builtin_bit_cast(uint4, __builtin_bit_cast(h16x8, a) + __builtin_bit_cast(h16x8, b));
}

__device__ __forceinline__ double mx_squares8(const float *f)
{
    double s = 0.0;
#pragma unroll
    for (int e = 0; e < 8; e++) s = __builtin_fma((double)f[e], (double)f[e], s);
    return s;
}

template <int W>
__device__ __forceinline__ double mx_sum(double ss, double *red)
{
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) ss += __shfl_xor(ss, off, 64);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = ss;
    __syncthreads();
    double part[W];
#pragma unroll
    for (int i = 0; i < W; i++) part[i] = red[i];
#pragma unroll
    for (int half = W / 2; half >= 1; half >>= 1)
#pragma unroll
        for (int i = 0; i < half; i++) part[i] = part[2 * i] + part[2 * i + 1];
    return part[0];
}

// 1 / sqrt(a) to 2^-45 at least: the hardware's (2^-23 at least) and one step of Newton's method, whose error is 3/2 of the square.  A
// quotient and a root to the last bit, in every thread, are 2 us of 2048 x 8192.
__device__ __forceinline__ double mx_rsqrt(double a)
{
    const double r = __builtin_amdgcn_rsq(a), next = r * __builtin_fma(-0.5 * a * r, r, 1.5);
    return a > 0.0 && a < __builtin_inf() ? next : r;  // (0: infinite, infinite: 0, NaN)
}

// Piece i (eight values) of a row into its place.
template <int TYPE>
__device__ __forceinline__ void mx_store8(const uint4 v, const uint4 g, double r, size_t i, void *codes, uint8_t *scales)
{
    float f[8], gf[8];
    sqp_widen8(v, f);
    sqp_widen8(g, gf);
    uint32_t amax = 0;
#pragma unroll
    for (int e = 0; e < 8; e++) {
        f[e] = mx_sticky((double)(f[e] * gf[e]) * r);  // (11 bits by 11: exact in fp32)
        amax = max(amax, sqp_abs_bits(f[e]));
    }
    const uint32_t byte = sqp_mx_byte<TYPE>(sqp_quad_max(amax));
    if constexpr (TYPE == SQP_E2M1) ((uint32_t *)codes)[i] = sqp_mx_e2m1_codes8(f, byte);
    else ((uint2 *)codes)[i] = sqp_mx_e4m3_codes8(f, byte);
    if ((i & 3) == 0) scales[i >> 2] = (uint8_t)byte;
}

// One workgroup of W waves per row, NI pieces of eight values per thread, which stay in registers between the sum of squares and the codes.
// Bound: HBM (2048 x 8192, e2m1: 23.6 us, 110 MB, 4.7 TB/s, the 8-bit form with a scale per row 22.4), for few rows the launch and a chain of
// latencies (2.7 us on 1 x 4096).  A z in 32 bits, with 64 only for lanes near a border, is slower (28.7 us).
template <int W, int NI, int TYPE>
__global__ void __launch_bounds__(64 * W) add_rmsnorm_mx_kernel(int H8, double inv_h, double eps, const uint4 *x, const uint4 *residual, const uint4 *__restrict__ gamma,
                                                                void *__restrict__ codes, uint8_t *__restrict__ scales, uint4 *sum)
{
    __shared__ double red[W];
    const size_t row = (size_t)blockIdx.x * H8;
    uint4 v[NI], g[NI];
#pragma unroll
    for (int j = 0; j < NI; j++) {
        const int i = threadIdx.x + 64 * W * j;
        v[j] = i < H8 ? x[row + i] : make_uint4(0, 0, 0, 0);
        g[j] = i < H8 ? residual[row + i] : make_uint4(0, 0, 0, 0);
    }
    double ss = 0.0;
#pragma unroll
    for (int j = 0; j < NI; j++) {
        const int i = threadIdx.x + 64 * W * j;
        v[j] = mx_add8(v[j], g[j]);
        g[j] = i < H8 ? gamma[i] : make_uint4(0, 0, 0, 0);
        if (i < H8) sum[row + i] = v[j];
        float f[8];
        sqp_widen8(v[j], f);
        ss += mx_squares8(f);
    }
    const double r = mx_rsqrt(__builtin_fma(mx_sum<W>(ss, red), inv_h, eps));
#pragma unroll
    for (int j = 0; j < NI; j++) {
        const int i = threadIdx.x + 64 * W * j;
        if (i < H8) mx_store8<TYPE>(v[j], g[j], r, row + i, codes, scales);
    }
}

// Rows too long for registers: the sums are read back from where this thread has written them.
template <int TYPE>
__global__ void __launch_bounds__(1024) add_rmsnorm_mx_long_kernel(int H8, double inv_h, double eps, const uint4 *x, const uint4 *residual, const uint4 *__restrict__ gamma,
                                                                   void *__restrict__ codes, uint8_t *__restrict__ scales, uint4 *sum)
{
    __shared__ double red[16];
    const size_t row = (size_t)blockIdx.x * H8;
    double ss = 0.0;
    for (int i = threadIdx.x; i < H8; i += 1024) {
        const uint4 v = mx_add8(x[row + i], residual[row + i]);
        sum[row + i] = v;
        float f[8];
        sqp_widen8(v, f);
        ss += mx_squares8(f);
    }
    const double r = mx_rsqrt(__builtin_fma(mx_sum<16>(ss, red), inv_h, eps));
    for (int i = threadIdx.x; i < H8; i += 1024) mx_store8<TYPE>(sum[row + i], gamma[i], r, row + i, codes, scales);
}

template <int TYPE>
int launch_norm(int M, int H, const void *x, const void *residual, const void *gamma, float eps, void *codes, uint8_t *scales, void *sum, hipStream_t st)
{
    constexpr int MOST = 1 << 21;  // rows of a launch, which has fewer than 2^32 threads
    const int H8 = H / 8;
    const uint4 *gp = (const uint4 *)gamma;
    for (int first = 0; first < M; first += MOST) {
        const size_t at = (size_t)first * H8;
        const uint4 *xp = (const uint4 *)x + at, *rp = (const uint4 *)residual + at;
        uint4 *sp = (uint4 *)sum + at;
        uint8_t *cp = (uint8_t *)codes + at * (TYPE == SQP_E2M1 ? 4 : 8), *bp = scales + at / 4;
        const dim3 grid((unsigned)min(M - first, MOST));
#define ADD_RMSNORM_MX(W, NI) add_rmsnorm_mx_kernel<W, NI, TYPE><<<grid, 64 * W, 0, st>>>(H8, 1.0 / H, (double)eps, xp, rp, gp, cp, bp, sp)
        if (H8 <= 256) ADD_RMSNORM_MX(4, 1);
        else if (H8 <= 512) ADD_RMSNORM_MX(8, 1);
        else if (H8 <= 1024) ADD_RMSNORM_MX(16, 1);
        else if (H8 <= 2048) ADD_RMSNORM_MX(16, 2);
        else if (H8 <= 4096) ADD_RMSNORM_MX(16, 4);
        else add_rmsnorm_mx_long_kernel<TYPE><<<grid, 1024, 0, st>>>(H8, 1.0 / H, (double)eps, xp, rp, gp, cp, bp, sp);
#undef ADD_RMSNORM_MX
    }
    return sqp_launch_status();
}

int check_blocks(int R, int K, int type, const void *x, const void *codes, const void *scales)
{
    if (!x || !codes || !scales) return SQP_ERR_NULL;
    if (type != SQP_E2M1 && type != SQP_E4M3) return SQP_ERR_ARG;
    if (R <= 0 || K <= 0 || (K % SQP_MX_BLOCK) || sqp_too_big(R, K)) return SQP_ERR_SHAPE;
    if (sqp_misaligned(x) || sqp_misaligned(codes) || sqp_misaligned(scales)) return SQP_ERR_ALIGN;
    return SQP_OK;
}

}  // namespace

extern "C" int sqp_mx_quantize(int R, int K, int type, const void *x, void *codes, uint8_t *scales, void *stream)
{
    const int rc = check_blocks(R, K, type, x, codes, scales);
    if (rc) return rc;
    const long pieces = (long)R * K / 8;
    const unsigned grid = (unsigned)((pieces + 255) / 256);
    hipStream_t st = (hipStream_t)stream;
    if (type == SQP_E2M1) mx_quantize_kernel<SQP_E2M1><<<grid, 256, 0, st>>>(pieces, (const uint4 *)x, codes, scales);
    else mx_quantize_kernel<SQP_E4M3><<<grid, 256, 0, st>>>(pieces, (const uint4 *)x, codes, scales);
    return sqp_launch_status();
}

extern "C" int sqp_mx_dequantize(int R, int K, int type, const void *codes, const uint8_t *scales, void *x, void *stream)
{
    const int rc = check_blocks(R, K, type, x, codes, scales);
    if (rc) return rc;
    const long pieces = (long)R * K / 8;
    const unsigned grid = (unsigned)((pieces + 255) / 256);
    hipStream_t st = (hipStream_t)stream;
    if (type == SQP_E2M1) mx_dequantize_kernel<SQP_E2M1><<<grid, 256, 0, st>>>(pieces, codes, scales, (uint4 *)x);
    else mx_dequantize_kernel<SQP_E4M3><<<grid, 256, 0, st>>>(pieces, codes, scales, (uint4 *)x);
    return sqp_launch_status();
}

extern "C" int sqp_mx_quantize_weight(int N, int K, const void *w, void *codes, uint8_t *scales, void *stream)
{
    const int rc = check_blocks(N, K, SQP_E2M1, w, codes, scales);
    if (rc) return rc;
    if (N % 8) return SQP_ERR_SHAPE;
    const dim3 grid((unsigned)((N + 127) / 128), (unsigned)((K + 255) / 256));
    if (grid.y > 65535u) return SQP_ERR_SHAPE;
    mx_quantize_weight_kernel<<<grid, 256, 0, (hipStream_t)stream>>>(N, K, (const h16 *)w, (uint4 *)codes, scales);
    return sqp_launch_status();
}

extern "C" int sqp_add_rmsnorm_mx(int M, int H, int type, const void *x, const void *residual, const void *gamma, float eps, void *codes, uint8_t *scales,
                                  void *sum, void *stream)
{
    if (!residual || !gamma || !sum) return SQP_ERR_NULL;
    const int rc = check_blocks(M, H, type, x, codes, scales);
    if (rc) return rc;
    if (!(eps >= 0.0f) || !(eps < 1.0f)) return SQP_ERR_ARG;
    if (sqp_misaligned(residual) || sqp_misaligned(gamma) || sqp_misaligned(sum)) return SQP_ERR_ALIGN;
    hipStream_t st = (hipStream_t)stream;
    if (type == SQP_E2M1) return launch_norm<SQP_E2M1>(M, H, x, residual, gamma, eps, codes, scales, sum, st);
    return launch_norm<SQP_E4M3>(M, H, x, residual, gamma, eps, codes, scales, sum, st);
}
