// Microscaled product for few rows: every weight is read once, straight into the registers that the matrix instruction takes it
// from (no unpacking: the matrix cores multiply the codes and both scales themselves).
// 1 x 4096 x 4096: 4.0 us, a launch, one round of loads and the waves' join; 1 x 44032 x 8192: 43.4 us, 191 MB, 4.4 TB/s.  What bounds it is how
// its loads follow each other, not the memory: a wave asks for a round of 512 k, waits, multiplies and asks for the next, and 5120 columns are
// 320 workgroups on 256 compute units (1 x 5120 x 13824: 12.8 us).  The kernels for integer weights, which load ahead, read at up to 5.6 TB/s
// (one row, these layers: 33 and 11.2 us).  From 16 rows on small tiles read large weights as fast and the activations once (16 x 44032 x
// 8192: 53.2 us here, 40.5 in tiles of 32 x 64).
//
// A workgroup takes 16 NT columns and all rows (16 MT); its KW waves take 512 k in turn and add their sums through shared
// memory at the end.  Per 512 k and 16 columns a wave has four 16x16x128 instructions: lane (c, g) holds the 32 codes of
// column c, block 4 s + g of the 16, for step s, so that a load of the wave is 16 columns x 64 bytes.  Its scales come 16 bytes at a time
// (a row's 16 blocks); the four that are this lane's are picked into one register, whose byte s step s takes.
// Weights are the instruction's rows and activations its columns: a lane's four results are neighbouring columns of y, so that gate and
// up lie in one lane.  e4m3 activations: of a block of 128 k a lane holds 16 g .. + 15 and 64 + 16 g .. + 15.
#include "sqp_mx_gemm.h"

namespace {

// Bytes s of the lane's scales: block 4 s + g.
__device__ __forceinline__ uint32_t pick_scales(const u32x4 v, uint32_t lo, uint32_t hi)
{
    return __builtin_amdgcn_perm(v.y, v.x, lo) | __builtin_amdgcn_perm(v.w, v.z, hi);
}

template <int XT, int MT, int NT, int KW>
__global__ void __launch_bounds__(64 * KW) mx_few_kernel(const SqpMxGemm a)
{
    constexpr int XL = XT == SQP_E2M1 ? 1 : 2;      // 16-byte loads per lane and step
    constexpr int XBITS = XT == SQP_E2M1 ? 4 : 8;
    constexpr int XFMT = XT == SQP_E2M1 ? 4 : 0;    // of the matrix instruction
    __shared__ f32x4 s_sum[KW][MT * NT][64];
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
    const int n0 = blockIdx.x * 16 * NT, m0 = blockIdx.y * 16 * MT;
    const int blocks = a.K / SQP_MX_BLOCK, rounds = (blocks + 15) / 16;
    const uint32_t lo = (uint32_t)g | (uint32_t)(4 + g) << 8 | 0x0c0c0000u, hi = (uint32_t)g << 16 | (uint32_t)(4 + g) << 24 | 0x0c0cu;

    const uint8_t *wp[NT], *wsp[NT], *xp[MT], *xsp[MT];
#pragma unroll
    for (int t = 0; t < NT; t++) {
        const size_t n = min(n0 + 16 * t + c, a.N - 1);
        wp[t] = (const uint8_t *)a.w + n * (size_t)(a.K / 2);
        wsp[t] = a.ws + n * blocks;
    }
#pragma unroll
    for (int t = 0; t < MT; t++) {
        const size_t m = min(m0 + 16 * t + c, a.M - 1);
        xp[t] = (const uint8_t *)a.x + m * (size_t)(a.K / 8 * XBITS);
        xsp[t] = a.xs + m * blocks;
    }
    f32x4 acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; i++)
#pragma unroll
        for (int j = 0; j < NT; j++) acc[i][j] = (f32x4)(0.f);

    for (int r = wave; r < rounds; r += KW) {
        const int first = 16 * r, left = blocks - first;
        u32x4 wv[NT][4], xv[MT][4 * XL], wsv[NT], xsv[MT];
#pragma unroll
        for (int t = 0; t < NT; t++) {
#pragma unroll
            for (int s = 0; s < 4; s++) {
                const int block = min(first + 4 * s + g, blocks - 1);
                const u32x4 v = __builtin_nontemporal_load((const u32x4 *)(wp[t] + (size_t)block * 16));
                wv[t][s] = 4 * s + g < left ? v : (u32x4)(0u);
            }
            wsv[t] = sqp_mx_load_scales(wsp[t] + first, left);
        }
#pragma unroll
        for (int t = 0; t < MT; t++) {
#pragma unroll
            for (int s = 0; s < 4; s++) {
                if constexpr (XT == SQP_E2M1) {
                    xv[t][s] = *(const u32x4 *)(xp[t] + (size_t)min(first + 4 * s + g, blocks - 1) * 16);
                } else {
                    // pieces of 16: g and 4 + g of the step's eight (past the end any: the weight's codes are zeros there)
#pragma unroll
                    for (int e = 0; e < 2; e++) xv[t][2 * s + e] = *(const u32x4 *)(xp[t] + (size_t)min(2 * (first + 4 * s) + 4 * e + g, 2 * blocks - 1) * 16);
                }
            }
            xsv[t] = sqp_mx_load_scales(xsp[t] + first, left);
        }
        uint32_t wsc[NT], xsc[MT];
#pragma unroll
        for (int t = 0; t < NT; t++) wsc[t] = pick_scales(wsv[t], lo, hi);
#pragma unroll
        for (int t = 0; t < MT; t++) xsc[t] = pick_scales(xsv[t], lo, hi);
#define SQP_MX_STEP(s)                                                                                                                      \
    for (int i = 0; i < MT; i++) {                                                                                                           \
        i32x8 b;                                                                                                                             \
        if constexpr (XT == SQP_E2M1) b = sqp_mx_operand(xv[i][s]);                                                                          \
        else b = sqp_mx_operand(xv[i][XL * s], xv[i][XL * s + XL - 1]);                                                                      \
        for (int j = 0; j < NT; j++)                                                                                                         \
            acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(sqp_mx_operand(wv[j][s]), b, acc[i][j], 4, XFMT, s, (int)wsc[j], s, \
                                                                         (int)xsc[i]);                                                       \
    }
        _Pragma("unroll") SQP_MX_STEP(0)
        _Pragma("unroll") SQP_MX_STEP(1)
        _Pragma("unroll") SQP_MX_STEP(2)
        _Pragma("unroll") SQP_MX_STEP(3)
#undef SQP_MX_STEP
    }
#pragma unroll
    for (int i = 0; i < MT; i++)
#pragma unroll
        for (int j = 0; j < NT; j++) s_sum[wave][i * NT + j][lane] = acc[i][j];
    __syncthreads();
    for (int u = threadIdx.x; u < MT * NT * 64; u += 64 * KW) {
        const int tile = u >> 6, l = u & 63;
        f32x4 s = s_sum[0][tile][l];
#pragma unroll
        for (int k = 1; k < KW; k++) s += s_sum[k][tile][l];
        const int m = m0 + 16 * (tile / NT) + (l & 15), n = n0 + 16 * (tile % NT) + 4 * (l >> 4);
        if (m < a.M && n < a.N) sqp_mx_store4(a, m, n, s);
    }
}

template <int XT, int MT, int NT, int KW>
int launch(const SqpMxGemm &a, hipStream_t st)
{
    const dim3 grid((unsigned)((a.N + 16 * NT - 1) / (16 * NT)), (unsigned)((a.M + 16 * MT - 1) / (16 * MT)));
    mx_few_kernel<XT, MT, NT, KW><<<grid, 64 * KW, 0, st>>>(a);
    return sqp_launch_status();
}

template <int XT>
int pick(const SqpMxFewPlan &p, const SqpMxGemm &a, hipStream_t st)
{
#define FEW(MT, NT, KW) \
    if (p.mt == MT && p.nt == NT && p.kw == KW) return launch<XT, MT, NT, KW>(a, st)
    FEW(1, 1, 8);
    FEW(1, 2, 8);
    FEW(2, 1, 8);
    FEW(2, 2, 4);
    FEW(4, 1, 8);
#undef FEW
    return SQP_ERR_SHAPE;
}

}  // namespace

int sqp_mx_few(int x_type, const SqpMxFewPlan &p, const SqpMxGemm &a, hipStream_t st)
{
    return x_type == SQP_E2M1 ? pick<SQP_E2M1>(p, a, st) : pick<SQP_E4M3>(p, a, st);
}
