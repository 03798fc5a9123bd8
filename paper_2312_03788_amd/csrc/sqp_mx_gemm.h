// The product of microscaled activations and weights: what its kernels share.
#pragma once
#include "sqp_mx.h"

struct SqpMxGemm {
    int M, N, K;
    int silu;  // columns alternate (gate, up): y [M][N / 2]
    int first_col, cols;  // of this launch (tiles)
    const void *x, *w;
    const uint8_t *xs, *ws;
    h16 *y;
    float *part;  // fp32 sums of the K parts, [part][M][N]; null: one part, y is written
};

// Few rows: weights stream through registers, K split over the waves of a workgroup.
struct SqpMxFewPlan {
    int mt, nt, kw;  // 16-row tiles, 16-column tiles per workgroup, waves
};
// Tiles through shared memory.
struct SqpMxTilePlan {
    int tile;   // index of the tile's shape (sqp_mx_tiles.hip)
    int parts;  // of K
};
int sqp_mx_few(int x_type, const SqpMxFewPlan &p, const SqpMxGemm &a, hipStream_t stream);
int sqp_mx_tiles(int x_type, const SqpMxTilePlan &p, const SqpMxGemm &a, hipStream_t stream);
struct SqpMxTileShape {
    int rows, cols;
    bool direct;  // for K of whole 128, 512 at least
};
// The tiles' shapes; those of the same shape differ in how far ahead they load (sqp_mx_tiles.hip).
constexpr int SQP_MX_TILES = 8, SQP_MX_DIRECT_TILES = 7;
constexpr SqpMxTileShape SQP_MX_TILE[SQP_MX_TILES] = {{256, 256, true}, {128, 256, true}, {128, 128, true}, {128, 128, true}, {64, 128, true}, {32, 128, true}, {32, 64, true},
                                                          {128, 128, false}};

#ifdef __HIPCC__
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

// Operands of the scaled matrix instructions: 32 codes per lane, e2m1 in the first half of the registers.
__device__ __forceinline__ i32x8 sqp_mx_operand(u32x4 a) { return __builtin_bit_cast(i32x8, __builtin_shufflevector(a, a, 0, 1, 2, 3, -1, -1, -1, -1)); }
__device__ __forceinline__ i32x8 sqp_mx_operand(u32x4 a, u32x4 b)
{
    return i32x8{(int)a.x, (int)a.y, (int)a.z, (int)a.w, (int)b.x, (int)b.y, (int)b.z, (int)b.w};
}

// Up to 16 scales of a row from p on (`left` of them are there, the others become 2^-127, and their codes zeros).
__device__ __forceinline__ u32x4 sqp_mx_load_scales(const uint8_t *p, int left)
{
    u32x4 v;
    if (left >= 16) {
        __builtin_memcpy(&v, p, 16);  // (rows of scales begin at any byte)
    } else {
        uint32_t w[4] = {0, 0, 0, 0};
        for (int i = 0; i < left; i++) w[i >> 2] |= (uint32_t)p[i] << (8 * (i & 3));
        v = u32x4{w[0], w[1], w[2], w[3]};
    }
    return v;
}

// 16 bytes moved down by `by` (the same for the whole wave), zeros behind.
__device__ __forceinline__ u32x4 sqp_mx_shift_down(u32x4 v, int by)
{
    const bool eight = by & 8, four = by & 4;
    v = u32x4{eight ? v.z : v.x, eight ? v.w : v.y, eight ? 0u : v.z, eight ? 0u : v.w};
    v = u32x4{four ? v.y : v.x, four ? v.z : v.y, four ? v.w : v.z, four ? 0u : v.w};
    return u32x4{__builtin_amdgcn_alignbyte(v.y, v.x, by & 3), __builtin_amdgcn_alignbyte(v.z, v.y, by & 3), __builtin_amdgcn_alignbyte(v.w, v.z, by & 3),
                 __builtin_amdgcn_alignbyte(0u, v.w, by & 3)};
}

// Four neighbouring columns of a row, already summed.
__device__ __forceinline__ void sqp_mx_store4(const SqpMxGemm &a, int m, int n, const f32x4 &s)
{
    if (a.silu) {
        *(uint32_t *)(a.y + (size_t)m * (a.N >> 1) + (n >> 1)) = sqp_half2(sqp_silu(s.x) * s.y, sqp_silu(s.z) * s.w);
    } else {
        *(uint2 *)(a.y + (size_t)m * a.N + n) = make_uint2(sqp_half2(s.x, s.y), sqp_half2(s.z, s.w));
    }
}
#endif
