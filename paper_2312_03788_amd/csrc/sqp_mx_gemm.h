// The product of microscaled activations and weights: what its kernels share.
#pragma once
#include "sqp_mx.h"

struct SqpMxGemm {
    int M, N, K;
    int silu;  // columns alternate (gate, up): y [M][N / 2]
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
void sqp_mx_tile_shape(int tile, int *rows, int *cols);
constexpr int SQP_MX_TILES = 4;

#ifdef __HIPCC__
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

// Operands of the scaled matrix instructions: 32 codes per lane, e2m1 in the first half of the registers.
__device__ __forceinline__ i32x8 sqp_mx_operand(u32x4 a) { return i32x8{(int)a.x, (int)a.y, (int)a.z, (int)a.w, 0, 0, 0, 0}; }
__device__ __forceinline__ i32x8 sqp_mx_operand(u32x4 a, u32x4 b)
{
    return i32x8{(int)a.x, (int)a.y, (int)a.z, (int)a.w, (int)b.x, (int)b.y, (int)b.z, (int)b.w};
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
