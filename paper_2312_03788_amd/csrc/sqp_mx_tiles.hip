// Microscaled product in tiles: 32x32x64 scaled matrix instructions on operands that lie in shared memory as they do in memory.
// Bound: the matrix cores.
//
// A workgroup of four waves takes BM rows x BN columns, a wave 32 RT x 32 CT of them (weights are the instruction's rows, activations
// its columns).  K goes in stages of 128 bytes of activations (256 k of e2m1, 128 of e4m3) through two slots that are filled by direct
// loads into shared memory, the next stage while one is consumed; pieces of 16 bytes change places within 128 bytes, so that
// the eight rows that are read at once lie in different banks.  The order of blocks within a stage is free as long as both
// operands and their scales have the same: of 256 k lane half h takes blocks 4 h + s in step s, so that its four scales are one word.
// Scales come 16 bytes (512 k) of a row at a time through registers, since rows of them begin at any byte.
#include <algorithm>

#include "sqp_mx_gemm.h"

namespace {

typedef int rsrc_t __attribute__((ext_vector_type(4)));
__device__ __forceinline__ rsrc_t buffer_of(const void *p, uint32_t bytes)
{
    const uint64_t at = reinterpret_cast<uint64_t>(p);
    return rsrc_t{(int)(uint32_t)at, (int)(uint32_t)(at >> 32), (int)bytes, 0x00020000};
}

// 16 bytes per lane from base + lane_offset + offset to shared memory at dst + 16 lane (beyond the buffer: zeros).  In assembly, since
// the compiler would wait for it at the next read of shared memory; the kernel waits itself.
__device__ __forceinline__ void copy_piece(rsrc_t base, uint32_t lane_offset, uint32_t offset, uint32_t dst)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(dst), "v"(lane_offset), "s"(base), "s"(offset) : "memory");
}

constexpr int XCDS = 8;

// Workgroup w of `total`: its place when every XCD has one run of consecutive places.
__device__ __forceinline__ uint32_t xcd_run(uint32_t w, uint32_t total)
{
    const uint32_t xcd = w % XCDS, len = total / XCDS, more = total % XCDS;
    return xcd * len + (xcd < more ? xcd : more) + w / XCDS;
}

template <int XT, int RT, int CT, int WM, int WN>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(RT * CT > 8 ? 1 : 2)))
mx_tiles_kernel(const SqpMxGemm a, int tiles_m, int tiles_n, int group_m, int stages_per_part)
{
    constexpr bool FOUR = XT == SQP_E2M1;
    constexpr int XFMT = FOUR ? 4 : 0;
    constexpr int BM = 32 * RT * WM, BN = 32 * CT * WN;
    constexpr int BLOCKS = FOUR ? 8 : 4;            // of 32 k per stage
    constexpr int STEPS = BLOCKS / 2;
    constexpr int WB = 16 * BLOCKS;                 // bytes of a weight row per stage
    constexpr int SPC = 16 / BLOCKS;                // stages per chunk of 16 scales
    constexpr int XCOPIES = BM / 32, WCOPIES = BN * WB / 4096;  // copies of 1 KB per wave and stage
    constexpr int SROWS = (BM + BN + 255) / 256;    // rows of scales per thread
    __shared__ __attribute__((aligned(1024))) uint8_t s_x[2][BM * 128];
    __shared__ __attribute__((aligned(1024))) uint8_t s_w[2][BN * WB];
    __shared__ __attribute__((aligned(16))) uint8_t s_s[2][(BM + BN) * 16];

    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63, l32 = lane & 31, h = lane >> 5;
    const int wm = wave / WN, wn = wave % WN;
    const int blocks = a.K / SQP_MX_BLOCK, all_stages = (blocks + BLOCKS - 1) / BLOCKS;
    // the tile: groups of group_m rows of tiles, row index fastest
    int m0, n0;
    {
        const uint32_t i = xcd_run(blockIdx.x, gridDim.x), g = i / (uint32_t)(group_m * tiles_n), in = i - g * (uint32_t)(group_m * tiles_n);
        const uint32_t rows = min((uint32_t)group_m, (uint32_t)tiles_m - g * group_m), col = in / rows;
        m0 = (int)(g * group_m + in - col * rows) * BM;
        n0 = (int)col * BN;
    }
    const int first = blockIdx.y * stages_per_part, stages = min(all_stages - first, stages_per_part);

    const uint32_t x_row = (uint32_t)a.K / (FOUR ? 2 : 1), w_row = (uint32_t)a.K / 2;
    const rsrc_t xbuf = buffer_of(a.x, (uint32_t)a.M * x_row), wbuf = buffer_of(a.w, (uint32_t)a.N * w_row);
    // this lane's pieces: row and piece within the stage's bytes of that row
    uint32_t xoff[XCOPIES], woff[WCOPIES];
    int xpiece[XCOPIES], wpiece[WCOPIES];
#pragma unroll
    for (int j = 0; j < XCOPIES; j++) {
        const int row = 8 * (wave + 4 * j) + (lane >> 3);
        xpiece[j] = (lane & 7) ^ (row & 7);
        xoff[j] = (uint32_t)min(m0 + row, a.M - 1) * x_row + 16u * (uint32_t)xpiece[j];
    }
#pragma unroll
    for (int j = 0; j < WCOPIES; j++) {
        int row;
        if constexpr (FOUR) {
            row = 8 * (wave + 4 * j) + (lane >> 3);
            wpiece[j] = (lane & 7) ^ (row & 7);
        } else {
            row = 16 * (wave + 4 * j) + (lane >> 2);
            wpiece[j] = (lane & 3) ^ (row >> 1 & 3);
        }
        woff[j] = (uint32_t)min(n0 + row, a.N - 1) * w_row + 16u * (uint32_t)wpiece[j];
    }
    const uint32_t sx = (uint32_t)(size_t)&s_x[0][0], sw = (uint32_t)(size_t)&s_w[0][0];
    auto copy_stage = [&](int t, int slot) {
        const int st = first + t;
        const bool whole = (st + 1) * BLOCKS <= blocks;
        const uint32_t xat = (uint32_t)st * 128u, wat = (uint32_t)st * WB;
        const int xleft = FOUR ? blocks - st * BLOCKS : 2 * (blocks - st * BLOCKS), wleft = blocks - st * BLOCKS;
#pragma unroll
        for (int j = 0; j < XCOPIES; j++)
            copy_piece(xbuf, whole || xpiece[j] < xleft ? xoff[j] : 0xfff00000u, xat, __builtin_amdgcn_readfirstlane(sx + slot * (BM * 128) + (wave + 4 * j) * 1024));
#pragma unroll
        for (int j = 0; j < WCOPIES; j++)
            copy_piece(wbuf, whole || wpiece[j] < wleft ? woff[j] : 0xfff00000u, wat, __builtin_amdgcn_readfirstlane(sw + slot * (BN * WB) + (wave + 4 * j) * 1024));
    };
    u32x4 sv[SROWS];
    auto load_scales = [&](int chunk) {  // of the whole K
#pragma unroll
        for (int i = 0; i < SROWS; i++) {
            const int row = (int)threadIdx.x + 256 * i;
            const uint8_t *p = row < BM ? a.xs + (size_t)min(m0 + row, a.M - 1) * blocks : a.ws + (size_t)min(n0 + row - BM, a.N - 1) * blocks;
            const int at = 16 * chunk, left = blocks - at;
            if (left >= 16) {
                __builtin_memcpy(&sv[i], p + at, 16);
            } else {
                uint32_t v[4] = {0, 0, 0, 0};
                for (int b = 0; b < left; b++) v[b >> 2] |= (uint32_t)p[at + b] << (8 * (b & 3));
                sv[i] = u32x4{v[0], v[1], v[2], v[3]};
            }
        }
    };
    auto store_scales = [&](int chunk) {
#pragma unroll
        for (int i = 0; i < SROWS; i++) {
            const int row = (int)threadIdx.x + 256 * i;
            if (row < BM + BN) *(u32x4 *)&s_s[chunk & 1][16 * row] = sv[i];
        }
    };

    f32x16 acc[RT][CT];
#pragma unroll
    for (int i = 0; i < RT; i++)
#pragma unroll
        for (int j = 0; j < CT; j++) acc[i][j] = (f32x16)(0.f);

    const int xr = 32 * RT * wm + l32, wr = 32 * CT * wn + l32;  // this lane's row of the wave's first tile
    u32x4 xf[2][RT][FOUR ? 1 : 2], wf[2][CT];
    uint32_t xsc[RT], wsc[CT];
    auto fetch = [&](int slot, int s, int to) {
#pragma unroll
        for (int i = 0; i < RT; i++) {
            const int row = xr + 32 * i;
            const uint8_t *p = &s_x[slot][row * 128];
            if constexpr (FOUR) {
                xf[to][i][0] = *(const u32x4 *)(p + 16 * ((4 * h + s) ^ (row & 7)));
            } else {  // the lane's first 16 values belong to block s, the others to block 2 + s
                xf[to][i][0] = *(const u32x4 *)(p + 16 * ((2 * s + h) ^ (row & 7)));
                xf[to][i][FOUR ? 0 : 1] = *(const u32x4 *)(p + 16 * ((4 + 2 * s + h) ^ (row & 7)));
            }
        }
#pragma unroll
        for (int j = 0; j < CT; j++) {
            const int row = wr + 32 * j;
            const uint8_t *p = &s_w[slot][row * WB];
            if constexpr (FOUR) wf[to][j] = *(const u32x4 *)(p + 16 * ((4 * h + s) ^ (row & 7)));
            else wf[to][j] = *(const u32x4 *)(p + 16 * ((2 * h + s) ^ (row >> 1 & 3)));
        }
    };
    auto fetch_scales = [&](int t) {
        const int st = first + t;
        const uint8_t *p = &s_s[(st / SPC) & 1][(st % SPC) * BLOCKS + (FOUR ? 4 : 2) * h];
#pragma unroll
        for (int i = 0; i < RT; i++) xsc[i] = FOUR ? *(const uint32_t *)(p + 16 * (xr + 32 * i)) : *(const uint16_t *)(p + 16 * (xr + 32 * i));
#pragma unroll
        for (int j = 0; j < CT; j++) wsc[j] = FOUR ? *(const uint32_t *)(p + 16 * (BM + wr + 32 * j)) : *(const uint16_t *)(p + 16 * (BM + wr + 32 * j));
    };
#define SQP_MX_MFMA(s)                                                                                                                          \
    _Pragma("unroll") for (int i = 0; i < RT; i++)                                                                                              \
    {                                                                                                                                           \
        i32x8 b;                                                                                                                                \
        if constexpr (FOUR) b = sqp_mx_operand(xf[(s) & 1][i][0]);                                                                              \
        else b = sqp_mx_operand(xf[(s) & 1][i][0], xf[(s) & 1][i][FOUR ? 0 : 1]);                                                               \
        _Pragma("unroll") for (int j = 0; j < CT; j++) acc[i][j] =                                                                              \
            __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(sqp_mx_operand(wf[(s) & 1][j]), b, acc[i][j], 4, XFMT, s, (int)wsc[j], s, (int)xsc[i]); \
    }

    // the first stage, and the first chunk's scales
    copy_stage(0, 0);
    load_scales(first / SPC);
    store_scales(first / SPC);
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    if (stages > 1) copy_stage(1, 1);
    if ((first + 1) % SPC == 0 || SPC == 1 || first % SPC == 0) {}
    fetch_scales(0);
    fetch(0, 0, 0);
    for (int t = 0; t < stages; t++) {
        const int slot = t & 1, st = first + t;
        // scales of the next chunk: on their way while the chunk's last stage is consumed
        const bool turn = (st + 1) % SPC == 0 && t + 1 < stages;
        if (turn) load_scales((st + 1) / SPC);
#pragma unroll
        for (int s = 0; s < STEPS; s++) {
            if (s + 1 < STEPS) {
                fetch(slot, s + 1, (s + 1) & 1);
                if (s == 0) { SQP_MX_MFMA(0) }
                if constexpr (STEPS > 2) {
                    if (s == 1) { SQP_MX_MFMA(1) }
                    if (s == 2) { SQP_MX_MFMA(2) }
                }
            } else {
                uint32_t keep_x[RT], keep_w[CT];
#pragma unroll
                for (int i = 0; i < RT; i++) keep_x[i] = xsc[i];
#pragma unroll
                for (int j = 0; j < CT; j++) keep_w[j] = wsc[j];
                if (t + 1 < stages) {
                    if (turn) store_scales((st + 1) / SPC);
                    // every read of this slot has ended, the next stage has landed
                    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
                    if (t + 2 < stages) copy_stage(t + 2, slot);
                    fetch_scales(t + 1);
                    fetch(slot ^ 1, 0, 0);
                }
                uint32_t next_x[RT], next_w[CT];
#pragma unroll
                for (int i = 0; i < RT; i++) { next_x[i] = xsc[i]; xsc[i] = keep_x[i]; }
#pragma unroll
                for (int j = 0; j < CT; j++) { next_w[j] = wsc[j]; wsc[j] = keep_w[j]; }
                if constexpr (STEPS > 2) { SQP_MX_MFMA(3) } else { SQP_MX_MFMA(1) }
#pragma unroll
                for (int i = 0; i < RT; i++) xsc[i] = next_x[i];
#pragma unroll
                for (int j = 0; j < CT; j++) wsc[j] = next_w[j];
            }
        }
    }
    // result register r of tile (i, j): row 32 i + l32, columns 32 j + 8 (r >> 2) + 4 h + (r & 3)
#pragma unroll
    for (int i = 0; i < RT; i++) {
        const int m = m0 + xr + 32 * i;
        if (m >= a.M) continue;
#pragma unroll
        for (int j = 0; j < CT; j++)
#pragma unroll
            for (int r4 = 0; r4 < 4; r4++) {
                const int n = n0 + 32 * CT * wn + 32 * j + 8 * r4 + 4 * h;
                if (n >= a.N) continue;
                const f32x4 v = {acc[i][j][4 * r4], acc[i][j][4 * r4 + 1], acc[i][j][4 * r4 + 2], acc[i][j][4 * r4 + 3]};
                if (a.part) *(f32x4 *)(a.part + ((size_t)blockIdx.y * a.M + m) * a.N + n) = v;
                else sqp_mx_store4(a, m, n, v);
            }
    }
}

// The K parts' sums joined, in their order.
__global__ void __launch_bounds__(256) mx_join_kernel(const SqpMxGemm a, int parts)
{
    const long n4 = a.N / 4, all = a.M * n4, i = (long)blockIdx.x * 256 + threadIdx.x;
    if (i >= all) return;
    f32x4 s = ((const f32x4 *)a.part)[i];
    for (int p = 1; p < parts; p++) s += ((const f32x4 *)a.part)[i + p * all];
    sqp_mx_store4(a, (int)(i / n4), 4 * (int)(i % n4), s);
}

struct Shape {
    int rows, cols;
};
constexpr Shape SHAPES[SQP_MX_TILES] = {{256, 256}, {128, 128}, {64, 128}, {32, 128}};

template <int XT, int RT, int CT, int WM, int WN>
int launch(const SqpMxTilePlan &p, const SqpMxGemm &a, hipStream_t st)
{
    constexpr int BM = 32 * RT * WM, BN = 32 * CT * WN, BLOCKS = XT == SQP_E2M1 ? 8 : 4;
    const int tm = (a.M + BM - 1) / BM, tn = (a.N + BN - 1) / BN;
    const int stages = (a.K / SQP_MX_BLOCK + BLOCKS - 1) / BLOCKS, per = (stages + p.parts - 1) / p.parts, parts = (stages + per - 1) / per;
    if ((long)tm * tn > 0x7fffffffL || parts > 65535) return SQP_ERR_SHAPE;
    SqpMxGemm b = a;
    if (parts == 1) b.part = nullptr;
    mx_tiles_kernel<XT, RT, CT, WM, WN><<<dim3((unsigned)(tm * tn), (unsigned)parts), 256, 0, st>>>(b, tm, tn, std::min(tm, 4), per);
    if (parts > 1) mx_join_kernel<<<(unsigned)(((long)a.M * (a.N / 4) + 255) / 256), 256, 0, st>>>(b, parts);
    return sqp_launch_status();
}

template <int XT>
int pick(const SqpMxTilePlan &p, const SqpMxGemm &a, hipStream_t st)
{
    switch (p.tile) {
        case 0: return launch<XT, 4, 4, 2, 2>(p, a, st);
        case 1: return launch<XT, 2, 2, 2, 2>(p, a, st);
        case 2: return launch<XT, 2, 1, 1, 4>(p, a, st);
        case 3: return launch<XT, 1, 1, 1, 4>(p, a, st);
    }
    return SQP_ERR_SHAPE;
}

}  // namespace

void sqp_mx_tile_shape(int tile, int *rows, int *cols)
{
    *rows = SHAPES[tile].rows;
    *cols = SHAPES[tile].cols;
}

int sqp_mx_tiles(int x_type, const SqpMxTilePlan &p, const SqpMxGemm &a, hipStream_t st)
{
    return x_type == SQP_E2M1 ? pick<SQP_E2M1>(p, a, st) : pick<SQP_E4M3>(p, a, st);
}
