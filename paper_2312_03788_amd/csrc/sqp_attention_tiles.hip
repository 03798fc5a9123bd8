// Attention over the paged cache for many rows per cached head: prompts and chunks of them.  Bound: the matrix cores, and beside
// them the softmax's vector work.
//
// A workgroup takes 128 rows (new token, query head) of one (sequence, cached head, part), a wave 32 of them, and goes through
// the tokens 64 at a time.  S^T = K Q^T and O^T = V^T P^T on 32x32x16 matrix instructions: a lane has one query row's scores (half
// of them, the other half in lane ^ 32), so the softmax's row reductions stay in the lane and its p are the second product's operand
// as they stand: tokens 16c + 8 (j >> 2) + 4h + (j & 3), j = 0..7, are slot (h, j) of its step c, h the lane's half.
// K and V^T lie in shared memory in fp16 (codes are exact there; their scales are applied to scores and p in fp32), twice, so
// that the next tile is fetched, converted and transposed while this one is used: one barrier per tile.  V is transposed on the
// way: a thread holds the 8 tokens of a slot group and pairs them up with byte permutations.
#include <algorithm>

#include "sqp_attention.h"

namespace {

template <int TYPE, int D>
__global__ void __launch_bounds__(256, 2) attention_tiles_kernel(const SqpAttention a, const SqpParts parts, int above_rows, int tiles)
{
    constexpr int BYTES = SqpCode<TYPE>::BYTES;
    constexpr int KU = D * BYTES / 16;       // 16-byte pieces per token of K
    constexpr int KP = KU / 4;               // of them per lane (a wave stages 16 tokens)
    constexpr int AHEAD = 4;                 // operands fetched ahead of the matrix instructions
    constexpr int VD = D / 32;               // dimensions per lane of V
    constexpr int VB = VD * BYTES;           // bytes of them per token
    constexpr int VW = (VB + 3) / 4;         // words of them
    __shared__ __attribute__((aligned(16))) h16 s_k[2][64 * D];
    __shared__ __attribute__((aligned(16))) h16 s_v[2][64 * D];
    __shared__ __attribute__((aligned(16))) float s_ks[2][64], s_vs[2][64];
    __shared__ __attribute__((aligned(16))) float s_lv[2][4];
    __shared__ int s_bad;

    const int kv_head = blockIdx.x, b = blockIdx.z, part = blockIdx.y % parts.parts;
    if (blockIdx.y == 0) sqp_zero_strays<D>(a, b, kv_head);
    const SqpSequence s = sqp_sequence(a, b);
    const int rows = s.n * a.group;
    if (rows <= above_rows) return;
    const int *table = a.table + b * a.table_stride;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63, col = lane & 31, h = lane >> 5;
    const int before = s.len - s.n;  // token i of the new ones sees before + i + 1
    const int mask = (1 << a.page_shift) - 1;

    // the last tiles, which see most, first
    for (int tile = tiles - 1 - (int)blockIdx.y / parts.parts; tile * SQP_TILE_ROWS < rows; tile += tiles) {
        const int row0 = tile * SQP_TILE_ROWS, row_last = min(row0 + SQP_TILE_ROWS, rows) - 1;
        const int most = before + row_last / a.group + 1, least = before + row0 / a.group + 1;
        const int nparts = parts.of(most);
        if (part >= nparts) continue;
        const int lo = part * parts.chunk, hi = part == nparts - 1 ? most : lo + parts.chunk;
        const int row = min(row0 + 32 * wave + col, rows - 1), token = row / a.group, head = kv_head * a.group + row - token * a.group;
        const int sees = before + token + 1;
        // of this wave's rows (a wave past the last row has none)
        const int wave_row = row0 + 32 * wave, wave_least = before + min(wave_row, rows - 1) / a.group + 1;
        const int wave_most = wave_row >= rows ? 0 : before + min(wave_row + 31, rows - 1) / a.group + 1;

        h16x8 qf[D / 16];
        const h16 *q = a.q + (size_t)(s.first + token) * a.q_stride + head * D + 8 * h;
#pragma unroll
        for (int c = 0; c < D / 16; c++) qf[c] = *(const h16x8 *)(q + 16 * c);

        u32x4 kw[KP];
        uint32_t vw[8][VW];
        float kscale = 0.f, vscale = 0.f;
        // A wave stages the 16 tokens base + 16 wave ..; their page is looked up a tile ahead.
        auto place = [&](int base) { return min(base + 16 * wave, (hi - 1) & ~15); };
        int page = lo < hi ? sqp_page(a, table, place(lo)) : 0;
        auto load = [&](int base) {
            const int t = place(base);
            const size_t r = (((size_t)__builtin_amdgcn_readfirstlane(page) * a.kv_heads + kv_head) << a.page_shift) + (t & mask);
            page = sqp_page(a, table, place(base + 64));
            const uint8_t *kp = (const uint8_t *)a.k + r * (D * BYTES) + lane * 16;
#pragma unroll
            for (int i = 0; i < KP; i++) kw[i] = *(const u32x4 *)(kp + 1024 * i);
            const uint8_t *vp = (const uint8_t *)a.v + r * (D * BYTES) + 4 * h * (D * BYTES) + col * VB;
#pragma unroll
            for (int j = 0; j < 8; j++) sqp_words<VB>(vp + (8 * (j >> 2) + (j & 3)) * (D * BYTES), vw[j]);
            if constexpr (TYPE != SQP_FP16) {
                kscale = a.k_scales[r + (lane & 15)];
                vscale = a.v_scales[r + (lane & 15)];
            }
        };
        bool bad = false;
        auto store = [&](int base, int buf) {
            if (base + 64 > least) {  // tokens that not all rows see, or that are none (memory past the length)
#pragma unroll
                for (int j = 0; j < 8; j++) {
                    const int key = base + 16 * wave + 8 * (j >> 2) + 4 * h + (j & 3);
#pragma unroll
                    for (int e = 0; e < VW; e++) {
                        if (key >= s.len) vw[j][e] = 0;
                        else bad = bad || sqp_not_finite<TYPE>(vw[j][e]);
                    }
                }
                if constexpr (TYPE != SQP_FP16) {
                    if (base + 16 * wave + (lane & 15) >= s.len) vscale = 0.f;
                    bad = bad || !(__builtin_fabsf(vscale) < INFINITY);
                }
            }
#pragma unroll
            for (int i = 0; i < KP; i++) {
                const int unit = lane + 64 * i, key = 16 * wave + unit / KU, piece = unit % KU;
                if constexpr (TYPE == SQP_FP16) {
                    *(u32x4 *)&s_k[buf][key * D + 8 * (piece ^ (key & (D / 8 - 1)))] = kw[i];
                } else {
                    const uint32_t w[4] = {kw[i].x, kw[i].y, kw[i].z, kw[i].w};
#pragma unroll
                    for (int e = 0; e < 2; e++) {
                        h16x2 p[4];
                        sqp_halves4<TYPE>(w[2 * e], p[0], p[1]);
                        sqp_halves4<TYPE>(w[2 * e + 1], p[2], p[3]);
                        const h16x8 x = {p[0].x, p[0].y, p[1].x, p[1].y, p[2].x, p[2].y, p[3].x, p[3].y};
                        *(h16x8 *)&s_k[buf][key * D + 8 * ((2 * piece + e) ^ (key & (D / 8 - 1)))] = x;
                    }
                }
            }
            uint32_t pairs[4][VB < 4 ? 4 : VD];
#pragma unroll
            for (int j = 0; j < 4; j++) {
#pragma unroll
                for (int e = 0; e < VW; e++) sqp_pair_up<TYPE>(vw[2 * j][e], vw[2 * j + 1][e], &pairs[j][e * (4 / BYTES)]);
            }
#pragma unroll
            for (int d = 0; d < VD; d++) {
                const int dim = VD * col + d;
                const u32x4 x = {pairs[0][d], pairs[1][d], pairs[2][d], pairs[3][d]};
                *(u32x4 *)&s_v[buf][dim * 64 + 8 * ((2 * wave + h) ^ ((dim ^ (dim >> 2)) & 7))] = x;
            }
            if constexpr (TYPE != SQP_FP16) {
                float top = __builtin_fabsf(vscale);
#pragma unroll
                for (int off = 8; off >= 1; off >>= 1) top = fmaxf(top, __shfl_xor(top, off, 64));
                if (lane < 16) {
                    s_ks[buf][16 * wave + lane] = kscale * a.scale2;
                    s_vs[buf][16 * wave + lane] = vscale;
                }
                if (lane == 0) s_lv[buf][wave] = ceilf(__builtin_amdgcn_logf(top));
            }
        };

        float m = SQP_LOWEST, l = 0.f, lv = TYPE == SQP_FP16 ? 0.f : -60.f;
        f32x16 o[D / 32];
#pragma unroll
        for (int d = 0; d < D / 32; d++) o[d] = (f32x16)(0.f);
        if (threadIdx.x == 0) s_bad = 0;
        if (lo < hi) {
            load(lo);
            store(lo, 0);
        }
        // Q's loads end here: left to the loop, the wait for them would also be one for the next tile's loads, in every round.
#pragma unroll
        for (int c = 0; c < D / 16; c++) asm volatile("" : "+v"(qf[c]));
        int buf = 0;
        for (int base = lo; base < hi; base += 64, buf ^= 1) {
            __syncthreads();
            const bool more = base + 64 < hi;
            if (more) load(base + 64);
            if (base < wave_most) {
                // The order of instructions is fixed: the compiler's own waits for every operand as soon as it is asked for.
                // Operands are fetched four matrix instructions ahead, and what has to be done to the first 32 tokens' scores is
                // done beside the next 32's products.
                f32x16 t[2];
                t[0] = t[1] = (f32x16)(0.f);
                h16x8 kf[AHEAD];
                f32x4 ks[4];
                auto fetch_k = [&](int n) {
                    const int key = 32 * (n / (D / 16)) + col, c = n % (D / 16);
                    kf[n % AHEAD] = *(const h16x8 *)&s_k[buf][key * D + 8 * ((2 * c + h) ^ (key & (D / 8 - 1)))];
                };
                // result register r of block i: token base + 32 i + 8 (r >> 2) + 4 h + (r & 3)
                auto fetch_ks = [&](int i, int r4) { ks[r4] = *(const f32x4 *)&s_ks[buf][32 * i + 8 * r4 + 4 * h]; };
                auto scale = [&](int i, int r4) {
#pragma unroll
                    for (int e = 0; e < 4; e++) t[i][4 * r4 + e] *= ks[r4][e];
                };
#pragma unroll
                for (int n = 0; n < AHEAD; n++) fetch_k(n);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int n = 0; n < D / 8; n++) {
                    t[n / (D / 16)] = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf[n % AHEAD], qf[n % (D / 16)], t[n / (D / 16)], 0, 0, 0);
                    if (n + AHEAD < D / 8) fetch_k(n + AHEAD);
                    if constexpr (TYPE != SQP_FP16) {  // (fp16: scores are scaled as p is formed)
                        const int j = n - D / 16;
                        if (j >= 0 && j < 4) fetch_ks(0, j);
                        if (j == D / 16 - 1) {
#pragma unroll
                            for (int r4 = 0; r4 < 4; r4++) {
                                scale(0, r4);
                                fetch_ks(1, r4);
                            }
                        }
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
                if constexpr (TYPE != SQP_FP16) {
#pragma unroll
                    for (int r4 = 0; r4 < 4; r4++) scale(1, r4);
                }
                if (base + 64 > wave_least) {
#pragma unroll
                    for (int i = 0; i < 2; i++)
#pragma unroll
                        for (int r = 0; r < 16; r++)
                            if (base + 32 * i + 8 * (r >> 2) + 4 * h + (r & 3) >= sees) t[i][r] = -INFINITY;
                }
                float top = t[0][0];
#pragma unroll
                for (int r = 1; r < 32; r++) top = fmaxf(top, t[r >> 4][r & 15]);
                if constexpr (TYPE == SQP_FP16) top *= a.scale2;
                float tile_lv = lv;
                if constexpr (TYPE != SQP_FP16) {
                    const f32x4 x = *(const f32x4 *)s_lv[buf];
                    tile_lv = fmaxf(lv, fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])));
                }
                // as in the few-rows kernel: p 2^-lv times a value's scale inside fp16's range
                if (__any(top + tile_lv > m + 12.f)) {
                    top = fmaxf(top, __shfl_xor(top, 32, 64));
                    const float next = top + tile_lv > m + 12.f ? top + tile_lv - 4.f : m, keep = sqp_exp2(m - next);
                    m = next;
                    l *= keep;
#pragma unroll
                    for (int d = 0; d < D / 32; d++) o[d] *= keep;
                }
                lv = tile_lv;
                // p of step c + 1 is formed beside the matrix instructions of step c
                h16x8 pf[2], vf[AHEAD];
                f32x4 vs[2];
                auto fetch_v = [&](int n) {
                    const int c = n / (D / 32), dim = 32 * (n % (D / 32)) + col;
                    vf[n % AHEAD] = *(const h16x8 *)&s_v[buf][dim * 64 + 8 * ((2 * c + h) ^ ((dim ^ (dim >> 2)) & 7))];
                };
                auto fetch_vs = [&](int c) {
                    if constexpr (TYPE != SQP_FP16) {
                        vs[0] = *(const f32x4 *)&s_vs[buf][16 * c + 4 * h];
                        vs[1] = *(const f32x4 *)&s_vs[buf][16 * c + 8 + 4 * h];
                    }
                };
                auto form = [&](int c, int from, int to) {
#pragma unroll
                    for (int j = from; j < to; j++) {
                        const float x = t[c >> 1][8 * (c & 1) + j];
                        const float p = sqp_exp2(TYPE == SQP_FP16 ? __builtin_fmaf(x, a.scale2, -m) : x - m);
                        l += p;
                        pf[c & 1][j] = (h16)(TYPE == SQP_FP16 ? p : p * vs[j >> 2][j & 3]);
                    }
                };
                fetch_vs(0);
#pragma unroll
                for (int n = 0; n < AHEAD; n++) fetch_v(n);
                __builtin_amdgcn_sched_barrier(0);
                form(0, 0, 8);
                fetch_vs(1);
                __builtin_amdgcn_sched_barrier(0);
                constexpr int ND = D / 32, SHARE = 8 / ND;
#pragma unroll
                for (int n = 0; n < 4 * ND; n++) {
                    const int c = n / ND, d = n % ND;
                    o[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf[n % AHEAD], pf[c & 1], o[d], 0, 0, 0);
                    if (n + AHEAD < 4 * ND) fetch_v(n + AHEAD);
                    if (c < 3) form(c + 1, SHARE * d, SHARE * (d + 1));
                    if (c < 2 && d == ND - 1) fetch_vs(c + 2);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            if (more) store(base + 64, buf ^ 1);
        }
        l += __shfl_xor(l, 32, 64);
        if (bad) s_bad = 1;
        __syncthreads();
        if (s_bad) {
            for (int r = row0 + wave; r <= row_last; r += 4) {
                const int tk = r / a.group;
                sqp_attend_row_of_part<TYPE, D>(a, parts, part, s.first + tk, kv_head * a.group + r - tk * a.group, before + tk + 1, table, lo, hi);
            }
        } else if (row0 + 32 * wave + col < rows) {
            const long at = (long)(s.first + token) * a.heads + head;
            float *partial;
            if (sqp_target<D>(parts, sees, part, at, partial)) {
                const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
                for (int d = 0; d < D / 32; d++)
#pragma unroll
                    for (int r4 = 0; r4 < 4; r4++) {
                        const int dim = 32 * d + 8 * r4 + 4 * h;
                        if (partial) {
                            *(f32x4 *)(partial + dim) = f32x4{o[d][4 * r4], o[d][4 * r4 + 1], o[d][4 * r4 + 2], o[d][4 * r4 + 3]};
                        } else {
                            h16x4 y;
#pragma unroll
                            for (int e = 0; e < 4; e++) y[e] = (h16)(l == 0.f ? 0.f : o[d][4 * r4 + e] * inv);
                            *(h16x4 *)(a.out + at * D + dim) = y;
                        }
                    }
                if (partial && h == 0) {
                    partial[D] = m;
                    partial[D + 1] = l;
                }
            }
        }
        __syncthreads();  // (s_bad and the tiles are written again for the next rows)
    }
}

template <int TYPE, int D>
void launch(const SqpAttention &a, const SqpParts &p, int above_rows, int max_q, hipStream_t st)
{
    const long rows = (long)max_q * a.group;
    const long tiles = std::min((rows + SQP_TILE_ROWS - 1) / SQP_TILE_ROWS, 65535L / p.parts);
    attention_tiles_kernel<TYPE, D><<<dim3((unsigned)a.kv_heads, (unsigned)(tiles * p.parts), (unsigned)a.B), 256, 0, st>>>(a, p, above_rows, (int)tiles);
}

}  // namespace

void sqp_attention_tiles(int type, int D, const SqpAttention &a, const SqpParts &p, int above_rows, int max_q, hipStream_t st)
{
#define TILES(TYPE) (D == 128 ? launch<TYPE, 128>(a, p, above_rows, max_q, st) : launch<TYPE, 64>(a, p, above_rows, max_q, st))
    if (type == SQP_FP16) TILES(SQP_FP16);
    else if (type == SQP_INT8) TILES(SQP_INT8);
    else TILES(SQP_E4M3);
#undef TILES
}
