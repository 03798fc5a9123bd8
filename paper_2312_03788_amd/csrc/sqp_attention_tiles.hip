// Attention over the paged cache for many rows per cached head: prompts and chunks of them.  Bound: the matrix cores, and beside
// them the softmax's vector work.
//
// A workgroup of W = 4 or 8 waves takes 32 W rows (new token, query head) of one (sequence, cached head, part), a wave 32 of them,
// and goes through the tokens 64 at a time.  S^T = K Q^T and O^T = V^T P^T on 32x32x16 matrix instructions: a lane has one query
// row's scores (half of them, the other half in lane ^ 32), so the softmax's row reductions stay in the lane and its p are the
// second product's operand as they stand: tokens 16c + 8 (j >> 2) + 4h + (j & 3), j = 0..7, are slot (h, j) of its step c, h the
// lane's half.
//
// Work goes in steps of 32 tokens whose order of instructions is fixed (left alone, the compiler waits for every operand as soon
// as it has asked for it): the next step's scores and this step's output are computed by the matrix cores beside this
// step's softmax, an exponential or two behind each matrix instruction, operands fetched some instructions ahead.
//
// K and V^T lie in shared memory in fp16 (codes are exact there).  The scale of a token's key multiplies its scores in fp32;
// the scale of its value is part of the exponent, p' = 2^(s + lv - m) with lv its logarithm, and leaves the sum again by its
// inverse, so that what is rounded to fp16 is the weight of the value's codes and stays inside fp16's range whatever the
// scales.  V is transposed on the way into shared memory: a thread holds the 8 tokens of a slot and pairs them up with
// byte permutations.  What is stored between two barriers is read after the second, and values come from memory a whole
// tile ahead of their storing; with three tiles of V (8 waves) that is one barrier per 64 tokens, with two (4 waves, two
// workgroups per compute unit) it is two.
//
// Measured: 2048 tokens behind 14336, 64 heads on 8, e4m3: 1080 to 1170 us from box to box, 880 to 950 TFLOP/s, where a large dense
// fp16 product of the library reaches 1134 and a loop of matrix instructions alone 1572: all of them run at the clock that the
// power limit leaves (1.8 of 2.4 GHz here).  A tile of 64 tokens takes a compute unit 2.2 to 2.35 us; without staging, maxima,
// exponentials and barriers it still takes 1.8 to 2.0.  A 2048-token prompt of 32 heads: 59.4 us; its longest tile goes through
// 32 steps of 64 tokens alone on its compute unit at 1.4 to 1.9 us each, in which latencies show that a second wave would hide.
// Over e2m1 blocks (fp16 values by the time they are in shared memory, so that the products are those of an fp16 cache): 1024 tokens behind
// 7168, 64 heads on 8, 282 us, 910 TFLOP/s.
// Dropped (figures of the kernel as it was then): 64 rows per wave with one wave per SIMD (half the reads of shared memory, but nothing hides what the order of
// instructions does not: 1288 us where 128-row tiles took 1240); stores spread over a step (their loads have less time: the
// prompt 68.6 -> 74.6 us); K in shared memory with its scale multiplied in (a rounding more in the scores); p cut to 11 bits before
// the sum takes it too, so that its error leaves rows that a few tokens rule (worst of 70 cases 1.37 times the output's rounding
// instead of 1.45, but the chunk 1090 -> 1119 us).
#include <algorithm>

#include "sqp_attention.h"

namespace {

template <int TYPE, int D, int W>
__global__ void __launch_bounds__(64 * W, 2) attention_tiles_kernel(const SqpAttention a, const SqpParts parts, int above_rows, int fold)
{
    constexpr bool BLOCKS = TYPE == SQP_E2M1, CODES = TYPE != SQP_FP16 && !BLOCKS;  // (codes with a scale per token)
    constexpr int ROWS = 32 * W, BYTES = TYPE == SQP_FP16 ? 2 : 1, ROW = SQP_ROW_BYTES<TYPE, D>;
    constexpr int SB = D / 32;                      // bytes of scales per token (blocks)
    constexpr int TOKENS = 64 / W;                  // that a wave stages
    constexpr int KU = ROW / 16;                    // 16-byte pieces per token of K
    constexpr int KL = (TOKENS * KU + 63) / 64;     // of them per lane
    constexpr int KPIECES = KL * (BLOCKS ? 4 : CODES ? 2 : 1);  // its stores
    constexpr int VD = W == 4 ? D / 32 : D / 64;    // dimensions per lane of V (4 waves: half a wave holds a token, 8 waves: a wave)
    constexpr int VSUB = D / 32 / VD;               // blocks of 32 rows of V^T per dimension of a lane
    constexpr int VB = BLOCKS ? (VD + 1) / 2 : VD * BYTES, VW = (VB + 3) / 4;  // (blocks, one dimension per lane: a byte, and half of it)
    constexpr int NK = D / 16, NV = D / 32;         // operands per step: of K, of V per 16 tokens
    constexpr int AHEAD = CODES && W == 4 ? 3 : 4;  // operands fetched ahead (as many as the registers hold)
    constexpr int KROW = D + 8, VROW = 64 + 8;      // 16 bytes between rows: eight lanes' operands lie in eight different sets of banks
    constexpr int VBUFS = W == 8 ? 3 : 2;
    __shared__ __attribute__((aligned(16))) h16 s_k[2][64 * KROW];
    __shared__ __attribute__((aligned(16))) h16 s_v[VBUFS][D * VROW];
    __shared__ __attribute__((aligned(16))) float s_ks[2][64], s_lv[2][64], s_rv[VBUFS][64];

    const int kv_head = blockIdx.x, part = blockIdx.y % parts.parts, ranks = gridDim.y / parts.parts;
    if (blockIdx.y == 0) sqp_zero_strays<D>(a, kv_head);
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63, col = lane & 31, h = lane >> 5;
    const int mask = (1 << a.page_shift) - 1;
    // what this thread stages of a tile: K's tokens first_token .., V's slots (v_half, j) of 16 tokens, dimensions VD v_lane ..
    const int block16 = TOKENS * wave / 16, first_token = TOKENS * wave % 16;
    const int v_half = W == 4 ? h : wave & 1, v_lane = W == 4 ? col : lane;

    for (int rank = blockIdx.y / parts.parts;; rank += ranks) {  // (once, as long as the starts are in order)
        const SqpTile at_tile = sqp_pick_tile(a, above_rows, ROWS, rank, fold);
        const int b = __builtin_amdgcn_readfirstlane(at_tile.b), tile = __builtin_amdgcn_readfirstlane(at_tile.tile);
        if (b < 0) break;
        const SqpSequence s = sqp_one_sequence(a, b);
        const int rows = s.n * a.group;
        const int *table = a.table + b * a.table_stride;
        const int before = s.len - s.n;  // token i of the new ones sees before + i + 1
        const int row0 = tile * ROWS, row_last = min(row0 + ROWS, rows) - 1;
        const int most = before + row_last / a.group + 1;
        const int nparts = parts.of(most);
        if (part >= nparts) continue;
        const int lo = part * parts.chunk, hi = part == nparts - 1 ? most : lo + parts.chunk;
        const int row = min(row0 + 32 * wave + col, rows - 1), token = row / a.group, head = kv_head * a.group + row - token * a.group;
        const int sees = before + token + 1;
        // of this wave's rows (a wave past the last row has none)
        const int wave_row = row0 + 32 * wave, wave_least = before + min(wave_row, rows - 1) / a.group + 1;
        const int wave_most = wave_row >= rows ? 0 : before + min(wave_row + 31, rows - 1) / a.group + 1;

        h16x8 qf[NK];
        auto load_q = [&] {
            const h16 *q = a.q + (size_t)(s.first + token) * a.q_stride + head * D + 8 * h;
#pragma unroll
            for (int c = 0; c < NK; c++) qf[c] = *(const h16x8 *)(q + 16 * c);
        };
        // ---- staging; pages are looked up a tile ahead
        uint32_t kw[4 * KL], vw[8 * VW];
        uint32_t kb = 0, vb[2 * SB];  // blocks: the scale of this lane's piece of K, the scales of its 8 tokens' values
#pragma unroll
        for (int i = 0; i < 2 * SB; i++) vb[i] = 0;
        float kscale = 0.f, kvscale = 0.f, vscale = 0.f;
        auto place = [&](int base) { return min(base + 16 * block16, (hi - 1) & ~15); };
        auto look_up = [&](int base) { return lo < hi ? sqp_page(a, table, place(base)) : 0; };
        auto cache_row = [&](int page, int base) {
            return (((size_t)__builtin_amdgcn_readfirstlane(page) * a.kv_heads + kv_head) << a.page_shift) + (place(base) & mask);
        };
        int page_k = look_up(lo), page_v = page_k;
        auto load_k = [&](int base) {
            const size_t r = cache_row(page_k, base) + first_token;
            page_k = look_up(base + 64);
            const uint8_t *kp = (const uint8_t *)a.k + r * ROW + lane % (TOKENS * KU) * 16;
#pragma unroll
            for (int i = 0; i < KL; i++) sqp_words<16>(kp + 1024 * i, &kw[4 * i]);
            if constexpr (CODES) {
                kscale = ((const float *)a.k_scales)[r + lane % TOKENS];
                kvscale = ((const float *)a.v_scales)[r + lane % TOKENS];
            }
            if constexpr (BLOCKS) kb = ((const uint8_t *)a.k_scales)[r * SB + lane % (TOKENS * KU)];
        };
        auto load_v = [&](int base) {
            const size_t r = cache_row(page_v, base);
            page_v = look_up(base + 64);
            const uint8_t *vp = (const uint8_t *)a.v + (r + 4 * v_half) * ROW + (BLOCKS ? v_lane * VD / 2 : v_lane * VB);
#pragma unroll
            for (int j = 0; j < 8; j++) sqp_words<VB>(vp + (8 * (j >> 2) + (j & 3)) * ROW, &vw[j * VW]);
            if constexpr (CODES) vscale = ((const float *)a.v_scales)[r + first_token + lane % TOKENS];
            if constexpr (BLOCKS) {
                const uint8_t *bp = (const uint8_t *)a.v_scales + (r + 4 * v_half) * SB;
                sqp_words<4 * SB>(bp, &vb[0]);
                sqp_words<4 * SB>(bp + 8 * SB, &vb[SB]);
            }
        };
        // (The empty statements keep a piece's work, and with it the wait for its loads, where the piece is.)
        auto store_k = [&](int buf, int piece) {
            const int i = BLOCKS ? piece / 4 : CODES ? piece / 2 : piece, unit = lane % (TOKENS * KU) + 64 * i;
#pragma unroll
            for (int e = 0; e < 4; e++) asm volatile("" : "+v"(kw[4 * i + e]));
            h16 *to = &s_k[buf][(16 * block16 + first_token + unit / KU) * KROW];
            if constexpr (BLOCKS) {
                *(h16x8 *)&to[32 * (unit % KU) + 8 * (piece & 3)] = sqp_e2m1_halves8(kw[4 * i + (piece & 3)], sqp_key_scale(kb));
            } else if constexpr (CODES) {
                h16x2 p[4];
                sqp_halves4<TYPE>(kw[4 * i + 2 * (piece & 1)], p[0], p[1]);
                sqp_halves4<TYPE>(kw[4 * i + 2 * (piece & 1) + 1], p[2], p[3]);
                *(h16x8 *)&to[16 * (unit % KU) + 8 * (piece & 1)] = h16x8{p[0].x, p[0].y, p[1].x, p[1].y, p[2].x, p[2].y, p[3].x, p[3].y};
                if (piece == KPIECES - 1 && lane < TOKENS) {
                    s_ks[buf][16 * block16 + first_token + lane] = kscale * a.scale2;
                    s_lv[buf][16 * block16 + first_token + lane] = kvscale >= 0.f && kvscale < 0x1p40f ? sqp_log_scale(kvscale) : __builtin_nanf("");
                }
            } else {
                *(u32x4 *)&to[8 * (unit % KU)] = u32x4{kw[4 * i], kw[4 * i + 1], kw[4 * i + 2], kw[4 * i + 3]};
            }
        };
        // Tokens past the length, whatever memory holds there.
        auto clear_v = [&](int base) {
            if (__builtin_expect(base + 64 > s.len, 0)) {
#pragma unroll
                for (int j = 0; j < 8; j++) {
                    const int key = base + 16 * block16 + 8 * (j >> 2) + 4 * v_half + (j & 3);
#pragma unroll
                    for (int e = 0; e < VW; e++) vw[j * VW + e] = key >= s.len ? 0 : vw[j * VW + e];
                    if constexpr (BLOCKS) {
                        if constexpr (SB == 4) vb[j] = key >= s.len ? 0 : vb[j];
                        else vb[j / 2] &= key >= s.len ? (j & 1 ? 0xffffu : 0xffff0000u) : 0xffffffffu;
                    }
                }
            }
        };
        auto store_v = [&](int buf, int d) {
            u32x4 x;
#pragma unroll
            for (int j = 0; j < 8; j++) asm volatile("" : "+v"(vw[j * VW + (BLOCKS ? 0 : d * BYTES / 4)]));
            if constexpr (BLOCKS) {
                auto one = [&](int j) {  // dimensions d and its neighbour of token j
                    const uint32_t s = SB == 4 ? vb[j] : vb[j / 2] >> (j & 1 ? 16 : 0);
                    const uint32_t w = VD == 1 ? vw[j] >> (4 * (v_lane & 1)) : vw[j];
                    return sqp_e2m1_halves2(w, sqp_value_scale(s >> (8 * (VD * v_lane / 32)) & 255u), d / 2);
                };
#pragma unroll
                for (int j = 0; j < 4; j++) x[j] = __builtin_amdgcn_perm(one(2 * j + 1), one(2 * j), d & 1 ? 0x07060302u : 0x05040100u);
            } else {
#pragma unroll
                for (int j = 0; j < 4; j++) x[j] = sqp_pair<TYPE>(&vw[2 * j * VW], &vw[(2 * j + 1) * VW], d);
            }
            *(u32x4 *)&s_v[buf][(32 * VSUB * d + v_lane) * VROW + 16 * block16 + 8 * v_half] = x;
            if (CODES && d == VD - 1 && lane < TOKENS) s_rv[buf][16 * block16 + first_token + lane] = 1.f / fmaxf(vscale, SQP_LEAST_SCALE);
        };

        // ---- steps
        float m = SQP_LOWEST, l = 0.f, l2 = 0.f, top = 0.f;  // l2: every second one's share of the sum
        f32x16 o[NV], t, u;
#pragma unroll
        for (int d = 0; d < NV; d++) o[d] = (f32x16)(0.f);
        h16x8 kf[AHEAD], vf[AHEAD], pf[2];
        f32x4 ks[2], lv[2], rv[2];
        auto fetch_k = [&](int buf, int half, int c) { kf[c % AHEAD] = *(const h16x8 *)&s_k[buf][(32 * half + col) * KROW + 16 * c + 8 * h]; };
        auto fetch_v = [&](int buf, int half, int n) {
            vf[n % AHEAD] = *(const h16x8 *)&s_v[buf][(32 * (n % NV) + col) * VROW + 32 * half + 16 * (n / NV) + 8 * h];
        };
        // result register r of a step's scores: token 8 (r >> 2) + 4 h + (r & 3) of its 32
        auto fetch_ks = [&](int buf, int half, int r4) {
            if constexpr (CODES) {
                ks[r4 & 1] = *(const f32x4 *)&s_ks[buf][32 * half + 8 * r4 + 4 * h];
                lv[r4 & 1] = *(const f32x4 *)&s_lv[buf][32 * half + 8 * r4 + 4 * h];
            }
        };
        auto fetch_rv = [&](int buf, int half, int r4) {
            if constexpr (CODES) rv[r4 & 1] = *(const f32x4 *)&s_rv[buf][32 * half + 8 * r4 + 4 * h];
        };
        // A fourth of a step's scores: their scales, and the row's largest (fp16: scores are scaled as p is formed).
        auto take_max = [&](f32x16 &x, int r4) {
#pragma unroll
            for (int e = 0; e < 4; e++) {
                if constexpr (CODES) x[4 * r4 + e] = __builtin_fmaf(x[4 * r4 + e], ks[r4 & 1][e], lv[r4 & 1][e]);
                top = r4 == 0 && e == 0 ? x[0] : fmaxf(top, x[4 * r4 + e]);
            }
            asm volatile("" : "+v"(top));
        };
        // p of result register n (8 of either 16 tokens) comes about in three stages, which the steps keep apart: one that follows
        // the other at once would wait for it.
        f32x16 e;
        auto stage1 = [&](const f32x16 &x, int n) {
            float v = CODES ? x[n] - m : __builtin_fmaf(x[n], a.scale2, -m);
            asm volatile("" : "+v"(v));
            e[n] = v;
        };
        auto stage2 = [&](int n) {
            float p = sqp_exp2(e[n]);
            asm volatile("" : "+v"(p));
            e[n] = p;
        };
        auto stage3 = [&](int n) {  // two of them
            const h16x2 p = {(h16)e[n], (h16)e[n + 1]};
            pf[n >> 3][n & 7] = p.x;
            pf[n >> 3][(n & 7) + 1] = p.y;
            if constexpr (CODES) {
                l = __builtin_fmaf(e[n], rv[n >> 2 & 1][n & 3], l);
                l2 = __builtin_fmaf(e[n + 1], rv[n >> 2 & 1][(n & 3) + 1], l2);
                asm volatile("" : "+v"(l2));
            } else {
                l = __builtin_amdgcn_fdot2(p, h16x2{(h16)1.f, (h16)1.f}, l, false);
            }
            asm volatile("" : "+v"(l));
        };
        // Masks and the running maximum, once a step's scores are there (SQP_WEIGHT_TOP: the maximum is changed at the first tokens, and
        // where a score outgrows it).
        auto settle = [&](f32x16 &x, int base) {
            if (__builtin_expect(base + 32 > wave_least, 0)) {
                top = -INFINITY;
#pragma unroll
                for (int r = 0; r < 16; r++) {
                    int left = sees - base - 4 * h;
                    asm volatile("" : "+v"(left));  // (known to be the same sixteen times, the comparisons become one chain)
                    x[r] = 8 * (r >> 2) + (r & 3) >= left ? -INFINITY : x[r];
                    top = fmaxf(top, x[r]);
                }
            }
            const float reach = CODES ? top : top * a.scale2;
            if (__builtin_expect(__any(reach > m + SQP_WEIGHT_MOST), 0)) {
                const float both = fmaxf(reach, __shfl_xor(reach, 32, 64)), next = both > m + SQP_WEIGHT_MOST ? both - SQP_WEIGHT_TOP : m, keep = sqp_exp2(m - next);
                m = next;
                l *= keep;
                l2 *= keep;
#pragma unroll
                for (int d = 0; d < NV; d++) o[d] *= keep;
            }
        };
        // One step: the softmax and output of the scores x with V of (vbuf, vhalf), and the next step's scores y with K of
        // (kbuf, khalf).  The matrix instructions are NK/2 of the scores, then the others in turn with the first 16
        // tokens' output, then the last 16 tokens' output; pieces of the staged tile are stored beside the last ones.
        auto step = [&](f32x16 &x, f32x16 &y, int vbuf, int vhalf, int kbuf, int khalf, int pieces, auto store) {
            constexpr int MIXED = NK / 2 + NK / 2 + NV, ALL = NK + 2 * NV;
#pragma unroll
            for (int c = 0; c < AHEAD; c++) fetch_k(kbuf, khalf, c);
#pragma unroll
            for (int r4 = 0; r4 < 2; r4++) fetch_rv(vbuf, vhalf, r4);
            y = (f32x16)(0.f);
            __builtin_amdgcn_sched_barrier(0);
            // stage 2 of how many p is done behind matrix instruction n: the first 8 before the first output asks for them, the other 8
            // before the last 16 tokens'; stage 1 an instruction before, stage 3 one after
            auto due = [](int n) {
                return n < 0 ? 0 : n < NK / 2 ? (n + 1) * 8 / (NK / 2) : n < MIXED - 1 ? 8 + (n + 1 - NK / 2) * 8 / (MIXED - 1 - NK / 2) : 16;
            };
            int kn = 0, vn = 0, done1 = 0, done2 = 0, done3 = 0;
#pragma unroll
            for (; done1 < 8; done1++) stage1(x, done1);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int n = 0; n < ALL; n++) {
                if (n < NK / 2 || (n < MIXED && (n - NK / 2) % 2 == 0)) {
                    y = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf[kn % AHEAD], qf[kn], y, 0, 0, 0);
                    asm volatile("" : "+v"(y));  // (keeps the instruction here)
                    if (kn < AHEAD) fetch_v(vbuf, vhalf, kn);
                    if (kn + AHEAD < NK) fetch_k(kbuf, khalf, kn + AHEAD);
                    kn++;
                } else {
                    o[vn % NV] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf[vn % AHEAD], pf[vn / NV], o[vn % NV], 0, 0, 0);
                    asm volatile("" : "+v"(o[vn % NV]));
                    if (vn + AHEAD < 2 * NV) fetch_v(vbuf, vhalf, vn + AHEAD);
                    vn++;
                }
#pragma unroll
                for (; done1 < due(n + 1); done1++) stage1(x, done1);
#pragma unroll
                for (; done2 < due(n); done2++) stage2(done2);
#pragma unroll
                for (; done3 + 2 <= due(n - 1); done3 += 2) {
                    stage3(done3);
                    if (done3 % 4 == 2 && done3 < 8) fetch_rv(vbuf, vhalf, done3 / 4 + 2);
                }
                if (n >= MIXED - 2 && n < MIXED) fetch_ks(kbuf, khalf, n - (MIXED - 2));
                if (n >= MIXED) {
                    const int i = n - MIXED;  // of NV
#pragma unroll
                    for (int r4 = i * 4 / NV; r4 < (i + 1) * 4 / NV; r4++) {
                        take_max(y, r4);
                        if (r4 < 2) fetch_ks(kbuf, khalf, r4 + 2);
                    }
#pragma unroll
                    for (int piece = i * pieces / NV; piece < (i + 1) * pieces / NV; piece++) store(piece);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        };

        if (lo < hi) {  // the first tile, and the second one's K; the third one's K and the second one's V are on their way then
            load_k(lo);
            load_v(lo);
            load_q();
            uint32_t first_kw[4 * KL];
            const float first_kscale = kscale, first_kvscale = kvscale;
            const uint32_t first_kb = kb;
#pragma unroll
            for (int i = 0; i < 4 * KL; i++) first_kw[i] = kw[i];
            load_k(lo + 64);
            clear_v(lo);
#pragma unroll
            for (int i = 0; i < VD; i++) store_v(0, i);
            load_v(lo + 64);
#pragma unroll
            for (int i = 0; i < KPIECES; i++) store_k(1, i);
#pragma unroll
            for (int i = 0; i < 4 * KL; i++) kw[i] = first_kw[i];
            kscale = first_kscale;
            kvscale = first_kvscale;
            kb = first_kb;
#pragma unroll
            for (int i = 0; i < KPIECES; i++) store_k(0, i);
            load_k(lo + 128);
        } else {
            load_q();
        }
        // (Q's loads end here: left to the loop, the wait for them would also be one for the tiles' loads, in every round)
#pragma unroll
        for (int c = 0; c < NK; c++) asm volatile("" : "+v"(qf[c]));
        __syncthreads();
        if (lo < wave_most && lo < hi) {
            t = (f32x16)(0.f);
#pragma unroll
            for (int c = 0; c < NK; c++) {
                fetch_k(0, 0, c);
                t = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf[c % AHEAD], qf[c], t, 0, 0, 0);
            }
#pragma unroll
            for (int r4 = 0; r4 < 4; r4++) {
                fetch_ks(0, 0, r4);
                take_max(t, r4);
            }
            settle(t, lo);
        }
        int kbuf = 0, vbuf = 0;
        for (int base = lo; base < hi; base += 64) {
            const int vnext = vbuf == VBUFS - 1 ? 0 : vbuf + 1;
            const bool active = base < wave_most;
            clear_v(base + 64);
            auto keep_v = [&](int i) { store_v(vnext, i); };
            if (active) {
                step(t, u, vbuf, 0, kbuf, 1, VD, keep_v);
                settle(u, base + 32);
            } else {
#pragma unroll
                for (int i = 0; i < VD; i++) keep_v(i);
            }
            load_v(base + 128);
            __syncthreads();
            auto keep_k = [&](int i) { store_k(kbuf, i); };
            if (active) {
                step(u, t, vbuf, 1, kbuf ^ 1, 0, KPIECES, keep_k);
                settle(t, base + 64);
            } else {
#pragma unroll
                for (int i = 0; i < KPIECES; i++) keep_k(i);
            }
            load_k(base + 192);
            if (VBUFS == 2) __syncthreads();
            kbuf ^= 1;
            vbuf = vnext;
        }
        l += l2;
        l += __shfl_xor(l, 32, 64);
        // A value that is infinite or NaN makes NaN of the rows that do not see it too (zero times it), and so does one whose p
        // is too small for fp16, and any whose scale is negative or large: then the wave's rows are computed one by one.
        float all = 0.f;
#pragma unroll
        for (int d = 0; d < NV; d++) {
            float some = o[d][0];
#pragma unroll
            for (int r = 1; r < 16; r++) some += o[d][r];  // (finite ones stay far below the largest float)
            all += some;
        }
        if (__any(!(__builtin_fabsf(all) < INFINITY))) {
            for (int r = wave_row; r <= min(wave_row + 31, row_last); r++) {
                const int tk = r / a.group, hd = kv_head * a.group + r - tk * a.group;
                sqp_attend_row_of_part<TYPE, D>(a, parts, part, (long)(s.first + tk) * a.heads + hd, s.first + tk, hd, before + tk + 1, table, lo, hi);
            }
        } else if (row0 + 32 * wave + col < rows) {
            const long at = (long)(s.first + token) * a.heads + head;
            float *partial;
            if (sqp_target<D>(parts, sees, part, at, partial)) {
                const float inv = l == 0.f ? 0.f : 1.f / l;
                // result register r of block VSUB d + sub: dimension VD (32 sub + i) + d, i = 8 (r >> 2) + 4 h + (r & 3)
#pragma unroll
                for (int sub = 0; sub < VSUB; sub++)
#pragma unroll
                    for (int r4 = 0; r4 < 4; r4++)
#pragma unroll
                        for (int n = 0; n < VD; n++) {
                            const int dim = VD * (32 * sub + 8 * r4 + 4 * h) + 4 * n;
                            f32x4 x;
#pragma unroll
                            for (int e = 0; e < 4; e++) x[e] = o[VSUB * ((4 * n + e) % VD) + sub][4 * r4 + (4 * n + e) / VD];
                            if (partial) {
                                *(f32x4 *)(partial + dim) = x;
                            } else {
                                h16x4 y;
#pragma unroll
                                for (int e = 0; e < 4; e++) y[e] = (h16)(l == 0.f ? 0.f : x[e] * inv);
                                *(h16x4 *)(a.out + at * D + dim) = y;
                            }
                        }
                if (partial && h == 0) {
                    partial[D] = m;
                    partial[D + 1] = l;
                }
            }
        }
        __syncthreads();  // (the tiles are written again for the next rows)
    }
}

template <int TYPE, int D, int W>
void launch(const SqpAttention &a, const SqpParts &p, int above_rows, int fold, hipStream_t st)
{
    // every sequence may end inside a tile
    const long tiles = std::min((long)a.T * a.group / (32 * W) + a.B, 65535L / p.parts);
    attention_tiles_kernel<TYPE, D, W><<<dim3((unsigned)a.kv_heads, (unsigned)(tiles * p.parts)), 64 * W, 0, st>>>(a, p, above_rows, fold);
}

template <int TYPE, int D>
void launch(const SqpAttention &a, const SqpParts &p, int tile_rows, int above_rows, int fold, hipStream_t st)
{
    if (tile_rows == 256) launch<TYPE, D, 8>(a, p, above_rows, fold, st);
    else launch<TYPE, D, 4>(a, p, above_rows, fold, st);
}

}  // namespace

void sqp_attention_tiles(int type, int D, const SqpAttention &a, const SqpParts &p, int tile_rows, int above_rows, int fold, hipStream_t st)
{
#define TILES(TYPE) (D == 128 ? launch<TYPE, 128>(a, p, tile_rows, above_rows, fold, st) : launch<TYPE, 64>(a, p, tile_rows, above_rows, fold, st))
    if (type == SQP_FP16) TILES(SQP_FP16);
    else if (type == SQP_INT8) TILES(SQP_INT8);
    else if (type == SQP_E4M3) TILES(SQP_E4M3);
    else TILES(SQP_E2M1);
#undef TILES
}
