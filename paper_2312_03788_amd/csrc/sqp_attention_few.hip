// Attention over the paged cache for few rows per cached head: decode steps, a few tokens at a time.  Bound: the bytes of the
// cache.
//
// Four waves of a workgroup share a (sequence, cached head, part) and take 32 (codes: 64) tokens of it in turn; nothing passes between them
// before the end.  Both products run on 16x16x32 matrix instructions with the up to 16 query rows as columns:
//   S^T = K Q^T   a lane's A operand is 8 values of one key, as they lie in memory (a lane's 16-byte loads: 16 keys x 64 bytes);
//                 the values' order within D is free as long as Q has the same.
//   O^T = V^T P^T the columns of S^T are those of P^T, so p goes from one instruction's result to the other's operand
//                 without leaving its lane: token 4g + j (j < 4) of either 16 is slot (g, j), g the lane's row of 16.  V^T's operand
//                 wants 8 tokens' values of one dimension in a lane: a lane loads D / 16 dimensions of its 8 tokens (a load of
//                 16 lanes is a token's whole row) and pairs tokens up with one byte permutation per word.
// So nothing goes through shared memory but the four waves' results.  Registers hold a step's K and V while the next one's are on
// their way: 64 KB per compute unit, two workgroups of four waves.  With three (168 registers) values spill and 32 sequences
// at up to 2500 tokens take 286 us instead of 147.
//
// The matrix cores wait for memory here, so p goes through them twice: rounded to fp16, and what that leaves, in fp16 again (2^-22
// of p then, or 2^-35 of the row's largest where that is more).  The output's rounding is the only one left: the error of the 32
// sequences' outputs below is 2.1e-4 of them instead of 2.6e-4, in the same time (149.2 us and 149.4); over codes it costs up to 3 % (16
// sequences 39.0 us instead of 38.3, called again and again on the same cache).
//
// Measured, kernel alone: those 800 MB in 149 us (5.4 TB/s; a streaming read alone reaches 5.9 on this chip); one sequence of 32000
// tokens, 40 heads, int8, 338 MB in 61 us (5.5 TB/s); 16 at up to 8192, 8 cached heads, e4m3, 166 MB in 36 us (4.6 TB/s, parts of unequal
// length).  32 heads over 129 tokens: 6.1 us, the chain length, page, K, V.
#include "sqp_attention.h"

namespace {

template <int TYPE, int D>
__global__ void __launch_bounds__(256, 2) attention_few_kernel(const SqpAttention a, SqpParts parts, int most_rows, int slots)
{
    constexpr int BYTES = SqpCode<TYPE>::BYTES;
    constexpr int KL = D * BYTES / 64;       // 16-byte loads per lane and 16 keys
    constexpr int VW = D * BYTES / 64;       // words per lane and token of V
    constexpr int DPL = D / 16;              // dimensions per lane of V
    constexpr int NB = TYPE == SQP_FP16 ? 2 : 4;  // blocks of 16 tokens per step: codes are half as long, so twice as many keep
                                                  // the same number of bytes on their way
    __shared__ float s_o[4][SQP_FEW_ROWS][D + 4];
    __shared__ float s_m[4][SQP_FEW_ROWS], s_l[4][SQP_FEW_ROWS];
    __shared__ int s_bad;

    const int kv_head = blockIdx.x, b = blockIdx.y, part = blockIdx.z;
    if (part == 0 && b == 0) sqp_zero_strays<D>(a, kv_head);
    const SqpSequence s = sqp_one_sequence(a, b);
    const int rows = s.n * a.group;
    if (rows > most_rows) return;
    if (rows > slots) parts.parts = 1;
    auto slot = [&](int r) { return ((long)b * a.kv_heads + kv_head) * slots + r; };
    const int *table = a.table + b * a.table_stride;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63, col = lane & 15, g = lane >> 4;
    const int before = s.len - s.n;  // token i of the new ones sees before + i + 1
    const int mask = (1 << a.page_shift) - 1, reach = a.table_width << a.page_shift;
    for (int row0 = 0; row0 < rows; row0 += SQP_FEW_ROWS) {  // (once, unless this kernel serves sequences of more rows)
        const int count = min(rows - row0, SQP_FEW_ROWS), fewest = before + row0 / a.group + 1, most = before + (row0 + count - 1) / a.group + 1;
        const int nparts = parts.of(most);
        if (part >= nparts) continue;
        const int lo = part * parts.chunk, hi = part == nparts - 1 ? most : lo + parts.chunk;
        const int row = row0 + min(col, count - 1), token = row / a.group, head = kv_head * a.group + row - token * a.group;
        const int sees = before + token + 1;
        if (threadIdx.x == 0) s_bad = 0;

        h16x8 qf[D / 32];
        {
            const h16 *q = a.q + (size_t)(s.first + token) * a.q_stride + head * D;
#pragma unroll
            for (int i = 0; i < D / 32; i++) qf[i] = *(const h16x8 *)(q + (BYTES == 2 ? 32 * i + 8 * g : 64 * (i >> 1) + 16 * g + 8 * (i & 1)));
        }
        // Rows in the caches of a step's blocks of 16 tokens (pages are whole blocks, so all 16 rows are there).  A block past the
        // end is whatever the table has there, kept inside the cache.  Pages are looked up a step ahead.
        auto look_up = [&](int base, int *page) {
#pragma unroll
            for (int i = 0; i < NB; i++) page[i] = sqp_uniform(table + (min(base + 16 * i, reach - 16) >> a.page_shift));
        };
        auto block = [&](int base, int i, const int *page) {
            const size_t at = (size_t)min(max(page[i], 0), a.pages - 1) * a.kv_heads + kv_head;
            return (at << a.page_shift) + ((base + 16 * i) & mask);
        };
        u32x4 kw[NB][KL];
        uint32_t vw[4 * NB][VW];
        f32x4 ks[NB], vs[NB];
        auto load_k = [&](int base, const int *page) {
#pragma unroll
            for (int i = 0; i < NB; i++) {
                const size_t r = block(base, i, page);
                const uint8_t *p = (const uint8_t *)a.k + r * (D * BYTES) + col * (D * BYTES) + 16 * g;
#pragma unroll
                for (int j = 0; j < KL; j++) kw[i][j] = *(const u32x4 *)(p + 64 * j);
                if constexpr (TYPE != SQP_FP16) ks[i] = *(const f32x4 *)(a.k_scales + r + 4 * g);
            }
        };
        auto load_v = [&](int base, const int *page) {
#pragma unroll
            for (int i = 0; i < NB; i++) {
                const size_t r = block(base, i, page);
                const uint8_t *p = (const uint8_t *)a.v + r * (D * BYTES) + col * (DPL * BYTES);
#pragma unroll
                for (int j = 0; j < 4; j++) sqp_words<4 * VW>(p + (4 * g + j) * (D * BYTES), vw[4 * i + j]);
                if constexpr (TYPE != SQP_FP16) vs[i] = *(const f32x4 *)(a.v_scales + r + 4 * g);
            }
        };

        float m = SQP_LOWEST, l = 0.f;
        f32x4 o[DPL];
#pragma unroll
        for (int t = 0; t < DPL; t++) o[t] = (f32x4)(0.f);
        int base = lo + 16 * NB * wave;
        int page[NB], ahead[NB];
        look_up(base, page);
        if (base < hi) {
            load_k(base, page);
            load_v(base, page);
            look_up(base + 64 * NB, page);
        }
        for (; base < hi; base += 64 * NB) {
            float t[4 * NB];
#pragma unroll
            for (int i = 0; i < NB; i++) {
                f32x4 acc = (f32x4)(0.f);
#pragma unroll
                for (int j = 0; j < KL; j++) {
                    if constexpr (TYPE == SQP_FP16) {
                        acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h16x8, kw[i][j]), qf[j], acc, 0, 0, 0);
                    } else {
                        const uint32_t w[4] = {kw[i][j].x, kw[i][j].y, kw[i][j].z, kw[i][j].w};
#pragma unroll
                        for (int e = 0; e < 2; e++) {
                            h16x2 p[4];
                            sqp_halves4<TYPE>(w[2 * e], p[0], p[1]);
                            sqp_halves4<TYPE>(w[2 * e + 1], p[2], p[3]);
                            const h16x8 x = {p[0].x, p[0].y, p[1].x, p[1].y, p[2].x, p[2].y, p[3].x, p[3].y};
                            acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(x, qf[2 * j + e], acc, 0, 0, 0);
                        }
                    }
                }
#pragma unroll
                for (int r = 0; r < 4; r++) t[4 * i + r] = TYPE == SQP_FP16 ? acc[r] * a.scale2 : acc[r] * (ks[i][r] * a.scale2);
            }
            const bool more = base + 64 * NB < hi;
            look_up(base + 128 * NB, ahead);
            if (more) load_k(base + 64 * NB, page);
            if (base + 16 * NB > fewest) {  // some row does not see all of these tokens
#pragma unroll
                for (int i = 0; i < 4 * NB; i++) {
                    const int key = base + 16 * (i >> 2) + 4 * g + (i & 3);
                    if (key >= sees) t[i] = -INFINITY;
                    if (key >= s.len) {  // memory past the length, whatever it holds
#pragma unroll
                        for (int e = 0; e < VW; e++) vw[i][e] = 0;
                        if (TYPE != SQP_FP16) vs[i >> 2][i & 3] = 0.f;
                    }
                }
            }
            // What goes through the matrix cores is p times the value's scale, so the running maximum is taken of that: t + log2 of
            // the token's own scale (SQP_WEIGHT_TOP: changed only now and then).
            float top = 0.f;
#pragma unroll
            for (int i = 0; i < 4 * NB; i++) {
                float weight = t[i];
                if constexpr (TYPE != SQP_FP16) {
                    weight += sqp_log_scale(vs[i >> 2][i & 3]);
                    vs[i >> 2][i & 3] = sqp_known_scale(vs[i >> 2][i & 3]);
                }
                top = i == 0 ? weight : fmaxf(top, weight);
            }
            if (__any(top > m + SQP_WEIGHT_MOST)) {
                top = fmaxf(top, __shfl_xor(top, 16, 64));
                top = fmaxf(top, __shfl_xor(top, 32, 64));
                const float next = top > m + SQP_WEIGHT_MOST ? top - SQP_WEIGHT_TOP : m, keep = sqp_exp2(m - next);
                m = next;
                l *= keep;
#pragma unroll
                for (int d = 0; d < DPL; d++) o[d] *= keep;
            }
            h16x8 pf[NB / 2], pr[NB / 2];  // p to fp16's 11 bits, and to the next 11
#pragma unroll
            for (int i = 0; i < 4 * NB; i++) {
                const float p = sqp_exp2(t[i] - m);
                l += p;
                const float pv = TYPE == SQP_FP16 ? p : p * vs[i >> 2][i & 3];
                pf[i >> 3][i & 7] = (h16)pv;
                pr[i >> 3][i & 7] = (h16)(pv - (float)pf[i >> 3][i & 7]);
            }
#pragma unroll
            for (int q = 0; q < NB / 2; q++) {
                uint32_t pairs[4][DPL];  // [pair of tokens][dimension]
#pragma unroll
                for (int j = 0; j < 4; j++)
#pragma unroll
                    for (int e = 0; e < VW; e++) sqp_pair_up<TYPE>(vw[8 * q + 2 * j][e], vw[8 * q + 2 * j + 1][e], &pairs[j][e * (4 / BYTES)]);
                if (more && q == NB / 2 - 1) load_v(base + 64 * NB, page);
#pragma unroll
                for (int d = 0; d < DPL; d++) {
                    const u32x4 x = {pairs[0][d], pairs[1][d], pairs[2][d], pairs[3][d]};
                    o[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h16x8, x), pf[q], o[d], 0, 0, 0);
                    o[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h16x8, x), pr[q], o[d], 0, 0, 0);
                }
            }
#pragma unroll
            for (int i = 0; i < NB; i++) page[i] = ahead[i];
        }
        l += __shfl_xor(l, 16, 64);
        l += __shfl_xor(l, 32, 64);
        if (g == 0) {
            s_m[wave][col] = m;
            s_l[wave][col] = l;
        }
#pragma unroll
        for (int r = 0; r < 4; r++)
#pragma unroll
            for (int d = 0; d < DPL; d++) s_o[wave][col][DPL * (4 * g + r) + d] = o[d][r];
        // A value that is infinite or NaN makes NaN of the rows that do not see it too (zero times it), or of an infinity (times the
        // two parts of p), and so does one whose scale is 2^40 or more: then the rows are computed one by one.
        f32x4 all = o[0];
#pragma unroll
        for (int d = 1; d < DPL; d++) all += o[d];  // (finite ones stay far below the largest float)
        __syncthreads();
        if (!(__builtin_fabsf((all.x + all.y) + (all.z + all.w)) < INFINITY)) s_bad = 1;
        __syncthreads();
        if (s_bad) {
            for (int r = row0 + wave; r < row0 + count; r += 4) {
                const int tk = r / a.group;
                sqp_attend_row_of_part<TYPE, D>(a, parts, part, slot(r), s.first + tk, kv_head * a.group + r - tk * a.group, before + tk + 1, table, lo, hi);
            }
        }
        for (int i = s_bad ? count * (D / 4) : (int)threadIdx.x; i < count * (D / 4); i += 256) {
            const int r = i / (D / 4), d = 4 * (i % (D / 4)), tk = (row0 + r) / a.group;
            const long at = (long)(s.first + tk) * a.heads + kv_head * a.group + row0 + r - tk * a.group;
            float *partial;
            if (!sqp_target<D>(parts, before + tk + 1, part, slot(row0 + r), partial)) continue;
            const float top = fmaxf(fmaxf(s_m[0][r], s_m[1][r]), fmaxf(s_m[2][r], s_m[3][r]));
            float sum = 0.f;
            f32x4 x = (f32x4)(0.f);
#pragma unroll
            for (int w = 0; w < 4; w++) {
                const float c = sqp_exp2(s_m[w][r] - top);
                sum += c * s_l[w][r];
                x += c * *(const f32x4 *)&s_o[w][r][d];
            }
            if (partial) {
                *(f32x4 *)(partial + d) = x;
                if (d == 0) {
                    partial[D] = top;
                    partial[D + 1] = sum;
                }
            } else {
                const float inv = sum == 0.f ? 0.f : 1.f / sum;
                h16x4 y;
#pragma unroll
                for (int e = 0; e < 4; e++) y[e] = (h16)(sum == 0.f ? 0.f : x[e] * inv);
                *(h16x4 *)(a.out + at * D + d) = y;
            }
        }
        __syncthreads();  // (the results and s_bad are written again for the next rows)
    }
}

template <int TYPE, int D>
void launch(const SqpAttention &a, const SqpParts &p, int most_rows, int slots, hipStream_t st)
{
    attention_few_kernel<TYPE, D><<<dim3((unsigned)a.kv_heads, (unsigned)a.B, (unsigned)p.parts), 256, 0, st>>>(a, p, most_rows, slots);
}

}  // namespace

void sqp_attention_few(int type, int D, const SqpAttention &a, const SqpParts &p, int most_rows, int slots, hipStream_t st)
{
#define FEW(TYPE) (D == 128 ? launch<TYPE, 128>(a, p, most_rows, slots, st) : launch<TYPE, 64>(a, p, most_rows, slots, st))
    if (type == SQP_FP16) FEW(SQP_FP16);
    else if (type == SQP_INT8) FEW(SQP_INT8);
    else FEW(SQP_E4M3);
#undef FEW
}
