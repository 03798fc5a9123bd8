// Attention over the paged cache: what its kernels share.
//
//   o[t][h] = sum_j p_j v_j,  p = softmax_j (scale q[t][h] . k_j)  over the cached tokens j that token t sees,
//
// t being one of the n newest tokens of a sequence of `len` cached ones (the new ones among them): token i of the n sees
// j <= len - n + i.  Query head h reads the cached head h / (heads / kv_heads).
#pragma once
#include "sqp_rows.h"

struct SqpAttention {
    int T, B, heads, kv_heads, group;  // group: query heads per cached head
    int page_shift, pages, table_width;
    long q_stride, table_stride;
    const h16 *q;
    const void *k, *v;
    const float *k_scales, *v_scales;
    const int *table, *lens, *starts;  // starts == nullptr: one new token per sequence
    h16 *out;
    float scale2;  // scale log2(e): the softmax is taken in powers of two
};

#ifdef __HIPCC__
constexpr float SQP_LOWEST = -3e38f;  // the running maximum of a row that has seen nothing: finite, so that differences are

__device__ __forceinline__ float sqp_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// The new tokens of a sequence, its length in the cache.  What the device arrays say is kept inside the tensors.
struct SqpSequence {
    int first, n, len;
};
__device__ __forceinline__ SqpSequence sqp_sequence(const SqpAttention &a, int b)
{
    SqpSequence s;
    s.first = b;
    s.n = 1;
    if (a.starts) {
        s.first = min(max(a.starts[b], 0), a.T);
        s.n = max(min(a.starts[b + 1], a.T) - s.first, 0);
    }
    s.len = min(max(a.lens[b], 0), a.table_width << a.page_shift);
    return s;
}

// The sequence of a new token: how many sequences end at or before it.  B if none holds it.
__device__ __forceinline__ int sqp_sequence_of(const SqpAttention &a, int token)
{
    if (!a.starts) return token;
    if (token < a.starts[0]) return a.B;
    int b = 0;
    for (int i = 0; i < a.B; i += 64) {
        const int at = i + (int)(threadIdx.x & 63);
        b += __popcll(__ballot(at < a.B && a.starts[min(at, a.B - 1) + 1] <= token));
    }
    return b;
}

// A page's number as the table has it, kept inside the cache.
__device__ __forceinline__ int sqp_page(const SqpAttention &a, const int *table_row, int token)
{
    return min(max(table_row[token >> a.page_shift], 0), a.pages - 1);
}

// Row (of D values) of a token and head in the caches.
__device__ __forceinline__ size_t sqp_cache_row(const SqpAttention &a, const int *table_row, int token, int kv_head)
{
    const size_t block = (size_t)sqp_page(a, table_row, token) * a.kv_heads + kv_head;
    return (block << a.page_shift) + (token & ((1 << a.page_shift) - 1));
}

// One query row over the keys lo .. hi - 1, by one wave: a lane takes every 64th key's score, and D / 64 values of the
// output.  Reads nothing of any other key.  m, l: the row's maximum (in powers of two) and sum; o: not divided by it.
template <int TYPE, int D>
__device__ __forceinline__ void sqp_attend_row(const SqpAttention &a, const h16 *q, const int *table_row, int kv_head, int lo, int hi, float &m, float &l, float *o)
{
    constexpr int PER = D / 64;
    const int lane = threadIdx.x & 63;
    m = SQP_LOWEST;
    l = 0.f;
#pragma unroll
    for (int e = 0; e < PER; e++) o[e] = 0.f;
    for (int base = lo; base < hi; base += 64) {
        const int key = min(base + lane, hi - 1);
        const size_t row = sqp_cache_row(a, table_row, key, kv_head);
        float s = 0.f, vs = 1.f;
        if constexpr (TYPE == SQP_FP16) {
            const uint4 *kp = (const uint4 *)((const h16 *)a.k + row * D);
#pragma unroll 2
            for (int i = 0; i < D / 8; i++) {
                float x[8];
                sqp_widen8(kp[i], x);
#pragma unroll
                for (int e = 0; e < 8; e++) s += x[e] * (float)q[8 * i + e];
            }
            s *= a.scale2;
        } else {
            const uint4 *kp = (const uint4 *)((const uint8_t *)a.k + row * D);
#pragma unroll 1
            for (int i = 0; i < D / 16; i++) {
                const uint4 w = kp[i];
                const uint32_t c[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    h16x2 x, y;
                    sqp_halves4<TYPE>(c[e], x, y);
                    const h16 *qe = q + 16 * i + 4 * e;
                    s += (float)x.x * (float)qe[0] + (float)x.y * (float)qe[1] + (float)y.x * (float)qe[2] + (float)y.y * (float)qe[3];
                }
            }
            s *= a.k_scales[row] * a.scale2;
            vs = a.v_scales[row];
        }
        if (base + lane >= hi) s = -INFINITY;
        float top = s;
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) top = fmaxf(top, __shfl_xor(top, off, 64));
        const float next = fmaxf(m, top), keep = sqp_exp2(m - next);
        float p = sqp_exp2(s - next);
        if (base + lane >= hi) p = 0.f;
        m = next;
        float sum = p;
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) sum += __shfl_xor(sum, off, 64);
        l = l * keep + sum;
#pragma unroll
        for (int e = 0; e < PER; e++) o[e] *= keep;
        const int count = min(64, hi - base);
        for (int j = 0; j < count; j++) {
            const float pj = __shfl(p * vs, j, 64);
            const size_t vrow = sqp_cache_row(a, table_row, base + j, kv_head);
            if constexpr (TYPE == SQP_FP16) {
                const h16 *vp = (const h16 *)a.v + vrow * D + PER * lane;
#pragma unroll
                for (int e = 0; e < PER; e++) o[e] += pj * (float)vp[e];
            } else {
                const uint8_t *vp = (const uint8_t *)a.v + vrow * D + PER * lane;
                const uint32_t w = PER == 2 ? *(const uint16_t *)vp : *vp;
                h16x2 x, y;
                sqp_halves4<TYPE>(w, x, y);
                o[0] += pj * (float)x.x;
                if constexpr (PER == 2) o[1] += pj * (float)x.y;
            }
        }
    }
}
#endif
