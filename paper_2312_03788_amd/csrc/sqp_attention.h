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

// A long sequence is read in parts of `chunk` tokens by workgroups of their own (at most `parts` of them, the last one takes
// what is left).  A row that sees one part only is written at once; of the others every part leaves its maximum, sum and
// output, which sqp_attention_combine joins.  A partial result is D + 4 floats: the output, the maximum, the sum; a row has
// `parts` of them, at its slot.
struct SqpParts {
    int chunk, parts;
    float *part;
    __host__ __device__ int of(int sees) const
    {
        const int n = sees <= chunk ? 1 : (sees + chunk - 1) / chunk;
        return n < parts ? n : parts;
    }
};

// Sequences whose new tokens make at most this many rows per cached head are for the few-rows kernel (one tile of the
// 16-column matrix instruction), the others for the tile kernel.  A kernel that is launched alone serves all of them: the few-rows
// kernel those of up to `most_rows` rows, the tile kernel those of more than `above_rows`.
constexpr int SQP_FEW_ROWS = 16;

// Slots: the tile kernel's rows have them in the order of the output; the few-rows kernel has `slots` for every sequence and cached
// head (a sequence of more rows than that is not split), so that they cost what its rows need and not all rows of a prompt beside them.
void sqp_attention_few(int type, int D, const SqpAttention &a, const SqpParts &p, int most_rows, int slots, hipStream_t stream);
void sqp_attention_tiles(int type, int D, const SqpAttention &a, const SqpParts &p, int tile_rows, int above_rows, int fold, hipStream_t stream);

#ifdef __HIPCC__
constexpr float SQP_LOWEST = -3e38f;  // the running maximum of a row that has seen nothing: finite, so that differences are

// Weights go through the matrix cores in fp16, relative to a running maximum that is changed only now and then: when it is, the
// largest weight becomes 2^10, and as long as no later one passes 2^15.9 (61147; fp16 ends at 65504) it stays.  Weights down to 2^-24 of
// the row's largest are normal numbers of fp16 then, and below its smallest step are only those under 2^-35 of it.  At 2^0
// instead of 2^10 a long tail behind one large weight is lost from 2^-25 on (it is still in the sum); the maximum is changed
// less often, the error of the outputs is larger: 2048-token prompt 60.1 us and 2.53e-4 instead of 61.9 and 2.48e-4, the mixed step 144.3 and
// 2.73e-4 instead of 149.7 and 2.49e-4, 2048 tokens behind 14336 1111 and 2.92e-4 instead of 1120 and 2.51e-4; few rows take the same time.
constexpr float SQP_WEIGHT_TOP = 10.f, SQP_WEIGHT_MOST = 15.9f;

__device__ __forceinline__ float sqp_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// A value's scale in the exponent of its token's weight: its logarithm, of 2^-40 at least (any code times that is below half of
// fp16's smallest number), so that a token of tiny or zero values keeps its place in the sum of the weights (with 2^-100 it lost
// it beside a weight times scale 2^26 above: fp32's exponents end there).
constexpr float SQP_LEAST_SCALE = 0x1p-40f;
__device__ __forceinline__ float sqp_log_scale(float scale) { return __builtin_amdgcn_logf(fmaxf(__builtin_fabsf(scale), SQP_LEAST_SCALE)); }

// A scale of 2^40 or more as NaN, which shows in the sums and leads to the slow way (by arithmetic: with a comparison
// and its mask per token a decode step of 16 sequences at up to 8192 tokens takes 39.1 us instead of 38.8).
__device__ __forceinline__ float sqp_known_scale(float scale)
{
    const float far = scale * 0x1p88f;  // infinite then
    return scale + (far - far);
}

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// BYTES bytes as words.
template <int BYTES>
__device__ __forceinline__ void sqp_words(const void *p, uint32_t *w)
{
    if constexpr (BYTES == 1) {
        w[0] = *(const uint8_t *)p;
    } else if constexpr (BYTES == 2) {
        w[0] = *(const uint16_t *)p;
    } else if constexpr (BYTES == 4) {
        w[0] = *(const uint32_t *)p;
    } else if constexpr (BYTES == 8) {
        const u32x2 v = *(const u32x2 *)p;
        w[0] = v.x;
        w[1] = v.y;
    } else {
        const u32x4 v = *(const u32x4 *)p;
        w[0] = v.x;
        w[1] = v.y;
        w[2] = v.z;
        w[3] = v.w;
    }
}

// Words i of two tokens' values to the pairs (token, next token) of fp16 values: 2 dimensions per word (fp16), 4 (codes).
template <int TYPE>
__device__ __forceinline__ void sqp_pair_up(uint32_t a, uint32_t b, uint32_t *pairs)
{
    if constexpr (TYPE == SQP_FP16) {
        pairs[0] = __builtin_amdgcn_perm(b, a, 0x05040100u);
        pairs[1] = __builtin_amdgcn_perm(b, a, 0x07060302u);
    } else if constexpr (TYPE == SQP_E4M3) {
        const uint32_t lo = __builtin_amdgcn_perm(b, a, 0x05010400u), hi = __builtin_amdgcn_perm(b, a, 0x07030602u);
        pairs[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)lo, 1.0f, false));
        pairs[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)lo, 1.0f, true));
        pairs[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)hi, 1.0f, false));
        pairs[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)hi, 1.0f, true));
    } else {
        const h16x2 off = {(h16)1152.0f, (h16)1152.0f};
        const uint32_t sel[4] = {0x0c040c00u, 0x0c050c01u, 0x0c060c02u, 0x0c070c03u};
#pragma unroll
        for (int i = 0; i < 4; i++)
            pairs[i] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(h16x2, __builtin_amdgcn_perm(b, a, sel[i]) ^ 0x64806480u) - off);
    }
}

// One of those pairs: dimension d of the tokens' words a, b.
template <int TYPE>
__device__ __forceinline__ uint32_t sqp_pair(const uint32_t *a, const uint32_t *b, int d)
{
    if constexpr (TYPE == SQP_FP16) {
        return __builtin_amdgcn_perm(b[d / 2], a[d / 2], d & 1 ? 0x07060302u : 0x05040100u);
    } else if constexpr (TYPE == SQP_E4M3) {
        const uint32_t both = __builtin_amdgcn_perm(b[d / 4], a[d / 4], 0x0c0c0400u + 0x0101u * (uint32_t)(d % 4));
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)both, 1.0f, false));
    } else {
        const h16x2 off = {(h16)1152.0f, (h16)1152.0f};
        const uint32_t both = __builtin_amdgcn_perm(b[d / 4], a[d / 4], 0x0c040c00u + 0x00010001u * (uint32_t)(d % 4));
        return __builtin_bit_cast(uint32_t, __builtin_bit_cast(h16x2, both ^ 0x64806480u) - off);
    }
}

// An index array's element at the same place for a whole wave, through the scalar cache (no kernel writes these arrays).
__device__ __forceinline__ int sqp_uniform(const int *p) { return *(const __attribute__((address_space(4))) int *)(uintptr_t)p; }

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

// The same where b is the same for the whole wave.
__device__ __forceinline__ SqpSequence sqp_one_sequence(const SqpAttention &a, int b)
{
    SqpSequence s;
    s.first = b;
    s.n = 1;
    if (a.starts) {
        s.first = min(max(sqp_uniform(a.starts + b), 0), a.T);
        s.n = max(min(sqp_uniform(a.starts + b + 1), a.T) - s.first, 0);
    }
    s.len = min(max(sqp_uniform(a.lens + b), 0), a.table_width << a.page_shift);
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

// Where a row's result of one part goes (null: the output); false: this part has nothing of the row.
template <int D>
__device__ __forceinline__ bool sqp_target(const SqpParts &p, int sees, int part, long slot, float *&partial)
{
    const int n = p.of(sees);
    partial = n > 1 ? p.part + ((size_t)slot * p.parts + part) * (D + 4) : nullptr;
    return part < n;
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
        if (l != 0.f && __all(o[0] != o[0] && o[PER - 1] != o[PER - 1])) break;  // NaN as a whole, whatever follows (a sum of zero would
                                                                                 // make zeros of it: a row all of whose scores are minus infinity)
    }
}

// The same for a row of a part, result included: the slow way of the kernels below where a value is infinite or NaN (zero times
// it is not zero, so the matrix instructions cannot keep it from the rows that do not see it).
template <int TYPE, int D>
__device__ __forceinline__ void sqp_attend_row_of_part(const SqpAttention &a, const SqpParts &parts, int part, long slot, int token, int head, int sees,
                                                       const int *table_row, int lo, int hi)
{
    constexpr int PER = D / 64;
    const long row = (long)token * a.heads + head;
    float *partial, m, l, o[PER];
    if (!sqp_target<D>(parts, sees, part, slot, partial)) return;
    sqp_attend_row<TYPE, D>(a, a.q + token * a.q_stride + head * D, table_row, head / a.group, lo, min(hi, sees), m, l, o);
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int e = 0; e < PER; e++) {
        if (partial) partial[PER * lane + e] = o[e];
        else a.out[row * D + PER * lane + e] = (h16)(l == 0.f ? 0.f : o[e] / l);
    }
    if (partial && lane == 0) {
        partial[D] = m;
        partial[D + 1] = l;
    }
}

// Rows in front of the first sequence's and behind the last one's: zeros.
template <int D>
__device__ __forceinline__ void sqp_zero_strays(const SqpAttention &a, int kv_head)
{
    if (!a.starts) return;
    const int width8 = a.group * D / 8, pitch8 = a.heads * D / 8;
    const int front = min(max(a.starts[0], 0), a.T), back = max(min(a.starts[a.B], a.T), 0);
    for (int side = 0; side < 2; side++) {
        const int from = side == 0 ? 0 : back, to = side == 0 ? front : a.T;
        for (long i = threadIdx.x; i < (long)max(to - from, 0) * width8; i += blockDim.x)
            ((uint4 *)a.out)[(from + i / width8) * pitch8 + kv_head * width8 + i % width8] = make_uint4(0, 0, 0, 0);
    }
}

// Sum over a wave's lanes (row by row, then across the rows), the same in all of them.
__device__ __forceinline__ int sqp_wave_sum(int x)
{
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);  // row_shr:1, 2, 4, 8
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
    return __builtin_amdgcn_readlane(x, 15) + __builtin_amdgcn_readlane(x, 31) + __builtin_amdgcn_readlane(x, 47) + __builtin_amdgcn_readlane(x, 63);
}

// The same for floats, and the largest (a lane exchange through the data-sharing unit takes a hundred cycles a step, these a few).
template <bool MAX>
__device__ __forceinline__ float sqp_wave_join(float x)
{
    auto lane = [](float v, int i) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), i)); };
    auto join = [](float a, float b) { return MAX ? fmaxf(a, b) : a + b; };
    const int none = __builtin_bit_cast(int, MAX ? SQP_LOWEST : 0.f);
#define SQP_ROW_SHR(n) x = join(x, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(none, __builtin_bit_cast(int, x), 0x110 + n, 0xf, 0xf, false)))
    SQP_ROW_SHR(1);
    SQP_ROW_SHR(2);
    SQP_ROW_SHR(4);
    SQP_ROW_SHR(8);
#undef SQP_ROW_SHR
    return join(join(lane(x, 15), lane(x, 31)), join(lane(x, 47), lane(x, 63)));
}

// The tile (of `height` rows) that is rank-th in the order of work, over all sequences of more than above_rows rows: those first
// that see most, so that the long ones do not begin last.  From `fold` on the order is turned round: with as many
// workgroups as fit the chip at once, the shortest share their compute units with the longest.  b < 0: no such tile.
struct SqpTile {
    int b, tile;
};
__device__ __forceinline__ SqpTile sqp_pick_tile(const SqpAttention &a, int above_rows, int height, int rank, int fold)
{
    const int lane = threadIdx.x & 63;
    auto tiles_of = [&](int b) {
        const SqpSequence s = sqp_sequence(a, b);
        const int rows = s.n * a.group;
        return rows > above_rows ? (rows + height - 1) / height : 0;
    };
    if (a.B > 64) {  // in the sequences' order
        int first = 0;
        for (int i = 0; i < a.B; i += 64) {
            const int n = i + lane < a.B ? tiles_of(i + lane) : 0, all = sqp_wave_sum(n);
            if (rank < first + all) {
                for (int j = 0; j < 64; j++) {
                    const int nj = __builtin_amdgcn_readlane(n, j);
                    if (rank < first + nj) return {i + j, nj - 1 - (rank - first)};
                    first += nj;
                }
            }
            first += all;
        }
        return {-1, 0};
    }
    if (a.B == 1) {
        const int rows = sqp_one_sequence(a, 0).n * a.group, all = rows > above_rows ? (rows + height - 1) / height : 0;
        if (rank >= all) return {-1, 0};
        return {0, fold > 0 && rank >= fold ? rank - fold : all - 1 - rank};
    }
    const int n = lane < a.B ? tiles_of(lane) : 0, all = sqp_wave_sum(n);
    if (rank >= all) return {-1, 0};
    if (fold > 0 && rank >= fold) rank = all - 1 - (rank - fold);
    // A tile's key: its sequence's length, less a power of two near the tokens per tile for every tile behind it.
    int shift = 0;
    while ((a.group << (shift + 1)) <= height) shift++;
    const int len = lane < a.B ? sqp_sequence(a, lane).len : 0;
    auto above = [&](int x) {  // tiles of this lane's sequence with a key greater than x
        return len <= x ? 0 : min(n, ((len - x - 1) >> shift) + 1);
    };
    int lo = -(all << shift) - 1, hi = a.table_width << a.page_shift;  // no key beyond hi, all above lo (a sequence has at most `all` tiles)
    while (lo < hi) {
        const int mid = lo + ((hi - lo) >> 1);
        if (sqp_wave_sum(above(mid)) <= rank) hi = mid;
        else lo = mid + 1;
    }
    const int here = above(lo - 1) - above(lo);  // 1: this lane's sequence has a tile with the key lo
    unsigned long long who = __ballot(here > 0);
    for (int skip = rank - sqp_wave_sum(above(lo)); skip > 0; skip--) who &= who - 1;
    const int b = __ffsll((long long)who) - 1;
    return {b, __builtin_amdgcn_readlane(n, b) - 1 - __builtin_amdgcn_readlane(above(lo), b)};
}
#endif
