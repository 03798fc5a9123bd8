// The paged cache of keys and values: [pages][kv_heads][page][D] in fp16, or as 8-bit codes with one fp32 scale per token and
// head ([pages][kv_heads][page]), or in e2m1 blocks ([..][D/2] bytes, scales [..][D/32]).  Writing rotates queries and keys (positions as angles: y = x e^{i angle} on the pairs
// (x_j, x_{j + D/2})) and quantises on the way, so that the projection's output is read once and nothing lies in memory in between.
#include "sqp_mx.h"

namespace {

struct CacheArgs {
    int heads, kv_heads, page_shift, slots_total, n_positions;
    const h16 *q, *k, *v;
    long q_stride, k_stride, v_stride;
    const int *slots, *positions;
    const float *cos_sin;
    void *k_cache, *v_cache, *k_scales, *v_scales;
    h16 *q_out;
};

// Where the row of (slot, head) begins, in rows of D elements; the caches may hold more than 2^31 elements.
__device__ __forceinline__ size_t cache_row(int slot, int head, int kv_heads, int page_shift)
{
    const size_t block = (size_t)(slot >> page_shift) * kv_heads + head;
    return (block << page_shift) + (slot & ((1 << page_shift) - 1));
}

// D / 16 lanes per row, each with the values j .. j + 7 and D/2 + j .. D/2 + j + 7, whose pairs it turns.  A workgroup takes
// 4096 / D rows of one token's heads + 2 kv_heads; the group's maximum is exchanged between those lanes alone.
// Bound: HBM, or for a few tokens the launch (3.3 us for 16 tokens of 64 + 16 heads).  1001 tokens of 40 + 80 heads into int8:
// 12.5 us, 52 MB, 4.1 TB/s; reading them back 6.5 us, 31 MB, 4.8 TB/s.  Into e2m1 blocks 11.1 us, 47 MB, 4.3 TB/s; back 6.8 us, 26 MB; 16 tokens of
// 64 + 16 heads 3.1 and 2.6 us.
template <int TYPE, int D, bool ROTATE>
__global__ void __launch_bounds__(256) kv_write_kernel(const CacheArgs a)
{
    constexpr int LANES = D / 16, ROWS = 256 / LANES;
    const int token = blockIdx.x, lane = threadIdx.x % LANES;
    const int row = blockIdx.y * ROWS + threadIdx.x / LANES;
    if (row >= a.heads + 2 * a.kv_heads) return;  // (a whole group of LANES lanes)
    const bool is_q = row < a.heads, is_v = row >= a.heads + a.kv_heads;
    const int head = is_q ? row : is_v ? row - a.heads - a.kv_heads : row - a.heads;
    const int slot = is_q ? 0 : a.slots[token];
    if (!is_q && (unsigned)slot >= (unsigned)a.slots_total) return;
    const h16 *src = (is_q ? a.q + (size_t)token * a.q_stride : is_v ? a.v + (size_t)token * a.v_stride : a.k + (size_t)token * a.k_stride) + (size_t)head * D + 8 * lane;
    float f[16];
    const uint4 lo = *(const uint4 *)src, hi = *(const uint4 *)(src + D / 2);
    sqp_widen8(lo, f);
    sqp_widen8(hi, f + 8);
    if constexpr (ROTATE) {
        if (!is_v) {
            const int pos = a.positions[token];
            if ((unsigned)pos < (unsigned)a.n_positions) {
                const float *cs = a.cos_sin + (size_t)pos * D + 8 * lane;
#pragma unroll
                for (int j = 0; j < 8; j++) {
                    // every product and sum rounded for itself: codes at a rounding's edge are those of plain 32-bit arithmetic
#pragma clang fp contract(off)
                    const float c = cs[j], s = cs[D / 2 + j], x = f[j], y = f[8 + j];
                    f[j] = x * c - y * s;
                    f[8 + j] = y * c + x * s;
                }
            } else {
#pragma unroll
                for (int j = 0; j < 16; j++) f[j] = __builtin_bit_cast(float, 0x7fc00000u);
            }
        }
    }
    if (is_q) {
        h16 *dst = a.q_out + ((size_t)token * a.heads + head) * D + 8 * lane;
        *(uint4 *)dst = sqp_narrow8(f);
        *(uint4 *)(dst + D / 2) = sqp_narrow8(f + 8);
        return;
    }
    const size_t at = cache_row(slot, head, a.kv_heads, a.page_shift);
    void *cache = is_v ? a.v_cache : a.k_cache;
    if constexpr (TYPE == SQP_FP16) {
        h16 *dst = (h16 *)cache + at * D + 8 * lane;
        *(uint4 *)dst = sqp_narrow8(f);
        *(uint4 *)(dst + D / 2) = sqp_narrow8(f + 8);
    } else if constexpr (TYPE == SQP_E2M1) {
        // four neighbouring lanes have a block of either half of the row
#pragma unroll
        for (int half = 0; half < 2; half++) {
            uint32_t amax = 0;
#pragma unroll
            for (int j = 0; j < 8; j++) amax = max(amax, sqp_abs_bits(f[8 * half + j]));
            const uint32_t byte = sqp_mx_byte<SQP_E2M1>(sqp_quad_max(amax));
            ((uint32_t *)cache)[at * (D / 8) + half * (D / 16) + lane] = sqp_mx_e2m1_codes8(f + 8 * half, byte);
            if (lane % 4 == 0) ((uint8_t *)(is_v ? a.v_scales : a.k_scales))[at * (D / 32) + half * (D / 64) + lane / 4] = (uint8_t)byte;
        }
    } else {
        uint32_t amax = 0;
#pragma unroll
        for (int j = 0; j < 16; j++) amax = max(amax, sqp_abs_bits(f[j]));
#pragma unroll
        for (int off = LANES / 2; off >= 1; off >>= 1) amax = max(amax, (uint32_t)__shfl_xor((int)amax, off, 64));
        float step, inverse;
        sqp_row_step<TYPE>(amax, step, inverse);
        uint8_t *dst = (uint8_t *)cache + at * D + 8 * lane;
        *(uint2 *)dst = sqp_codes8<TYPE>(f, inverse);
        *(uint2 *)(dst + D / 2) = sqp_codes8<TYPE>(f + 8, inverse);
        if (lane == 0) ((float *)(is_v ? a.v_scales : a.k_scales))[at] = step;
    }
}

// The same rows back as fp16: D / 8 lanes per row.
template <int TYPE, int D>
__global__ void __launch_bounds__(256) kv_read_kernel(int kv_heads, int page_shift, int slots_total, const int *__restrict__ slots, const void *__restrict__ k_cache,
                                                      const void *__restrict__ v_cache, const void *__restrict__ k_scales,
                                                      const void *__restrict__ v_scales, h16 *__restrict__ k, h16 *__restrict__ v)
{
    constexpr int LANES = D / 8, ROWS = 256 / LANES;
    const int token = blockIdx.x, lane = threadIdx.x % LANES;
    const int row = blockIdx.y * ROWS + threadIdx.x / LANES;
    if (row >= 2 * kv_heads) return;
    const bool is_v = row >= kv_heads;
    const int head = is_v ? row - kv_heads : row, slot = slots[token];
    uint4 *dst = (uint4 *)((is_v ? v : k) + ((size_t)token * kv_heads + head) * D + 8 * lane);
    if ((unsigned)slot >= (unsigned)slots_total) {
        *dst = make_uint4(0, 0, 0, 0);
        return;
    }
    const size_t at = cache_row(slot, head, kv_heads, page_shift);
    const void *cache = is_v ? v_cache : k_cache;
    if constexpr (TYPE == SQP_FP16) {
        *dst = *(const uint4 *)((const h16 *)cache + at * D + 8 * lane);
    } else if constexpr (TYPE == SQP_E2M1) {
        const uint32_t byte = ((const uint8_t *)(is_v ? v_scales : k_scales))[at * (D / 32) + lane / 4];
        float f[8];
        sqp_mx_e2m1_values8(((const uint32_t *)cache)[at * (D / 8) + lane], __builtin_bit_cast(float, byte << 23), f);
        *dst = sqp_narrow8(f);
    } else {
        const uint2 c = *(const uint2 *)((const uint8_t *)cache + at * D + 8 * lane);
        const float step = ((const float *)(is_v ? v_scales : k_scales))[at];
        h16x2 p[4];
        sqp_halves4<TYPE>(c.x, p[0], p[1]);
        sqp_halves4<TYPE>(c.y, p[2], p[3]);
        float f[8];
#pragma unroll
        for (int i = 0; i < 4; i++) {
            f[2 * i] = (float)p[i].x * step;
            f[2 * i + 1] = (float)p[i].y * step;
        }
        *dst = sqp_narrow8(f);
    }
}

template <int TYPE, int D>
void write(int T, const CacheArgs &a, hipStream_t st)
{
    const dim3 grid((unsigned)T, (unsigned)((a.heads + 2 * a.kv_heads + 4096 / D - 1) / (4096 / D)));
    if (a.cos_sin) kv_write_kernel<TYPE, D, true><<<grid, 256, 0, st>>>(a);
    else kv_write_kernel<TYPE, D, false><<<grid, 256, 0, st>>>(a);
}

template <int TYPE, int D>
void read(int T, int kv_heads, int shift, int total, const int *slots, const void *kc, const void *vc, const void *ks, const void *vs, void *k, void *v, hipStream_t st)
{
    const dim3 grid((unsigned)T, (unsigned)((2 * kv_heads + 2048 / D - 1) / (2048 / D)));
    kv_read_kernel<TYPE, D><<<grid, 256, 0, st>>>(kv_heads, shift, total, slots, kc, vc, ks, vs, (h16 *)k, (h16 *)v);
}

}  // namespace

int sqp_check_cache(int kv_heads, int D, int type, int page, int pages, const void *k_cache, const void *v_cache, const void *k_scales, const void *v_scales)
{
    if (!k_cache || !v_cache) return SQP_ERR_NULL;
    if (type != SQP_FP16 && type != SQP_INT8 && type != SQP_E4M3 && type != SQP_E2M1) return SQP_ERR_ARG;
    if (type != SQP_FP16 && (!k_scales || !v_scales)) return SQP_ERR_NULL;
    if (kv_heads <= 0 || kv_heads > 65535 || (D != 64 && D != 128) || pages <= 0) return SQP_ERR_SHAPE;
    if (page < 16 || page > 65536 || (page & (page - 1)) || (long)pages * page >= (1L << 31) || sqp_too_big((long)kv_heads * page, D)) return SQP_ERR_SHAPE;
    if (sqp_misaligned(k_cache) || sqp_misaligned(v_cache)) return SQP_ERR_ALIGN;
    if (type != SQP_FP16 && (sqp_misaligned(k_scales) || sqp_misaligned(v_scales))) return SQP_ERR_ALIGN;
    return SQP_OK;
}

extern "C" int sqp_kv_cache_write(int T, int heads, int kv_heads, int D, int type, int page, int pages, const void *q, long q_stride, const void *k,
                                  long k_stride, const void *v, long v_stride, const int *slots, const float *cos_sin, const int *positions,
                                  int n_positions, void *k_cache, void *v_cache, void *k_scales, void *v_scales, void *q_out, void *stream)
{
    const int rc = sqp_check_cache(kv_heads, D, type, page, pages, k_cache, v_cache, k_scales, v_scales);
    if (rc) return rc;
    if (!k || !v || !slots || (heads > 0 && (!q || !q_out)) || (cos_sin && !positions)) return SQP_ERR_NULL;
    if (T < 0 || heads < 0 || heads > 65535 || (cos_sin && n_positions <= 0)) return SQP_ERR_SHAPE;
    if ((k_stride % 8) || (v_stride % 8) || (heads > 0 && (q_stride % 8))) return SQP_ERR_ALIGN;
    if (k_stride < (long)kv_heads * D || v_stride < (long)kv_heads * D || (heads > 0 && q_stride < (long)heads * D)) return SQP_ERR_SHAPE;
    if (sqp_misaligned(k) || sqp_misaligned(v) || (cos_sin && sqp_misaligned(cos_sin)) || (((uintptr_t)slots | (uintptr_t)positions) & 3)) return SQP_ERR_ALIGN;
    if (heads > 0 && (sqp_misaligned(q) || sqp_misaligned(q_out))) return SQP_ERR_ALIGN;
    if (T == 0) return SQP_OK;
    int shift = 0;
    while ((1 << shift) < page) shift++;
    CacheArgs a = {};
    a.heads = heads; a.kv_heads = kv_heads; a.page_shift = shift; a.slots_total = pages * page; a.n_positions = n_positions;
    a.q = (const h16 *)q; a.k = (const h16 *)k; a.v = (const h16 *)v;
    a.q_stride = q_stride; a.k_stride = k_stride; a.v_stride = v_stride;
    a.slots = slots; a.positions = positions; a.cos_sin = cos_sin;
    a.k_cache = k_cache; a.v_cache = v_cache; a.k_scales = k_scales; a.v_scales = v_scales; a.q_out = (h16 *)q_out;
    hipStream_t st = (hipStream_t)stream;
#define KV_WRITE(TYPE) (D == 128 ? write<TYPE, 128>(T, a, st) : write<TYPE, 64>(T, a, st))
    if (type == SQP_FP16) KV_WRITE(SQP_FP16);
    else if (type == SQP_INT8) KV_WRITE(SQP_INT8);
    else if (type == SQP_E4M3) KV_WRITE(SQP_E4M3);
    else KV_WRITE(SQP_E2M1);
#undef KV_WRITE
    return sqp_launch_status();
}

extern "C" int sqp_kv_cache_read(int T, int kv_heads, int D, int type, int page, int pages, const int *slots, const void *k_cache, const void *v_cache,
                                 const void *k_scales, const void *v_scales, void *k, void *v, void *stream)
{
    const int rc = sqp_check_cache(kv_heads, D, type, page, pages, k_cache, v_cache, k_scales, v_scales);
    if (rc) return rc;
    if (!slots || !k || !v) return SQP_ERR_NULL;
    if (T < 0) return SQP_ERR_SHAPE;
    if (((uintptr_t)slots & 3) || sqp_misaligned(k) || sqp_misaligned(v)) return SQP_ERR_ALIGN;
    if (T == 0) return SQP_OK;
    int shift = 0;
    while ((1 << shift) < page) shift++;
    hipStream_t st = (hipStream_t)stream;
#define KV_READ(TYPE) (D == 128 ? read<TYPE, 128>(T, kv_heads, shift, pages * page, slots, k_cache, v_cache, k_scales, v_scales, k, v, st) \
                                : read<TYPE, 64>(T, kv_heads, shift, pages * page, slots, k_cache, v_cache, k_scales, v_scales, k, v, st))
    if (type == SQP_FP16) KV_READ(SQP_FP16);
    else if (type == SQP_INT8) KV_READ(SQP_INT8);
    else if (type == SQP_E4M3) KV_READ(SQP_E4M3);
    else KV_READ(SQP_E2M1);
#undef KV_READ
    return sqp_launch_status();
}
