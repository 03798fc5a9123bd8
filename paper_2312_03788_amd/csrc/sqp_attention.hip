// Entry point of the attention over the paged cache: argument checks and launches.
#include "sqp_attention.h"

int sqp_check_cache(int kv_heads, int D, int type, int page, int pages, const void *k_cache, const void *v_cache, const float *k_scales, const float *v_scales);

namespace {

// One wave per query row.
template <int TYPE, int D>
__global__ void __launch_bounds__(256) attention_rows_kernel(const SqpAttention a)
{
    constexpr int PER = D / 64;
    const long row = (long)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= (long)a.T * a.heads) return;
    const int token = __builtin_amdgcn_readfirstlane((int)(row / a.heads)), head = __builtin_amdgcn_readfirstlane((int)(row % a.heads));
    const int b = __builtin_amdgcn_readfirstlane(sqp_sequence_of(a, token));
    float m, l = 0.f, o[PER] = {};
    if (b < a.B) {
        const SqpSequence s = sqp_sequence(a, b);
        const int sees = min(s.len, s.len - s.n + (token - s.first) + 1);
        sqp_attend_row<TYPE, D>(a, a.q + token * a.q_stride + head * D, a.table + b * a.table_stride, head / a.group, 0, sees, m, l, o);
    }
    h16 *out = a.out + row * D + PER * (threadIdx.x & 63);
#pragma unroll
    for (int e = 0; e < PER; e++) out[e] = (h16)(l == 0.f ? 0.f : o[e] / l);
}

template <int TYPE, int D>
void rows(const SqpAttention &a, hipStream_t st)
{
    attention_rows_kernel<TYPE, D><<<(unsigned)(((long)a.T * a.heads + 3) / 4), 256, 0, st>>>(a);
}

}  // namespace

extern "C" size_t sqp_paged_attention_scratch_bytes(int T, int B, int heads, int kv_heads, int D, int max_q, int max_len)
{
    return 0;
}

extern "C" int sqp_paged_attention(int T, int B, int heads, int kv_heads, int D, int type, int page, int pages, int table_width, int max_q, int max_len,
                                   float scale, const void *q, long q_stride, const void *k_cache, const void *v_cache, const float *k_scales,
                                   const float *v_scales, const int *page_table, long table_stride, const int *seq_lens, const int *q_starts, void *out,
                                   void *scratch, size_t scratch_bytes, void *stream)
{
    const int rc = sqp_check_cache(kv_heads, D, type, page, pages, k_cache, v_cache, k_scales, v_scales);
    if (rc) return rc;
    if (!q || !page_table || !seq_lens || !out) return SQP_ERR_NULL;
    if (T < 0 || B < 0 || B > 65535 || heads <= 0 || heads > 65535 || (heads % kv_heads) || max_q < 0 || max_len < 0) return SQP_ERR_SHAPE;
    if ((!q_starts && T != B) || (B == 0 && T > 0)) return SQP_ERR_SHAPE;
    if (table_width <= 0 || (long)table_width * page >= (1L << 31) || (B > 1 && table_stride < table_width)) return SQP_ERR_SHAPE;
    if (q_stride < (long)heads * D || sqp_too_big(T, (long)heads * D)) return SQP_ERR_SHAPE;
    if (!(scale > 0.0f) || !(scale < 1e30f)) return SQP_ERR_ARG;
    if ((q_stride % 8) || sqp_misaligned(q) || sqp_misaligned(out) || (scratch && sqp_misaligned(scratch))) return SQP_ERR_ALIGN;
    if (((uintptr_t)page_table | (uintptr_t)seq_lens | (uintptr_t)q_starts) & 3) return SQP_ERR_ALIGN;
    if (T == 0) return SQP_OK;
    SqpAttention a = {};
    a.T = T; a.B = B; a.heads = heads; a.kv_heads = kv_heads; a.group = heads / kv_heads;
    while ((1 << a.page_shift) < page) a.page_shift++;
    a.pages = pages; a.table_width = table_width;
    a.q_stride = q_stride; a.table_stride = table_stride;
    a.q = (const h16 *)q; a.k = k_cache; a.v = v_cache; a.k_scales = k_scales; a.v_scales = v_scales;
    a.table = page_table; a.lens = seq_lens; a.starts = q_starts; a.out = (h16 *)out;
    a.scale2 = scale * 1.44269504088896340736f;
    hipStream_t st = (hipStream_t)stream;
#define ATTEND(TYPE) (D == 128 ? rows<TYPE, 128>(a, st) : rows<TYPE, 64>(a, st))
    if (type == SQP_FP16) ATTEND(SQP_FP16);
    else if (type == SQP_INT8) ATTEND(SQP_INT8);
    else ATTEND(SQP_E4M3);
#undef ATTEND
    return sqp_launch_status();
}
