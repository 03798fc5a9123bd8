// Entry point of the attention over the paged cache: argument checks and launches.
#include <limits.h>

#include <algorithm>

#include "sqp_attention.h"

int sqp_check_cache(int kv_heads, int D, int type, int page, int pages, const void *k_cache, const void *v_cache, const float *k_scales, const float *v_scales);

namespace {

// Joins the parts of the rows that have more than one: a wave per slot (the few-rows kernel's `few_slots`, then the tile kernel's),
// a lane per part for the weights; then D / 4 lanes have four values of a part each, so that two (D = 128) or four parts are read at
// once.
template <int D>
__global__ void __launch_bounds__(256) attention_combine_kernel(const SqpAttention a, const SqpParts few, const SqpParts tiles, int most_rows, int slots,
                                                                int few_slots, int all_slots)
{
    constexpr int LANES = D / 4, AT_ONCE = 64 / LANES;
    const int at = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * 4 + (threadIdx.x >> 6)));
    if (at >= all_slots) return;
    const bool is_few = at < few_slots;
    const int slot = is_few ? at : at - few_slots;
    const SqpParts &p = is_few ? few : tiles;
    const int lane = threadIdx.x & 63, d = 4 * (lane % LANES), which = lane / LANES;
    // read before it is known how many parts there are: the chain of loads is what this kernel takes
    const float *part = p.part + (size_t)slot * p.parts * (D + 4);
    const float m0 = part[min(lane, p.parts - 1) * (D + 4) + D], l0 = part[min(lane, p.parts - 1) * (D + 4) + D + 1];
    f32x4 x[4];
#pragma unroll
    for (int j = 0; j < 4; j++) x[j] = *(const f32x4 *)&part[min(j * AT_ONCE + which, p.parts - 1) * (D + 4) + d];
    int b, row, sees;
    if (is_few) {
        const int kv_head = slot / slots % a.kv_heads, r = slot % slots, token = r / a.group;
        b = slot / (a.kv_heads * slots);
        const SqpSequence s = sqp_one_sequence(a, b);
        const int rows = s.n * a.group;
        if (r >= rows || rows > slots || rows > most_rows) return;
        row = (s.first + token) * a.heads + kv_head * a.group + r - token * a.group;  // (T heads D < 2^31)
        sees = s.len - s.n + token + 1;
    } else {
        const int token = slot / a.heads;
        row = slot;
        b = __builtin_amdgcn_readfirstlane(sqp_sequence_of(a, token));
        if (b >= a.B) return;
        const SqpSequence s = sqp_one_sequence(a, b);
        if (s.n * a.group <= most_rows) return;
        sees = s.len - s.n + (token - s.first) + 1;
    }
    const int n = p.of(sees);
    if (n == 1) return;
    const float m = lane < n ? m0 : SQP_LOWEST;
    const float top = sqp_wave_join<true>(m);
    const float w = lane < n ? sqp_exp2(m - top) : 0.f;
    const float sum = sqp_wave_join<false>(lane < n ? w * l0 : 0.f);
    f32x4 o = (f32x4)(0.f);
    for (int i = 0; i < n; i += 4 * AT_ONCE) {
        if (i > 0) {
#pragma unroll
            for (int j = 0; j < 4; j++) x[j] = *(const f32x4 *)&part[min(i + j * AT_ONCE + which, n - 1) * (D + 4) + d];
        }
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const int from = i + j * AT_ONCE + which;
            const float wj = __shfl(w, from & 63, 64);
            if (from < n) o += wj * x[j];
        }
    }
#pragma unroll
    for (int off = 32; off >= LANES; off >>= 1)
#pragma unroll
        for (int e = 0; e < 4; e++) o[e] += __shfl_xor(o[e], off, 64);
    if (which == 0) {
        h16x4 y;
#pragma unroll
        for (int e = 0; e < 4; e++) y[e] = (h16)(sum == 0.f ? 0.f : o[e] / sum);
        *(h16x4 *)(a.out + (size_t)row * D + d) = y;
    }
}

// What a call launches.
struct Plan {
    bool few, tiles;    // which kernels
    int tile_rows;      // 128 or 256
    SqpParts f, t;      // their parts
    int slots;          // of the few-rows kernel, per sequence and cached head
    int few_slots, tile_slots;  // of rows that may have more than one part
    int fold;           // tiles on the first half of the places, the shortest then share theirs (0: none)
    size_t bytes;       // of partial results
};

constexpr int MOST_PARTS = 64;  // a lane each when they are joined

// Parts: as many as make `wanted` workgroups of these groups, each of at least `least` tokens.  512 workgroups, two per compute unit,
// are what runs at once: decoding at 8192 (16 sequences, 8 cached heads, e4m3) takes 47 us with parts for 512, 53 with 768, 48.5
// with 1024, one sequence at 32000 (int8) 82, 89 and 82.  The tile kernel's parts cost their partial results besides (a 2048-token
// prompt in parts of 1024 takes 92 us instead of 66), so its tiles are only split where they leave half the chip empty.
SqpParts split(long groups, long wanted, int least, int max_len, int most_parts)
{
    const long parts = std::max(1L, std::min((long)most_parts, wanted / std::max(groups, 1L)));
    SqpParts p = {};
    const long chunk = std::max((long)least, (((long)max_len + parts - 1) / parts + 127) / 128 * 128);
    p.chunk = (int)std::min(chunk, 1L << 30);
    p.parts = (int)std::max(1L, std::min((long)most_parts, ((long)max_len + chunk - 1) / chunk));
    return p;
}

Plan plan(int T, int B, int heads, int kv_heads, int D, int max_q, int max_len, int most_parts)
{
    Plan p = {};
    const int group = heads / kv_heads;
    max_q = std::max(1, std::min(max_q > 0 ? max_q : T, T));
    max_len = std::max(max_len, 1);
    const long rows = (long)max_q * group;
    // Single tokens beside prompts: the few-rows kernel reads their cache faster, but its launch waits for the other one's end. Up to
    // 8 sequences the tile kernel takes them along (four prompts and two tokens of 64 heads on 8: 194 -> 171 us).
    p.few = rows <= SQP_FEW_ROWS || (group <= SQP_FEW_ROWS && (long)B * max_q > T && B > 8);
    p.tiles = rows > SQP_FEW_ROWS;
    // Tiles of 256 rows are the quicker ones where they fill the chip (a workgroup per compute unit) twice or more: 2048 tokens behind
    // 14336, 64 heads on 8, 1240 -> 1155 us.  Below that tiles of 128 rows (two per compute unit) spread better: a 2048-token prompt
    // of 32 heads 75 -> 68 us.
    auto count = [&](int height) { return (B == 1 ? ((long)T * group + height - 1) / height : (long)T * group / height + B) * kv_heads; };
    p.tile_rows = count(256) >= 2 * 256 ? 256 : 128;
    const long blocks = count(p.tile_rows);
    p.f = split((long)B * kv_heads, 512, 256, max_len, most_parts);
    p.t = split(blocks, 512, 512, max_len, most_parts);
    const int at_once = p.tile_rows == 128 ? 512 : 256;
    p.fold = blocks * p.t.parts <= at_once && p.tile_rows == 128 ? 256 / (kv_heads * p.t.parts) : 0;
    // (Parts are only made of few groups: at most 256 of a sequence and cached head, or of tiles, so the slots are few as well.)
    p.slots = p.tiles ? SQP_FEW_ROWS : (int)rows;
    p.few_slots = p.few && p.f.parts > 1 ? B * kv_heads * p.slots : 0;
    p.tile_slots = p.tiles && p.t.parts > 1 ? T * heads : 0;
    p.bytes = ((size_t)p.few_slots * p.f.parts + (size_t)p.tile_slots * p.t.parts) * (D + 4) * sizeof(float);
    return p;
}

template <int D>
void combine(const SqpAttention &a, const Plan &p, int most_rows, hipStream_t st)
{
    const int all = p.few_slots + p.tile_slots;
    attention_combine_kernel<D><<<(unsigned)((all + 3) / 4), 256, 0, st>>>(a, p.f, p.t, most_rows, p.slots, p.few_slots, all);
}

}  // namespace

extern "C" size_t sqp_paged_attention_scratch_bytes(int T, int B, int heads, int kv_heads, int D, int max_q, int max_len)
{
    if (T <= 0 || B <= 0 || heads <= 0 || kv_heads <= 0 || heads % kv_heads || max_q < 0 || max_len < 0 || (D != 64 && D != 128)) return 0;
    return plan(T, B, heads, kv_heads, D, max_q, max_len, MOST_PARTS).bytes;
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
    if (table_width <= 0 || (long)table_width * page > (1L << 30) || (B > 1 && table_stride < table_width)) return SQP_ERR_SHAPE;
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
    const int reach = max_len > 0 ? max_len : table_width * page, most_q = q_starts ? max_q : 1;
    Plan p = plan(T, B, heads, kv_heads, D, most_q, reach, MOST_PARTS);
    const size_t room = scratch ? scratch_bytes : 0;
    for (int most = room ? MOST_PARTS - 1 : 1; p.bytes > room; most--) p = plan(T, B, heads, kv_heads, D, most_q, reach, most);  // (one part takes none)
    p.f.part = (float *)scratch;
    p.t.part = p.f.part + (size_t)p.few_slots * p.f.parts * (D + 4);
    const int most_rows = !p.few ? -1 : !p.tiles ? INT_MAX : SQP_FEW_ROWS;  // of the few-rows kernel
    if (p.few) sqp_attention_few(type, D, a, p.f, most_rows, p.slots, st);
    if (p.tiles) sqp_attention_tiles(type, D, a, p.t, p.tile_rows, std::max(most_rows, 0), p.fold, st);
    if (p.few_slots + p.tile_slots > 0) D == 128 ? combine<128>(a, p, most_rows, st) : combine<64>(a, p, most_rows, st);
    return sqp_launch_status();
}
