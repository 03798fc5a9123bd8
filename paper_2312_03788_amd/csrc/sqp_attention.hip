// Entry point of the attention over the paged cache: argument checks and launches.
#include <limits.h>

#include <algorithm>

#include "sqp_attention.h"

int sqp_check_cache(int kv_heads, int D, int type, int page, int pages, const void *k_cache, const void *v_cache, const void *k_scales, const void *v_scales);

namespace {

// Joins the parts of the rows that have more than one: a wave per slot (the few-rows kernel's, `slots` per sequence and cached head, or
// with slots == 0 the tile kernel's), a lane per part for the weights; then D / 4 lanes have four values of a part each, so that two
// (D = 128) or four parts are read at once.
template <int D>
__global__ void __launch_bounds__(256) attention_combine_kernel(const SqpAttention a, const SqpParts p, int most_rows, int slots, int all_slots)
{
    constexpr int LANES = D / 4, AT_ONCE = 64 / LANES;
    const int slot = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * 4 + (threadIdx.x >> 6)));
    if (slot >= all_slots) return;
    const int lane = threadIdx.x & 63, d = 4 * (lane % LANES), which = lane / LANES;
    // read before it is known how many parts there are: the chain of loads is what this kernel takes
    const float *part = p.part + (size_t)slot * p.parts * (D + 4);
    const float m0 = part[min(lane, p.parts - 1) * (D + 4) + D], l0 = part[min(lane, p.parts - 1) * (D + 4) + D + 1];
    f32x4 x[4];
#pragma unroll
    for (int j = 0; j < 4; j++) x[j] = *(const f32x4 *)&part[min(j * AT_ONCE + which, p.parts - 1) * (D + 4) + d];
    int row, sees;
    if (slots) {
        const int b = slot / (a.kv_heads * slots), kv_head = slot / slots % a.kv_heads, r = slot % slots, token = r / a.group;
        const SqpSequence s = sqp_one_sequence(a, b);
        const int rows = s.n * a.group;
        if (r >= rows || rows > slots || rows > most_rows) return;
        row = (s.first + token) * a.heads + kv_head * a.group + r - token * a.group;  // (T heads D < 2^31)
        sees = s.len - s.n + token + 1;
    } else {
        const int token = slot / a.heads, b = __builtin_amdgcn_readfirstlane(sqp_sequence_of(a, token));
        if (b >= a.B) return;
        const SqpSequence s = sqp_one_sequence(a, b);
        row = slot;
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
    int few_slots, tile_slots;  // of rows that may have more than one part: of one kernel at most
    int fold;           // tiles on the first half of the places, the shortest then share theirs (0: none)
    size_t bytes;       // of partial results
};

constexpr int MOST_PARTS = 64;  // a lane each when they are joined

// Parts: as many as make `wanted` workgroups of these groups, each of at least `least` tokens.  512 workgroups, two per compute unit,
// are what runs at once: 16 sequences of up to 8192 tokens (8 cached heads, e4m3) take 38.9 us with parts for 512, 41.3 with 768, 40.8
// with 1024; one of 32000 (40 cached heads, int8) 67.1, 67.2, 66.4; 33 of up to 1570 (8 cached heads, int8) 25.4, 25.4, 23.4; 43 of up to
// 5152 (one cached head, int8) 18.3, 17.2, 19.0.  Where max_len is far above the lengths more would be better: one sequence of 2048 tokens,
// 32 heads, takes 9.8 us with its own length as max_len and 25.1, 20.4, 16.8 with 32768.  The tile kernel's parts cost their partial
// results besides, so its tiles are only split where they leave half the chip empty: wanting 1024, a 2048-token prompt takes 84.9 us
// instead of 65.2, a mixed step of six sequences 199 instead of 156.
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
    // Tiles of 256 rows are the quicker ones where they fill the chip (a workgroup per compute unit) twice or more: 2048 tokens behind
    // 14336, 64 heads on 8, 1166 us against 1237.  Below that tiles of 128 rows (two per compute unit) spread better: a 2048-token prompt
    // of 32 heads 65.3 us against 84.5.  (Many short prompts would rather have the small ones: 64 of 17 to 100 tokens 116 against 110.)
    auto count = [&](int height) { return (B == 1 ? ((long)T * group + height - 1) / height : (long)T * group / height + B) * kv_heads; };
    p.tile_rows = count(256) >= 2 * 256 ? 256 : 128;
    const long blocks = count(p.tile_rows);
    // Single tokens beside prompts: the tile kernel takes them along, a tile each, unless that costs more than a launch of the few-rows
    // kernel and the wait for its end.  It does where every head has a cache of its own, so that a tile holds one row, and there
    // are as many tiles as the chip takes at once (18 sequences of up to 393 tokens, 32 heads, e4m3: 34.5 us against 26.9; with two
    // sequences there is little to gain, 85 against 89), and where a long sequence's one row may be the longest tile, tiles being too
    // many to be split (a token at 16000 beside a chunk of 512 at 2048, 64 heads on 8: 351 against 81; 15 at 5000 to 14800 beside 2048 at
    // 16384: 1578 against 1244).  Elsewhere taking them along is mostly the quicker (60 sequences of up to 224 tokens, 16 heads on 1: 13.2
    // against 20.7; 25 of up to 5163, 64 on 8: 234 against 293), though not always (six sequences whose tokens are at 3000 and 5000, the
    // prompts short: 130 against 67).  Over 70 drawn mixed calls this is 1 % from the better choice on average, two kernels for all 21 %.
    const bool mixed = rows > SQP_FEW_ROWS && group <= SQP_FEW_ROWS && (long)B * max_q > T;
    p.few = rows <= SQP_FEW_ROWS || (mixed && ((group == 1 && B > 8 && blocks >= 512) || (blocks > 256 && max_len >= 8192)));
    p.tiles = rows > SQP_FEW_ROWS;
    p.f = split((long)B * kv_heads, 512, 256, max_len, most_parts);
    p.t = split(blocks, p.few ? 1 : 512, 512, max_len, most_parts);  // (beside the few-rows kernel tiles are whole: one joining kernel, one layout)
    const int at_once = p.tile_rows == 128 ? 512 : 256;
    p.fold = blocks * p.t.parts <= at_once && p.tile_rows == 128 ? 256 / (kv_heads * p.t.parts) : 0;
    // Parts are only made of few groups, at most 256 of a sequence and cached head or of tiles, so that the slots are few as well.
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
    attention_combine_kernel<D><<<(unsigned)((all + 3) / 4), 256, 0, st>>>(a, p.few_slots ? p.f : p.t, most_rows, p.few_slots ? p.slots : 0, all);
}

}  // namespace

extern "C" size_t sqp_paged_attention_scratch_bytes(int T, int B, int heads, int kv_heads, int D, int max_q, int max_len)
{
    if (T <= 0 || B <= 0 || heads <= 0 || kv_heads <= 0 || heads % kv_heads || max_q < 0 || max_len < 0 || (D != 64 && D != 128)) return 0;
    return plan(T, B, heads, kv_heads, D, max_q, max_len, MOST_PARTS).bytes;
}

extern "C" int sqp_paged_attention(int T, int B, int heads, int kv_heads, int D, int type, int page, int pages, int table_width, int max_q, int max_len,
                                   float scale, const void *q, long q_stride, const void *k_cache, const void *v_cache, const void *k_scales,
                                   const void *v_scales, const int *page_table, long table_stride, const int *seq_lens, const int *q_starts, void *out,
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
    a.scale2 = scale * (type == SQP_E2M1 ? 2.0f : 1.0f) * 1.44269504088896340736f;  // (blocks' keys are taken at half their size)
    hipStream_t st = (hipStream_t)stream;
    const int reach = max_len > 0 ? max_len : table_width * page, most_q = q_starts ? max_q : 1;
    Plan p = plan(T, B, heads, kv_heads, D, most_q, reach, MOST_PARTS);
    const size_t room = scratch ? scratch_bytes : 0;
    for (int most = room ? MOST_PARTS - 1 : 1; p.bytes > room; most--) p = plan(T, B, heads, kv_heads, D, most_q, reach, most);  // (one part takes none)
    p.f.part = p.t.part = (float *)scratch;
    const int most_rows = !p.few ? -1 : !p.tiles ? INT_MAX : SQP_FEW_ROWS;  // of the few-rows kernel
    if (p.few) sqp_attention_few(type, D, a, p.f, most_rows, p.slots, st);
    if (p.tiles) sqp_attention_tiles(type, D, a, p.t, p.tile_rows, std::max(most_rows, 0), p.fold, st);
    if (p.few_slots + p.tile_slots > 0) D == 128 ? combine<128>(a, p, most_rows, st) : combine<64>(a, p, most_rows, st);
    return sqp_launch_status();
}
