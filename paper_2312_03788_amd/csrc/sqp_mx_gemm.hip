// Entry point of the microscaled product: argument checks and the choice of kernel, tile and K parts.
#include <algorithm>

#include "sqp_mx_gemm.h"

namespace {

int g_hook_kind = 0, g_hook_a = 0, g_hook_b = 0, g_hook_c = 0;

struct Plan {
    bool few;
    SqpMxFewPlan f;
    SqpMxTilePlan t;     // of the first columns
    int cols;            // how many
    SqpMxTilePlan rest;  // of the others (whole K), if there are any
    size_t bytes;        // of partial sums
};

// What a call takes in us, by the number of its workgroups: the least squares over 1799 timed calls (e2m1) and 1202 (e4m3) of every tile in one
// to eight K parts, row counts from 1 to 4096 on eight layers from 1024 x 4096 to 44032 x 8192.  A round of workgroups, as many
// as run at once, takes `tile` and for every 512 k `chunk[n - 1]` with n workgroups on a compute unit; a joining kernel takes `join`
// and `join_mb` per MB of partial sums; the few-rows kernel `few` and per million weights `few_w` + rows * `few_mw`.  A call is off by 10 %
// (root mean square).  Over the 207 sizes what is chosen now takes 2 % more than the best of all forms on average, 28 % at worst (1000 x 1024 x 4096,
// e4m3: 18.3 us in four parts, 14.3 in one); over 28 sizes of layers that the fit does not know (4096 x 11008, 11008 x 4096) 4 %, 28 % at worst
// (333 x 11008 x 4096, e2m1: 24.6 us in tiles of 128 x 256, 19.3 in 128 x 128).
struct Costs {
    float launch, join, join_mb, few, few_w, few_mw;
    struct {
        float tile, chunk[4];
        int at_once;  // per compute unit
    } tile[SQP_MX_DIRECT_TILES];
};
constexpr Costs COSTS4 = {1.27f, 3.95f, 0.357f, 3.4f, 0.120f, 0.0045f,
                          {{4.59f, {2.92f}, 1}, {2.94f, {2.28f}, 1}, {1.37f, {1.64f, 2.54f}, 2}, {1.98f, {1.25f}, 1}, {1.19f, {1.20f, 2.82f}, 2},
                           {1.17f, {1.00f, 2.46f}, 2}, {1.12f, {0.75f, 1.27f, 2.17f, 3.22f}, 4}}};
constexpr Costs COSTS8 = {0.67f, 4.09f, 0.331f, 3.4f, 0.130f, 0.0085f,
                          {{6.65f, {4.08f}, 1}, {4.40f, {2.63f}, 1}, {2.18f, {1.78f, 3.54f}, 2}, {2.55f, {1.70f}, 1}, {2.54f, {1.31f}, 1},
                           {1.59f, {1.19f, 2.82f}, 2}, {0.84f, {1.11f, 1.75f, 2.65f, 3.37f}, 4}}};
constexpr int CUS = 256;

int up(int a, int b) { return (a + b - 1) / b; }

float tile_cost(const Costs &c, int t, int M, int N, int K, int parts)
{
    const auto &k = c.tile[t];
    const int chunks = up(K, 512), per = up(chunks, parts), real = up(chunks, per);
    const long groups = (long)up(M, SQP_MX_TILE[t].rows) * up(N, SQP_MX_TILE[t].cols) * real, room = CUS * k.at_once;
    const long full = groups / room, rest = groups % room;
    float us = full * (k.tile + per * k.chunk[k.at_once - 1]);
    if (rest) us += k.tile + per * k.chunk[up((int)rest, CUS) - 1];
    if (real > 1) us += c.join + c.join_mb * 4e-6f * M * N * real;
    return us + c.launch;
}

Plan plan(int M, int N, int K, int x_type, size_t room)
{
    Plan p = {};
    p.cols = N;
    p.t.parts = p.rest.parts = 1;
    p.f.mt = M <= 16 ? 1 : M <= 32 ? 2 : 4;
    p.f.nt = N >= 16384 && M <= 32 ? 2 : 1;  // (16 x 44032 x 8192: 51 us with two, 57 with one; 16 x 8192 x 8192 11.5, 11.0)
    p.f.kw = p.f.mt == 2 && p.f.nt == 2 ? 4 : 8;
    const int chunks = up(K, 512);
    const size_t one = (size_t)M * N * sizeof(float);
    const int most = (int)std::min((size_t)8, std::max(room / one, (size_t)1));
    if (K % 128 || K < 512) {  // scales that do not begin at words, or no 16 of a row: no direct copies
        // By the number of rows alone, which is not always the quicker: over 42 sizes 12 % more than the better of the two on average.  Up to 16 rows the
        // few-rows kernel is, but for short K on many columns (1 x 4096 x 11040, e2m1: 10.7 us, tiles 14.5; 16 x 16384 x 480: 9.2, 6.3); up to
        // 64 on up to 4096 columns mostly (64 x 2048 x 4128: 9.7, 11.1; but 64 x 4096 x 480: 9.3, 6.1), on more columns and long K tiles are (64 x 8192 x
        // 1376: 16.8, 8.4; 64 x 4096 x 11040: 24.3, 17.5).  Parts: as many as fill two workgroups per compute unit (100 x 4096 x 11040: 19.1 us
        // in eight, 55.6 whole), which a short K does not want (333 x 5120 x 4128: 24.9 in four, 18.3 whole).
        p.few = M <= 64;
        p.t.tile = SQP_MX_DIRECT_TILES;
        const long groups = (long)up(M, 128) * up(N, 128);
        if (!p.few) p.t.parts = (int)std::max(1L, std::min({2L * CUS / groups, (long)chunks / 2, (long)most}));
    } else {
        const Costs &c = x_type == SQP_E2M1 ? COSTS4 : COSTS8;
        float best = 1e30f;
        if (M <= (x_type == SQP_E2M1 ? 64 : 32)) {  // (e4m3, 33 to 64 rows: tiles are as quick on all sizes timed, 64 x 1024 x 4096 7.7 us instead of 11.8)
            best = c.few + 1e-6f * N * K * (c.few_w + c.few_mw * M);
            p.few = true;
        }
        auto offer = [&](int t, int parts, int cols, int rest, float us) {
            if (us >= best) return;
            best = us;
            p.few = false;
            p.t = {t, parts};
            p.cols = cols;
            p.rest.tile = rest;
        };
        const int lo = M > 96 ? 0 : M > 64 ? 1 : M > 32 ? 3 : 5, hi = M > 256 ? 3 : M > 64 ? 4 : 6;  // tiles of the rows' size
        for (int t = lo; t <= hi; t++) {
            const SqpMxTileShape &s = SQP_MX_TILE[t];
            const long groups = (long)up(M, s.rows) * up(N, s.cols), at_once = CUS * c.tile[t].at_once;
            // K parts up to one and a half times what runs at once (which bounds their sums: 96 MiB in the largest tile): 16 x 44032 x 8192, e4m3, 45.5 us
            // in 688 workgroups on 512 places, 51 in smaller tiles without parts.
            for (int parts : {1, 2, 3, 4, 6, 8})
                if (parts == 1 || (parts <= most && parts <= chunks && 2 * groups * parts <= 3 * at_once)) offer(t, parts, N, 0, tile_cost(c, t, M, N, K, parts));
            // Whole rounds of this tile, and the columns left over in tiles of another shape.  (Not for few rows, which wait for memory in either
            // launch: 33 x 44032 x 8192, e2m1, 54.7 us in two, 49.8 in one.)
            if (M > 64 && groups > at_once && groups % at_once) {
                const int cols = (int)(groups / at_once * at_once / up(M, s.rows)) * s.cols;
                for (int r = t + 1; r <= hi && cols > 0 && cols < N; r++)
                    offer(t, 1, cols, r, tile_cost(c, t, M, cols, K, 1) + tile_cost(c, r, M, N - cols, K, 1) + 1.0f);
            }
        }
    }
    if (g_hook_kind == 1) {
        p.few = true;
        p.f = {g_hook_a, g_hook_b, g_hook_c};
    } else if (g_hook_kind == 2) {
        p.few = false;
        p.t = {std::min(g_hook_a, SQP_MX_TILES - 1), std::min(std::max(1, g_hook_b), (int)std::min((size_t)64, std::max(room / one, (size_t)1)))};
        p.cols = N;
    } else if (g_hook_kind == 3) {
        p.few = false;
        p.t = {g_hook_a, 1};
        p.cols = std::min(N, g_hook_c * SQP_MX_TILE[g_hook_a].cols);
        p.rest.tile = g_hook_b;
    }
    p.bytes = !p.few && p.t.parts > 1 ? p.t.parts * one : 0;
    return p;
}

bool shape_ok(int M, int N, int K)
{
    return M > 0 && N > 0 && K > 0 && !(N % 8) && !(K % SQP_MX_BLOCK) && !sqp_too_big(M, K) && !sqp_too_big(N, K) && !sqp_too_big(M, N);
}

}  // namespace

extern "C" void sqp_debug_set_mx_plan(int kind, int a, int b, int c)
{
    g_hook_kind = kind;
    g_hook_a = a;
    g_hook_b = b;
    g_hook_c = c;
}

extern "C" int sqp_debug_mx_plan(int M, int N, int K, int x_type, int *to)
{
    if (!to) return SQP_ERR_NULL;
    if (!shape_ok(M, N, K) || (x_type != SQP_E2M1 && x_type != SQP_E4M3)) return SQP_ERR_SHAPE;
    const Plan p = plan(M, N, K, x_type, (size_t)-1);
    const int few[5] = {1, p.f.mt, p.f.nt, p.f.kw, 0}, tiles[5] = {2, p.t.tile, p.t.parts, p.cols, p.rest.tile};
    std::copy_n(p.few ? few : tiles, 5, to);
    return SQP_OK;
}

extern "C" size_t sqp_mx_gemm_scratch_bytes(int M, int N, int K, int x_type)
{
    if (!shape_ok(M, N, K) || (x_type != SQP_E2M1 && x_type != SQP_E4M3)) return 0;
    return plan(M, N, K, x_type, (size_t)-1).bytes;
}

extern "C" int sqp_mx_gemm(int M, int N, int K, int x_type, int silu_mul, const void *x, const uint8_t *x_scales, const void *w, const uint8_t *w_scales,
                           void *y, void *scratch, size_t scratch_bytes, void *stream)
{
    if (!x || !x_scales || !w || !w_scales || !y) return SQP_ERR_NULL;
    if (x_type != SQP_E2M1 && x_type != SQP_E4M3) return SQP_ERR_ARG;
    if (!shape_ok(M, N, K) || (silu_mul && (N % 16))) return SQP_ERR_SHAPE;
    if (sqp_misaligned(x) || sqp_misaligned(x_scales) || sqp_misaligned(w) || sqp_misaligned(w_scales) || sqp_misaligned(y)) return SQP_ERR_ALIGN;
    if (scratch && sqp_misaligned(scratch)) return SQP_ERR_ALIGN;
    SqpMxGemm a = {};
    a.M = M; a.N = N; a.K = K; a.silu = silu_mul != 0;
    a.x = x; a.w = w; a.xs = x_scales; a.ws = w_scales; a.y = (h16 *)y; a.part = (float *)scratch;
    const Plan p = plan(M, N, K, x_type, scratch ? scratch_bytes : 0);
    hipStream_t st = (hipStream_t)stream;
    if (p.few) return sqp_mx_few(x_type, p.f, a, st);
    a.cols = p.cols;
    const int rc = sqp_mx_tiles(x_type, p.t, a, st);
    if (rc || p.cols == N) return rc;
    a.first_col = p.cols;
    a.cols = N - p.cols;
    return sqp_mx_tiles(x_type, p.rest, a, st);
}
