// Entry point of the microscaled product: argument checks and the choice of kernel, tile and K parts.
#include <algorithm>

#include "sqp_mx_gemm.h"

namespace {

int g_hook_kind = 0, g_hook_a = 0, g_hook_b = 0, g_hook_c = 0;

struct Plan {
    bool few;
    SqpMxFewPlan f;
    SqpMxTilePlan t;
    size_t bytes;
};

Plan plan(int M, int N, int K, int x_type, size_t room)
{
    Plan p = {};
    const long cus = 256;
    const int stages = (K + (x_type == SQP_E2M1 ? 255 : 127)) / (x_type == SQP_E2M1 ? 256 : 128);
    p.few = M <= 32;
    p.f.mt = M <= 16 ? 1 : M <= 32 ? 2 : 4;
    p.f.nt = N >= 16384 ? 2 : 1;
    p.f.kw = K > 2048 ? 8 : 4;
    p.t.parts = 1;
    if (!p.few) {
        p.t.tile = SQP_MX_TILES - 1;
        for (int t = 0; t < SQP_MX_TILES; t++) {
            int rows, cols;
            sqp_mx_tile_shape(t, &rows, &cols);
            const long tiles = (long)((M + rows - 1) / rows) * ((N + cols - 1) / cols);
            if (tiles >= cus * 3 / 4 || t == SQP_MX_TILES - 1 || (M > 64 && t == 1)) {
                p.t.tile = t;
                p.t.parts = (int)std::max(1L, std::min({2 * cus / std::max(tiles, 1L), (long)stages / 4, 16L}));
                break;
            }
        }
    }
    if (g_hook_kind == 1) {
        p.few = true;
        p.f = {g_hook_a, g_hook_b, g_hook_c};
    } else if (g_hook_kind == 2) {
        p.few = false;
        p.t = {g_hook_a, std::max(1, g_hook_b)};
    }
    if (p.few) return p;
    const size_t one = (size_t)M * N * sizeof(float);
    if (p.t.parts > 1 && (size_t)p.t.parts * one > room) p.t.parts = (int)std::max((size_t)1, room / one);
    p.bytes = p.t.parts > 1 ? p.t.parts * one : 0;
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
    return p.few ? sqp_mx_few(x_type, p.f, a, (hipStream_t)stream) : sqp_mx_tiles(x_type, p.t, a, (hipStream_t)stream);
}
