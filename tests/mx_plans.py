"""Sizes of the microscaled product, smallest first, and what the library makes of them by itself."""
import ctypes

E2M1, E4M3 = 4, 2

# M, N, K, activations, the plan: ("few", 16-row tiles, 16-column tiles, waves) or ("tiles", tile, K parts, tile of the columns left over)
CHOSEN = [
    (1, 8, 640, "e2m1", ("few", 1, 1, 8)), (16, 40, 1376, "e4m3", ("few", 1, 1, 8)), (3, 16392, 96, "e2m1", ("few", 1, 2, 8)), (1, 32960, 640, "e4m3", ("few", 1, 2, 8)),
    (17, 8, 640, "e4m3", ("few", 2, 1, 8)), (20, 16392, 288, "e2m1", ("few", 2, 2, 4)), (30, 16400, 96, "e4m3", ("few", 2, 2, 4)), (33, 8, 640, "e2m1", ("few", 4, 1, 8)),
    (64, 72, 1312, "e4m3", ("few", 4, 1, 8)),
    (33, 8, 512, "e4m3", ("tiles", 6, 1, None)), (33, 8, 2688, "e4m3", ("tiles", 6, 6, None)), (1, 16664, 512, "e2m1", ("tiles", 5, 1, None)),
    (1, 10600, 4480, "e4m3", ("tiles", 5, 3, None)), (65, 8, 512, "e2m1", ("tiles", 4, 1, None)), (100, 264, 11008, "e2m1", ("tiles", 4, 8, None)),
    (65, 8, 2688, "e4m3", ("tiles", 4, 6, None)), (257, 8, 640, "e2m1", ("tiles", 3, 1, None)), (257, 8, 3200, "e2m1", ("tiles", 3, 4, None)),
    (259, 8, 512, "e4m3", ("tiles", 2, 1, None)), (259, 8, 1664, "e4m3", ("tiles", 2, 4, None)), (70, 136, 1376, "e2m1", ("tiles", 7, 1, None)),
    (90, 264, 11040, "e4m3", ("tiles", 7, 8, None)), (66, 35096, 1152, "e4m3", ("tiles", 1, 1, None)), (133, 16408, 3200, "e2m1", ("tiles", 1, 1, None)),
    (149, 32856, 640, "e2m1", ("tiles", 0, 1, None)), (390, 32776, 640, "e2m1", ("tiles", 0, 1, 3)), (390, 32776, 640, "e4m3", ("tiles", 0, 1, 2)),
    (415, 35272, 640, "e2m1", ("tiles", 0, 1, 3)), (292, 47576, 1152, "e4m3", ("tiles", 0, 1, 1)), (579, 45184, 1664, "e4m3", ("tiles", 1, 1, 2))]


def chosen(L, M, N, K, kind):
    """The automatic plan as CHOSEN has it, with the number of columns in the first tile's launch."""
    p = (ctypes.c_int * 5)()
    assert L.sqp_debug_mx_plan(M, N, K, E2M1 if kind == "e2m1" else E4M3, p) == 0
    return (("few", *p[1:4]), N) if p[0] == 1 else (("tiles", p[1], p[2], p[4] if p[3] != N else None), p[3])
