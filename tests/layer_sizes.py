"""Sizes of the products on a layer by the way that they go to the GPU, one for each way that there is (not collected by pytest): the CPU tests hold the plans to this
table, the GPU tests run all of it.  Contractions are long enough that rings of tiles come round (nine steps and more a part) and that each wave of few rows has two chunks
and more, and they end inside a step."""
import paper_1706_07191_amd as B


def way_of(plan):
    """What of a plan decides which kernels run: few rows by their tiles, or tiles of 256 rows, of 64 times so many rows, and a contraction in parts."""
    rows, mt, nt, tiles, large, nq, parts, _ = plan
    return ("rows", mt, nt) if rows else ("tiles", 256 if large else 0, 64 * nq, parts > 1)


# (rows, columns, contraction) = m, n, k
LINEAR = {
    ("rows", 1, 1): (1, 68, 2394), ("rows", 1, 2): (3, 4124, 2199), ("rows", 1, 3): (16, 8481, 2281), ("rows", 1, 5): (7, 17775, 2475),
    ("rows", 2, 1): (17, 79, 2156), ("rows", 2, 2): (18, 4659, 2279), ("rows", 2, 3): (20, 8354, 2177), ("rows", 2, 5): (17, 12307, 2239),
    ("rows", 3, 1): (33, 67, 2275), ("rows", 3, 2): (35, 4481, 2160), ("rows", 3, 3): (33, 9393, 2139), ("rows", 3, 5): (40, 12658, 2178),
    ("rows", 4, 1): (51, 66, 2223), ("rows", 4, 2): (49, 4323, 2244), ("rows", 4, 3): (50, 9278, 2121), ("rows", 4, 5): (50, 20001, 2100),
    ("tiles", 0, 64, False): (1964, 138, 518), ("tiles", 0, 64, True): (1369, 79, 7004), ("tiles", 0, 128, False): (8749, 261, 563), ("tiles", 0, 128, True): (6594, 65, 2714),
    ("tiles", 256, 0, False): (146, 33784, 551), ("tiles", 256, 0, True): (8296, 68, 4437), ("tiles", 256, 64, False): (405, 32961, 551), ("tiles", 256, 128, False): (520, 29566, 564),
}
# (rows, contraction, columns) = m, n, k
BACKWARD = {
    ("tiles", 0, 64, False): (5505, 513, 93), ("tiles", 0, 64, True): (72, 11164, 65), ("tiles", 0, 128, False): (8435, 527, 273), ("tiles", 0, 128, True): (1404, 9587, 68),
    ("tiles", 256, 0, False): (8661, 519, 770), ("tiles", 256, 0, True): (2960, 11141, 67), ("tiles", 256, 64, False): (3392, 525, 4647), ("tiles", 256, 128, False): (6498, 513, 2820),
}
# tokens, dim, width
GLU = {
    ("rows", 1, 1): (5, 4211, 68), ("rows", 2, 1): (18, 2201, 87), ("rows", 4, 1): (50, 2203, 69),
    ("tiles", 0, 64, False): (84, 513, 1359), ("tiles", 0, 64, True): (1268, 7709, 68), ("tiles", 0, 128, False): (65, 554, 16495), ("tiles", 0, 128, True): (130, 1919, 4219),
    ("tiles", 256, 0, False): (142, 515, 17155), ("tiles", 256, 0, True): (8344, 1880, 141), ("tiles", 256, 64, False): (135, 577, 32846), ("tiles", 256, 128, False): (268, 519, 23802),
}
GLU_DX = {
    ("tiles", 0, 64, False): (433, 520, 261), ("tiles", 0, 64, True): (69, 70, 5186), ("tiles", 0, 128, False): (8254, 261, 275), ("tiles", 0, 128, True): (1347, 68, 5062),
    ("tiles", 256, 0, False): (8274, 808, 267), ("tiles", 256, 0, True): (8777, 65, 2183), ("tiles", 256, 64, False): (3331, 4637, 259), ("tiles", 256, 128, False): (8409, 2073, 262),
}
GLU_DW = {
    ("tiles", 0, 64, False): (518, 88, 1293), ("tiles", 0, 64, True): (8421, 67, 577), ("tiles", 0, 128, False): (546, 65, 8716), ("tiles", 0, 128, True): (1376, 65, 5558),
    ("tiles", 256, 0, False): (524, 66, 17585), ("tiles", 256, 0, True): (2097, 68, 8230), ("tiles", 256, 64, False): (524, 1574, 4674), ("tiles", 256, 128, False): (515, 546, 11962),
}
PLANS = {
    "linear": (LINEAR, lambda m, n, k: B.brsvd_linear_e2m1_plan(m, n, k), lambda m, n, k: k),
    "backward": (BACKWARD, lambda m, n, k: B.brsvd_linear_e2m1_plan(m, n, k, True), lambda m, n, k: n),
    "glu": (GLU, lambda t, d, f: B.brsvd_glu_plan(0, t, d, f), lambda t, d, f: d),
    "dX": (GLU_DX, lambda t, d, f: B.brsvd_glu_plan(1, t, d, f), lambda t, d, f: 2 * (-(-f // 64) * 64)),
    "dW": (GLU_DW, lambda t, d, f: B.brsvd_glu_plan(2, t, d, f), lambda t, d, f: t),
}
