"""Which code of gemm_i8's kernels a product runs through, and products that run through all of it.

A kernel is a tile shape; beside it count whether the last K tile (128 inputs) is a partial one, whether rows are dealt to groups, whether
K is long enough for the unrolled loop of the large tiles, and which copy of the loop a tile takes: `once` for a group of one row tile
whose weights are past the caches, `tail WxH` for tiles behind the last whole round of 256 x 256."""
import paper_2405_13053_amd as m

KT = 128
# K tiles from which the unrolled loop of a tile shape is entered: a period of its two rings and the tiles that are on their way
UNROLLED_FROM = {(192, 128): 15, (224, 128): 15, (256, 128): 15, (256, 256): 8}


def deal(T, N):
    """Rows of N groups: a large one first, small, single and empty ones behind it, and a last row that is in none."""
    most, left, small = max(T // (4 * N), 1), T - 1, []
    for e in range(N - 1):
        small.append(max(min((0, 17, 1, 40, 63, 5, 16)[e % 7], most, left - 1), 0))
        left -= small[-1]
    return [left] + small


def code_of(T, d_in, d_out, counts=None):
    """The set of (kernel, rows, cols, per_cu, partial K tile, groups, unrolled, copy) that a call runs through; counts: rows of each group."""
    plan = m.gemm_i8_kernel(T, d_in, d_out, None if counts is None else len(counts))
    name, rows, cols, per_cu, read_once, tail = plan
    key = (name, rows, cols, per_cu, d_in % KT != 0, counts is not None, d_in // KT >= UNROLLED_FROM.get((rows, cols), 1 << 30))
    groups = [T] if counts is None else counts
    tiles = [-(-c // rows) for c in groups if c > 0]
    copies = set()
    if tail:
        total = sum(tiles) * -(-d_out // cols)
        rest = total % 256 if total > 256 and total % 256 <= 128 else 0
        if total > rest:
            copies.add("kept")
        if rest:
            copies.add("tail 64x64" if rest <= 16 else "tail 128x64" if rest <= 32 else "tail 128x128")
    else:
        copies = {"once" if read_once and t == 1 else "kept" for t in tiles}
    # the tail's tiles have loops of their own, none of them unrolled
    return {key + (c,) if not c.startswith("tail") else key[:6] + (False, c) for c in copies}


# (T, d_in, d_out, N): a product that runs through each of them (test_i8_kernels_host sees to it), small ones first
PRODUCTS = [
    (1, 256, 8, None), (340, 160, 360, None), (401, 256, 304, None), (614, 416, 200, None), (1, 10432, 8, None),
    (1, 10496, 8, None), (578, 832, 200, None), (330, 512, 392, None), (451, 768, 272, None), (40, 1040, 264, None),
    (10430, 784, 648, None), (142, 144, 8248, None), (77, 144, 8464, None), (106, 144, 8696, None), (136, 160, 9576, None),
    (2438, 1024, 1800, None), (65, 256, 8280, None), (97, 256, 8424, None), (130, 256, 8752, None), (3635, 1040, 2200, None),
    (139, 256, 9512, None), (3215, 1984, 1232, None), (1676, 272, 10392, None), (2571, 1024, 2784, None),
    (2334, 1024, 3368, None), (3030, 576, 8184, None), (1034, 896, 5544, None), (2188, 352, 14584, None), (544, 672, 8552, None),
    (1286, 1920, 3000, None), (1992, 1936, 3024, None), (4813, 896, 6688, None), (1286, 512, 12288, None), (650, 736, 8752, None),
    (1746, 2048, 3288, None), (1124, 1920, 5432, None), (1872, 896, 12192, None), (720, 2000, 8216, None),
    (17, 10752, 9304, None), (23, 6688, 14960, None), (68, 9792, 10248, None), (99, 8448, 11896, None), (68, 9216, 10944, None),
    (106, 11280, 8960, None), (670, 144, 168, 2), (606, 416, 200, 2), (2, 10624, 8, 2), (2, 10736, 8, 2), (451, 512, 264, 2),
    (574, 768, 200, 2), (7734, 896, 904, 2), (4053, 912, 1672, 2), (3, 256, 8216, 2), (201, 1536, 1560, 2), (5, 256, 9520, 2),
    (1446, 1952, 2480, 2), (1561, 528, 72, 3), (33, 272, 520, 3), (13, 144, 6280, 3), (7102, 1056, 1032, 3),
    (5243, 1024, 1448, 3), (4484, 2048, 776, 3), (43, 7008, 4800, 3), (70, 2048, 136, 5), (17, 144, 3304, 5),
    (2357, 400, 6304, 5), (1093, 400, 8800, 5), (1098, 512, 8280, 5), (143, 6528, 3088, 5), (593, 3920, 5192, 5),
    (766, 1712, 12056, 5), (735, 4224, 4968, 5), (753, 1792, 12072, 5), (165, 256, 1808, 8), (9608, 512, 1544, 8),
    (3302, 288, 3584, 8), (1527, 512, 5728, 8), (930, 4224, 2960, 8), (9, 1984, 6304, 8), (4, 1136, 11032, 8), (3, 896, 13992, 8),
    (113, 7296, 1720, 8), (4, 896, 14016, 8), (1163, 4176, 3040, 8), (120, 7104, 1800, 8), (220, 3328, 3880, 8),
    (223, 3248, 3976, 8), (129, 7296, 1800, 8), (181, 7008, 1888, 8), (1358, 1536, 11872, 8), (1650, 1712, 11536, 8),
]
# dense ones with 1, 16, 17, 32, 33 and 128 tiles of 256 x 256 behind a whole round, with whole K tiles and with a partial one
TAILS = {1: [(4813, 896, 6688), (2188, 352, 14584)], 16: [(4053, 384, 4344), (3993, 592, 4352)],
         17: [(5263, 512, 3176), (3076, 496, 5192)], 32: [(4038, 384, 4496), (1289, 416, 12224)],
         33: [(4306, 1280, 4128), (4149, 720, 4288)], 128: [(1872, 896, 12192), (3030, 576, 8184)]}
