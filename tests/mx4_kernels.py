"""Which code of gemm_mx4's kernels a product runs through, and products that run through all of it: those of tests.i8_kernels, whose
tiles lie in rows of as many bytes, and more where the choice of the tile differs."""
import paper_2405_13053_amd as m
from tests import i8_kernels

KT = 128   # bytes
# K tiles from which the unrolled loop of a tile shape is entered: a period of its two rings and the tiles that are on their way
UNROLLED_FROM = {(192, 128): 15, (224, 128): 8, (256, 128): 8, (256, 256): 8}


def code_of(T, half, d_out, counts=None):
    """The set of (kernel, rows, cols, per_cu, partial K tile, groups, unrolled, copy) that a call runs through, with rows of `half` bytes."""
    name, rows, cols, per_cu, read_once, tail = m.gemm_mx4_kernel(T, 2 * half, d_out, None if counts is None else len(counts))
    key = (name, rows, cols, per_cu, half % KT != 0, counts is not None, half // KT >= UNROLLED_FROM.get((rows, cols), 1 << 30))
    tiles = [-(-c // rows) for c in ([T] if counts is None else counts) if c > 0]
    if not tail:
        return {key + ("once" if read_once and t == 1 else "kept",) for t in tiles}
    total = sum(tiles) * -(-d_out // cols)
    rest = total % 256 if total > 256 and total % 256 <= 128 else 0
    codes = {key + ("kept",)} if total > rest else set()
    if rest:
        codes.add(key[:6] + (False, "tail 64x64" if rest <= 16 else "tail 128x64" if rest <= 32 else "tail 128x128"))
    return codes


# (T, half, d_out, N), small ones first
MORE = [
    (1444, 160, 2712, None), (2664, 160, 1488, 2), (1415, 256, 2728, None), (2913, 144, 1808, 2), (2940, 256, 1808, 2), (2850, 640, 2608, None),
    (2544, 1888, 1568, None), (2032, 1792, 2328, None), (2819, 1792, 1352, 2), (2640, 1824, 1584, 2), (5, 880, 14216, 8),
    (262, 3152, 10616, 3), (187, 3968, 12696, 2), (762, 1792, 12920, 5),
]
PRODUCTS = i8_kernels.PRODUCTS + [(*c, None) for cases in i8_kernels.TAILS.values() for c in cases] + MORE
