"""Products that go through tiles, for tests on the GPU, and what each of them reaches: test_product_choice.py holds the
choice of the library (256 compute units) against these tables."""
from collections import namedtuple

Shape = namedtuple("Shape", "sizes N row_bytes width height")        # rows of each group; the tiles that are chosen

# rows that are cut into tiles of every height, the lowest ones of groups with few rows and of a long group's end among them
_TALL = (256, 200, 180, 150, 100, 70, 64, 33, 20, 5, 0, 512, 700, 900, 110, 1800)
_LOW = (128, 100, 70, 64, 33, 20, 5, 0, 300, 130)

# a slab; two, the second one cut; more slabs than any ring of stages holds
ROW_BYTES = (128, 208, 1168)

# by is_gated; fp32 may have lower tiles where the matrix instructions, four times as long there, count
SHAPES = {
    False: [Shape(_TALL, 5003, b, 256, 256) for b in ROW_BYTES] + [Shape(_LOW, 2045, 128, 128, 128), Shape(_LOW, 2045, 208, 128, 128), Shape(_LOW, 2500, 1168, 128, 128)],
    True: [Shape(_TALL, 2045, b, 256, 256) for b in ROW_BYTES] + [Shape(_LOW, 1000, b, 128, 128) for b in ROW_BYTES],
}
FRONT, SPARE = 3, 7                                # places in front of the first group and behind the last

# calls whose offsets change between replays or are none: groups, places, columns, bytes of a row
CHANGING = (5, 2200, 1540, 528)
# rows far apart: rows of x, bytes from one to the next, places, columns; through a permutation, and in order
FAR_GATHERED = (4095, 1 << 20, 700, 2052)
FAR_IN_ORDER = (512, (1 << 24) - 16, 512, 32768)
FAR_BYTES = 256

_BYTES = {"i8": 1, "bf16": 2, "f32": 4}


def elements(fmt: str, row_bytes: int) -> int:
    return row_bytes // _BYTES[fmt]


def tiles_of(sizes, width: int, height: int):
    """(fragments of weights, of rows) a wave of every tile: groups of up to 64 rows have one of half the width, others equal
    tiles of as few as hold them, in whole fragments of 32 rows."""
    for rows in sizes:
        if 0 < rows <= 64:
            yield 4, 2 if rows > 32 else 1
        elif rows:
            n = -(-rows // height)
            h = -(-(-(-rows // n)) // 32) * 32
            for at in range(0, rows, h):
                r = min(h, rows - at)
                yield width // 32, (2 if r <= 64 else 4 if r <= 128 else -(-r // 32))
