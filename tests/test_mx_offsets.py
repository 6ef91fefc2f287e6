"""Products by groups whose offsets make no sense, on the host: the tiles and rows that the kernels find in them, with the arithmetic of 32 bits that they
use, stay inside X, Y and the workspace."""
import os
import sys

import pytest

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import hip_stub
import mx_offsets

U32 = 0xffffffff


def find_item(offsets, B, R, item):
    """(group, first row, rows, tiles before) of stretch `item` of R rows, as a wavefront finds it: 64 groups at a time, 32 bits"""
    count = len(offsets) - 1
    items = tiles = 0
    for base in range(0, count, 64):
        upto = upto16 = 0
        for e in range(base, min(base + 64, count)):
            a, b = (min(max(o, 0), B) for o in offsets[e:e + 2])
            rows = max(b - a, 0)
            mine, mine16 = (rows + R - 1) // R, (rows + 15) // 16
            upto, upto16 = upto + mine & U32, upto16 + mine16 & U32
            if items + upto & U32 > item:
                within = item - (items + upto - mine) & U32
                return e, a + within * R & U32, min(R, rows - within * R & U32), tiles + upto16 - mine16 + within * (R // 16) & U32
        items, tiles = items + upto & U32, tiles + upto16 & U32
    return 0, 0, 0, 0


# the arguments of a launch: where the tile kernel finds the number of tiles laid out, the rows of a stretch and the stretches
PLANS = """
sys.path.insert(0, TESTS)
import mx_offsets
at = lambda x: C.c_void_p(x << 40)
out = []
for dtype, both, n, m, B in mx_offsets.SIZES:
    d = hac.mx_describe(n, m, mx_offsets.COUNT)
    type = int(dtype == "bfloat16")
    need = lib.mx_workspace_bytes(C.byref(d), type, B, int(both), 1)
    for X in (2 << 40, (2 << 40) + 4):
        def call(launch, arg):
            stub.stub_reset()
            if launch >= 0: stub.stub_copy_arg(launch, arg, 4)
            assert lib.mx_grouped_dot(C.byref(d), at(1), type, C.c_void_p(X), B, n, at(3), at(4), m, int(both), at(5), need, None) == 0
            return events()[launch][3] if launch >= 0 else [k.split("<")[0] for k in lib.hac_last_kernels().decode().split("; ")]
        lib.hac_last_kernels.restype = C.c_char_p
        names = call(-1, 0)
        tile = names.index("mx_tile_kernel")
        out.append([B, names, call(tile, 4), call(tile, 9), call(tile, 10)])
print(json.dumps(out))
"""


def test_tiles_and_rows_of_offsets_that_make_no_sense(tmp_path):
    plans = hip_stub.run(tmp_path, f"TESTS = {os.path.dirname(os.path.abspath(__file__))!r}\n" + PLANS)
    laid_out = [p for p in plans if "mx_lay_out_kernel" in p[1]]
    assert laid_out and any("mx_sum_kernel" in p[1] for p in laid_out) and len(laid_out) < len(plans)
    left_out = 0
    for B, names, tiles, R, stretches in plans:
        assert R % 16 == 0 and stretches * R >= B and tiles * 16 >= B
        for offsets in mx_offsets.offsets(B):
            for item in range(tiles):                            # laid out: a tile of the workspace each
                e, row0, rows, tile = find_item(offsets, B, 16, item)
                assert rows <= 16 and row0 + rows <= B and (not rows or tile == item), (offsets, item)
            for item in range(stretches):
                e, row0, rows, tile = find_item(offsets, B, R, item)
                assert e < mx_offsets.COUNT and rows <= R and row0 + rows <= B, (offsets, item)
                if "mx_lay_out_kernel" in names and tile + (rows + 15) // 16 > tiles:
                    left_out += 1                                # (not read: the kernel leaves such a stretch)
    assert left_out                                              # groups that overlap claim more tiles than there are


@pytest.mark.parametrize("count", [1, 63, 64, 65, 200])
def test_stretches_of_groups_that_do_make_sense(count):
    """The same arithmetic on ascending offsets: every row of a group is in one stretch, tiles are numbered without a gap."""
    import numpy as np
    rng = np.random.default_rng(count)
    sizes = rng.multinomial(1500, rng.dirichlet(np.full(count, 0.3)))
    B = int(sizes.sum()) + 20
    offsets = [int(v) for v in np.cumsum([9] + list(sizes))]
    for R in (16, 32, 64, 128):
        item = seen = tiles = 0
        while True:
            e, row0, rows, tile = find_item(offsets, B, R, item)
            if not rows:
                break
            assert offsets[e] <= row0 and row0 + rows <= offsets[e + 1] and tile == tiles
            seen, tiles, item = seen + rows, tiles + (rows + 15) // 16, item + 1
        assert seen == sizes.sum() and item <= (B + (R - 1) * count) // R
