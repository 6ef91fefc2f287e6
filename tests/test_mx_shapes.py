"""The sizes that the GPU tests of tiled 4-bit products use reach every form of their kernel that any call reaches: plans of a hundred thousand calls
over the whole range, without a GPU."""
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import hip_stub
import mx_shapes

# the kernels of a product, its workspace left out of account
PLAN = """
lib.hac_last_kernels.restype = C.c_char_p
at = lambda x: C.c_void_p(x << 40)
def plan(count, n, m, B, type, flags, X=2 << 40):
    d = hac.mx_describe(n, m, max(count, 1))
    need = lib.mx_workspace_bytes(C.byref(d), type, B, flags, int(count > 0))
    stub.stub_reset()
    X = C.c_void_p(X)
    if count: rc = lib.mx_grouped_dot(C.byref(d), at(1), type, X, B, n, at(3), at(4), m, flags, at(5), need, None)
    else: rc = lib.mx_dot(C.byref(d), at(1), type, X, B, n, at(4), m, flags, at(5), need, None)
    assert rc == 0, (count, n, m, B, type, flags, rc)
    names = lib.hac_last_kernels().decode().split("; ")
    tiles = [k[len("mx_tile_kernel<"):-1] for k in names if k.startswith("mx_tile_kernel")]
    return (tiles[0] if tiles else None), any(k.startswith("mx_sum_kernel") for k in names)
"""

# (rows of bfloat16 also from an odd entry on: those that were planned to be read where they lie are laid out)
LISTED = PLAN + """
sys.path.insert(0, TESTS)
import mx_shapes
seen = set()
for dtype, both, count, n, m, B in mx_shapes.TILES:
    for X in (2 << 40, (2 << 40) + 2) if dtype == "bfloat16" else (2 << 40,):
        kernel, split = plan(count, n, m, B, int(dtype == "bfloat16"), int(both), X)
        seen.add((kernel or "", count > 0, split))
print(json.dumps(sorted(seen)))
"""

DRAWN = PLAN + """
import math, random
rng = random.Random(7)
def li(a, b): return min(b, max(a, round(math.exp(rng.uniform(math.log(a), math.log(b))))))
seen = set()
for i in range(100000):
    count = 0 if i % 2 else li(2, 300)
    n, m, B = li(1, 30000), li(1, 30000), li(16, 1 << 20)
    if i % 3 == 0: n = (n + 7) // 8 * 8
    if max(count, 1) * n * m > 1 << 33: continue
    kernel, split = plan(count, n, m, B, i // 2 % 2, i // 4 % 2)
    if kernel: seen.add((kernel, count > 0, split))
print(json.dumps(sorted(seen)))
"""


def test_no_call_takes_a_kernel_that_no_listed_size_takes(tmp_path):
    listed = hip_stub.run(tmp_path, f"TESTS = {os.path.dirname(os.path.abspath(__file__))!r}\n" + LISTED)
    drawn = hip_stub.run(tmp_path, DRAWN)
    kernels = {k for k, *_ in listed}
    grouped = {k for k, in_groups, _ in listed if in_groups}
    kind = lambda k: k.rsplit(", ", 2)[0]                       # all but the tiles' numbers
    splits = {(kind(k), in_groups) for k, in_groups, split in listed if split}
    assert len({k for k, *_ in drawn}) >= 25
    for kernel, in_groups, split in drawn:
        assert kernel in kernels and (not in_groups or kernel in grouped), (kernel, in_groups)
        assert not split or (kind(kernel), in_groups) in splits, (kernel, in_groups)
