"""Offsets of groups that make no sense (they descend, overlap, lie outside the rows), and sizes of eight groups whose products go to tiles, whole
columns and split ones, in each way that X enters.  test_mx_offsets.py follows every index that the kernels form of them, without a GPU."""

MOST, LEAST = 2 ** 31 - 1, -2 ** 31

# (type, quantize, n, m, rows)
SIZES = [("float32", False, 1000, 600, 4000), ("float32", False, 6600, 400, 1200), ("float32", True, 1000, 600, 4000), ("float32", True, 16000, 130, 1500),
         ("bfloat16", False, 1000, 600, 4000), ("bfloat16", False, 8000, 200, 1500), ("bfloat16", True, 1000, 600, 4000), ("bfloat16", True, 16000, 130, 1500)]
COUNT = 8


def offsets(B):
    return [[0, B, 0, B, 0, B, 0, B, 0], [B, B - 1, 900, 700, 501, 300, 100, 3, 0], [0, 500, 3, 400, 6, 7, 1100, 9, B], [-5, 2, B + 9, 40, 100000, 0, 17, 900, B],
            [MOST] * 9, [LEAST] * 9, [LEAST, MOST] * 4 + [LEAST], [0, 16, 0, 33, 1, B, B - 15, B, B], [0] * 8 + [MOST], [7, 6, 5, 4, 3, 2, 1, 0, LEAST]]
