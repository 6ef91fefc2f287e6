"""Pins of the oracle of 4-bit microscaled matrices: blocks worked by hand, nearest by exhaustive search, the layout of a tile."""
import numpy as np
import pytest

from oracle import mx


def test_a_block_by_hand():
    # a = 10: floor(log2 10) = 3, scale 2^(3 - 2) = 2; in units of 2: 5 is halfway between 4 and 6 (codes 6, 7), even: 4
    w = np.zeros((32, 1))
    w[:9, 0] = [10.0, -10.0, 0.4, 0.5, 1.5, -2.5, 3.5, 7.0, -0.0]
    codes, exps, vals = mx.quantise(w)
    assert exps.tolist() == [[1]]
    # units: 5 -> 4; 0.2 -> 0; 0.25 halfway 0 / 0.5 -> 0; 0.75 halfway 0.5 / 1 -> 1; 1.25 halfway 1 / 1.5 -> 1;
    # 1.75 halfway 1.5 / 2 -> 2; 3.5 halfway 3 / 4 -> 4
    assert vals[:9, 0].tolist() == [8.0, -8.0, 0.0, 0.0, 2.0, -2.0, 4.0, 8.0, -0.0]
    assert codes[:9, 0].tolist() == [6, 14, 0, 0, 2, 10, 4, 6, 8]


def test_largest_entries_saturate_at_six():
    # a just below 8 units rounds down to 6
    w = np.full((32, 1), 7.99)
    assert mx.values(w)[0, 0] == 6.0
    w[0, 0] = 8.0                                             # the scale doubles: 4 units of 2
    assert mx.values(w)[0, 0] == 8.0 and mx.values(w)[1, 0] == 8.0


@pytest.mark.parametrize("n,m", [(1, 1), (31, 2), (32, 3), (33, 2), (100, 5)])
def test_both_forms_agree_and_are_nearest(n, m):
    rng = np.random.default_rng(n)
    w = (rng.standard_normal((n, m)) * 10.0 ** rng.integers(-6, 6, (1, m))).astype(np.float32)
    w[rng.random((n, m)) < 0.1] = 0
    for a, b in zip(mx.quantise(w), mx.quantise_slow(w)):
        assert np.array_equal(a, b)
    _, exps, vals = mx.quantise(w)
    scale = np.exp2(np.repeat(exps, 32, axis=0)[:n].astype(np.float64))
    near = np.abs(np.abs(w)[..., None] - mx.GRID * scale[..., None]).min(-1)
    assert np.array_equal(np.abs(w - vals), near)


def test_small_and_zero_blocks():
    w = np.zeros((64, 1))
    w[32, 0] = 2.0 ** -130
    codes, exps, vals = mx.quantise(w)
    assert exps.ravel().tolist() == [-127, -127]
    assert vals[32, 0] == 0.0                                 # an eighth of the scale
    w[32, 0] = 2.0 ** -127
    assert mx.values(w)[32, 0] == 2.0 ** -127


def test_layout_of_a_tile():
    w = np.zeros((130, 17))
    w[0, 0], w[33, 0], w[129, 16] = 4.0, 6.0, -1.0
    scales, codes = mx.sections(w)
    # two tiles of columns x (one group of scales, two steps)
    assert scales.size == 2 * 256 and codes.size == 4 * 1024
    assert scales[0] == 127 and scales[16 * 4] == 127         # floor(log2 4) - 2 = floor(log2 6) - 2 = 0
    assert codes[0] == 6 and codes[16 * 16] == 7 << 4         # row 0; row 33: second entry of the second block
    assert scales[256 + 1] == 125                             # column 16, step 1: floor(log2 1) - 2 = -2
    assert codes[3 * 1024] == (8 + 6) << 4                    # row 129: -4 times 2^-2
    assert np.count_nonzero(codes) == 3
