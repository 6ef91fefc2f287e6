"""4-bit microscaled matrices, written from their definition in 64 bits.

Blocks of 32 consecutive rows of a column; with a the largest magnitude of a block its scale is 2^s, s = floor(log2 a) - 2,
not below -127; an entry is the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 times the scale with a sign, a tie going to the code that
is even (codes 0 .. 7 in this order, 8 added for a negative entry), everything larger to 6.
"""
from __future__ import annotations

import numpy as np

BLOCK = 32
GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def exponent(a):
    """s of a block whose largest magnitude is a."""
    if a == 0:
        return -127
    f, e = np.frexp(np.float64(a))                           # a = f 2^e, 0.5 <= f < 1
    return max(int(e) - 1 - 2, -127)


def code_of(u):
    """Code of a magnitude u given in units of the scale: by distance, ties to the even code."""
    d = np.abs(GRID - u)
    best = np.flatnonzero(d == d.min())
    return int(best[0] if best[0] % 2 == 0 else best[-1])


def quantise_slow(w):
    """(codes, scale exponents, values) of an n x m matrix, entry by entry."""
    n, m = w.shape
    nb = (n + BLOCK - 1) // BLOCK
    codes, exps, vals = np.zeros((n, m), np.int64), np.zeros((nb, m), np.int64), np.zeros((n, m))
    for j in range(m):
        for b in range(nb):
            block = w[b * BLOCK:(b + 1) * BLOCK, j].astype(np.float64)
            s = exponent(np.abs(block).max())
            exps[b, j] = s
            for i, v in enumerate(block):
                c = code_of(abs(v) * 2.0 ** -s)
                codes[b * BLOCK + i, j] = c + (8 if np.signbit(v) else 0)
                vals[b * BLOCK + i, j] = (-1 if np.signbit(v) else 1) * GRID[c] * 2.0 ** s
    return codes, exps, vals


def quantise(w):
    """The same, whole arrays at a time."""
    n, m = w.shape
    nb = (n + BLOCK - 1) // BLOCK
    full = np.zeros((nb * BLOCK, m))
    full[:n] = w
    blocks = full.reshape(nb, BLOCK, m)
    a = np.abs(blocks).max(axis=1)
    _, e = np.frexp(a)
    exps = np.where(a == 0, -127, np.maximum(e.astype(np.int64) - 3, -127))
    u = np.abs(blocks) * np.exp2(-exps.astype(np.float64))[:, None, :]
    border = (GRID[1:] + GRID[:-1]) / 2
    c = np.zeros(blocks.shape, np.int64)
    for i, x in enumerate(border):                           # borders between codes i and i + 1
        c += (u > x) if i % 2 == 0 else (u >= x)
    sign = np.signbit(blocks)
    vals = np.where(sign, -1.0, 1.0) * GRID[c] * np.exp2(exps.astype(np.float64))[:, None, :]
    codes = c + 8 * sign
    return codes.reshape(-1, m)[:n], exps, vals.reshape(-1, m)[:n]


def values(w):
    """w as its 4-bit entries stand for it (any leading axes)."""
    w = np.asarray(w)
    if w.ndim == 2:
        return quantise(w)[2]
    return np.stack([values(e) for e in w])


def rows(x):
    """x with its rows rounded, blocks along a row."""
    return quantise(np.asarray(x).T)[2].T


def sections(w):
    """The two sections of a blob of one matrix, (scales, codes) as bytes, laid out entry by entry from the format's text."""
    n, m = w.shape
    codes, exps, _ = quantise(w)
    steps = (n + 127) // 128
    groups, tiles = (steps + 3) // 4, (m + 15) // 16
    out_codes = np.zeros(tiles * steps * 1024, np.uint8)
    out_scales = np.zeros(tiles * groups * 256, np.uint8)
    for j in range(m):
        for b in range(exps.shape[0]):
            t, c, s, g = j // 16, j % 16, b // 4, b % 4
            out_scales[(t * groups + s // 4) * 256 + (16 * g + c) * 4 + s % 4] = exps[b, j] + 127
            at = ((t * steps + s) * 64 + 16 * g + c) * 16
            for i, q in enumerate(codes[b * BLOCK:(b + 1) * BLOCK, j]):
                out_codes[at + i // 2] |= int(q) << (4 * (i % 2))
    return out_scales, out_codes


def product(x, w, both=False):
    """(Y, sum of the magnitudes) of X . W, W's entries in 4 bits, X's too where `both`."""
    x = rows(x) if both else np.asarray(x, np.float64)
    v = values(w)
    return x @ v, np.abs(x) @ np.abs(v)
