"""Products of 4-bit layers where values end: scales from the lowest to the highest, subnormal entries, borders between codes, blocks of zeros.

One side holds a single power of two in every column (row), so that a result is one entry of the other side times that power: no sum rounds but
among fp32's subnormal numbers, and the expected result is the oracle's value, rounded once where fp32 or bfloat16 does not hold it (below their least
numbers, above their largest)."""
import numpy as np
import pytest

from oracle import mx

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
DEV = "cuda:0"
# (type, quantize, n, m, rows): the kernel for few rows, and tiles in each way that X enters
SIZES = [(F32, False, 200, 90, 28), (F32, False, 1080, 644, 2262), (F32, True, 200, 90, 28), (F32, True, 400, 644, 2221), (BF16, False, 200, 90, 28),
         (BF16, False, 203, 90, 28), (BF16, False, 392, 354, 2170), (BF16, False, 515, 788, 4323), (BF16, True, 200, 90, 28), (BF16, True, 323, 645, 2517)]
SCALES = (-149, -140, -133, -130, -127, -126, -125, -100, -20, 0, 1, 20, 100, 120, 125)
POWERS = (100, 0, -100)


def values(shape, dtype, seed):
    """Rows of entries around the borders between codes, in units of a scale that goes with the row; one block in eight zero."""
    rng = np.random.default_rng(seed)
    at = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
    step = 2.0 ** (-7 if dtype == BF16 else -23)
    units = np.concatenate([np.arange(0, 64) / 8.0, at * (1 + step), at * (1 - step / 2), [7.9375, 7.9999995]])
    v = rng.choice(units, shape) * np.where(rng.random(shape) < 0.5, -1, 1)
    v[:, ::32] = np.where(rng.random(v[:, ::32].shape) < 0.5, 7.5, v[:, ::32])
    zero = np.repeat(rng.random((shape[0], -(-shape[1] // 32))) < 0.125, 32, axis=1)[:, :shape[1]]
    v = np.where(zero, 0, v) * 2.0 ** np.resize(SCALES, shape[0])[:, None]
    with np.errstate(under="ignore"):
        return torch.from_numpy(v.astype(np.float32)).to(dtype)


def once(ref, dtype):
    """ref (64 bits) rounded to fp32, and on to bfloat16 where that is the result's type"""
    with np.errstate(under="ignore", over="ignore"):
        return torch.from_numpy(ref.astype(np.float32)).to(dtype)


def same(Y, want, what, parts=1):
    """parts: that a result is the sum of.  Where results are subnormal each of the sums rounds to a multiple of 2^-149, by at most half of it, and so does
    the expected result: 1.5 of them + 0.5 for three parts."""
    got = Y.cpu()
    bad = (got != want) & ~(torch.isnan(got) & torch.isnan(want))
    if parts > 1:
        bad &= (want.abs() >= 2.0 ** -126) | ((got.double() - want.double()).abs() > (parts + 1) / 2 * 2.0 ** -149)
    if not bad.any():
        return
    bad = bad.nonzero()
    r, j = bad[0].tolist()
    assert False, (what, len(bad), (r, j), float(got[r, j]).hex(), float(want[r, j]).hex())


def picking(n, m, p):
    """a matrix whose column j holds 2^p in row j % n and else zeros"""
    w = np.zeros((n, m), np.float32)
    w[np.arange(m) % n, np.arange(m)] = 2.0 ** p
    return w


@pytest.mark.parametrize("dtype,both,n,m,B", SIZES)
def test_entries_of_x(dtype, both, n, m, B):
    """quantize: the codes and scales that rows of X get.  Otherwise their bits: all of them, in fp32 but for those below 2^-133."""
    import paper_2108_12704_amd as hac
    rng = np.random.default_rng(n + B)
    if both:
        X = values((B, n), dtype, 3)
        finite = torch.isfinite(X)                               # (7.9999995 times 2^125 is an infinity in bfloat16: its row is NaN)
        x = np.where(finite.all(1, keepdim=True).numpy(), mx.rows(torch.where(finite, X, 0).double().numpy()), np.nan)
    else:
        v = rng.integers(1 << 23, 1 << 24, (B, n)) * np.where(rng.random((B, n)) < 0.5, -1, 1) * 2.0 ** rng.integers(-172, 104, (B, n))
        with np.errstate(under="ignore"):
            X = torch.from_numpy(v.astype(np.float32))
        if dtype == BF16:
            X = (X.view(torch.int32) & -65536).view(torch.float32).to(BF16)
        x = np.trunc(X.double().numpy() * 2.0 ** 133) * 2.0 ** -133
    for p in POWERS:
        print(f"[case] ends of X {dtype} both={both} {n} x {m} B={B} 2^{p}", flush=True)
        db = hac.mx_encode(picking(n, m, p)).to_device(DEV)
        same(hac.mx_dot(db, X.to(DEV), quantize=both), once(x[:, np.arange(m) % n] * 2.0 ** p, dtype), p, 3 if dtype == F32 and not both else 1)


@pytest.mark.parametrize("dtype,both,n,m,B", SIZES)
def test_entries_of_w(dtype, both, n, m, B):
    """What the products make of W's codes and scales."""
    import paper_2108_12704_amd as hac
    w = np.ascontiguousarray(values((m, n), F32, 4).numpy().T)
    db, v = hac.mx_encode(w).to_device(DEV), mx.values(w)
    pick = np.random.default_rng(B).integers(0, n, B)
    for p in POWERS:
        print(f"[case] ends of W {dtype} both={both} {n} x {m} B={B} 2^{p}", flush=True)
        X = torch.zeros((B, n), dtype=dtype)
        X[torch.arange(B), torch.from_numpy(pick)] = 2.0 ** p
        same(hac.mx_dot(db, X.to(DEV), quantize=both), once(v[pick] * 2.0 ** p, dtype), p)
