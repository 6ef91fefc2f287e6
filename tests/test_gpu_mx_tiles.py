"""4-bit products of sizes that go to tiles, in every form of that kernel: against the oracle's 4-bit values multiplied in 64 bits.

Tolerance, from the additions: a result is a chain of matrix instructions (32 products each, or 128 of 4-bit entries; fp32 rows of X take three
per 32) and at most 16 sums of parts of k.  Products are exact; each step rounds a partial sum, at most S = sum |x w|, by at most
2^-23 S.  So |Y - Yref| <= (steps + 64) 2^-23 S, and a bfloat16 result is rounded once more, by half of its eps: 2^-8 |Yref|."""
import numpy as np
import pytest

import mx_shapes
from oracle import mx

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
DEV = "cuda:0"


@pytest.fixture(scope="module")
def hac():
    import paper_2108_12704_amd as lib
    lib.load_library()
    assert torch.cuda.is_available(), "GPU tests need a device"
    return lib


def layer(n, m, seed=0, count=None):
    rng = np.random.default_rng(seed + 100 * n + m)
    shape = (n, m) if count is None else (count, n, m)
    w = rng.standard_normal(shape, np.float32) * np.float32(10.0) ** rng.integers(-2, 3, shape[:-2] + (1, m)).astype(np.float32)
    w[rng.random(shape, np.float32) < 0.05] = 0
    return w


def batch(B, n, dtype, seed=1):
    rng = np.random.default_rng(seed + B + n)
    x = rng.standard_normal((B, n), np.float32) * np.exp(rng.standard_normal(n, np.float32))
    return torch.from_numpy(x).to(dtype)                     # on the host


def place(X, left, ldx):
    """X in a matrix of rows of ldx entries, from entry `left` of a row on, NaN around it"""
    wide = torch.full((X.shape[0], ldx), float("nan"), dtype=X.dtype, device=DEV)
    at = wide[:, left:left + X.shape[1]]
    at.copy_(X)
    return at


def reference(X, v, both):
    """(Y, sum of the magnitudes) in 64 bits on the device; v: W's 4-bit values"""
    x = torch.from_numpy(mx.rows(X.double().numpy()) if both else X.double().numpy()).to(DEV)
    v = torch.from_numpy(v).to(DEV)
    return x @ v, x.abs() @ v.abs()


def check(Y, ref, size, n, both, what):
    steps = -(-n // 128) if both else -(-n // 32) * (3 if Y.dtype == F32 else 1)
    bound = (steps + 64) * 2.0 ** -23 * size
    if Y.dtype == BF16:
        bound = bound + 2.0 ** -8 * ref.abs() + 1e-40
    err = (Y.double() - ref).abs()
    assert bool((err <= bound).all()), (what, float((err - bound).max()), float(err.max()))


def tiled(hac):
    """the kernel on tiles that the last call launched, as its template arguments"""
    return [k[len("mx_tile_kernel<"):-1] for k in hac.hac_last_kernels() if k.startswith("mx_tile_kernel<")]


def whole(n, dtype, both):
    return dtype == BF16 and not both and n % 8 == 0


# ---- every form ------------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype,both,n,m,B", [(d, q, n, m, B) for d, q, count, n, m, B in mx_shapes.TILES if not count])
def test_products_on_tiles(hac, dtype, both, n, m, B):
    """... of rows that lie apart, NaN between them, at 16 bytes and at an odd entry; what lies around Y stays."""
    dtype = getattr(torch, dtype)
    print(f"[case] tiles {n} x {m} B={B} {dtype} both={both}", flush=True)
    w, X = layer(n, m), batch(B, n, dtype)
    db = hac.mx_encode_dev(torch.from_numpy(w).to(DEV))
    ref, size = reference(X, mx.values(w), both)
    Y = hac.mx_dot(db, place(X, 8, (n + 23) // 8 * 8), quantize=both)
    check(Y, ref, size, n, both, "aligned")
    if whole(n, dtype, both):
        assert all(", true," in k for k in tiled(hac)), tiled(hac)
    y = torch.full((B + 2, m + 3), 9.0, dtype=dtype, device=DEV)
    for ldx in (n + 1, n + 2):
        y[1:-1, 2:2 + m].fill_(float("nan"))
        hac.mx_dot(db, place(X, 1, ldx), Y=y[1:-1, 2:2 + m], quantize=both)
        assert all(", false," in k for k in tiled(hac)) and torch.equal(y[1:-1, 2:2 + m], Y), ldx
        assert bool((y[0] == 9).all()) and bool((y[-1] == 9).all()) and bool((y[:, :2] == 9).all()) and bool((y[:, 2 + m:] == 9).all())


@pytest.mark.parametrize("dtype,both,count,n,m,B", [c for c in mx_shapes.TILES if c[2]])
def test_groups_on_tiles(hac, dtype, both, count, n, m, B):
    """... ragged, with empty groups, with all rows in one, rows before the first and behind the last."""
    dtype = getattr(torch, dtype)
    w, X = layer(n, m, count=count), batch(B, n, dtype)
    db = hac.mx_encode_dev(torch.from_numpy(w).to(DEV))
    xd = place(X, 8, (n + 23) // 8 * 8)
    rng = np.random.default_rng(B)
    p = rng.random(count) ** 2 + 0.01
    if count > 2:
        p[count // 2] = 0
    ragged = rng.multinomial(B - 40, p / p.sum())
    ragged[0] += 17 - ragged[0] % 16 if ragged[0] % 16 > 1 else 0       # a last tile of one row
    ragged[-1] = B - 40 - ragged[:-1].sum()
    last = np.zeros(count, np.int64)
    last[-1] = B
    v, xs = [mx.values(e) for e in w], [(23, ragged), (0, last)]
    for before, sizes in xs:
        print(f"[case] tiles {count} x {n} x {m} B={B} {dtype} both={both} {list(sizes)}", flush=True)
        assert (sizes >= 0).all()
        off = np.cumsum([before] + list(sizes)).astype(np.int32)
        offd = torch.from_numpy(off).to(DEV)
        Y = torch.full((B, m + 1), 5.0, dtype=dtype, device=DEV)
        hac.mx_grouped_dot(db, xd, offd, Y=Y[:, :m], quantize=both)
        if whole(n, dtype, both):
            assert all(", true," in k for k in tiled(hac)), tiled(hac)
        for e in range(count):
            at = slice(off[e], off[e + 1])
            if sizes[e]:
                ref, size = reference(X[at], v[e], both)
                check(Y[at, :m], ref, size, n, both, (before, e))
        assert bool((Y[:before] == 5).all()) and bool((Y[off[-1]:] == 5).all()) and bool((Y[:, m] == 5).all())
        again = torch.full((B, m), 5.0, dtype=dtype, device=DEV)
        hac.mx_grouped_dot(db, place(X, 1, n + 2), offd, Y=again, quantize=both)
        assert torch.equal(again, Y[:, :m])


# ---- values that are not numbers -------------------------------------------------------------------------

# one size for each way that X enters, whole columns and split ones; n is no multiple of 128
SPECIAL = [(F32, False, 1080, 644, 2262), (F32, False, 9066, 598, 311), (F32, True, 400, 644, 2221), (F32, True, 5759, 194, 339),
           (BF16, False, 392, 354, 2170), (BF16, False, 7784, 99, 363), (BF16, False, 515, 788, 4323), (BF16, False, 8987, 344, 435),
           (BF16, True, 323, 645, 2517), (BF16, True, 10779, 599, 136)]


@pytest.mark.parametrize("dtype,both,n,m,B", SPECIAL)
def test_nan_and_infinity_on_tiles(hac, dtype, both, n, m, B):
    """In X they reach their rows only, a block of NaN in W its column only; all other results are what they are without."""
    w, X = layer(n, m), batch(B, n, dtype)
    print(f"[case] NaN on tiles {n} x {m} B={B} {dtype} both={both}", flush=True)
    wd = torch.from_numpy(w).to(DEV)
    db = hac.mx_encode_dev(wd)
    clean = hac.mx_dot(db, X.to(DEV), quantize=both)
    assert tiled(hac)
    v = mx.values(w)
    bad = X.clone()
    nan_rows, inf_rows = (0, B - 1), ((5, n - 1, 1.0), (17, 3, -1.0), (B // 2, n // 2, 1.0))
    bad[0, n - 1] = bad[B - 1, 0] = float("nan")
    for r, i, sign in inf_rows:
        bad[r, i] = sign * float("inf")
    Y = hac.mx_dot(db, bad.to(DEV), quantize=both)
    for r in nan_rows:
        assert torch.isnan(Y[r]).all()
    for r, i, sign in inf_rows:
        with np.errstate(invalid="ignore"):
            want = torch.from_numpy(sign * np.inf * v[i]).to(DEV)
        if both:
            want = torch.full_like(want, float("nan"))
        assert torch.equal(torch.isnan(Y[r]), torch.isnan(want)) and torch.equal(Y[r][~torch.isnan(want)].double(), want[~torch.isnan(want)])
    rest = torch.ones(B, dtype=torch.bool, device=DEV)
    rest[list(nan_rows) + [r for r, *_ in inf_rows]] = False
    assert torch.equal(Y[rest], clean[rest])
    wd[n - 1, 2], wd[40, m - 1], wd[0, m // 2] = float("nan"), float("inf"), -float("inf")
    Y = hac.mx_dot(hac.mx_encode_dev(wd), X.to(DEV), quantize=both)
    rest = torch.ones(m, dtype=torch.bool, device=DEV)
    rest[[2, m - 1, m // 2]] = False
    assert torch.isnan(Y[:, ~rest]).all() and torch.equal(Y[:, rest], clean[:, rest])


# ---- past 32 bits ----------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype,both,n,m,B", [(BF16, False, 512, 8192, 300000), (BF16, True, 512, 8192, 300000), (F32, False, 512, 8192, 150000),
                                              (BF16, False, 4096, 72, 530000), (BF16, True, 4096, 72, 530000)])
def test_rows_and_results_past_32_bits(hac, dtype, both, n, m, B):
    """4.3 to 4.9 GB of X or of results: the last rows, and the same rows further up give the same."""
    w = layer(n, m)
    few = batch(1000, n, dtype)
    X = few.to(DEV).repeat(B // 1000, 1)
    db = hac.mx_encode_dev(torch.from_numpy(w).to(DEV))
    print(f"[case] {B} rows, {n} x {m} {dtype} both={both}", flush=True)
    Y = hac.mx_dot(db, X, quantize=both)
    assert tiled(hac)
    ref, size = reference(few, mx.values(w), both)
    for at in (0, B // 2000 * 1000, B - 1000):
        check(Y[at:at + 1000], ref, size, n, both, at)
    assert torch.equal(Y[B - 1000:], Y[:1000])
    if dtype == BF16 and not both and m == 72:               # ... laid out in a workspace of as much
        assert all(", true," in k for k in tiled(hac))
        X = torch.empty((B, n + 1), dtype=dtype, device=DEV)[:, 1:].copy_(X)
        again = hac.mx_dot(db, X)
        assert all(", false," in k for k in tiled(hac)) and torch.equal(again, Y)


@pytest.mark.parametrize("both", [False, True])
def test_a_blob_past_32_bits_on_tiles(hac, both):
    """520 matrices of 4096 x 4096, 4.6 GB of codes: the first and the last multiplied."""
    count, n, rows = 520, 4096, 3000
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    W = torch.zeros((count, n, n), dtype=BF16, device=DEV)
    W[0].normal_(generator=g)
    W[-1].normal_(generator=g)
    print(f"[case] 520 matrices of 4096 x 4096 both={both}", flush=True)
    db = hac.mx_encode_dev(W)
    v = [mx.values(W[e].float().cpu().numpy()) for e in (0, -1)]
    del W
    X = batch(2 * rows, n, BF16)
    off = torch.full((count + 1,), rows, dtype=torch.int32, device=DEV)
    off[0], off[-1] = 0, 2 * rows
    Y = hac.mx_grouped_dot(db, X.to(DEV), off, quantize=both)
    assert tiled(hac)
    for e, at in enumerate((slice(0, rows), slice(rows, 2 * rows))):
        ref, size = reference(X[at], v[e], both)
        check(Y[at], ref, size, n, both, e)


# ---- captured --------------------------------------------------------------------------------------------


@pytest.mark.parametrize("both", [False, True])
def test_groups_on_tiles_captured_and_replayed(hac, both):
    """One graph over a split and a whole product by groups, whose rows and offsets change from replay to replay."""
    sizes = ((2, 8704, 140, 2383), (2, 400, 452, 1733)) if both is False else ((2, 8645, 132, 371), (2, 643, 322, 2752))
    calls = []
    for count, n, m, B in sizes:
        db = hac.mx_encode_dev(torch.from_numpy(layer(n, m, count=count)).to(DEV))
        calls.append((db, torch.zeros((B, n), dtype=BF16, device=DEV), torch.zeros(count + 1, dtype=torch.int32, device=DEV), torch.zeros((B, m), dtype=BF16, device=DEV)))

    def fill(seed):
        for db, x, off, y in calls:
            x.copy_(batch(x.shape[0], x.shape[1], BF16, seed))
            part = np.random.default_rng(seed).multinomial(x.shape[0] - seed, np.full(db.count, 1 / db.count))
            off.copy_(torch.from_numpy(np.cumsum([seed] + list(part)).astype(np.int32)))
            y.fill_(seed)

    def run():
        for db, x, off, y in calls:
            hac.mx_grouped_dot(db, x, off, Y=y, quantize=both)
    print(f"[case] graph of groups on tiles both={both}", flush=True)
    fill(1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for seed in (2, 3, 4, 5):
        fill(seed)
        graph.replay()
        torch.cuda.synchronize()
        got = [y.clone() for *_, y in calls]
        fill(seed)
        run()
        torch.cuda.synchronize()
        for (db, x, off, y), replayed in zip(calls, got):
            assert torch.equal(replayed, y) and bool((y[:seed] == seed).all())
