"""4-bit microscaled layers on the GPU: the encoder byte for byte against the host's, values and products against the oracle in 64 bits.

Tolerance of a product, from its additions: a result is a chain of matrix instructions (32 products each, or 128 of 4-bit entries; fp32 rows of X
take three per 32), then at most 64 sums of wavefronts or K splits.  Products are exact; each step rounds a partial sum, which is at
most S = sum |x w|, by at most 2^-23 S.  So |Y - Yref| <= (steps + 64) 2^-23 S, and a bfloat16 result is rounded once more, by half of its
eps: 2^-8 |Yref|."""
import numpy as np
import pytest

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
    w = (rng.standard_normal(shape) * 10.0 ** rng.integers(-2, 3, shape[:-2] + (1, m))).astype(np.float32)
    w[rng.random(shape) < 0.05] = 0
    return w


def batch(B, n, dtype, seed=1):
    rng = np.random.default_rng(seed + B + n)
    x = (rng.standard_normal((B, n)) * np.exp(rng.standard_normal(n))).astype(np.float32)
    return torch.from_numpy(x).to(dtype)                     # on the host


def check(Y, X, w, both, what):
    """Y (device) against X (host) times the rounded w."""
    x = X.double().numpy()
    ref, size = mx.product(x, w, both)
    steps = -(-x.shape[1] // 128) if both else -(-x.shape[1] // 32) * (3 if X.dtype == F32 else 1)
    bound = (steps + 64) * 2.0 ** -23 * size
    if Y.dtype == BF16:
        bound = bound + 2.0 ** -8 * np.abs(ref) + 1e-40
    err = np.abs(Y.double().cpu().numpy() - ref)
    assert Y.dtype == X.dtype and not (err > bound).any(), (what, float((err - bound).max()), float(err.max()))


# ---- quantisation ------------------------------------------------------------------------------------


@pytest.mark.parametrize("n,m", [(1, 1), (31, 3), (32, 16), (33, 17), (127, 64), (128, 65), (500, 300), (513, 16), (640, 70), (2100, 130)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_encoder_writes_the_host_encoders_bytes(hac, n, m, dtype):
    print(f"[case] mx_encode_dev {n} x {m} {dtype}", flush=True)
    w = torch.from_numpy(layer(n, m)).to(dtype)
    want = hac.mx_encode(w.float().numpy())
    db = hac.mx_encode_dev(w.to(DEV))
    assert bytes(db.desc) == bytes(want.desc) and db.n == n and db.m == m and db.count == 1
    assert np.array_equal(db.tensor.cpu().numpy(), want.data)
    # rows that are part of a wider matrix, from an odd column on
    wide = torch.full((n, m + 5), 7.0, dtype=dtype, device=DEV)
    wide[:, 3:3 + m] = w.to(DEV)
    assert torch.equal(hac.mx_encode_dev(wide[:, 3:3 + m]).tensor, db.tensor)
    for out in (F32, BF16):
        got = hac.mx_decode_dev(db, dtype=out)
        assert got.dtype == out and np.array_equal(got.double().cpu().numpy(), mx.values(w.float().numpy()))
    # into the middle of a wider matrix, whose other entries stay
    wide.fill_(7.0)
    assert hac.mx_decode_dev(db, W=wide[:, 3:3 + m]) is not None
    assert torch.equal(wide[:, 3:3 + m].double().cpu(), torch.from_numpy(mx.values(w.float().numpy())))
    assert bool((wide[:, :3] == 7.0).all()) and bool((wide[:, 3 + m:] == 7.0).all())


def test_borders_and_ends_of_the_range(hac):
    units = np.concatenate([np.arange(0, 64) / 8.0, [7.9999995, 5.0000005, 0.24999999]])
    rng = np.random.default_rng(5)
    w = np.zeros((96, 40), np.float32)
    for j in range(40):
        scale = 2.0 ** [-149, -140, -133, -127, -126, -125, -100, -20, 0, 1, 20, 100, 120, 125][j % 14]
        w[:, j] = (rng.choice(units, 96) * np.where(rng.random(96) < 0.5, -1, 1) * scale).astype(np.float32)
    w[40, 3] = -0.0
    db = hac.mx_encode_dev(torch.from_numpy(w).to(DEV))
    assert np.array_equal(db.tensor.cpu().numpy(), hac.mx_encode(w).data)
    for out in (F32, BF16):
        assert np.array_equal(hac.mx_decode_dev(db, dtype=out).double().cpu().numpy(), mx.values(w))


def test_experts_of_a_layer(hac):
    w = torch.from_numpy(layer(200, 40, count=5))
    room = torch.zeros((5, 260, 48), device=DEV)
    room[:, 30:230, :40] = w.to(DEV)
    db = hac.mx_encode_dev(room[:, 30:230, :40])
    assert db.count == 5 and np.array_equal(db.tensor.cpu().numpy(), hac.mx_encode(w.numpy()).data)
    got = hac.mx_decode_dev(db)
    assert got.shape == (5, 200, 40) and np.array_equal(got.double().cpu().numpy(), mx.values(w.numpy()))
    room.zero_()
    hac.mx_decode_dev(db, W=room[:, 30:230, :40])
    assert torch.equal(room[:, 30:230, :40], got) and float(room.abs().sum()) == float(got.abs().sum())


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_blocks_with_a_nan_or_infinity(hac, dtype):
    w = torch.from_numpy(layer(100, 20)).to(dtype)
    w[5, 3], w[40, 4], w[99, 5] = float("nan"), float("inf"), -float("inf")
    db = hac.mx_encode_dev(w.to(DEV))
    got = hac.mx_decode_dev(db).cpu().numpy()
    assert hac.Blob(db.tensor.cpu().numpy()).validate() == 0
    bad = np.zeros((100, 20), bool)
    bad[:32, 3], bad[32:64, 4], bad[96:, 5] = True, True, True
    clean = w.float().numpy().copy()
    clean[bad] = 0
    assert np.array_equal(np.isnan(got), bad) and np.array_equal(got[~bad], mx.values(clean)[~bad].astype(np.float32))
    for B in (3, 100):                                        # ... make their columns NaN, no others
        for both in (False, True):
            print(f"[case] NaN blocks {dtype} B={B} both={both}", flush=True)
            Y = hac.mx_dot(db, batch(B, 100, dtype).to(DEV), quantize=both)
            assert torch.isnan(Y).cpu().numpy().tolist() == [[j in (3, 4, 5) for j in range(20)]] * B


# ---- product -----------------------------------------------------------------------------------------

SIZES = [(1, 1), (32, 16), (33, 17), (127, 5), (128, 64), (500, 300), (513, 70), (1000, 130), (2100, 257)]


@pytest.mark.parametrize("n,m", SIZES)
@pytest.mark.parametrize("both", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_products(hac, n, m, both, dtype):
    w = layer(n, m)
    db = hac.mx_encode_dev(torch.from_numpy(w).to(DEV))
    for B in (1, 2, 8, 15, 16, 17, 31, 32, 33, 64, 65, 100, 128, 129, 300):
        print(f"[case] mx_dot {n} x {m} B={B} {dtype} both={both}", flush=True)
        X = batch(B, n, dtype)
        Y = hac.mx_dot(db, X.to(DEV), quantize=both)
        check(Y, X, w, both, (n, m, B))
        again = torch.full_like(Y, float("nan"))
        assert hac.mx_dot(db, X.to(DEV), Y=again, quantize=both) is again and torch.equal(again, Y)


@pytest.mark.parametrize("n,m,B", [(4096, 4096, 1), (25088, 512, 5), (9973, 1511, 137), (4608, 512, 784), (4096, 1000, 64), (300, 5000, 260)])
@pytest.mark.parametrize("both", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_larger_products(hac, n, m, B, both, dtype):
    print(f"[case] mx_dot {n} x {m} B={B} {dtype} both={both}", flush=True)
    w = layer(n, m)
    X = batch(B, n, dtype)
    check(hac.mx_dot(hac.mx_encode_dev(torch.from_numpy(w).to(DEV)), X.to(DEV), quantize=both), X, w, both, (n, m, B))


@pytest.mark.parametrize("B", [1, 7, 30, 50, 200])
@pytest.mark.parametrize("both", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_inside_wider_matrices(hac, B, both, dtype):
    """X and Y start at odd elements, with rows an odd number of elements apart; what lies around Y stays."""
    n, m = 301, 77
    w, X = layer(n, m), batch(B, n, dtype)
    db = hac.mx_encode(w).to_device(DEV)
    for left, more in ((0, 3), (1, 2), (3, 7), (4, 4), (8, 11)):
        print(f"[case] strides B={B} {dtype} both={both} left={left} more={more}", flush=True)
        x = torch.full((B, n + left + more), float("nan"), dtype=dtype, device=DEV)
        x[:, left:left + n] = X.to(DEV)
        y = torch.full((B + 1, m + left + more), 9.0, dtype=dtype, device=DEV)
        hac.mx_dot(db, x[:, left:left + n], Y=y[:B, left:left + m], quantize=both)
        check(y[:B, left:left + m], X, w, both, (left, more))
        assert bool((y[:, :left] == 9).all()) and bool((y[:, left + m:] == 9).all()) and bool((y[B] == 9).all())
    turned = X.t().contiguous().t()                           # rows of X not contiguous
    check(hac.mx_dot(db, turned.to(DEV), quantize=both), X, w, both, "turned")


@pytest.mark.parametrize("B", [5, 60])
def test_fp32_rows_enter_whole(hac, B):
    """Entries of X with all 24 bits, of very different sizes: one non-zero of W per column picks them out exactly."""
    n, m = 200, 200
    w = np.zeros((n, m), np.float32)
    w[np.arange(n), np.random.default_rng(0).permutation(m)] = 1.0
    rng = np.random.default_rng(B)
    x = (rng.integers(1 << 23, 1 << 24, (B, n)) * 2.0 ** rng.integers(-110, 100, (B, n))).astype(np.float32)
    x[0, :4] = [3.4028234663852886e38, -3.4028234663852886e38, 0.0, 1.0 + 2.0 ** -23]
    Y = hac.mx_dot(hac.mx_encode_dev(torch.from_numpy(w).to(DEV)), torch.from_numpy(x).to(DEV))
    assert np.array_equal(Y.cpu().numpy(), x @ w)


@pytest.mark.parametrize("B", [6, 100])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_nan_and_infinity_in_x(hac, B, dtype):
    n, m = 150, 40
    w = np.abs(layer(n, m)) + np.float32(0.01)
    X = batch(B, n, dtype).abs() + 0.01
    X[1, 7], X[2, 140], X[3, 0] = float("inf"), float("nan"), -float("inf")
    db = hac.mx_encode_dev(torch.from_numpy(w).to(DEV))
    Y = hac.mx_dot(db, X.to(DEV)).float().cpu().numpy()
    v = mx.values(w)
    for r, i in ((1, 7), (3, 0)):
        with np.errstate(invalid="ignore"):
            want = float(X[r, i]) * v[i]
        assert np.array_equal(np.isnan(Y[r]), np.isnan(want)) and np.array_equal(Y[r][~np.isnan(want)], want[~np.isnan(want)])
    assert np.isnan(Y[2]).all()
    Y = hac.mx_dot(db, X.to(DEV), quantize=True)
    assert torch.isnan(Y).all(1).cpu().tolist() == [r in (1, 2, 3) for r in range(B)] and not torch.isnan(Y[4:]).any()


def test_no_rows_and_no_workspace_of_ones_own(hac):
    db = hac.mx_encode(layer(300, 40)).to_device(DEV)
    assert hac.mx_dot(db, torch.zeros((0, 300), device=DEV)).shape == (0, 40)
    w = layer(2048, 2048)
    db, X = hac.mx_encode(w).to_device(DEV), batch(2000, 2048, F32)
    need = hac.mx_workspace_bytes(db.desc, 2000)
    assert need
    ws = torch.full((need + 256,), 0xff, dtype=torch.uint8, device=DEV)
    Y = hac.mx_dot(db, X.to(DEV), workspace=ws[:need])
    check(Y, X, w, False, "workspace")
    assert bool((ws[need:] == 0xff).all())
    with pytest.raises(hac.HacError) as e:
        hac.mx_dot(db, X.to(DEV), workspace=ws[:need - 1])
    assert e.value.status == -6
    with pytest.raises(hac.HacError) as e:
        hac.mx_dot(db, X.to(DEV), workspace=ws[16:])
    assert e.value.status == -1


def test_refusals(hac):
    db, many = hac.mx_encode(layer(300, 40)).to_device(DEV), hac.mx_encode(layer(300, 40, count=2)).to_device(DEV)
    x = torch.zeros((4, 300), device=DEV)
    off = torch.tensor([0, 2, 4], dtype=torch.int32, device=DEV)
    for bad in (x.double(), x.half(), x.cpu(), x[0], None):
        with pytest.raises(TypeError, match="X must be"):
            hac.mx_dot(db, bad)
    with pytest.raises(ValueError, match="wrong width"):
        hac.mx_dot(db, x[:, 1:])
    for bad in (torch.zeros((4, 40), device=DEV, dtype=BF16), torch.zeros((5, 40), device=DEV), torch.zeros((4, 40)),
                torch.zeros((40, 4), device=DEV).t()):
        with pytest.raises(TypeError, match="Y must be"):
            hac.mx_dot(db, x, Y=bad)
    with pytest.raises(hac.HacError):
        hac.mx_dot(many, x)                                   # experts need groups
    with pytest.raises(ValueError, match="must be an MX blob"):
        hac.mx_dot(hac.im_encode(layer(300, 40)).to_device(DEV), x)
    for bad in (off.long(), off[:2], off.cpu(), off.repeat(2)[::2], off.view(1, 3), [0, 2, 4]):
        with pytest.raises(TypeError, match="offsets must be"):
            hac.mx_grouped_dot(many, x, bad)
    with pytest.raises(hac.HacError) as e:
        hac.im_dot(db, x)
    assert e.value.status == -1
    for bad in (x[0], x.double(), x.t()):
        with pytest.raises(TypeError, match="W must be"):
            hac.mx_encode_dev(bad)
    with pytest.raises(hac.HacError):
        hac.mx_encode_dev(x[:1].expand(4, 300))               # rows that are all the same memory
    with pytest.raises(TypeError, match="dtype must be"):
        hac.mx_decode_dev(db, dtype=torch.float16)


# ---- groups ------------------------------------------------------------------------------------------


def grouped_check(hac, w, sizes, dtype, both, before=0, behind=0, what=""):
    count, n, m = w.shape
    T = before + sum(sizes) + behind
    print(f"[case] mx_grouped_dot {count} x {n} x {m} rows={T} {dtype} both={both} {what}", flush=True)
    db = hac.mx_encode(w).to_device(DEV)
    X = batch(T, n, dtype, seed=7)
    off = np.cumsum([before] + list(sizes)).astype(np.int32)
    Y = torch.full((T, m), 5.0, dtype=dtype, device=DEV)
    assert hac.mx_grouped_dot(db, X.to(DEV), torch.from_numpy(off).to(DEV), Y=Y, quantize=both) is Y
    for e in range(count):
        if sizes[e]:
            check(Y[off[e]:off[e + 1]], X[off[e]:off[e + 1]], w[e], both, (what, e))
    assert bool((Y[:before] == 5).all()) and bool((Y[T - behind:] == 5).all()), what
    return db, X, off, Y


@pytest.mark.parametrize("both", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_groups(hac, both, dtype):
    w = layer(257, 83, count=6)
    for sizes in ([1, 0, 0, 0, 0, 0], [0, 0, 0, 0, 0, 1], [0] * 6, [1, 2, 3, 0, 1, 1], [16, 17, 0, 15, 1, 33], [100, 0, 3, 0, 0, 260],
                  [0, 0, 700, 0, 0, 0], [64, 128, 129, 127, 65, 63], [40, 40, 40, 40, 40, 40]):
        for before, behind in ((0, 0), (3, 20)):
            if before + sum(sizes) + behind:
                grouped_check(hac, w, sizes, dtype, both, before, behind, sizes)


@pytest.mark.parametrize("count,rows", [(1, 5), (1, 90), (64, 64), (65, 40), (130, 700), (200, 9000)])
@pytest.mark.parametrize("both", [False, True])
def test_many_groups(hac, count, rows, both):
    rng = np.random.default_rng(count)
    p = np.exp(2 * rng.standard_normal(count)) * (rng.random(count) > 0.2)
    sizes = rng.multinomial(rows, p / p.sum() if p.any() else np.full(count, 1 / count))
    grouped_check(hac, layer(130, 36, count=count), [int(s) for s in sizes], BF16, both)


@pytest.mark.parametrize("count,n,m,rows", [(4, 2048, 300, 1000), (8, 4096, 64, 24)])
@pytest.mark.parametrize("both", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_larger_groups(hac, count, n, m, rows, both, dtype):
    sizes = np.random.default_rng(3).multinomial(rows, np.arange(1, count + 1) / (count * (count + 1) / 2))
    db, X, off, Y = grouped_check(hac, layer(n, m, count=count), [int(s) for s in sizes], dtype, both)
    # a group's rows are what the product with its own matrix makes of them, within both bounds
    one = hac.mx_dot(hac.mx_encode(layer(n, m, count=count)[-1]).to_device(DEV), X[off[-2]:off[-1]].to(DEV), quantize=both)
    check(one, X[off[-2]:off[-1]], layer(n, m, count=count)[-1], both, "alone")


def test_offsets_that_make_no_sense_stay_inside(hac):
    """Held to 0 .. B by the kernels; only what lies around X and Y is looked at."""
    w = layer(100, 20, count=4)
    db = hac.mx_encode(w).to_device(DEV)
    for B in (6, 200):
        for off in ([0, 500, 3, 4, 6], [-5, 2, 2, 9, 100000], [6, 5, 4, 2, 0], [2 ** 31 - 1] * 5, [-2 ** 31] * 5, [0, B, 0, B, B]):
            for both in (False, True):
                print(f"[case] offsets {off} B={B} both={both}", flush=True)
                y = torch.full((B + 2, 20), 3.0, device=DEV)
                hac.mx_grouped_dot(db, batch(B, 100, F32).to(DEV), torch.tensor(off, dtype=torch.int32, device=DEV), Y=y[1:-1], quantize=both)
                torch.cuda.synchronize()
                assert bool((y[0] == 3).all()) and bool((y[-1] == 3).all())


@pytest.mark.parametrize("m", [1496, 1500, 1501])
@pytest.mark.parametrize("both", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_of_results_that_are_padded(hac, m, both, dtype):
    """Rows of Y start at 16 bytes, their last entries do not fill them; what lies between two rows stays."""
    B, n = 1030, 1024
    w, X = layer(n, m), batch(B, n, dtype)
    y = torch.full((B, 1504), 5.0, dtype=dtype, device=DEV)
    print(f"[case] padded {dtype} m={m} both={both}", flush=True)
    hac.mx_dot(hac.mx_encode_dev(torch.from_numpy(w).to(DEV)), X.to(DEV), y[:, :m], quantize=both)
    assert dtype == F32 or "mx_tile_kernel" in str(hac.hac_last_kernels())        # (the kernel whose results leave eight at a time)
    check(y[:, :m], X, w, both, m)
    assert bool((y[:, m:] == 5).all())


@pytest.mark.parametrize("both", [False, True])
def test_a_million_rows(hac, both):
    """More than 65535 stretches of 16 rows; the same rows in smaller calls, within both bounds."""
    B, n, m = 65535 * 16 + 40, 40, 12
    w = layer(n, m)
    X = batch(1000, n, BF16).to(DEV).repeat(B // 1000 + 1, 1)[:B]
    db = hac.mx_encode_dev(torch.from_numpy(w).to(DEV))
    print(f"[case] {B} rows both={both}", flush=True)
    Y = hac.mx_dot(db, X, quantize=both)
    for at in (slice(0, 300), slice(B // 2, B // 2 + 300), slice(B - 300, B)):
        check(Y[at], X[at].cpu(), w, both, at)
    off = torch.tensor([0, B], dtype=torch.int32, device=DEV)
    assert torch.equal(hac.mx_grouped_dot(db, X, off, quantize=both), Y)


def test_results_past_32_bits(hac):
    """4.9 GB of results: the last rows are what the same rows give alone, within both bounds."""
    B, n, m = 300000, 32, 8192
    w = layer(n, m)
    X = batch(1000, n, BF16).to(DEV).repeat(B // 1000, 1)
    db = hac.mx_encode_dev(torch.from_numpy(w).to(DEV))
    print("[case] 300000 x 8192 results", flush=True)
    Y = hac.mx_dot(db, X)
    for at in (slice(0, 40), slice(B - 40, B)):
        check(Y[at], X[at].cpu(), w, False, at)
    assert torch.equal(Y[1000:1040], Y[B - 1000:B - 960])


@pytest.mark.parametrize("dtype,n", [(F32, 20001), (BF16, 40001)])
def test_a_matrix_larger_than_the_cache(hac, dtype, n):
    """Streamed past the last-level cache; its column halves, which are not, have the same bytes and values."""
    m = 4100
    g = torch.Generator(device=DEV)
    g.manual_seed(2)
    W = torch.randn((n, m), generator=g, device=DEV).to(dtype)
    print(f"[case] {n} x {m} {dtype}", flush=True)
    values = hac.mx_decode_dev(hac.mx_encode_dev(W), dtype)
    assert hac.hac_last_kernels()[0].endswith("true>")
    for part in (slice(0, 2048), slice(2048, m)):
        half = hac.mx_decode_dev(hac.mx_encode_dev(W[:, part]), dtype)
        assert hac.hac_last_kernels()[0].endswith("false>") and torch.equal(values[:, part], half)
    assert np.array_equal(values[:700, -5:].double().cpu().numpy()[:672], mx.values(W[:700, -5:].float().cpu().numpy())[:672])


def test_a_blob_past_32_bits(hac):
    """520 matrices of 4096 x 4096, 4.6 GB of codes: encoded, decoded and multiplied where offsets do not fit 32 bits."""
    count, n = 520, 4096
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    W = torch.empty((count, n, n), dtype=BF16, device=DEV)
    W[:2].normal_(generator=g)
    W[2:] = 0
    W[-1].normal_(generator=g)
    print("[case] 520 matrices of 4096 x 4096", flush=True)
    db = hac.mx_encode_dev(W)
    alone = [hac.mx_encode_dev(W[e]) for e in (0, count - 1)]
    back = hac.mx_decode_dev(db, BF16)
    for e, one in zip((0, count - 1), alone):
        assert torch.equal(back[e], hac.mx_decode_dev(one, BF16))
    assert not bool(back[2:-1].any())
    del back, W
    for rows in (5, 300):
        for both in (False, True):
            X = batch(2 * rows, n, BF16).to(DEV)
            off = torch.full((count + 1,), rows, dtype=torch.int32, device=DEV)
            off[0], off[-1] = 0, 2 * rows
            Y = hac.mx_grouped_dot(db, X, off, quantize=both)
            for e, one, at in zip((0, count - 1), alone, (slice(0, rows), slice(rows, 2 * rows))):
                check(Y[at], X[at].cpu(), hac.mx_decode_dev(one).cpu().numpy(), both, (e, rows))


# ---- as they are used ----------------------------------------------------------------------------------


@pytest.mark.parametrize("rows", [12, 600])
def test_a_layer_of_experts_captured_and_replayed(hac, rows):
    """Encode, two products per expert with an activation between them, in one graph whose inputs change from replay to replay."""
    count, n, hidden = 6, 192, 320
    up, down = layer(n, hidden, 1, count), layer(hidden, n, 2, count) * np.float32(0.01)
    a, b = hac.mx_encode_dev(torch.from_numpy(up).to(DEV)), hac.mx_encode_dev(torch.from_numpy(down).to(DEV))
    x = torch.zeros((rows, n), dtype=BF16, device=DEV)
    off = torch.zeros(count + 1, dtype=torch.int32, device=DEV)

    def run():
        h = hac.mx_grouped_dot(a, x, off)
        return h, hac.mx_grouped_dot(b, torch.relu(h), off, quantize=True)

    def fill(seed):
        x.copy_(batch(rows, n, BF16, seed))
        sizes = np.random.default_rng(seed).multinomial(rows, np.full(count, 1 / count))
        off.copy_(torch.from_numpy(np.cumsum([0] + list(sizes)).astype(np.int32)))
    fill(1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    print(f"[case] graph of a layer of experts, {rows} rows", flush=True)
    with torch.cuda.graph(graph):
        h, y = run()
    for seed in (1, 2, 3, 4):
        fill(seed)
        graph.replay()
        torch.cuda.synchronize()
        h0, y0 = run()
        assert torch.equal(h, h0) and torch.equal(y, y0), seed
        ends = off.cpu().tolist()
        for e in range(count):
            at = slice(ends[e], ends[e + 1])
            if ends[e + 1] > ends[e]:
                check(h[at], x[at].cpu(), up[e], False, (seed, e))
                check(y[at], torch.relu(h[at]).cpu(), down[e], True, (seed, e))


@pytest.mark.parametrize("B", [4, 90])
def test_a_stream_of_ones_own(hac, B):
    w, X = layer(700, 96), batch(B, 700, F32)
    xd, other = X.to(DEV), torch.cuda.Stream()
    torch.cuda.synchronize()
    print("[case] another stream", flush=True)
    torch.cuda._sleep(20_000_000)                             # the current stream is late
    db = hac.mx_encode_dev(torch.from_numpy(w).to(DEV, non_blocking=True), stream=None)
    other.wait_stream(torch.cuda.current_stream())
    y = hac.mx_dot(db, xd, stream=other)
    back = hac.mx_decode_dev(db, stream=other)
    other.synchronize()
    with torch.cuda.stream(other):
        check(y, X, w, False, "stream")
        assert np.array_equal(back.double().cpu().numpy(), mx.values(w))


@pytest.mark.parametrize("B", [3, 40, 200])
def test_a_chain_with_such_layers(hac, B):
    """hac_forward over MX, sHAC and MX layers is the calls one after the other; and near the chain in 64 bits."""
    w = [layer(300, 200, 1), np.where(np.abs(layer(200, 120, 2)) > 1.0, np.float32(0.5), np.float32(0.0)), layer(120, 37, 3)]
    blobs = [hac.mx_encode(w[0]).to_device(DEV), hac.shac_encode(w[1]).to_device(DEV), hac.mx_encode(w[2]).to_device(DEV)]
    bias = [torch.from_numpy(np.random.default_rng(i).standard_normal(m.shape[1]).astype(np.float32)) for i, m in enumerate(w)]
    relu, X = (True, False, True), batch(B, 300, F32)
    print(f"[case] chain B={B}", flush=True)
    Y = hac.hac_forward([(b, None if i == 1 else v.to(DEV), r) for i, (b, v, r) in enumerate(zip(blobs, bias, relu))], X.to(DEV))
    a = X.to(DEV)
    for i, (blob, call) in enumerate(zip(blobs, (hac.mx_dot, hac.shac_dot, hac.mx_dot))):
        a = call(blob, a)
        if i != 1:
            a = a + bias[i].to(DEV)
        a = torch.relu(a) if relu[i] else a
    assert torch.equal(Y, a)


def test_calls_from_two_threads(hac):
    import threading
    w = layer(900, 200)
    db = hac.mx_encode_dev(torch.from_numpy(w).to(DEV))
    xs = [batch(B, 900, BF16, B) for B in (9, 120)]
    want = [hac.mx_dot(db, x.to(DEV)) for x in xs]
    torch.cuda.synchronize()
    bad = []

    def work(i):
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            xd = xs[i].to(DEV)
            for _ in range(20):
                if not torch.equal(hac.mx_dot(db, xd), want[i]):
                    bad.append(i)
    print("[case] two threads", flush=True)
    threads = [threading.Thread(target=work, args=(i,)) for i in (0, 1)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not bad
