"""4-bit layers at sizes that no other test calls with: very short rows in very many, the most matrices a blob can have, large matrices whose rows
lie apart, chains of such layers in a graph."""
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
    return rng.standard_normal((n, m) if count is None else (count, n, m), np.float32)


def check(Y, X, v, both, what):
    """Y against X (both on the device) times the 4-bit values v; each of `steps` instructions and 64 sums rounds by at most 2^-23 of sum |x w|."""
    x = X.double()
    if both:
        x = torch.from_numpy(mx.rows(x.cpu().numpy())).to(DEV)
    w = torch.from_numpy(v).to(DEV)
    ref, size = x @ w, x.abs() @ w.abs()
    steps = -(-x.shape[1] // 128) if both else -(-x.shape[1] // 32) * (3 if X.dtype == F32 else 1)
    bound = (steps + 64) * 2.0 ** -23 * size + (2.0 ** -8 * ref.abs() + 1e-40 if Y.dtype == BF16 else 0)
    err = (Y.double() - ref).abs()
    assert bool((err <= bound).all()), (what, float((err - bound).max()))


@pytest.mark.parametrize("n,m", [(1, 1), (3, 5), (4, 2), (7, 3), (9, 1)])
@pytest.mark.parametrize("both", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_million_very_short_rows(hac, n, m, both, dtype):
    """More rows than the kernel for few rows takes, shorter than one load of 16 bytes or hardly longer."""
    B = 65535 * 16 + 21
    g = torch.Generator(device=DEV)
    g.manual_seed(n)
    w = layer(n, m)
    X = torch.randn((B, n), generator=g, device=DEV).to(dtype)
    db = hac.mx_encode(w).to_device(DEV)
    print(f"[case] {B} rows of {n}, {m} columns {dtype} both={both}", flush=True)
    Y = hac.mx_dot(db, X, quantize=both)
    check(Y, X, mx.values(w), both, (n, m))
    off = torch.tensor([5, B - 9], dtype=torch.int32, device=DEV)
    Z = torch.full((B, m), 2.0, dtype=dtype, device=DEV)
    hac.mx_grouped_dot(db, X, off, Y=Z, quantize=both)
    assert torch.equal(Z[5:B - 9], Y[5:B - 9]) and bool((Z[:5] == 2).all()) and bool((Z[B - 9:] == 2).all())


@pytest.mark.parametrize("rows", [70, 3000])
def test_the_most_experts(hac, rows):
    count, n, m = 65535, 33, 5
    w = layer(n, m, count=count)
    db = hac.mx_encode_dev(torch.from_numpy(w).to(DEV))
    assert db.count == count
    rng = np.random.default_rng(rows)
    of = np.sort(np.concatenate([rng.integers(0, count, rows - 4), [0, 0, count - 1, count - 1]]))     # a row's expert
    off = torch.from_numpy(np.searchsorted(of, np.arange(count + 1)).astype(np.int32)).to(DEV)
    X = torch.from_numpy(rng.standard_normal((rows, n), np.float32)).to(DEV)
    v = {e: mx.values(w[e]) for e in set(of)}
    for dtype in (F32, BF16):
        for both in (False, True):
            print(f"[case] {count} experts, {rows} rows {dtype} both={both}", flush=True)
            x = X.to(dtype)
            Y = hac.mx_grouped_dot(db, x, off, quantize=both)
            # every row with its own matrix, as one product of rows that are zero but for their expert's place
            xs = x.double() if not both else torch.from_numpy(mx.rows(x.double().cpu().numpy())).to(DEV)
            vs = torch.from_numpy(np.stack([v[e] for e in of])).to(DEV)
            ref, size = (xs[:, :, None] * vs).sum(1), (xs[:, :, None] * vs).abs().sum(1)
            bound = (6 + 64) * 2.0 ** -23 * size + (2.0 ** -8 * ref.abs() + 1e-40 if dtype == BF16 else 0)
            assert bool(((Y.double() - ref).abs() <= bound).all())


@pytest.mark.parametrize("dtype,n", [(F32, 18001), (BF16, 36001)])
def test_large_matrices_whose_rows_lie_apart(hac, dtype, n):
    """Streamed past the cache from and into a wider matrix, from an odd column on; what lies around stays."""
    m = 4001
    g = torch.Generator(device=DEV)
    g.manual_seed(6)
    room = torch.randn((n, m + 6), generator=g, device=DEV).to(dtype)
    print(f"[case] {n} x {m} {dtype} in {m + 6} columns", flush=True)
    W = room[:, 3:3 + m]
    db = hac.mx_encode_dev(W)
    assert hac.hac_last_kernels()[0].endswith("true>") and torch.equal(db.tensor, hac.mx_encode_dev(W.contiguous()).tensor)
    values = hac.mx_decode_dev(db, dtype)
    left, right = room[:, :3].clone(), room[:, 3 + m:].clone()
    hac.mx_decode_dev(db, W=W)
    assert torch.equal(W, values) and torch.equal(room[:, :3], left) and torch.equal(room[:, 3 + m:], right)


@pytest.mark.parametrize("B", [1, 19, 2300])
def test_a_chain_of_such_layers_captured_on_a_stream_of_its_own(hac, B):
    """hac_forward over MX layers only, the last without bias and activation, replayed on new inputs; each replay is the calls one after the other."""
    sizes = (400, 644, 130, 17)
    blobs = [hac.mx_encode(layer(n, m) * np.float32(0.05)).to_device(DEV) for n, m in zip(sizes, sizes[1:])]
    bias = [torch.randn(m, device=DEV) for m in sizes[1:]]
    layers = [(blobs[0], bias[0], True), (blobs[1], None, True), (blobs[2], None, False)]
    x, y = torch.zeros((B, sizes[0]), device=DEV), torch.zeros((B, sizes[-1]), device=DEV)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    print(f"[case] chain in a graph B={B}", flush=True)
    with torch.cuda.stream(stream):
        hac.hac_forward(layers, x, Y=y)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            hac.hac_forward(layers, x, Y=y)
        for seed in range(4):
            x.copy_(torch.from_numpy(np.random.default_rng(seed).standard_normal((B, sizes[0]), np.float32)))
            y.fill_(float("nan"))
            graph.replay()
            stream.synchronize()
            a = torch.relu(hac.mx_dot(blobs[0], x) + bias[0])
            a = torch.relu(hac.mx_dot(blobs[1], a))
            a = hac.mx_dot(blobs[2], a)
            stream.synchronize()
            assert torch.equal(y, a), seed
