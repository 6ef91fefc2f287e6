"""Products of 4-bit layers with rows of bfloat16 of odd length that all begin at a word: a row's last 16 bytes begin inside one."""
import numpy as np
import pytest

from oracle import mx

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("n,m,B", [(9, 20, 3), (129, 40, 17), (301, 77, 200), (385, 3161, 763), (8987, 344, 435)])
@pytest.mark.parametrize("both", [False, True])
def test_rows_of_odd_length_in_a_matrix_of_even_width(n, m, B, both):
    """One non-zero of W per column picks entries of X out, so results are X's values without any rounding; NaN lies between the rows."""
    import paper_2108_12704_amd as hac
    rng = np.random.default_rng(n)
    X = torch.from_numpy(rng.standard_normal((B, n)).astype(np.float32)).to(torch.bfloat16)
    pick = np.concatenate([np.arange(n - 1, -1, -1)] * (m // n + 1))[:m]
    w = np.zeros((n, m), np.float32)
    w[pick, np.arange(m)] = 1.0
    db = hac.mx_encode(w).to_device(DEV)
    x = torch.full((B, n + 1), float("nan"), dtype=torch.bfloat16, device=DEV)
    x[:, :n] = X.to(DEV)
    print(f"[case] rows of {n} in {n + 1}, {m} columns, B={B} both={both}", flush=True)
    want = mx.rows(X.double().numpy()) if both else X.double().numpy()
    assert np.array_equal(hac.mx_dot(db, x[:, :n], quantize=both).double().cpu().numpy(), want[:, pick])
