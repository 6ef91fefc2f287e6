"""Products by groups on tiles whose offsets make no sense write nothing outside the rows of Y and the workspace (what they write there is undefined);
test_mx_offsets.py follows the indices of the same calls without a GPU."""
import pytest

import mx_offsets

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype,both,n,m,B", mx_offsets.SIZES)
def test_offsets_that_make_no_sense_stay_inside_on_tiles(dtype, both, n, m, B):
    import paper_2108_12704_amd as hac
    dtype = getattr(torch, dtype)
    g = torch.Generator(device=DEV)
    g.manual_seed(n)
    db = hac.mx_encode_dev(torch.randn((mx_offsets.COUNT, n, m), generator=g, device=DEV))
    need = hac.mx_workspace_bytes(db.desc, B, dtype, both, grouped=True)
    ws = torch.empty(need + 8192, dtype=torch.uint8, device=DEV)
    flat = torch.randn(B * n + 64, generator=g, device=DEV).to(dtype)
    good = torch.linspace(0, B, mx_offsets.COUNT + 1).to(torch.int32).to(DEV)
    for left in (0, 4 // flat.element_size()):                    # (rows of bfloat16 where they lie, and laid out)
        x = flat[left:left + B * n].view(B, n)
        want = hac.mx_grouped_dot(db, x, good, quantize=both)
        for off in mx_offsets.offsets(B):
            print(f"[case] offsets {off} {n} x {m} B={B} {dtype} both={both} from entry {left}", flush=True)
            ws.fill_(0xa5)
            y = torch.full((B + 40, m + 6), 3.0, dtype=dtype, device=DEV)
            inner = y[20:-20, 4:4 + m]
            hac.mx_grouped_dot(db, x, torch.tensor(off, dtype=torch.int32, device=DEV), Y=inner, workspace=ws[4096:4096 + need], quantize=both)
            torch.cuda.synchronize()
            assert any(k.startswith("mx_tile_kernel") for k in hac.hac_last_kernels())
            assert bool((ws[:4096] == 0xa5).all()) and bool((ws[4096 + need:] == 0xa5).all())
            assert bool((y[:20] == 3).all()) and bool((y[-20:] == 3).all()) and bool((y[:, :4] == 3).all()) and bool((y[:, 4 + m:] == 3).all())
        # a call with offsets that do make sense, in the same workspace, is not affected by what the others left there
        assert torch.equal(hac.mx_grouped_dot(db, x, good, workspace=ws[4096:4096 + need], quantize=both), want)
