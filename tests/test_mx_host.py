"""4-bit microscaled layers without a GPU: the host encoder against the oracle byte for byte, validation, accounting, plans and refusals."""
import ctypes as C
import os
import re
import shutil
import subprocess
import sys

import numpy as np
import pytest

import paper_2108_12704_amd as hac
from oracle import mx

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import hip_stub

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def layer(n, m, seed=0, count=None):
    rng = np.random.default_rng(seed + 100 * n + m)
    shape = (n, m) if count is None else (count, n, m)
    w = (rng.standard_normal(shape) * 10.0 ** rng.integers(-3, 4, shape[:-2] + (1, m))).astype(np.float32)
    w[rng.random(shape) < 0.05] = 0
    return w


def test_every_declared_function_is_exported():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "hac.h")).read(), flags=re.S)
    assert set(re.findall(r"\b(mx_[a-z_]+)\s*\(", text)) == set(hac.MX_EXPORTS)


@pytest.mark.parametrize("n,m", [(1, 1), (32, 16), (33, 17), (128, 1), (129, 40), (500, 30), (640, 5), (1100, 64)])
def test_host_encoder_writes_what_the_oracle_lays_out(n, m):
    w = layer(n, m)
    blob = hac.mx_encode(w)
    d = blob.desc
    assert (d.format, d.n, d.m, d.k_sym, d.ent_bits, d.chunk, d.nnz) == (hac.HAC_FORMAT_MX, n, m, 1, 4, 32, 0)
    scales, codes = mx.sections(w)
    assert np.array_equal(blob.data[d.off_codebook:d.off_stream], scales)
    assert np.array_equal(blob.data[d.off_stream:], codes)
    assert blob.nbytes == 256 + scales.size + codes.size
    assert blob.validate(True) == 0
    W, sym = blob.decode_host()
    c, _, v = mx.quantise(w)
    assert np.array_equal(W, v.astype(np.float32)) and np.array_equal(sym.reshape(m, n).T, c)
    assert bytes(blob.desc) == bytes(hac.mx_describe(n, m))


def test_values_on_borders_and_at_the_ends_of_the_range():
    rng = np.random.default_rng(5)
    units = np.concatenate([np.arange(0, 64) / 8.0, [7.9999995, 5.0, 5.0000005, 0.25, 0.24999999]])
    w = np.zeros((96, 40), np.float32)
    for j in range(40):
        scale = 2.0 ** [-149, -140, -133, -127, -126, -125, -100, -20, 0, 1, 20, 100, 120, 125][j % 14]
        col = rng.choice(units, 96) * np.where(rng.random(96) < 0.5, -1, 1)
        col[[0, 32, 64]] = [4.0, 7.5, 6.0]
        w[:, j] = (col * scale).astype(np.float32)
    blob = hac.mx_encode(w)
    scales, codes = mx.sections(w)
    assert np.array_equal(blob.data[256:], np.concatenate([scales, codes]))
    assert np.isfinite(blob.decode_host()[0]).all()


def test_experts_are_one_matrix_after_the_other():
    w = layer(200, 20, count=3)
    blob = hac.mx_encode(w)
    one = [hac.mx_encode(e) for e in w]
    d = blob.desc
    size_s, size_c = (d.off_stream - d.off_codebook) // 3, (d.blob_bytes - d.off_stream) // 3
    for e in range(3):
        o = one[e].desc
        assert np.array_equal(blob.data[d.off_codebook + e * size_s:][:size_s], one[e].data[o.off_codebook:o.off_stream])
        assert np.array_equal(blob.data[d.off_stream + e * size_c:][:size_c], one[e].data[o.off_stream:])
    assert blob.validate() == 0 and hac.DeviceBlob.count.fget(type("B", (), {"desc": d})()) == 3
    W, _ = blob.decode_host()
    assert np.array_equal(W, mx.values(w).astype(np.float32))


def test_accounting():
    w = layer(500, 30)
    st = hac.mx_encode(w).stats()
    assert st.stream_bits == 4 * 500 * 30 and st.paper_bits == 4 * 500 * 30 + 8 * 16 * 30
    assert st.avg_code_bits == 4.0 and 0 < st.entropy_bits <= 4.0
    assert st.stream_bytes == 2 * 4 * 1024 and st.table_bytes == 2 * 256 and st.blob_bytes == 256 + 2 * 4 * 1024 + 2 * 256


def test_damaged_blobs_are_refused():
    blob = hac.mx_encode(layer(100, 20))
    lib = hac.load_library()
    check = lambda b, deep=1: lib.hac_validate(b.ctypes.data, b.size, deep)
    assert check(blob.data[:-1]) == -3 and check(blob.data[:100]) == -3
    for field in ("n", "m", "k_sym", "off_stream", "off_codebook", "blob_bytes", "ent_bits", "chunk", "nnz", "total_bits", "dict_shared", "off_ri"):
        b = blob.data.copy()
        b[getattr(hac.Desc, field).offset] ^= 1
        assert check(b, 0) == -3, field
    d = blob.desc
    for at, value in ((d.off_codebook, 253), (d.off_codebook, 254),                  # a scale that no finite block has
                      (d.off_codebook + 1, 3),                                       # a scale behind row n
                      (d.off_codebook + 256 + 4 * 4, 3),                             # ... of column 20
                      (d.off_stream + 16 * 48 + 2, 1),                               # a code of row 100
                      (d.off_stream + 1024 + 16 * 4, 1)):                            # ... of column 20
        b = blob.data.copy()
        b[at] = value
        assert check(b, 0) == 0 and check(b, 1) == -3, (at, value)
    b = blob.data.copy()
    b[d.off_codebook] = 255                                                          # a block of NaN, as the device encoder marks it
    assert check(b) == 0 and np.isnan(hac.Blob(b).decode_host()[0][:32, 0]).all()


def test_encoder_refusals():
    for bad in (np.inf, -np.inf, np.nan):
        w = layer(40, 4)
        w[33, 2] = bad
        with pytest.raises(hac.HacError) as e:
            hac.mx_encode(w)
        assert e.value.status == -1
    for bad in (np.zeros((4, 4)), np.zeros(4, np.float32), np.zeros((1, 1, 2, 2), np.float32)):
        with pytest.raises(TypeError):
            hac.mx_encode(bad)
    for shape in ((0, 4), (4, 0), (0, 4, 4)):
        with pytest.raises(hac.HacError):
            hac.mx_encode(np.zeros(shape, np.float32))
    lib, d = hac.load_library(), hac.Desc()
    for args, rc in (((0, 1, 1), -1), ((65536, 1, 1), -1), ((1, 0, 1), -1), ((1, 1, 0), -1), ((1, 1 << 31, 1), -1), ((1, 1, 1 << 31), -1),
                     ((65535, 1 << 20, 1 << 20), -4), ((1, 0x7fffff00, 1 << 14), -4)):
        assert lib.mx_describe(*args, C.byref(d)) == rc, args
    assert lib.mx_describe(1, 1, 1, None) == -1
    w, out, size = layer(4, 4), C.c_void_p(), C.c_size_t()
    p = w.ctypes.data_as(C.POINTER(C.c_float))
    for args in ((1, 4, 4, 3, 16), (2, 2, 4, 4, 7), (2, 2, 4, 4, -8)):
        assert lib.mx_encode(p, *args, C.byref(out), C.byref(size)) == -1 and not out.value


def test_other_calls_refuse_the_format():
    blob = hac.mx_encode(layer(64, 32))
    assert hac.load_library().hac_dot_route(C.byref(blob.desc), 4, None) == -1
    with pytest.raises(hac.HacError):
        hac.hac_net_encode([layer(8, 8)], [hac.HAC_FORMAT_MX])


# calls of the C ABI on made-up addresses: what they refuse launches nothing
REFUSE = """
F32, BF16, Q = 0, 1, 1
d = hac.mx_describe(300, 40)
many = hac.mx_describe(300, 40, 3)
big, bigger = hac.mx_describe(4096, 4096), hac.mx_describe(4096, 4096, 2)      # 500 rows take a workspace
broken = hac.mx_describe(300, 40); broken.off_stream += 256
at = lambda x: C.c_void_p(x << 20)
def dot(desc=d, blob=at(1), type=F32, X=at(2), B=4, ldx=300, Y=at(3), ldy=40, flags=0, ws=at(4), bytes=1 << 30):
    return lib.mx_dot(C.byref(desc) if desc else None, blob, type, X, B, ldx, Y, ldy, flags, ws, bytes, None)
def grouped(desc=many, blob=at(1), type=F32, X=at(2), B=4, ldx=300, offsets=at(5), Y=at(3), ldy=40, flags=0, ws=at(4), bytes=1 << 30):
    return lib.mx_grouped_dot(C.byref(desc), blob, type, X, B, ldx, offsets, Y, ldy, flags, ws, bytes, None)
def encode(type=F32, W=at(1), count=1, n=300, m=40, ldw=40, stride=0, blob=at(2), room=1 << 30, desc=hac.Desc()):
    return lib.mx_encode_dev(type, W, count, n, m, ldw, stride, blob, room, C.byref(desc) if desc else None, None)
def decode(desc=d, blob=at(1), type=F32, W=at(2), ldw=40, stride=0):
    return lib.mx_decode_dev(C.byref(desc), blob, type, W, ldw, stride, None)
odd = C.c_void_p((2 << 20) + 1)
out = []
for call, rc in (
    (lambda: dot(desc=None), -1), (lambda: dot(desc=broken), -1), (lambda: dot(desc=many), -1), (lambda: dot(blob=None), -1),
    (lambda: dot(blob=C.c_void_p((1 << 20) + 16)), -1), (lambda: dot(type=2), -1), (lambda: dot(flags=2), -1), (lambda: dot(B=-1), -1),
    (lambda: dot(X=None), -1), (lambda: dot(Y=None), -1), (lambda: dot(ldx=299), -1), (lambda: dot(ldy=39), -1), (lambda: dot(X=odd), -1),
    (lambda: dot(type=BF16, X=odd), -1), (lambda: dot(Y=odd), -1), (lambda: dot(B=(1 << 27) + 1), -4),
    (lambda: dot(desc=big, B=500, ldx=4096, ldy=4096, ws=None), -6), (lambda: dot(desc=big, B=500, ldx=4096, ldy=4096, bytes=16), -6),
    (lambda: dot(desc=big, B=500, ldx=4096, ldy=4096, ws=C.c_void_p((4 << 20) + 16)), -1),
    (lambda: dot(B=0, X=None, Y=None), 0),
    (lambda: grouped(offsets=None), -1), (lambda: grouped(offsets=odd), -1), (lambda: grouped(desc=bigger, B=600, ldx=4096, ldy=4096, ws=None), -6), (lambda: grouped(B=0), 0),
    (lambda: encode(desc=None), -1), (lambda: encode(W=None), -1), (lambda: encode(type=7), -1), (lambda: encode(ldw=39), -1),
    (lambda: encode(count=2, stride=300 * 40 - 1), -1), (lambda: encode(count=0), -1), (lambda: encode(W=odd), -1),
    (lambda: encode(blob=None), -6), (lambda: encode(room=100), -6), (lambda: encode(blob=C.c_void_p((2 << 20) + 64)), -1),
    (lambda: decode(desc=broken), -1), (lambda: decode(blob=None), -1), (lambda: decode(W=None), -1), (lambda: decode(ldw=39), -1),
    (lambda: decode(desc=many, stride=11999), -1), (lambda: decode(type=3), -1)):
    stub.stub_reset()
    out.append([call(), rc, len(events())])
print(json.dumps(out))
"""


def test_refused_calls_launch_nothing(tmp_path):
    for i, (got, want, launches) in enumerate(hip_stub.run(tmp_path, REFUSE)):
        assert (got, launches) == (want, 0), (i, got, want, launches)


# every plan keeps to its workspace and to 32 bits of threads in a grid: sizes over the whole range
PLANS = """
out = []
for n, m in ((1, 1), (64, 10), (500, 300), (4096, 4096), (25088, 4096), (9973, 1511), (100, 100000)):
    for count in (1, 2, 64, 1000):
        d = hac.mx_describe(n, m, count)
        for B in (1, 2, 16, 17, 33, 100, 1000, 12544):
            for type in (0, 1):
                for flags in (0, 1):
                    need = lib.mx_workspace_bytes(C.byref(d), type, B, flags, 1)
                    stub.stub_reset()
                    at = lambda x: C.c_void_p(x << 40)
                    rc = lib.mx_grouped_dot(C.byref(d), at(1), type, at(2), B, n, at(3), at(4), m, flags, at(5), need, None)
                    short = lib.mx_grouped_dot(C.byref(d), at(1), type, at(2), B, n, at(3), at(4), m, flags, at(5), need - 1, None) if need else -6
                    seen = events()
                    out.append([n, m, count, B, rc, short, max(e[2] for e in seen), len(seen)])
print(json.dumps(out))
"""


def test_plans_over_the_range(tmp_path):
    for n, m, count, B, rc, short, lds, launches in hip_stub.run(tmp_path, PLANS):
        assert rc == 0 and short == -6 and lds <= 160 * 1024 and 1 <= launches <= 3, (n, m, count, B, rc, short, lds, launches)


torch = pytest.importorskip("torch")
X = "X must be a 2-D float32 or bfloat16 CUDA tensor"


@pytest.mark.parametrize("call,args,kw,error,text", [
    ("mx_dot", (), {}, TypeError, "missing argument 'dblob'"),
    ("mx_dot", (None, torch.zeros(2, 3)), {}, TypeError, X),                          # not on the GPU
    ("mx_dot", (None, torch.zeros(2, 3)), {"offsets": None}, TypeError, "unexpected keyword argument 'offsets'"),
    ("mx_dot", (None, torch.zeros(2, 3), None, None, False, None, None), {}, TypeError, "too many arguments"),
    ("mx_grouped_dot", (None, torch.zeros(2, 3)), {}, TypeError, "missing argument 'offsets'"),
    ("mx_grouped_dot", (None, [[1.0]], None), {}, TypeError, X),
    ("mx_encode_dev", (None, torch.zeros(2, 3)), {}, TypeError, "W must be a 2-D or 3-D float32 or bfloat16 CUDA tensor"),
    ("mx_decode_dev", (), {}, TypeError, "missing argument 'dblob'"),
])
def test_refused_arguments(call, args, kw, error, text):
    with pytest.raises(error, match=text):
        getattr(hac._native(), call)(*args, **kw)


def test_workspace_of_a_chain_with_such_a_layer():
    import ctypes
    w1, w2 = layer(2048, 2048), layer(2048, 40)
    a, b = hac.mx_encode(w1), hac.hac_encode(np.where(np.abs(w2) > 1, np.float32(0.5), np.float32(0)))
    layers = (hac.Layer * 2)()
    for l, blob in zip(layers, (a, b)):
        l.desc, l.d_blob = ctypes.pointer(blob.desc), 1 << 20
    lib = hac.load_library()
    assert lib.hac_forward_workspace_bytes(layers, 2, 2000) > 0
    assert hac.hac_workspace_bytes(a.desc, 2000) == hac.mx_workspace_bytes(a.desc, 2000) > 0
    many = hac.mx_encode(layer(2048, 2048, count=2))
    layers[0].desc = ctypes.pointer(many.desc)
    assert lib.hac_forward_workspace_bytes(layers, 2, 2000) == 0                        # a layer is one matrix


def test_reads_of_a_step_that_is_not_whole_stay_inside_the_row(tmp_path):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no g++")
    exe = str(tmp_path / "mx_reads")
    subprocess.run([gxx, "-std=c++17", "-O1", "-o", exe, os.path.join(ROOT, "tests", "native", "mx_reads.cpp")], check=True, timeout=120)
    run = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert run.returncode == 0 and " 0 failures" in run.stdout, run.stdout


# more rows than the kernel for few rows can count in a launch, whatever the layer
MANY_ROWS = """
out = []
for n, m, count in ((1, 1, 1), (64, 10, 1), (4096, 64, 1), (64, 10, 3), (64, 10, 65535)):
    d = hac.mx_describe(n, m, count)
    for B in (300000, 65535 * 16, 65535 * 16 + 1, 1 << 24, 1 << 27):
        for type in (0, 1):
            for flags in (0, 1):
                need = lib.mx_workspace_bytes(C.byref(d), type, B, flags, 1)
                at = lambda x: C.c_void_p(x << 48)
                stub.stub_reset()
                out.append([n, m, count, B, lib.mx_grouped_dot(C.byref(d), at(1), type, at(2), B, n, at(3), at(4), m, flags, at(5), need, None), len(events())])
print(json.dumps(out))
"""


def test_plans_of_many_rows(tmp_path):
    for case in hip_stub.run(tmp_path, MANY_ROWS):
        assert case[-2] == 0 and case[-1] >= 1, case
