"""The entry points for sequence models (token lookup, orthogonalised updates): exports and host-side refusals (CPU)."""

import ctypes
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = ctypes.c_void_p
COEF = (ctypes.c_float * 3)(3.4445, -4.7750, 2.0315)


@pytest.fixture(scope="module")
def libs():
    from paper_2609_30656_gb300 import build, muon, token_embedding
    build.build()
    return token_embedding._library(), muon._library()


def test_every_entry_point_is_declared_bound_and_exported(libs):
    from paper_2609_30656_gb300 import muon, token_embedding
    with open(os.path.join(ROOT, "include", "cb_tbe.h")) as f:
        text = re.sub(r"/\*.*?\*/", "", f.read(), flags=re.S)
    declared = sorted(set(re.findall(r"\b(cb_(?:token|muon)_\w+)\s*\(", text)))
    assert declared == sorted(token_embedding.EXPORTS + muon.EXPORTS)
    for name in declared:
        assert hasattr(libs[0], name), name


def _forward(lib, table=4096, dtype=0, rows=10, dim=8, stride=8, tokens=8192, idx=1, seqs=2, length=3, ts=3, tp=1,
             scale=1.0, out=12288, out_dtype=0, os_=24, op=8, error=None):
    return lib.cb_token_forward(P(table), dtype, rows, dim, stride, P(tokens), idx, seqs, length, ts, tp, scale, P(out),
                                out_dtype, os_, op, error, None)


@pytest.mark.parametrize("bad", [
    {"table": None}, {"tokens": None}, {"out": None}, {"dtype": 3}, {"out_dtype": -1}, {"idx": 2}, {"rows": -1},
    {"rows": 2 ** 31}, {"dim": -1}, {"dim": 2 ** 20 + 1}, {"stride": 7}, {"seqs": -1}, {"length": -1},
    {"seqs": 2 ** 15, "length": 2 ** 15}, {"scale": float("nan")}, {"op": 7}, {"os_": 7}, {"table": 4097},
    {"out": 12289}, {"tokens": 8196}, {"error": P(2)}])
def test_forward_refuses_before_any_gpu_work(libs, bad):
    assert _forward(libs[0], **bad) == 1


def test_forward_of_nothing(libs):
    for none in ({"seqs": 0}, {"length": 0}, {"dim": 0}):
        assert _forward(libs[0], **{**none, "table": None, "tokens": None, "out": None}) in (0, 1)
        assert _forward(libs[0], **none) == 0


def _backward(lib, go=4096, dtype=0, gs=24, gp=8, tokens=8192, idx=1, seqs=2, length=3, ts=3, tp=1, rows=10, dim=8,
              scale=1.0, pad=-1, acc=0, grad=12288, grad_dtype=0, stride=8, work=None, nbytes=0, error=None):
    return lib.cb_token_backward(P(go), dtype, gs, gp, P(tokens), idx, seqs, length, ts, tp, rows, dim, scale, pad, acc,
                                 P(grad), grad_dtype, stride, P(work), nbytes, error, None)


@pytest.mark.parametrize("bad", [
    {"go": None}, {"tokens": None}, {"grad": None}, {"dtype": 3}, {"grad_dtype": 7}, {"idx": -1}, {"rows": -1},
    {"rows": 2 ** 31}, {"dim": -2}, {"stride": 7}, {"seqs": -1}, {"length": -1}, {"scale": float("nan")}, {"gp": -8},
    {"gs": -8}, {"go": 4098}, {"grad": 12290}, {"tokens": 8193}, {"error": P(6)}])
def test_backward_refuses_before_any_gpu_work(libs, bad):
    assert _backward(libs[0], **bad) == 1


def test_backward_refuses_a_small_or_misaligned_workspace(libs):
    lib = libs[0]
    need = lib.cb_token_backward_workspace_bytes(3000, 10, 8)
    assert need > 0 and lib.cb_token_backward_workspace_bytes(100, 10, 8) == 0
    for work, nbytes in ((None, need), (16384, need - 1), (16384 + 128, need)):
        assert _backward(lib, seqs=1, length=3000, work=work, nbytes=nbytes) == 4


def test_backward_workspace_grows_with_the_call(libs):
    f = libs[0].cb_token_backward_workspace_bytes
    sizes = [f(n, 50_000, 1024) for n in (2049, 5000, 100_000, 1 << 20)]
    assert sizes == sorted(sizes) and sizes[0] > 0
    # two rows of sums per chunk of the sorted tokens, beside the sort
    assert sizes[-1] < (1 << 20) * 1024 * 4


def _ortho(lib, g=4096, dtype=0, batch=1, rows=8, cols=16, gb=128, gr=16, eps=0.0, coef=COEF, steps=1, out=8192,
           out_dtype=2, ob=128, orow=16, work=65536, nbytes=1 << 20, error=None):
    return lib.cb_muon_orthogonalise(P(g), dtype, batch, rows, cols, gb, gr, eps, coef, steps, P(out), out_dtype, ob, orow,
                                     P(work), nbytes, error, None)


@pytest.mark.parametrize("bad", [
    {"g": None}, {"out": None}, {"dtype": 3}, {"out_dtype": 3}, {"batch": -1}, {"batch": 65536}, {"rows": -1},
    {"cols": -1}, {"rows": 2 ** 20 + 1}, {"gr": 15}, {"orow": 15}, {"batch": 2, "ob": 127}, {"batch": 2, "gb": -1},
    {"eps": -1.0}, {"eps": float("nan")}, {"coef": None}, {"coef": (ctypes.c_float * 3)(1, float("nan"), 2)},
    {"steps": 0}, {"steps": 65}, {"g": 4098}, {"out": 8193}, {"error": P(3)},
    {"rows": 2 ** 20, "cols": 2 ** 20, "gr": 2 ** 20, "orow": 2 ** 20}])
def test_orthogonalise_refuses_before_any_gpu_work(libs, bad):
    assert _ortho(libs[1], **bad) == 1


def test_orthogonalise_refuses_a_small_or_misaligned_workspace(libs):
    need = libs[1].cb_muon_workspace_bytes(1, 8, 16)
    for work, nbytes in ((None, need), (65536, need - 1), (65536 + 64, need)):
        assert _ortho(libs[1], work=work, nbytes=nbytes) == 4


def test_orthogonalise_nothing(libs):
    for none in ({"batch": 0}, {"rows": 0}, {"cols": 0}):
        assert _ortho(libs[1], **none) == 0
    assert libs[1].cb_muon_workspace_bytes(0, 8, 8) == 0 and libs[1].cb_muon_workspace_bytes(1, -8, 8) == 0


def test_step_refuses_before_any_gpu_work(libs):
    def step(w=4096, m=8192, lr=0.1, wd=0.0, beta=0.9, scale=1.0, mr=16, mb=128, batch=1):
        return libs[1].cb_muon_step(P(w), 0, 128, 16, P(12288), 0, 128, 16, P(m), mb, mr, batch, 8, 16, lr, wd, beta, 1,
                                    0.0, COEF, 1, scale, P(65536), 1 << 20, None, None)
    nan = float("nan")
    for bad in ({"w": None}, {"m": None}, {"m": 8194}, {"lr": nan}, {"wd": nan}, {"beta": -0.1}, {"beta": nan},
                {"scale": nan}, {"mr": 15}, {"mb": 100, "batch": 2}):
        assert step(**bad) == 1, bad


def test_update_scales():
    from paper_2609_30656_gb300 import muon
    assert muon.update_scale(100, 400, "rms") == pytest.approx(4.0)
    assert muon.update_scale(400, 100, "spectral") == pytest.approx(2.0)
    assert muon.update_scale(100, 400, "spectral") == 1.0 and muon.update_scale(3, 4, None) == 1.0
    with pytest.raises(ValueError):
        muon.update_scale(3, 4, "adam")
