"""Layer normalisation and clipping: exports and host-side refusals (CPU)."""

import ctypes
import os
import re

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = ctypes.c_void_p
NAN = float("nan")


@pytest.fixture(scope="module")
def libs():
    from paper_2609_30656_gb300 import build, clip, layer_norm
    build.build()
    return layer_norm._library(), clip._library()


def test_every_entry_point_is_declared_bound_and_exported(libs):
    from paper_2609_30656_gb300 import clip, layer_norm
    with open(os.path.join(ROOT, "include", "cb_tbe.h")) as f:
        text = re.sub(r"/\*.*?\*/", "", f.read(), flags=re.S)
    declared = sorted(set(re.findall(r"\b(cb_(?:layer|grad)_\w+)\s*\(", text)))
    assert declared == sorted(layer_norm.EXPORTS + clip.EXPORTS)
    for name in declared:
        assert hasattr(libs[0], name), name


def _forward(lib, x=4096, dtype=0, rows=3, dim=8, stride=8, w=8192, wd=0, b=12288, bd=0, eps=1e-5, out=16384, od=0, os_=8,
             mean=20480, rstd=24576):
    return lib.cb_layer_norm_forward(P(x), dtype, rows, dim, stride, P(w), wd, P(b), bd, eps, P(out), od, os_, P(mean),
                                     P(rstd), None)


@pytest.mark.parametrize("bad", [
    {"x": None}, {"out": None}, {"dtype": 3}, {"od": -1}, {"wd": 5}, {"bd": 3}, {"rows": -1}, {"rows": 2 ** 40}, {"dim": -1},
    {"dim": 2 ** 20 + 1, "stride": 2 ** 21, "os_": 2 ** 21}, {"stride": 7}, {"os_": 7}, {"stride": 2 ** 60}, {"eps": -1.0},
    {"eps": NAN}, {"x": 4098}, {"out": 16385}, {"w": 8193}, {"b": 12290}, {"mean": 20481}, {"rstd": 24577}])
def test_forward_refuses_before_any_gpu_work(libs, bad):
    assert _forward(libs[0], **bad) == 1


def test_forward_of_nothing(libs):
    for none in ({"rows": 0}, {"dim": 0}):
        assert _forward(libs[0], **none, x=None, out=None) == 0


def _backward(lib, go=4096, x=8192, dtype=0, rows=3, dim=8, gs=8, xs=8, mean=12288, rstd=16384, w=20480, wd=0, dx=24576, dd=0,
              ds=8, dw=28672, db=32768, work=65536, nbytes=1 << 30):
    return lib.cb_layer_norm_backward(P(go), P(x), dtype, rows, dim, gs, xs, P(mean), P(rstd), P(w), wd, P(dx), dd, ds, P(dw),
                                      P(db), P(work), nbytes, None)


@pytest.mark.parametrize("bad", [
    {"go": None}, {"x": None}, {"dx": None}, {"mean": None}, {"rstd": None}, {"dtype": 3}, {"dd": 9}, {"wd": -1}, {"rows": -1},
    {"dim": -1}, {"gs": 7}, {"xs": 7}, {"ds": 7}, {"go": 4097}, {"x": 8194}, {"dx": 24578}, {"mean": 12290}, {"dw": 28674},
    {"db": 32769}, {"w": 20482}])
def test_backward_refuses_before_any_gpu_work(libs, bad):
    assert _backward(libs[0], **bad) == 1


def test_backward_refuses_a_small_or_misaligned_workspace(libs):
    need = libs[0].cb_layer_norm_backward_workspace_bytes(3, 8)
    assert need > 0
    for work, nbytes in ((None, need), (65536, need - 1), (65536 + 16, need)):
        assert _backward(libs[0], work=work, nbytes=nbytes) == 4
    assert libs[0].cb_layer_norm_backward_workspace_bytes(-1, 8) == 0


def _entry(data=4096, out=None, count=None, rows=1, cols=100, row=100, out_row=100, dtype=0, out_dtype=0):
    from paper_2609_30656_gb300 import clip
    return clip.CbGradTensor(data, data if out is None else out, count, rows, cols, row, out_row, dtype, out_dtype)


def _clip(lib, *entries, n=None, max_norm=1.0, eps=0.0, norm=1 << 20, work=1 << 21, nbytes=1 << 24):
    from paper_2609_30656_gb300 import clip
    table = (clip.CbGradTensor * max(1, len(entries)))(*entries)
    return lib.cb_grad_clip(table, len(entries) if n is None else n, max_norm, eps, P(norm), P(work), nbytes, None)


def test_clip_refuses_before_any_gpu_work(libs):
    lib = libs[1]
    for bad in ({"data": 4098}, {"dtype": 3}, {"out_dtype": 3}, {"rows": -1}, {"cols": -1}, {"rows": 4, "row": 99},
                {"rows": 4, "out_row": 99}, {"rows": 2 ** 30, "cols": 2 ** 30, "row": 2 ** 30, "out_row": 2 ** 30},
                {"count": 8192, "rows": 2}, {"count": 8193}, {"out": 8193}, {"data": 0, "out": 8192}):
        assert _clip(lib, _entry(**bad)) == 1, bad
    for bad in ({"max_norm": -1.0}, {"max_norm": NAN}, {"eps": -1.0}, {"eps": NAN}, {"norm": 3}, {"n": -1}, {"n": 2 ** 21}):
        assert _clip(lib, _entry(), **bad) == 1, bad
    for work, nbytes in ((None, 1 << 24), (1 << 21, 16), ((1 << 21) + 16, 1 << 24)):
        assert _clip(lib, _entry(), work=work, nbytes=nbytes) == 4


def test_clip_refuses_values_written_twice_or_read_elsewhere(libs):
    lib = libs[1]
    far = 1 << 16
    assert _clip(lib, _entry(4096), _entry(4096)) == 1                   # the same tensor twice
    assert _clip(lib, _entry(4096), _entry(4096 + 396)) == 1             # one value of it
    assert _clip(lib, _entry(4096, out=4100)) == 1                       # onto itself, moved
    assert _clip(lib, _entry(4096, out_dtype=1)) == 1                    # in place in another type
    assert _clip(lib, _entry(4096, out=far), _entry(far)) == 1           # a result onto another gradient
    # two halves of the columns of one matrix are apart; overlapping ones are not
    left = dict(rows=8, cols=50, row=100, out_row=100)
    assert _clip(lib, _entry(4096, **left), _entry(4096 + 196, **left)) == 1
    assert _clip(lib, _entry(4096, **left), _entry(4096 + 200, rows=8, cols=51, row=100, out_row=100)) == 1
    assert _clip(lib, _entry(4096, **left), _entry(4096 + 200, rows=8, cols=50, row=99, out_row=99)) == 1


def test_norm_refuses(libs):
    from paper_2609_30656_gb300 import clip
    table = (clip.CbGradTensor * 1)(_entry())
    assert libs[1].cb_grad_norm(table, 1, None, P(1 << 21), 1 << 24, None) == 1
    assert libs[1].cb_grad_norm(None, 1, P(4096), P(1 << 21), 1 << 24, None) == 1
    assert libs[1].cb_grad_norm_workspace_bytes(0) == 0 and libs[1].cb_grad_norm_workspace_bytes(1) > 0
    assert libs[1].cb_grad_norm_workspace_bytes(401) == 2 * libs[1].cb_grad_norm_workspace_bytes(400)


def test_the_bindings_refuse_host_tensors():
    from paper_2609_30656_gb300 import clip, layer_norm
    x = torch.zeros(3, 8)
    with pytest.raises(ValueError):
        layer_norm.layer_norm(x)
    with pytest.raises(ValueError):
        layer_norm.layer_norm_backward(x, x, x[:, 0], x[:, 0])
    with pytest.raises(ValueError):
        clip.grad_norm([x])
    with pytest.raises(ValueError):
        clip.clip_grad_norm([], 1.0)


def test_layouts_of_gradients():
    from paper_2609_30656_gb300 import clip
    t = torch.zeros(6, 8, 10)
    assert clip._as_rows(t, t) == (1, 480, 480, 480)
    p = t.permute(2, 0, 1)
    assert clip._as_rows(p, p) == (1, 480, 480, 480)
    s = t[:, :, :7]
    assert clip._as_rows(s, s) == (48, 7, 10, 10)
    assert clip._as_rows(s, torch.zeros(6, 8, 7)) == (48, 7, 10, 7)
    assert clip._as_rows(torch.zeros(6, 8, 7), s) == (48, 7, 7, 10)
    assert clip._as_rows(t[:, :3], t[:, :3]) == (6, 30, 80, 80)
    assert clip._as_rows(t[:, ::2, :7], t[:, ::2, :7]) == (24, 7, 20, 20)
    assert clip._as_rows(t[:, :3, :7], t[:, :3, :7]) is None
    assert clip._as_rows(t[:1].expand(6, 8, 10), t[:1].expand(6, 8, 10)) is None
    assert clip._as_rows(t, t.permute(2, 1, 0).contiguous().permute(2, 1, 0)) is None
    assert clip._as_rows(t[0, :, :1], t[0, :, :1]) == (8, 1, 10, 10)
