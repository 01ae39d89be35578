"""Windowed attention: exports and host-side refusals (CPU)."""

import ctypes
import os
import re

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = ctypes.c_void_p
NAN = float("nan")
MB = 1 << 20


@pytest.fixture(scope="module")
def lib():
    from paper_2609_30656_gb300 import build, window_attention
    build.build()
    return window_attention._library()


def test_every_entry_point_is_declared_bound_and_exported(lib):
    from paper_2609_30656_gb300 import window_attention
    with open(os.path.join(ROOT, "include", "cb_tbe.h")) as f:
        text = re.sub(r"/\*.*?\*/", "", f.read(), flags=re.S)
    declared = sorted(set(re.findall(r"\b(cb_attention_\w+)\s*\(", text)))
    assert declared == sorted(window_attention.EXPORTS)
    for name in declared:
        assert hasattr(lib, name), name


COMMON = dict(dtype=2, tokens=10, heads=4, kv=2, dim=64, off=8 * MB, idx=0, seqs=2, window=5, sinks=1, scale=0.1,
              work=16 * MB, nbytes=MB, error=None)


def _forward(lib, **kw):
    a = dict(COMMON, q=MB, k=2 * MB, v=3 * MB, qt=256, qh=64, kt=128, kh=64, vt=128, vh=64, out=4 * MB, ot=256, oh=64, lse=5 * MB)
    a.update(kw)
    return lib.cb_attention_forward(P(a["q"]), P(a["k"]), P(a["v"]), a["dtype"], a["tokens"], a["heads"], a["kv"], a["dim"],
                                    a["qt"], a["qh"], a["kt"], a["kh"], a["vt"], a["vh"], P(a["off"]), a["idx"], a["seqs"],
                                    a["window"], a["sinks"], a["scale"], P(a["out"]), a["ot"], a["oh"], P(a["lse"]),
                                    P(a["work"]), a["nbytes"], a["error"], None)


BAD = [{"dtype": 3}, {"tokens": -1}, {"tokens": 2 ** 31}, {"heads": 0}, {"heads": 3}, {"heads": 65536}, {"kv": 0}, {"dim": 0},
       {"dim": 257}, {"off": None}, {"off": 8 * MB + 2}, {"idx": 2}, {"seqs": -1}, {"window": 0}, {"window": -5}, {"sinks": -1},
       {"scale": NAN}, {"error": P(2)}, {"q": None}, {"k": None}, {"v": None}, {"q": MB + 1}, {"qt": -1}, {"kh": -1},
       {"vt": 2 ** 41}, {"lse": 5 * MB + 2}]


@pytest.mark.parametrize("bad", BAD + [{"out": None}, {"ot": 63}, {"oh": 63}, {"ot": 192, "oh": 64},
                                       {"out": MB}, {"out": 2 * MB}, {"out": 3 * MB}, {"lse": 4 * MB}])
def test_forward_refuses_before_any_gpu_work(lib, bad):
    assert _forward(lib, **bad) == 1


def test_forward_refuses_a_small_or_misaligned_workspace(lib):
    need = lib.cb_attention_workspace_bytes(10, 4, 2, 64, 5, 1, 0)
    assert need > 0
    for work, nbytes in ((None, need), (16 * MB, need - 1), (16 * MB + 64, need)):
        assert _forward(lib, work=work, nbytes=nbytes) == 4


def test_no_tokens(lib):
    assert _forward(lib, tokens=0) == 0


def _backward(lib, **kw):
    a = dict(COMMON, go=MB, q=2 * MB, k=3 * MB, v=4 * MB, out=5 * MB, lse=6 * MB, dq=9 * MB, dk=10 * MB, dv=11 * MB,
             gt=256, qt=256, kt=128, kh=64, vt=128, dqt=256, dkt=128, dvt=128)
    a.update(kw)
    return lib.cb_attention_backward(P(a["go"]), P(a["q"]), P(a["k"]), P(a["v"]), P(a["out"]), P(a["lse"]), a["dtype"], a["tokens"],
                                     a["heads"], a["kv"], a["dim"], a["gt"], 64, a["qt"], 64, a["kt"], a["kh"], a["vt"], 64, 256,
                                     64, P(a["off"]), a["idx"], a["seqs"], a["window"], a["sinks"], a["scale"], P(a["dq"]), P(a["dk"]),
                                     P(a["dv"]), a["dqt"], 64, a["dkt"], 64, a["dvt"], 64, P(a["work"]), a["nbytes"], a["error"],
                                     None)


@pytest.mark.parametrize("bad", BAD + [{"go": None}, {"out": None}, {"lse": None}, {"dq": None}, {"dk": None}, {"dv": None},
                                       {"dqt": 200}, {"dkt": 100}, {"dvt": 63}, {"dq": 9 * MB + 1},
                                       {"dq": 2 * MB}, {"dk": 11 * MB}, {"dv": MB}, {"dq": 5 * MB}, {"dk": 6 * MB}])
def test_backward_refuses_before_any_gpu_work(lib, bad):
    assert _backward(lib, **bad) == 1


def test_backward_refuses_a_small_or_misaligned_workspace(lib):
    need = lib.cb_attention_workspace_bytes(10, 4, 2, 64, 5, 1, 1)
    assert need > lib.cb_attention_workspace_bytes(10, 4, 2, 64, 5, 1, 0)
    for work, nbytes in ((None, need), (16 * MB, need - 1), (16 * MB + 64, need)):
        assert _backward(lib, work=work, nbytes=nbytes) == 4


def test_workspace_sizes(lib):
    size = lib.cb_attention_workspace_bytes
    assert size(0, 4, 2, 64, 5, 1, 1) == 0 and size(10, 4, 0, 64, 5, 1, 1) == 0 and size(10, 4, 2, 64, 0, 1, 1) == 0
    # places for parts of the first tokens' gradients: only where a session can be long, and no more than 256 MB
    without, some = size(100000, 16, 4, 128, 256, 0, 1), size(100000, 16, 4, 128, 256, 4, 1)
    assert without < some <= without + (256 << 20) + (1 << 20)
    assert size(100000, 16, 4, 128, 256, 10 ** 9, 1) <= without + (256 << 20) + (1 << 20)
    assert size(1000, 16, 4, 128, 256, 4, 1) == size(1000, 16, 4, 128, 256, 0, 1)


def _step(lib, **kw):
    a = dict(COMMON, q=MB, k=2 * MB, v=3 * MB, out=4 * MB, capacity=100, qs=256, qh=64, ks=12800, kt=128, kh=64, vs=12800, vt=128,
             vh=64, os=256, oh=64)
    a.update(kw)
    return lib.cb_attention_step(P(a["q"]), P(a["k"]), P(a["v"]), a["dtype"], a["seqs"], a["capacity"], a["heads"], a["kv"],
                                 a["dim"], a["qs"], a["qh"], a["ks"], a["kt"], a["kh"], a["vs"], a["vt"], a["vh"], P(a["off"]), a["idx"],
                                 a["window"], a["sinks"], a["scale"], P(a["out"]), a["os"], a["oh"], P(a["work"]), a["nbytes"],
                                 a["error"], None)


@pytest.mark.parametrize("bad", [b for b in BAD if not {"tokens", "lse", "vt", "qt"} & set(b)] + [
    {"out": None}, {"capacity": -1}, {"capacity": 2 ** 31}, {"os": 63}, {"oh": 10}, {"qs": -1}, {"ks": -1}, {"vt": 2 ** 41},
    {"out": MB}, {"out": 2 * MB}, {"out": 3 * MB}])
def test_step_refuses_before_any_gpu_work(lib, bad):
    assert _step(lib, **bad) == 1


def test_step_workspace(lib):
    assert _step(lib, seqs=0) == 0
    need = lib.cb_attention_step_workspace_bytes(1, 4, 2, 64, 100000, 50000, 4)
    assert need > 0 and lib.cb_attention_step_workspace_bytes(1, 4, 2, 64, 100, 50, 4) == 0
    big = dict(seqs=1, capacity=100000, window=50000, sinks=4)
    for work, nbytes in ((None, need), (16 * MB, need - 1), (16 * MB + 16, need)):
        assert _step(lib, **big, work=work, nbytes=nbytes) == 4


def test_the_bindings_refuse_host_tensors():
    from paper_2609_30656_gb300 import window_attention as wa
    q, off = torch.zeros(4, 2, 64, dtype=torch.bfloat16), torch.tensor([0, 4])
    with pytest.raises(ValueError):
        wa.window_attention(q, q, q, off)
    with pytest.raises(ValueError):
        wa.window_attention_step(q, q[:, None], q[:, None], torch.ones(4, dtype=torch.int64))
