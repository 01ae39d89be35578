"""Waits that run out: they end, are reported, and leave the caller's weights alone (GPU).

No kernel hangs here: the wait that runs out is on a barrier that nothing is to arrive on, with a limit of a few
polls and nothing in flight, and what follows a report is tried with the report's word set by the test.
"""

import ctypes
import os
import subprocess

import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TIMEOUT = 7  # CB_ERR_TIMEOUT


@pytest.fixture(scope="module")
def probe(tmp_path_factory):
    from paper_2609_30656_gb300 import build, tbe
    tbe.load_library()
    out = str(tmp_path_factory.mktemp("native") / "libwait_probe.so")
    source = os.path.join(os.path.dirname(os.path.abspath(__file__)), "native", "wait_probe.cu")
    subprocess.run([build.nvcc(), "-O2", "-std=c++17", "-shared", "-Xcompiler", "-fPIC", "-cudart", "shared", *build.ARCH,
                    "-I", build.INCLUDE, "-I", build.CSRC, source, build.LIB, "-o", out], check=True)
    lib = ctypes.CDLL(out)
    p, i, u, f = ctypes.c_void_p, ctypes.c_int, ctypes.c_uint32, ctypes.c_float
    lib.probe_wait.argtypes = [i, u, p, p, p]
    lib.probe_result.argtypes = [p, p, p, p, p, i, i, i, i, i, f, f, f, f, p]
    return lib


def _word(value):
    return torch.full((1,), value, dtype=torch.int32, device=DEV)


def test_a_wait_ends_and_is_reported(probe):
    for arrive, polls in ((0, 1), (0, 1000), (1, 1000)):
        complete, error = _word(5), _word(0)
        assert probe.probe_wait(arrive, polls, complete.data_ptr(), error.data_ptr(), None) == 0
        torch.cuda.synchronize()
        assert complete.item() == arrive and error.item() == (0 if arrive else TIMEOUT)


@pytest.mark.parametrize("batch,p,q", [(1, 200, 330), (40, 130, 264), (200, 136, 144)])  # tiles of 64, 128, pairs
def test_the_last_product_after_a_report_writes_nothing(probe, batch, p, q):
    g = torch.Generator(device=DEV)
    g.manual_seed(p)
    lda, ldx = -(-p // 64) * 64, -(-q // 64) * 64
    poly = torch.randn(batch, p, lda, generator=g, device=DEV).half()
    hi = torch.randn(batch, p, ldx, generator=g, device=DEV).half()
    lo = (torch.randn(batch, p, ldx, generator=g, device=DEV) * 2.0 ** -12).half()
    start = torch.randn(batch, p, q, generator=g, device=DEV)
    for fault in (TIMEOUT, 0):
        w, word = start.clone(), _word(fault)
        torch.cuda.synchronize()
        assert probe.probe_result(poly.data_ptr(), hi.data_ptr(), lo.data_ptr(), w.data_ptr(), word.data_ptr(), batch, p, q,
                                  lda, ldx, 3.0, 2.0, 0.5, 4.0, None) == 0
        torch.cuda.synchronize()
        assert word.item() == fault
        if fault:
            assert torch.equal(w, start)
        else:
            x, y = hi[..., :q].double(), lo[..., :q].double()
            o = (poly[..., :p].double() @ x / 2.0 ** 8 + x + 3.0 * y) / 2.0 ** 10
            # fp32 sums of p products, a few operations
            assert (w.double() - (0.5 * start.double() - 4.0 * o)).abs().max().item() <= 2.0 ** -18
