"""Strides of what the sequence calls write: rows in one place are refused, rows in turn are taken (CPU)."""

import ctypes

import pytest
import torch

P = ctypes.c_void_p
COEF = (ctypes.c_float * 3)(3.4445, -4.7750, 2.0315)
INVALID, CAPACITY = 1, 4


@pytest.fixture(scope="module")
def lib():
    from paper_2609_30656_gb300 import build, muon, token_embedding
    build.build()
    token_embedding._library()
    return muon._library()


def brute_apart(outer, s0, inner, s1, width):
    seen = set()
    for o in range(outer):
        for i in range(inner):
            at = range(o * s0 + i * s1, o * s0 + i * s1 + width)
            if not seen.isdisjoint(at):
                return False
            seen.update(at)
    return True


STRIDES = [(o, s0, i, s1) for o in (1, 2, 3) for i in (1, 2, 3) for s0 in (0, 3, 4, 5, 8, 9, 11, 12, 16, 24)
           for s1 in (4, 5, 8, 11, 12, 16)]


# Every argument is checked before the workspace, whose absence is the last refusal: no call gets to the GPU.
def _step(lib, batch, rows, cols, w, m):
    return lib.cb_muon_step(P(4096), 0, *w, P(12288), 0, rows * cols, cols, P(8192), *m, batch, rows, cols, 0.1, 0.0, 0.9,
                            1, 0.0, COEF, 1, 1.0, None, 0, None, None)


def test_matrices_that_are_written(lib):
    for batch, s0, rows, s1 in STRIDES:
        want = CAPACITY if brute_apart(batch, s0, rows, s1, 4) else INVALID
        fine = (rows * 4, 4)
        assert _step(lib, batch, rows, 4, (s0, s1), fine) == want, (batch, s0, rows, s1)
        assert _step(lib, batch, rows, 4, fine, (s0, s1)) == want, (batch, s0, rows, s1)
        assert lib.cb_muon_orthogonalise(P(4096), 0, batch, rows, 4, 0, 4, 0.0, COEF, 1, P(8192), 0, s0, s1, None, 0, None,
                                         None) == want, (batch, s0, rows, s1)
    huge = 2 ** 62  # (rows - 1) * stride passes 64 bits
    assert _step(lib, 2, 8, 4, (4, huge), (32, 4)) == CAPACITY
    assert _step(lib, 2, 8, 4, (huge, huge - 1), (32, 4)) == INVALID


def test_rows_of_a_lookup(lib):
    def forward(seqs, s0, length, s1, out_dtype=0):
        return lib.cb_token_forward(P(4096), 0, 10, 4, 4, P(8192), 1, seqs, length, 0, 0, 1.0, P(12288), out_dtype, s0, s1,
                                    None, None)
    for seqs, s0, length, s1 in STRIDES:
        if not brute_apart(seqs, s0, length, s1, 4):
            assert forward(seqs, s0, length, s1) == INVALID, (seqs, s0, length, s1)
    assert forward(2, 2 ** 62, 8, 2 ** 62 - 1) == INVALID and forward(8, 4, 2 ** 20, 16) == INVALID


def test_layouts_of_the_binding():
    from paper_2609_30656_gb300 import muon
    for batch, s0, rows, s1 in STRIDES:
        t = torch.zeros(256).as_strided((batch, rows, 4), (s0, s1, 1))
        want = brute_apart(batch, s0, rows, s1, 4)
        assert muon._layout(t)[3] == want, (batch, s0, rows, s1)
    w = torch.zeros(5, 3, 7)
    assert muon._layout(w.transpose(0, 1))[3]
