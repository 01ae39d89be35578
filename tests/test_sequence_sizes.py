"""Sizes past 32 bits at the entry points for sequence models: refused, not cut off (CPU)."""

import ctypes

import pytest

P = ctypes.c_void_p
COEF = (ctypes.c_float * 3)(3.4445, -4.7750, 2.0315)
INVALID = 1
PAST = [2 ** 30, 2 ** 31, 2 ** 32, 2 ** 32 + 5, 2 ** 40, 2 ** 62, 2 ** 63 - 1]


@pytest.fixture(scope="module")
def lib():
    from paper_2609_30656_gb300 import build, muon, token_embedding
    build.build()
    token_embedding._library()
    return muon._library()


@pytest.mark.parametrize("size", PAST)
@pytest.mark.parametrize("what", ["sequences", "length", "both", "dim"])
def test_token_calls(lib, size, what):
    seqs, length, dim = 2, 3, 8
    if what in ("sequences", "both"):
        seqs = size
    if what in ("length", "both"):
        length = size
    if what == "dim":
        dim = size
    assert lib.cb_token_forward(P(4096), 0, 10, dim, dim, P(8192), 1, seqs, length, 3, 1, 1.0, P(12288), 0, 3 * 8, dim,
                                None, None) == INVALID
    assert lib.cb_token_backward(P(4096), 0, 3 * 8, dim, P(8192), 1, seqs, length, 3, 1, 10, dim, 1.0, -1, 1, P(12288), 0,
                                 dim, P(16384), 1 << 62, None, None) == INVALID


@pytest.mark.parametrize("size", PAST)
def test_workspace_of_sizes_refused_is_none(lib, size):
    assert lib.cb_token_backward_workspace_bytes(size, 10, 8) == 0
    assert lib.cb_token_backward_workspace_bytes(5000, 10, size) == 0
    assert lib.cb_token_backward_workspace_bytes(5000, size * 2, 8) == 0
    for batch, rows, cols in ((size, 8, 8), (1, size, 8), (1, 8, size), (size, size, size)):
        assert lib.cb_muon_workspace_bytes(batch, rows, cols) == 0


@pytest.mark.parametrize("size", PAST)
@pytest.mark.parametrize("what", ["batch", "rows", "cols"])
def test_matrix_calls(lib, size, what):
    sizes = {"batch": 1, "rows": 8, "cols": 16, what: size}
    stride = max(sizes["cols"], 16)
    args = (sizes["batch"], sizes["rows"], sizes["cols"])
    assert lib.cb_muon_orthogonalise(P(4096), 0, *args, 1 << 62, stride, 0.0, COEF, 1, P(8192), 2, 1 << 62, stride,
                                     P(65536), 1 << 62, None, None) == INVALID
    assert lib.cb_muon_step(P(4096), 0, 1 << 62, stride, P(12288), 0, 1 << 62, stride, P(8192), 1 << 62, stride, *args, 0.1,
                            0.0, 0.9, 1, 0.0, COEF, 1, 1.0, P(65536), 1 << 62, None, None) == INVALID


def test_no_tokens_of_any_number_of_sequences(lib):
    for seqs, length in ((2 ** 40, 0), (0, 2 ** 40)):
        assert lib.cb_token_forward(P(4096), 0, 10, 8, 8, P(8192), 1, seqs, length, 3, 1, 1.0, P(12288), 0, 24, 8, None,
                                    None) == 0
