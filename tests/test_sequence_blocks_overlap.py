"""Results that share memory with what a call reads, or with one another, are refused before any GPU work, wherever the one
begins within the other (CPU)."""

import pytest

from tests.test_window_attention_abi import _backward, _forward, _step, MB, P, lib  # noqa: F401

SMALL = 2 * 64  # bytes of a head of a token: 10 tokens of 4 heads of q and out, of 2 of k and v


@pytest.mark.parametrize("bad", [
    {"out": MB + SMALL}, {"out": MB + 9 * 512}, {"out": MB - 512}, {"out": 2 * MB + SMALL}, {"out": 3 * MB + 256},
    {"lse": 4 * MB + 4}, {"lse": MB + 64}, {"out": 8 * MB}, {"out": 8 * MB - 512}, {"work": 4 * MB}, {"work": 2 * MB},
    {"error": P(4 * MB + 8)}, {"error": P(16 * MB)}, {"lse": 16 * MB},
    # columns of one matrix: q and out side by side, but for a value
    {"qt": 512, "ot": 512, "out": MB + 2 * 255, "tokens": 10}], ids=str)
def test_forward(lib, bad):  # noqa: F811
    assert _forward(lib, **bad) == 1


@pytest.mark.parametrize("bad", [
    {"dq": MB + SMALL}, {"dq": 2 * MB + 256}, {"dk": 3 * MB + SMALL}, {"dv": 4 * MB - 256}, {"dk": 5 * MB + 9 * 512},
    {"dv": 6 * MB + 32}, {"dk": 11 * MB + SMALL}, {"dv": 9 * MB + 512}, {"dq": 8 * MB}, {"work": 9 * MB}, {"error": P(10 * MB)},
    {"dqt": 512, "gt": 512, "dq": MB + 2 * 255}], ids=str)
def test_backward(lib, bad):  # noqa: F811
    assert _backward(lib, **bad) == 1


@pytest.mark.parametrize("bad", [
    {"out": MB + SMALL}, {"out": 2 * MB + 256}, {"out": 2 * MB + 12800 * 2}, {"out": 3 * MB + 99 * 256}, {"out": 8 * MB},
    {"error": P(4 * MB)}, {"out": 2 * MB - 64}], ids=str)
def test_step(lib, bad):  # noqa: F811
    assert _step(lib, **bad) == 1


@pytest.mark.parametrize("bad", [
    {"out": 4096 + 32}, {"out": 4096 - 32}, {"out": 4096, "od": 1}, {"out": 4096, "os_": 16}, {"out": 4096, "stride": 16},
    {"out": 4096 + 4 * 15, "stride": 16, "os_": 16}, {"out": 8192 + 16}, {"out": 12288 - 64}, {"mean": 4096 + 64}, {"rstd": 20480 + 8},
    {"mean": 16384}, {"rstd": 8192}], ids=str)
def test_layer_norm(lib, bad):  # noqa: F811
    from paper_2609_30656_gb300 import layer_norm
    from tests.test_norm_and_clip_abi import _forward as forward
    assert forward(layer_norm._library(), **bad) == 1


@pytest.mark.parametrize("bad", [
    {"dx": 4096 + 32}, {"dx": 8192 - 32}, {"dx": 8192, "dd": 1}, {"dx": 4096, "ds": 16}, {"dx": 20480}, {"dx": 12288 - 64},
    {"dw": 24576 + 64}, {"db": 28672 + 28}, {"dw": 8192 + 32}, {"db": 16384}, {"work": 8192}, {"dx": 65536 + 32}, {"db": 65536}],
    ids=str)
def test_layer_norm_backward(lib, bad):  # noqa: F811
    from paper_2609_30656_gb300 import layer_norm
    from tests.test_norm_and_clip_abi import _backward as backward
    assert backward(layer_norm._library(), **bad) == 1


@pytest.mark.parametrize("entry,call", [
    ({}, {"norm": 4096 + 8}), ({"out": 1 << 16}, {"norm": 4096}), ({"out": 1 << 16}, {"norm": (1 << 16) + 396}), ({}, {"work": 4096 - 256}),
    ({"count": 4096 + 16}, {}), ({"count": (1 << 16) + 392, "out": 1 << 16}, {}), ({"count": 1 << 20}, {}), ({}, {"norm": 1 << 21})], ids=str)
def test_clip(lib, entry, call):  # noqa: F811
    """The norm, the workspace and the counts too."""
    from paper_2609_30656_gb300 import clip
    from tests.test_norm_and_clip_abi import _clip, _entry
    assert _clip(clip._library(), _entry(**entry), **call) == 1
