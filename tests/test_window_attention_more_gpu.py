"""Windowed attention: a session among others at many places, infinities behind the mask in every type, caches at odd
places, one new token in a graph (GPU). The bounds are derived in attention_reference.py."""

import pytest
import torch

from tests.attention_reference import check, reference, visible
from tests.test_window_attention_gpu import run_and_check, step_reference

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
ALL = [torch.bfloat16, torch.float16, torch.float32]


def _wa():
    from paper_2609_30656_gb300 import window_attention
    return window_attention


def _rand(g, *shape, dtype):
    return torch.randn(shape, generator=g, device=DEV).to(dtype)


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


@pytest.mark.parametrize("dtype", ALL, ids=str)
@pytest.mark.parametrize("before", [[], [1], [100], [127], [128, 3], [300, 0, 29], [511]], ids=str)
def test_a_session_at_any_place_of_the_batch(before, dtype):
    """Its results are those that it has alone, and twice the same bits."""
    wa = _wa()
    n = 333
    one = [_rand(_gen(1), n, h, 64, dtype=dtype) for h in (4, 2, 2, 4)]
    want = reference(*one[:3], visible(n, [n], 90, 3), 0.125, one[3])
    lens = [*before, n, 77]
    at = sum(before)
    q, k, v, go = (_rand(_gen(2), sum(lens), h, 64, dtype=dtype) for h in (4, 2, 2, 4))
    for t, a in zip((q, k, v, go), one):
        t[at:at + n] = a
    off = torch.tensor([0, *lens], device=DEV).cumsum(0)

    def both():
        out, lse = wa.window_attention(q, k, v, off, 90, 3, stats=True)
        return (out, lse, *wa.window_attention_backward(go, q, k, v, out, lse, off, 90, 3))

    got = both()
    assert all(torch.equal(a, b) for a, b in zip(got, both()))
    for t, name in zip((got[0], *got[2:]), ("out", "dq", "dk", "dv")):
        check(t[at:at + n], want[name], name)
    check(got[1][:, at:at + n], want["lse"], "lse")


@pytest.mark.parametrize("dtype", ALL, ids=str)
@pytest.mark.parametrize("kind", ["nan", "inf"])
@pytest.mark.parametrize("dim,window,sinks", [(64, 30, 0), (128, None, 0), (72, 50, 5)])
def test_behind_the_mask(dim, window, sinks, kind, dtype):
    """NaNs or infinities of the session between take nothing from those beside it."""
    wa = _wa()
    g = _gen(12)
    lens = [100, 90, 320]
    q, k, v, go = (_rand(g, 510, h, dim, dtype=dtype) for h in (4, 2, 2, 4))
    want = reference(q, k, v, visible(510, lens, window or 510, sinks), dim ** -0.5, go)
    for t in (q, k, v, go):
        t[100:190] = float(kind)
    off = torch.tensor([0, 100, 190, 510], device=DEV)
    error = torch.zeros(1, dtype=torch.int32, device=DEV)
    out, lse = wa.window_attention(q, k, v, off, window, sinks, stats=True, error=error)
    grads = wa.window_attention_backward(go, q, k, v, out, lse, off, window, sinks, error=error)
    apart = torch.ones(510, dtype=torch.bool, device=DEV)
    apart[100:190] = False
    for got, name in zip((out, *grads), ("out", "dq", "dk", "dv")):
        check(got[apart], (want[name][0][apart], want[name][1][apart]), name)
        assert got[~apart].isnan().any()
    check(lse[:, apart], (want["lse"][0][:, apart], want["lse"][1][:, apart]), "lse")
    assert error.item() == 0


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=str)
@pytest.mark.parametrize("dim", [64, 63, 128])
def test_step_over_caches_at_odd_places(dim, dtype):
    """Rows that do not begin at 16 bytes go key by key: the same attention."""
    wa = _wa()
    g = _gen(62)
    lens = [50, 7, 64, 0]
    q = _rand(g, 4, 4, dim, dtype=dtype)
    k, v = (_rand(g, 4, 64, 2, dim, dtype=dtype) for _ in range(2))
    wide = torch.full((4, 64, 5, dim + 9), float("nan"), dtype=dtype, device=DEV)
    odd_k, odd_v = wide[:, :, 1:3, 1:dim + 1], wide[:, :, 3:5, 5:dim + 5]
    odd_k.copy_(k)
    odd_v.copy_(v)
    n = torch.tensor(lens, device=DEV)
    for window, sinks in ((20, 2), (None, 0)):
        want = step_reference(q, k, v, lens, window or 100, sinks, dim ** -0.5)
        check(wa.window_attention_step(q, odd_k, odd_v, n, window, sinks), want)
        check(wa.window_attention_step(q, k, odd_v, n, window, sinks), want)


@pytest.mark.parametrize("dtype", ALL, ids=str)
def test_step_by_step_in_a_graph(dtype):
    """One captured step, replayed for every token over a cache that grows, gives what the packed call gives."""
    wa = _wa()
    T, H, KV, D = 70, 4, 2, 64
    q, k, v, go, off, out, *_ = run_and_check([T], H, KV, D, dtype, 25, 3, seed=63)
    want = reference(q, k, v, visible(T, [T], 25, 3), D ** -0.5)["out"]
    caches = torch.zeros(2, 1, 80, KV, D, dtype=dtype, device=DEV)
    new = [torch.zeros_like(t[:1]) for t in (q, k, v)]
    n = torch.zeros(1, dtype=torch.int64, device=DEV)
    row = torch.zeros(1, dtype=torch.int64, device=DEV)

    def step():
        for i in (0, 1):
            caches[i, row, n] = new[1 + i]
        n.add_(1)
        return wa.window_attention_step(new[0], caches[0], caches[1], n, 25, 3)

    step()
    n.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    n.zero_()
    for t in range(T):
        for a, b in zip(new, (q, k, v)):
            a.copy_(b[t:t + 1])
        graph.replay()
        check(got[0], (want[0][t], want[1][t]), t)
    assert n.item() == T
