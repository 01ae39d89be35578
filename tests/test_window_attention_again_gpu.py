"""Values that are not finite in attention over long sessions and shared heads: what does not see them is right, all of
the results are written, and no wait runs out, however many rows are computed again (GPU).

The bounds are derived in attention_reference.py."""

import pytest
import torch

from tests.attention_reference import check, half, reference, visible

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HALVES = [torch.float16, torch.bfloat16]


def _inputs(T, heads, kv, dim, dtype, seed=1):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return [torch.randn(T, n, dim, generator=g, device=DEV).to(dtype) for n in (heads, kv, kv, heads)]


def _both(q, k, v, go, lens, window, sinks, take=None):
    """(out, lse, dq, dk, dv); what is not written would keep its 77s. take(out, lse): what the backward pass gets of them."""
    from paper_2609_30656_gb300 import window_attention as wa
    off = torch.tensor([0] + lens, device=DEV).cumsum(0)
    error = torch.zeros(1, dtype=torch.int32, device=DEV)
    out, *grads = (torch.full_like(t, 77) for t in (q, q, k, v))
    _, lse = wa.window_attention(q, k, v, off, window, sinks, out=out, stats=True, error=error)
    wa.window_attention_backward(go, q, k, v, *(take(out, lse) if take else (out, lse)), off, window, sinks, grads=grads, error=error)
    assert error.item() == 0
    assert all((t != 77).all() for t in (out, *grads))  # as good as no value of these is 77 by itself
    return out, lse, *grads


def _check(got, want, where, what):
    check(got[where], (want[0][where], want[1][where]), what)


@pytest.mark.parametrize("dtype", HALVES, ids=str)
@pytest.mark.parametrize("heads,kv,dim,window,sinks", [(8, 1, 64, None, 0), (4, 2, 128, 700, 3), (2, 2, 72, None, 0)])
@pytest.mark.parametrize("before,behind", [(300, 500), (0, 70), (130, 0)])
def test_a_session_beside_others_of_nan(before, behind, heads, kv, dim, window, sinks, dtype):
    n = 4000
    T = before + n + behind
    q, k, v, go = _inputs(T, heads, kv, dim, dtype)
    lens = [before, n, behind]
    want = reference(q, k, v, visible(T, lens, window or T, sinks), dim ** -0.5, go)
    for t in (q, k, v, go):
        t[:before] = float("nan")
        t[before + n:] = float("nan")
    out, lse, *grads = _both(q, k, v, go, lens, window, sinks)
    here = slice(before, before + n)
    for got, name in zip((out, *grads), ("out", "dq", "dk", "dv")):
        _check(got, want[name], here, name)
        assert got[:before].isnan().all() and got[before + n:].isnan().all()
    check(lse[:, here], (want["lse"][0][:, here], want["lse"][1][:, here]), "lse")


@pytest.mark.parametrize("dtype", HALVES, ids=str)
@pytest.mark.parametrize("at", [5, 1400, 2999])
@pytest.mark.parametrize("heads,kv,window,sinks", [(8, 2, None, 0), (4, 4, 500, 3), (3, 1, 100, 150)])
def test_an_infinite_value(heads, kv, window, sinks, at, dtype):
    """Of the tokens that see it one component is infinite; all else is right."""
    T, dim, c = 3000, 64, 17
    q, k, v, go = _inputs(T, heads, kv, dim, dtype)
    v[at, 0, c] = 0
    seen = visible(T, [T], window or T, sinks)
    want = reference(q, k, v, seen, dim ** -0.5)
    v[at, 0, c] = torch.inf
    out, lse, *_ = _both(q, k, v, go, [T], window, sinks)
    check(lse, want["lse"], "lse")
    met = torch.zeros(T, heads, dim, dtype=torch.bool, device=DEV)
    met[:, :heads // kv, c] = seen[:, at, None]
    _check(out, want["out"], ~met, "out")
    assert (~out[met].isfinite()).all()


@pytest.mark.parametrize("dtype", HALVES, ids=str)
@pytest.mark.parametrize("at", [5, 1400, 2999])
@pytest.mark.parametrize("heads,kv,window,sinks", [(8, 2, None, 0), (4, 4, 500, 3), (3, 1, 100, 150)])
def test_an_infinite_gradient(heads, kv, window, sinks, at, dtype):
    """As a loss scale that is too large gives: what does not come from it is right."""
    T, dim, c, h = 3000, 64, 17, 1
    q, k, v, go = _inputs(T, heads, kv, dim, dtype)
    go[at, h, c] = 0
    seen = visible(T, [T], window or T, sinks)
    want = reference(q, k, v, seen, dim ** -0.5, go)
    go[at, h, c] = -torch.inf
    _, _, dq, dk, dv = _both(q, k, v, go, [T], window, sinks)
    y = h // (heads // kv)
    met = torch.zeros(T, heads, dim, dtype=torch.bool, device=DEV)
    met[at, h] = True
    _check(dq, want["dq"], ~met, "dq")
    assert (~dq[met].isfinite()).any()
    met = torch.zeros(T, kv, dim, dtype=torch.bool, device=DEV)
    met[:, y] = seen[at, :, None]
    _check(dk, want["dk"], ~met, "dk")
    assert not dk[met].isfinite().any()
    met[:, y] = False
    met[:, y, c] = seen[at]
    _check(dv, want["dv"], ~met, "dv")
    assert not dv[met].isfinite().any()


def test_a_long_session_whose_every_key_is_computed_again():
    """One infinity in the last token's gradient: 40000 keys, each over 8 heads of up to 40000 tokens. The other components
    of dV are those of the clean run but for roundings: of the weights (half a step each, of a sum of random gradients that
    much of its norm; not where computed again) and of the results of both."""
    T, heads, dim, c = 40000, 8, 64, 3
    q, k, v, go = _inputs(T, heads, 1, dim, torch.float16)
    clean = _both(q, k, v, go, [T], None, 0)[-1]
    go[-1, 5, c] = torch.inf
    out, lse, dq, dk, dv = _both(q, k, v, go, [T], None, 0)
    assert not dv[..., c].isfinite().any() and not dk.isfinite().any()
    assert dq[:-1].isfinite().all()
    others = torch.arange(dim, device=DEV) != c
    a, b = dv[..., others].double(), clean[..., others].double()
    assert a.isfinite().all() and (a - b).norm() < 4 * half(torch.float16) * b.norm()


def test_replays_begin_anew():
    """A captured call notes its own rows each time."""
    from paper_2609_30656_gb300 import window_attention as wa
    T = 900
    q, k, v, go = _inputs(T, 4, 2, 64, torch.float16)
    off = torch.tensor([0, 400, T], device=DEV)

    def both():
        out, lse = wa.window_attention(q, k, v, off, 200, 4, stats=True)
        return (out, lse, *wa.window_attention_backward(go, q, k, v, out, lse, off, 200, 4))

    clean = both()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both()
    kept = [t.clone() for t in (q, k, v, go)]
    for broken in (False, True, True, False, True, False):
        for t, a in zip((q, k, v, go), kept):
            t.copy_(a)
            if broken:
                t[350:420] = float("nan")
        graph.replay()
        want = both()
        assert all(torch.equal(a.nan_to_num(55), b.nan_to_num(55)) for a, b in zip(got, want))
        if not broken:
            assert all(torch.equal(a, b) for a, b in zip(got, clean))


@pytest.mark.parametrize("dtype", HALVES, ids=str)
@pytest.mark.parametrize("heads,kv,dim,window,sinks", [(2, 1, 64, None, 0), (4, 4, 128, None, 0), (8, 2, 72, 600, 5), (3, 3, 64, 40, 200)])
@pytest.mark.parametrize("before,behind", [(300, 500), (0, 100), (130, 0)])
def test_only_rows_in_reach_of_another_session_are_computed_again(before, behind, heads, kv, dim, window, sinks, dtype):
    """Tiles that hold no token of a session of NaNs have the bits that they have beside one of numbers: their products meet
    none. The first keys and queries of a tile's block of 128, or pair of them, may lie beside a neighbour's. The session's
    rows there have other roundings, so both backward passes get one forward pass's."""
    n = 4000
    T = before + n + behind
    q, k, v, go = _inputs(T, heads, kv, dim, dtype)
    lens = [before, n, behind]
    clean = _both(q, k, v, go, lens, window, sinks)
    for t in (q, k, v, go):
        t[:before] = float("nan")
        t[before + n:] = float("nan")

    def take(out, lse):
        out, lse = out.clone(), lse.clone()
        out[before:before + n], lse[:, before:before + n] = clean[0][before:before + n], clean[1][:, before:before + n]
        return out, lse

    broken = _both(q, k, v, go, lens, window, sinks, take)
    inner = slice(-(-before // 256) * 256, (before + n) // 256 * 256 - 256)
    for a, b in zip(clean[:1] + clean[2:], broken[:1] + broken[2:]):
        assert torch.equal(a[inner], b[inner])


@pytest.mark.parametrize("dtype", HALVES, ids=str)
def test_unused_tokens_hold_anything(dtype):
    """NaNs behind the last session and before the first one, as of a buffer that is larger than the batch, and beside the
    first tokens that all see."""
    q, k, v, go = _inputs(3000, 4, 2, 64, dtype)
    from paper_2609_30656_gb300 import window_attention as wa
    off = torch.tensor([100, 2100, 2500], device=DEV)

    def both(take=None):
        out, lse = wa.window_attention(q, k, v, off, 50, 4, stats=True)
        return (out, lse.T, *wa.window_attention_backward(go, q, k, v, *(take or (out, lse)), off, 50, 4))

    clean = both()
    for t in (q, k, v, go):
        t[:100] = t[2500:] = float("nan")
    broken = both((clean[0], clean[1].T))
    for a, b in zip(clean, broken):
        assert torch.equal(a[256:2304], b[256:2304])
        assert torch.equal(a[:100], b[:100]) and torch.equal(a[2500:], b[2500:])
    # Of a session's keys 4 .. 127 the far tokens see none, whatever those hold.
    v[150] = torch.inf
    k[150] = torch.nan
    far = both()
    assert torch.equal(far[0][512:2048], clean[0][512:2048])
    assert torch.equal(far[2][512:2048], clean[2][512:2048])
