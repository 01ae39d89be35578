"""Views of one buffer as inputs and results: those that share a value are refused, those that lie between one another are
taken (GPU)."""

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _gen(seed=1):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _rand(*shape, dtype=torch.bfloat16, seed=1):
    return torch.randn(shape, generator=_gen(seed), device=DEV).to(dtype)


def _offsets(*values):
    return torch.tensor(values, device=DEV)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=str)
def test_attention_into_its_inputs(dtype):
    from paper_2609_30656_gb300 import tbe, window_attention as wa
    room = _rand(302, 4, 64, dtype=dtype)
    q, k, v = room[:300], _rand(300, 4, 64, dtype=dtype, seed=2), _rand(300, 4, 64, dtype=dtype, seed=3)
    off = _offsets(0, 300)
    for out in (room[1:301], room[2:302]):
        with pytest.raises(tbe.CbTbeError):
            wa.window_attention(q, k, v, off, 50, out=out)
    out, lse = wa.window_attention(q, k, v, off, 50, stats=True)
    go = _rand(300, 4, 64, dtype=dtype, seed=4)
    one = torch.empty(600, 4, 64, dtype=dtype, device=DEV)
    for grads in ((one[:300], one[299:599], torch.empty_like(v)), (room[1:301], one[:300], one[300:])):
        with pytest.raises(tbe.CbTbeError):
            wa.window_attention_backward(go, q, k, v, out, lse, off, 50, grads=grads)
    with pytest.raises(tbe.CbTbeError):
        wa.window_attention_step(q, k[:, None], v[:, None], torch.ones(300, dtype=torch.int64, device=DEV), out=room[1:301])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=str)
def test_attention_between_its_inputs(dtype):
    """Everything in one buffer: heads side by side, tokens apart; all in another order of dimensions too."""
    from paper_2609_30656_gb300 import window_attention as wa
    T, H, KV, D = 300, 4, 2, 64
    off = _offsets(0, 120, 300)
    want = None
    for turned in (False, True):
        n = 5 * H + 4 * KV
        room = torch.zeros(n, T, D, dtype=dtype, device=DEV).transpose(0, 1) if turned else torch.zeros(T, n, D, dtype=dtype, device=DEV)
        q, out, go, dq, _, k, v, dk, dv = room.split([H, H, H, H, H, KV, KV, KV, KV], dim=1)
        for i, t in enumerate((q, k, v, go)):
            t.copy_(_rand(T, t.shape[1], D, dtype=dtype, seed=i))
        _, lse = wa.window_attention(q, k, v, off, 50, 2, out=out, stats=True)
        wa.window_attention_backward(go, q, k, v, out, lse, off, 50, 2, grads=(dq, dk, dv))
        got = [t.clone() for t in (out, dq, dk, dv)]
        apart = [t.contiguous() for t in (q, k, v, go)]
        if want is None:
            o, lse = wa.window_attention(*apart[:3], off, 50, 2, stats=True)
            want = [o, *wa.window_attention_backward(apart[3], *apart[:3], o, lse, off, 50, 2)]
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    # one new token: queries, results and caches as slices of one row for each session
    room = torch.zeros(7, 2 * H + 2 * 20 * KV, D, dtype=dtype, device=DEV)
    q, out, rest = room.split([H, H, 40 * KV], dim=1)
    k, v = rest.view(7, 2, 20, KV, D).unbind(1) if rest.is_contiguous() else rest.unflatten(1, (2, 20, KV)).unbind(1)
    for i, t in enumerate((q, k, v)):
        t.copy_(_rand(*t.shape, dtype=dtype, seed=i))
    lengths = torch.tensor([20, 3, 0, 1, 7, 19, 11], device=DEV)
    wa.window_attention_step(q, k, v, lengths, 5, 2, out=out)
    assert torch.equal(out, wa.window_attention_step(q.contiguous(), k.contiguous(), v.contiguous(), lengths, 5, 2))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
def test_layer_norm_into_its_inputs(dtype):
    from paper_2609_30656_gb300 import layer_norm as ln, tbe
    room = _rand(40, 100, dtype=dtype)
    x = room[:30]
    for out in (room[1:31], room[5:35]):
        with pytest.raises(tbe.CbTbeError):
            ln.layer_norm(x, out=out)
    y, mean, rstd = ln.layer_norm(x, stats=True)
    for out in (room[1:31], room[10:40]):
        with pytest.raises(tbe.CbTbeError):
            ln.layer_norm_backward(y, x, mean, rstd, out=out)
    # columns of one matrix
    pair = torch.zeros(30, 250, dtype=dtype, device=DEV)
    pair[:, 20:120] = x
    with pytest.raises(tbe.CbTbeError):
        ln.layer_norm(pair[:, 20:120], out=pair[:, 119:219])
    want = ln.layer_norm(pair[:, 20:120], out=torch.zeros_like(pair)[:, 120:220])  # in the same order: alike in alignment
    assert torch.equal(ln.layer_norm(pair[:, 20:120], out=pair[:, 120:220]), want)
    assert (pair[:, :20] == 0).all() and (pair[:, 220:] == 0).all() and torch.equal(pair[:, 20:120], x)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16, torch.float32], ids=str)
@pytest.mark.parametrize("dim,stride", [(41, 41), (1001, 1001), (1027, 1030), (72, 80), (7, 9), (4099, 4099), (18001, 18001)])
def test_layer_norm_in_place(dim, stride, dtype):
    """Odd rows of halves read whole pieces, with their neighbours' values, while those are written."""
    from paper_2609_30656_gb300 import layer_norm as ln
    w = _rand(dim, dtype=torch.float32, seed=3)

    def wide(t):
        room = torch.full((700, stride), 5.0, dtype=dtype, device=DEV)
        room[:, :dim] = t
        return room[:, :dim]

    def kept(t):  # what lies between the rows
        return (t.as_strided((700, stride), (stride, 1))[:, dim:] == 5).all()

    x, go = wide(_rand(700, dim, dtype=dtype)), wide(_rand(700, dim, dtype=dtype, seed=2))
    y, mean, rstd = ln.layer_norm(x, w, stats=True, out=wide(x))
    want = ln.layer_norm_backward(go, x, mean, rstd, w, out=wide(x))
    for _ in range(3):
        a = wide(x)
        assert torch.equal(ln.layer_norm(a, w, out=a), y) and kept(a)
        for which in (0, 1):
            views = wide(go), wide(x)
            got = ln.layer_norm_backward(*views, mean, rstd, w, out=views[which])
            assert all(torch.equal(s, t) for s, t in zip(got, want)) and kept(views[which])
