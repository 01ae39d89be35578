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
