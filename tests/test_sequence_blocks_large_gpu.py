"""Layer norm and attention where places pass 32 bits (GPU): the last rows of a large call against a call on them
alone, or against 64 bits."""

import pytest
import torch

from tests.attention_reference import check, reference, visible

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


@pytest.fixture(autouse=True)
def _free():
    yield
    torch.cuda.empty_cache()


def test_layer_norm_rows():
    from paper_2609_30656_gb300 import layer_norm as ln
    rows, dim = (1 << 20) + 4096, 2048  # 2.2e9 values
    x, dy = (torch.zeros(rows, dim, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    for t in (x, dy):
        t[-64:] = torch.randn(64, dim, generator=_gen(1), device=DEV)
    y, mean, rstd = ln.layer_norm(x, stats=True)
    few, few_mean, few_rstd = ln.layer_norm(x[-64:].clone(), stats=True)
    assert torch.equal(y[-64:], few) and torch.equal(mean[-64:], few_mean) and torch.equal(rstd[-64:], few_rstd)
    dx = ln.layer_norm_backward(dy, x, mean, rstd, out=dy)[0]
    assert torch.equal(dx[-64:], ln.layer_norm_backward(x[-64:].clone(), x[-64:].clone(), few_mean, few_rstd)[0])


@pytest.mark.parametrize("sessions,capacity,window", [(40, 500000, 900), (1, 17_000_000, 900), (40, 500000, None)])
def test_step_caches(sessions, capacity, window):
    """The keys' places pass 32 bits over the sessions, or within one."""
    from paper_2609_30656_gb300 import window_attention as wa
    g = _gen(2)
    k, v = (torch.zeros(sessions, capacity, 1, 128, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    last = 1500
    for t in (k, v):
        t[-1, -last:] = torch.randn(last, 1, 128, generator=g, device=DEV)
    q = (8 * torch.randn(sessions, 4, 128, generator=g, device=DEV)).to(torch.bfloat16)  # few keys have all the weight
    lengths = torch.full((sessions,), capacity, device=DEV)
    if window is None:  # all others begin empty: the last keys are the only ones
        lengths[:-1] = 0
        k[-1, :last], v[-1, :last] = k[-1, -last:].clone(), v[-1, -last:].clone()
        lengths[-1] = last
    out = wa.window_attention_step(q, k, v, lengths, window)
    alone = wa.window_attention_step(q[-1:], k[-1:, -last:].clone(), v[-1:, -last:].clone(), lengths.new_full((1,), last), window)
    # The splits may differ. Both are off by the rounding of P (2^-8 of a mean of |v|) and their own (2^-8); the rest is fp32.
    most = v[-1].abs().max().item()
    assert (out[-1].float() - alone[0].float()).abs().max() <= 4 * 2 ** -8 * most * (1 + 2 ** -6)
    assert alone.float().abs().max() > most / 4


def _check_one_session(tokens, heads, dim, begin, last, dtype, runs=1):
    """A session of `last` tokens from `begin` on in a batch that holds nothing else."""
    from paper_2609_30656_gb300 import window_attention as wa
    g = _gen(3)
    q, k, v, go = (torch.zeros(tokens, heads, dim, dtype=dtype, device=DEV) for _ in range(4))
    here = slice(begin, begin + last)
    for t in (q, k, v, go):
        t[here] = torch.randn(last, heads, dim, generator=g, device=DEV)
    want = reference(*[t[here].clone() for t in (q, k, v)], visible(last, [last], 100, 0), dim ** -0.5, go[here].clone())
    off = torch.tensor([begin, begin + last], device=DEV)
    error = torch.zeros(1, dtype=torch.int32, device=DEV)
    for _ in range(runs):
        out, lse = wa.window_attention(q, k, v, off, 100, stats=True, error=error)
        grads = wa.window_attention_backward(go, q, k, v, out, lse, off, 100, error=error)
        assert error.item() == 0
        check(lse[:, here], want["lse"], "lse")
        assert (lse[:, :begin] == -torch.inf).all() and (lse[:, begin + last:] == -torch.inf).all()
        for got, name in zip((out, *grads), ("out", "dq", "dk", "dv")):
            check(got[here], want[name], name)
            assert (got[:begin] == 0).all() and (got[begin + last:] == 0).all()


@pytest.mark.parametrize("dim", [128, 63])
def test_packed_attention(dim):
    tokens = 17_000_000 * 128 // (128 * dim) // 128 * 128
    _check_one_session(tokens, 128, dim, tokens - 256, 256, torch.bfloat16)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=str)
@pytest.mark.parametrize("begin,behind", [(60000, 0), (0, 60000), (30000, 30000), (100, 20000)])
@pytest.mark.parametrize("dim", [64, 128])
def test_a_session_among_many_unused_tokens(begin, behind, dim, dtype):
    """Blocks of threads come through hundreds of tiles without a key, one after the other."""
    _check_one_session(begin + 900 + behind, 24, dim, begin, 900, dtype, runs=6)
