"""Gradients of attention where grad_out's magnitude varies from session to session and from token to token (GPU).

The bounds are derived in attention_reference.py: relative to what a row's own sums hold, with nothing for fp16's
subnormal numbers. A scaled dS is rounded by 2^-25 there, against 2^-11 of the largest of its row: they are in reach of
one another only where the row's token of the largest |grad_out| gives the key a weight under 2^-20 or so."""

import pytest
import torch

from tests.attention_reference import check, reference, visible

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _run(lens, factors, dtype, heads, kv, dim, window, sinks, std=1.0):
    from paper_2609_30656_gb300 import window_attention as wa
    g = torch.Generator(device=DEV)
    g.manual_seed(7)
    T = sum(lens)
    q, k, v, go = ((torch.randn(T, n, dim, generator=g, device=DEV) * std).to(dtype) for n in (heads, kv, kv, heads))
    go = (go.float() / std * factors(T, g)).to(dtype)
    assert go.isfinite().all()
    off = torch.tensor([0] + lens, device=DEV).cumsum(0)
    error = torch.zeros(1, dtype=torch.int32, device=DEV)
    out, lse = wa.window_attention(q, k, v, off, window, sinks, stats=True)
    grads = wa.window_attention_backward(go, q, k, v, out, lse, off, window, sinks, error=error)
    assert error.item() == 0
    want = reference(q, k, v, visible(T, lens, window or T, sinks), dim ** -0.5, go)
    for got, name in zip(grads, ("dq", "dk", "dv")):
        check(got, want[name], name)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=str)
@pytest.mark.parametrize("lens", [[200, 150, 300, 40], [60] * 12, [700, 3, 5]], ids=str)
@pytest.mark.parametrize("window,sinks", [(None, 0), (50, 2)])
@pytest.mark.parametrize("powers", [(10, 0), (10, -4, -10), (-10, 3)], ids=str)
def test_sessions_of_other_magnitudes(powers, window, sinks, lens, dtype):
    """Sessions from 2^-20 to 2^20 beside one another: none loses digits by another's."""
    def factors(T, g):
        f = [2.0 ** powers[i % len(powers)] for i in range(len(lens))]
        return torch.cat([torch.full((n,), x, device=DEV) for n, x in zip(lens, f)])[:, None, None]
    _run(lens, factors, dtype, 4, 2, 64, window, sinks)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=str)
@pytest.mark.parametrize("window,sinks", [(None, 0), (50, 2), (200, 130), (1, 0), (131, 1)])
@pytest.mark.parametrize("late", [False, True])
def test_tokens_of_other_magnitudes(late, window, sinks, dtype):
    """A key's gradient counts the tokens that see it: those before it, or behind its window, take no digits from it."""
    def factors(T, g):
        f = torch.full((T,), 2.0 ** -10, device=DEV)
        f[[150, 290, 401, 600] if late else [0, 20, 131]] = 2.0 ** 10
        return f[:, None, None]
    _run([450, 260], factors, dtype, 2, 1, 72, window, sinks)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=str)
@pytest.mark.parametrize("power", [-12, -6, 6, 10])
def test_common_factors(power, dtype):
    """As loss scales bring them about."""
    _run([300, 129], lambda T, g: torch.full((1, 1, 1), 2.0 ** power, device=DEV), dtype, 4, 1, 64, 100, 3)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=str)
def test_heads_of_other_magnitudes_and_first_tokens_in_parts(dtype):
    """Heads that share a key are one sum; a long session's first tokens are summed in parts, each with its own scale."""
    def factors(T, g):
        f = torch.full((T, 4, 1), 2.0 ** -8, device=DEV)
        f[:, 1] = 2.0 ** -3
        f[4000:4100] *= 2.0 ** 10
        return f
    _run([5000, 90], factors, dtype, 4, 2, 64, 60, 3)
