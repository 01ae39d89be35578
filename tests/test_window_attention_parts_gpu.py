"""First tokens of long sessions, which every later token sees: their gradients are summed in parts (GPU).

The bounds are derived in attention_reference.py."""

import pytest
import torch

from tests.attention_reference import check, reference, visible
from tests.test_window_attention_gpu import run_and_check

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=str)
@pytest.mark.parametrize("lens,begin,window,sinks,dim", [
    ([5000], 0, 40, 3, 64), ([4200, 30, 4500], 126, 300, 5, 64), ([6000], 0, 1, 1, 128), ([10, 4300], 0, 129, 140, 72)], ids=str)
def test_long_sessions(lens, begin, window, sinks, dim, dtype):
    first = run_and_check(lens, 2, 1, dim, dtype, window, sinks, begin=begin, seed=len(lens))
    again = run_and_check(lens, 2, 1, dim, dtype, window, sinks, begin=begin, seed=len(lens))
    assert all(torch.equal(a, b) for a, b in zip(first[-1], again[-1]))


def test_more_first_tokens_than_there_is_room_for():
    """Every tile of keys is seen to the end: some are summed in parts, the others in one piece."""
    from paper_2609_30656_gb300 import window_attention as wa
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    T, heads = 6000, 32
    q, k, v, go = (torch.randn(T, heads, 64, generator=g, device=DEV).to(torch.bfloat16) for _ in range(4))
    off = torch.tensor([0, T], device=DEV)
    out, lse = wa.window_attention(q, k, v, off, 10, T, stats=True)
    grads = wa.window_attention_backward(go, q, k, v, out, lse, off, 10, T)
    again = wa.window_attention_backward(go, q, k, v, out, lse, off, 10, T)
    assert all(torch.equal(a, b) for a, b in zip(grads, again))
    seen = visible(T, [T], 10, T)
    for h in (0, 31):
        part = [t[:, h:h + 1] for t in (q, k, v)]
        want = reference(*part, seen, 0.125, go[:, h:h + 1])
        for got, name in zip(grads, ("dq", "dk", "dv")):
            check(got[:, h:h + 1], want[name], name)


def test_infinities_elsewhere():
    from paper_2609_30656_gb300 import window_attention as wa
    g = torch.Generator(device=DEV)
    g.manual_seed(2)
    lens = [4500, 100]
    q, k, v, go = (torch.randn(4600, 1, 64, generator=g, device=DEV).to(torch.bfloat16) for _ in range(4))
    off = torch.tensor([0, 4500, 4600], device=DEV)
    want = reference(q, k, v, visible(4600, lens, 20, 2), 0.125, go)
    for t in (q, k, v, go):
        t[4500:] = float("nan")
    out, lse = wa.window_attention(q, k, v, off, 20, 2, stats=True)
    grads = wa.window_attention_backward(go, q, k, v, out, lse, off, 20, 2)
    for got, name in zip((out, *grads), ("out", "dq", "dk", "dv")):
        check(got[:4500], (want[name][0][:4500], want[name][1][:4500]), name)
