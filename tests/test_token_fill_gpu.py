"""The gradient's zeros, written beside the sort, call after call in one workspace (GPU)."""

import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


# 17 bits of keys in one tile of the sort and in several, one pass, and more tiles than the short passes take.
@pytest.mark.parametrize("n,rows,dim", [(3000, 70_000, 64), (30_000, 70_000, 64), (5000, 200, 256), (400_000, 20_000, 8)])
def test_calls_in_turn_leave_nothing_of_each_other(n, rows, dim):
    from paper_2609_30656_gb300 import token_embedding as te
    g = torch.Generator(device=DEV)
    g.manual_seed(n)
    calls = []
    for _ in range(3):
        tokens = torch.randint(0, rows, (1,), generator=g, device=DEV) + torch.randint(0, max(1, rows // 3), (n,), generator=g,
                                                                                      device=DEV)
        tokens = tokens % rows
        grad_out = torch.randn(n, dim, generator=g, device=DEV)
        want = te.token_backward(grad_out, tokens, rows)
        touched = torch.zeros(rows, dtype=torch.bool, device=DEV)
        touched[tokens] = True
        assert not want[~touched].any() and want[touched].any(1).all()
        calls.append((grad_out, tokens, want))
    out = [torch.full((rows, dim), 7.0, device=DEV) for _ in range(3)]
    torch.cuda.synchronize()
    for _ in range(30):
        for k, (grad_out, tokens, _) in enumerate(calls):
            out[k].fill_(7.0)
            te.token_backward(grad_out, tokens, rows, out=out[k])
    for k in range(3):
        assert torch.equal(out[k], calls[k][2])
