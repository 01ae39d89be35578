"""Adding into a gradient that ends where its allocation ends, at rows that a slab of columns reaches past (GPU)."""

import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.mark.parametrize("dim", [1, 24, 130, 257])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_the_last_row_of_the_tensor(dim, dtype):
    from paper_2609_30656_gb300 import token_embedding as te
    rows, n = 300, 4000
    tokens = torch.full((n,), rows - 1, device=DEV)
    tokens[:1000] = torch.arange(1000, device=DEV) % rows
    grad_out = torch.ones(n, dim, device=DEV)
    grad = torch.ones(rows, dim, device=DEV).to(dtype)
    te.token_backward(grad_out, tokens, rows, scale=0.25, out=grad, accumulate=True)
    count = torch.bincount(tokens, minlength=rows).float().unsqueeze(1)  # whole numbers of quarters: exact in fp32
    assert torch.equal(grad, (1 + 0.25 * count).expand(rows, dim).to(dtype))
