"""Token lookups into outputs whose rows lie in turn, or between one another's; refusals of rows in one place; infinite
scales (GPU)."""

import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def te():
    from paper_2609_30656_gb300 import token_embedding
    return token_embedding


def _randn(shape, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.randn(shape, generator=g, device=DEV)


@pytest.mark.parametrize("dim", [64, 63])
@pytest.mark.parametrize("strides", [(1, 5), (13, 4), (20, 1)])  # in rows: in turn, between one another, one after the other
def test_rows_apart_in_any_way(dim, strides):
    table, tokens = _randn((50, dim), 1), torch.arange(15, device=DEV).view(3, 5) * 3
    flat = torch.full((60 * dim,), 7.0, device=DEV)
    out = flat.as_strided((3, 5, dim), (strides[0] * dim, strides[1] * dim, 1))
    te().token_forward(table, tokens, out=out)
    assert torch.equal(out, table[tokens])
    out.fill_(7.0)
    assert bool((flat == 7.0).all())


def test_rows_in_one_place_are_refused():
    from paper_2609_30656_gb300 import tbe
    table, tokens = _randn((50, 8), 2), torch.arange(4, device=DEV).view(2, 2)
    with pytest.raises(tbe.CbTbeError):
        te().token_forward(table, tokens, out=torch.zeros(32, device=DEV).as_strided((2, 2, 8), (8, 8, 1)))


@pytest.mark.parametrize("dim", [1024, 64, 12, 6, 63])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("scale", [float("inf"), -float("inf"), 2.0])
def test_tokens_out_of_range_give_zeros_whatever_the_scale(dim, dtype, scale):
    table = _randn((50, dim), 3).to(dtype)
    table[7] = 0
    tokens = torch.tensor([[3, -1, 50, 7], [2 ** 40, 8, -2 ** 40, 49]], device=DEV)
    got = te().token_forward(table, tokens, scale=scale)
    inside = (tokens >= 0) & (tokens < 50)
    assert not got[~inside].any() and not got[~inside].isnan().any()
    want = (table[tokens[inside]].float() * scale).to(dtype)
    assert torch.equal(got[inside].nan_to_num(9.0), want.nan_to_num(9.0))  # 0 * inf is NaN, as multiplied
