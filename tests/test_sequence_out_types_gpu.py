"""An output's type named twice: alike, or refused (GPU)."""

import pytest
import torch

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
DEV = "cuda:0"


@pytest.mark.parametrize("own", [F32, F16, BF16])
@pytest.mark.parametrize("named", [None, F32, F16, BF16])
def test_outputs(own, named):
    from paper_2609_30656_gb300 import muon, token_embedding as te
    table, tokens = torch.ones(20, 8, device=DEV), torch.arange(5, device=DEV)
    calls = [lambda: te.token_forward(table, tokens, out=torch.empty(5, 8, dtype=own, device=DEV), out_dtype=named),
             lambda: te.token_backward(table[:5], tokens, 20, out=torch.empty(20, 8, dtype=own, device=DEV), out_dtype=named),
             lambda: muon.newton_schulz(table, out=torch.empty(20, 8, dtype=own, device=DEV), out_dtype=named),
             lambda: muon.newton_schulz(table, out=torch.empty(8, 20, dtype=own, device=DEV).T, out_dtype=named)]
    for call in calls:
        if named in (None, own):
            assert call().dtype == own
        else:
            with pytest.raises(TypeError):
                call()


def test_types_without_an_output():
    from paper_2609_30656_gb300 import muon, token_embedding as te
    table, tokens = torch.ones(20, 8, device=DEV).half(), torch.arange(5, device=DEV)
    assert te.token_forward(table, tokens).dtype == F16
    assert te.token_backward(table[:5], tokens, 20).dtype == F32
    assert muon.newton_schulz(table).dtype == BF16
    for dtype in (F32, F16, BF16):
        assert te.token_backward(table[:5], tokens, 20, out_dtype=dtype).dtype == dtype
        assert muon.newton_schulz(table, out_dtype=dtype).dtype == dtype
        assert muon.newton_schulz(table.T, out_dtype=dtype).dtype == dtype
