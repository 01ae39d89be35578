"""The next-item model on batches without a token, and serving no session (GPU)."""

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("heads", [0, 4])
@pytest.mark.parametrize("sessions,items", [(0, 6), (4, 1), (0, 1)])
def test_no_tokens(sessions, items, heads):
    """No gradient, and a mean loss of nothing, with attention as without."""
    from paper_2609_30656_gb300 import next_item
    model = next_item.NextItem(50, dim=64, hidden=96, heads=heads, window=5)
    batch = torch.zeros(sessions, items, dtype=torch.int32, device=DEV)
    loss, grads = model.loss_and_gradients(batch)
    leaves = [model.table, model.w1, model.w2, *((model.w_qkv, model.w_out, model.gain, model.shift) if heads else ())]
    assert loss.isnan() and [g.shape for g in grads] == [t.shape for t in leaves]
    assert all((g == 0).all() for g in grads)
    model.step(batch, max_norm=1.0)
    assert all(t.isfinite().all() for t in leaves)


def test_serving_no_session():
    from paper_2609_30656_gb300 import next_item
    serving = next_item.Serving(next_item.NextItem(50, dim=64, hidden=96, heads=4), 0, 3)
    assert serving.append(torch.zeros(0, dtype=torch.int32, device=DEV)).shape == (0, 50)
