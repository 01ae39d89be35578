"""The calls for sequence models together: a next-item model's gradients and its training (GPU)."""

import math

import pytest
import torch

pytestmark = pytest.mark.gpu


def test_gradients_match_autograd_in_64_bits():
    from paper_2609_30656_gb300 import next_item
    model = next_item.NextItem(300, dim=40, hidden=96, seed=3)
    sessions = next_item.make_sessions(300, 7, 11, seed=5)
    loss, grads = model.loss_and_gradients(sessions)
    e, w1, w2 = (t.detach().double().cpu().requires_grad_(True) for t in (model.table, model.w1, model.w2))
    tok = sessions.long().cpu()
    x = e[tok[:, :-1]] * math.sqrt(40)
    y = x + (x @ w1).relu() @ w2
    scores = (y @ e.T / math.sqrt(40)).reshape(-1, 300)
    want = torch.nn.functional.cross_entropy(scores, tok[:, 1:].reshape(-1))
    want.backward()
    # fp32 throughout: sums of at most 300 products, four deep
    assert abs(loss.item() - want.item()) < 1e-5
    for got, ref in zip(grads, (e.grad, w1.grad, w2.grad)):
        assert (got.double().cpu() - ref).norm() < 1e-5 * ref.norm()


def test_training_learns_the_successors():
    from paper_2609_30656_gb300 import next_item
    losses = next_item.train(steps=120, items=500, sessions=32, length=40)
    # A model that knew only how popular items are would stay near the entropy of the clicks,
    # over 5; the successors are worth most of that.
    assert losses[0] > 5.5
    assert sum(losses[-10:]) / 10 < 3.6
