"""The next-item model with a block of attention: lookup, layer norm, attention, their backward passes, clipping and Muon
steps together, and the same model served an item at a time (GPU)."""

import math

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _loss(model, sessions, table, w1, w2, w_qkv, w_out, gain, shift):
    """The model in 64 bits on the host, nothing rounded."""
    D, H = model.dim, model.heads
    tok = sessions.long().cpu()
    x = table[tok[:, :-1]] * math.sqrt(D)
    n = torch.nn.functional.layer_norm(x, (D,), gain, shift)
    B, L = tok.shape[0], tok.shape[1] - 1
    q, k, v = (n @ w_qkv).view(B, L, 3, H, D // H).permute(2, 0, 3, 1, 4)
    at = torch.arange(L)
    back = at[:, None] - at[None, :]
    seen = (back >= 0) & ((back < model.window) | (at < model.sinks)[None, :])
    p = torch.softmax((q @ k.mT / math.sqrt(D // H)).masked_fill(~seen, -torch.inf), -1)
    x = x + (p @ v).permute(0, 2, 1, 3).reshape(B, L, D) @ w_out
    y = x + (x @ w1).relu() @ w2
    scores = y @ table.T / math.sqrt(D)
    return torch.nn.functional.cross_entropy(scores.reshape(-1, model.items), tok[:, 1:].reshape(-1)), scores


def _model(**kw):
    from paper_2609_30656_gb300 import next_item
    return next_item.NextItem(300, dim=64, hidden=96, seed=3, heads=4, window=5, sinks=1, **kw), next_item


def test_gradients_match_autograd_in_64_bits():
    model, next_item = _model()
    sessions = next_item.make_sessions(300, 7, 19, seed=5)
    loss, grads = model.loss_and_gradients(sessions)
    leaves = [t.detach().double().cpu().requires_grad_(True)
              for t in (model.table, model.w1, model.w2, model.w_qkv, model.w_out, model.gain, model.shift)]
    want, _ = _loss(model, sessions, *leaves)
    want.backward()
    # bf16: q, k, v, the weights, the output, its gradient, dS and the three gradients, each off by 2^-9 of the norm at
    # most in the mean (2^-8 at worst): 8 x 2^-8.
    assert abs(loss.item() - want.item()) < 8 * 2 ** -8
    assert len(grads) == 7
    for got, ref in zip(grads, leaves):
        assert (got.double().cpu() - ref.grad).norm() < 8 * 2 ** -8 * ref.grad.norm()


def test_a_step_clips_all_gradients_together():
    model, next_item = _model()
    other, _ = _model()
    sessions = next_item.make_sessions(300, 7, 19, seed=6)
    _, grads = model.loss_and_gradients(sessions)
    norm = math.sqrt(sum(t.double().square().sum().item() for t in grads))
    model.step(sessions, max_norm=norm / 4)
    other.step(sessions)
    # The first step's momentum is its gradient: a quarter of the other's, which is computed again the same way.
    # The factor is norm / 4 over norm + 1e-6, its products in fp32, a few roundings.
    for a, b in zip(model.momentum, other.momentum):
        assert b.norm() > 0 and (a - b / 4).norm() < (2 ** -20 + 1e-6 / norm) * b.norm()


def test_training_and_serving_run():
    from paper_2609_30656_gb300 import next_item
    losses = next_item.train(steps=3, items=200, sessions=4, length=9, heads=2, window=4, max_norm=1.0)
    assert len(losses) == 3 and all(math.isfinite(x) for x in losses)
    with pytest.raises(ValueError):
        next_item.Serving(next_item.NextItem(50), 1, 4)
    with pytest.raises(ValueError):
        next_item.NextItem(50, dim=64, heads=3)


def test_serving_gives_the_scores_of_the_whole_sessions():
    model, next_item = _model()
    sessions = next_item.make_sessions(300, 5, 30, seed=8)
    with torch.no_grad():
        _, want = _loss(model, sessions, *[t.double().cpu() for t in (model.table, model.w1, model.w2, model.w_qkv, model.w_out,
                                                                      model.gain, model.shift)])
    serving = next_item.Serving(model, 5, 30)
    for t in range(30):
        scores = serving.append(sessions[:, t]).double().cpu()
        assert (scores - want[:, t]).norm() < 8 * 2 ** -8 * want[:, t].norm()
    with pytest.raises(ValueError, match="capacity"):
        serving.append(sessions[:, 0])
    with pytest.raises(ValueError, match="every session"):
        next_item.Serving(model, 5, 30).append(sessions[:3, 0])
