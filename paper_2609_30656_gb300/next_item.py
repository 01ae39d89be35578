"""Next-item prediction over sessions, trained with this library's calls for sequence models.

    python -m paper_2609_30656_gb300.next_item --steps 200

A user's session is a sequence of item ids, and the model scores the item that follows each:

    x = sqrt(D) E[items]                  token_forward
    h = relu(x W1),  y = x + h W2         two matrices, fp32 masters
    scores = y E^T / sqrt(D)              the table is the output head too (tied)

The gradient of the table has two parts: the head's, a dense product, and the lookup's, which
token_backward adds into it. The matrices are stepped by muon_step, the table by
row-wise Adagrad, the rule that the library applies to its pooled tables. Sessions are synthetic:
most items have one successor that follows them four times out of five, the rest of the clicks
are popular items (Zipf).
"""

from __future__ import annotations

import argparse
import math

import torch

from . import muon, token_embedding as te


class NextItem:
    """The model and its optimizer states, on one CUDA device."""

    def __init__(self, items: int, dim: int = 128, hidden: int = 512, seed: int = 0, device="cuda:0"):
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        self.items, self.dim = items, dim

        def normal(*shape, std):
            return torch.randn(shape, generator=g, device=device) * std

        self.table = normal(items, dim, std=dim ** -0.5)
        self.w1 = normal(dim, hidden, std=dim ** -0.5)
        self.w2 = normal(hidden, dim, std=0.1 * hidden ** -0.5)
        self.momentum = [torch.zeros_like(self.w1), torch.zeros_like(self.w2)]
        self.row_state = torch.zeros(items, 1, device=device)

    def loss_and_gradients(self, sessions: torch.Tensor):
        """Mean cross entropy of the next items of sessions [B, L + 1], and the gradients of
        (table, w1, w2)."""
        inputs, targets = sessions[:, :-1], sessions[:, 1:].reshape(-1)
        scale = math.sqrt(self.dim)
        x = te.token_forward(self.table, inputs, scale=scale).view(-1, self.dim)
        a = x @ self.w1
        h = a.relu()
        y = x + h @ self.w2
        scores = y @ self.table.T / scale
        log_p = scores.log_softmax(1)
        n = targets.numel()
        loss = -log_p.gather(1, targets.long().unsqueeze(1)).mean()
        d_scores = log_p.exp()
        d_scores.scatter_add_(1, targets.long().unsqueeze(1), torch.full((n, 1), -1.0, device=x.device))
        d_scores /= n * scale
        d_table = d_scores.T @ y  # the head's part
        d_y = d_scores @ self.table
        d_a = (d_y @ self.w2.T) * (a > 0)
        d_x = d_y + d_a @ self.w1.T
        te.token_backward(d_x.view(*inputs.shape, self.dim), inputs, self.items, scale=scale, out=d_table,
                          accumulate=True)
        return loss, (d_table, x.T @ d_a, h.T @ d_y)

    def step(self, sessions: torch.Tensor, lr: float = 0.02, table_lr: float = 0.1) -> torch.Tensor:
        """One training step; returns the loss before it (on the device)."""
        loss, (d_table, d_w1, d_w2) = self.loss_and_gradients(sessions)
        for w, d, m in ((self.w1, d_w1, self.momentum[0]), (self.w2, d_w2, self.momentum[1])):
            muon.muon_step(w, d, m, lr=lr, weight_decay=0.01, adjust="spectral")
        self.row_state += d_table.square().mean(1, keepdim=True)
        self.table -= table_lr * d_table / (self.row_state.sqrt() + 1e-8)
        return loss


def make_sessions(items: int, sessions: int, length: int, seed: int, device="cuda:0") -> torch.Tensor:
    """Synthetic sessions [sessions, length + 1] of int32 items, with the successors of one world (seed-independent)."""
    world = torch.Generator(device=device)
    world.manual_seed(1)
    successor = torch.randperm(items, generator=world, device=device)
    popular = torch.arange(1, items + 1, device=device, dtype=torch.float64).reciprocal()
    g = torch.Generator(device=device)
    g.manual_seed(seed)
    noise = torch.multinomial(popular, sessions * (length + 1), replacement=True, generator=g).view(sessions, -1)
    follow = torch.rand(sessions, length + 1, generator=g, device=device) < 0.8
    out = noise.clone()
    for t in range(1, length + 1):
        out[:, t] = torch.where(follow[:, t], successor[out[:, t - 1]], noise[:, t])
    return out.to(torch.int32)


def train(steps: int = 200, items: int = 2000, sessions: int = 64, length: int = 50, seed: int = 0) -> list[float]:
    model = NextItem(items, seed=seed)
    losses = [model.step(make_sessions(items, sessions, length, seed=1000 + k)) for k in range(steps)]
    return torch.stack(losses).tolist()


def main() -> None:
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--steps", type=int, default=200)
    p.add_argument("--items", type=int, default=2000)
    a = p.parse_args()
    losses = train(a.steps, a.items)
    for k in range(0, len(losses), max(1, len(losses) // 10)):
        print(f"step {k:5d}  loss {losses[k]:.4f}")
    print(f"step {len(losses) - 1:5d}  loss {losses[-1]:.4f}  (uniform {math.log(a.items):.4f})")


if __name__ == "__main__":
    main()
