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

With heads, a block of attention stands before the two matrices, so that a position knows more than its own item:

    n = layer_norm(x),  q, k, v = n W (rounded to bf16),  x <- x + window_attention(q, k, v) W'

and with max_norm all gradients together are clipped before the steps (clip_grad_norm). ``Serving``
scores sessions an item at a time over a cache of keys and values (window_attention_step).

    python -m paper_2609_30656_gb300.next_item --steps 200 --heads 4 --window 32 --sinks 2 --max-norm 1.0
"""

from __future__ import annotations

import argparse
import math

import torch

from . import clip, layer_norm as ln, muon, token_embedding as te, window_attention as wa


class NextItem:
    """The model and its optimizer states, on one CUDA device; heads > 0: with a block of attention."""

    def __init__(self, items: int, dim: int = 128, hidden: int = 512, seed: int = 0, device="cuda:0", heads: int = 0,
                 window: int = 32, sinks: int = 2):
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
        self.heads, self.window, self.sinks = heads, window, sinks
        if heads:
            if dim % heads:
                raise ValueError("dim must be a multiple of heads")
            self.w_qkv = normal(dim, 3 * dim, std=dim ** -0.5)
            self.w_out = normal(dim, dim, std=0.1 * dim ** -0.5)
            self.gain, self.shift = torch.ones(dim, device=device), torch.zeros(dim, device=device)
            self.momentum += [torch.zeros_like(self.w_qkv), torch.zeros_like(self.w_out)]

    def _projected(self, x: torch.Tensor):
        """(normalised rows, mean, rstd, (q, k, v)) of rows x [tokens, dim]; the three are slices of one product."""
        n, mean, rstd = ln.layer_norm(x, self.gain, self.shift, stats=True)
        return n, mean, rstd, (n @ self.w_qkv).to(torch.bfloat16).view(len(x), 3, self.heads, self.dim // self.heads).unbind(1)

    def _attend(self, x: torch.Tensor, offsets: torch.Tensor):
        """x + attention, and what its backward pass needs."""
        n, mean, rstd, qkv = self._projected(x)
        out, lse = wa.window_attention(*qkv, offsets, self.window, self.sinks, stats=True)
        o = out.view(len(x), self.dim).float()
        return x + o @ self.w_out, (x, n, mean, rstd, qkv, out, lse, o, offsets)

    def _attend_backward(self, d_y: torch.Tensor, saved):
        """(d_x, gradients of w_qkv, w_out, gain and shift)."""
        x, n, mean, rstd, qkv, out, lse, o, offsets = saved
        d_out = (d_y @ self.w_out.T).to(torch.bfloat16).view(out.shape)
        d_qkv = torch.empty(len(x), 3, *out.shape[1:], dtype=torch.bfloat16, device=x.device)
        wa.window_attention_backward(d_out, *qkv, out, lse, offsets, self.window, self.sinks, grads=d_qkv.unbind(1))
        d_qkv = d_qkv.view(len(x), 3 * self.dim).float()
        d_x, d_gain, d_shift = ln.layer_norm_backward(d_qkv @ self.w_qkv.T, x, mean, rstd, self.gain)
        return d_y + d_x, (n.T @ d_qkv, o.T @ d_y, d_gain, d_shift)

    def loss_and_gradients(self, sessions: torch.Tensor):
        """Mean cross entropy of the next items of sessions [B, L + 1], and the gradients of
        (table, w1, w2), with heads also of (w_qkv, w_out, gain, shift)."""
        inputs, targets = sessions[:, :-1], sessions[:, 1:].reshape(-1)
        scale = math.sqrt(self.dim)
        x = te.token_forward(self.table, inputs, scale=scale).view(-1, self.dim)
        if self.heads:
            length = inputs.shape[1]
            x, saved = self._attend(x, torch.arange(0, inputs.numel() + 1, max(length, 1), device=x.device))
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
        more = ()
        d_w1 = x.T @ d_a
        if self.heads:
            d_x, more = self._attend_backward(d_x, saved)
        te.token_backward(d_x.view(*inputs.shape, self.dim), inputs, self.items, scale=scale, out=d_table,
                          accumulate=True)
        return loss, (d_table, d_w1, h.T @ d_y, *more)

    def step(self, sessions: torch.Tensor, lr: float = 0.02, table_lr: float = 0.1,
             max_norm: float | None = None) -> torch.Tensor:
        """One training step; returns the loss before it (on the device). With max_norm the gradients are clipped to it."""
        loss, grads = self.loss_and_gradients(sessions)
        if max_norm is not None:
            clip.clip_grad_norm(grads, max_norm)
        d_table, matrices = grads[0], [self.w1, self.w2]
        if self.heads:
            matrices += [self.w_qkv, self.w_out]
            self.gain -= table_lr * grads[5]
            self.shift -= table_lr * grads[6]
        for w, d, m in zip(matrices, grads[1:], self.momentum):
            muon.muon_step(w, d, m, lr=lr, weight_decay=0.01, adjust="spectral")
        self.row_state += d_table.square().mean(1, keepdim=True)
        self.table -= table_lr * d_table / (self.row_state.sqrt() + 1e-8)
        return loss


class Serving:
    """Scores of the next item of `sessions` sessions, which grow an item at a time to at most `capacity`."""

    def __init__(self, model: NextItem, sessions: int, capacity: int):
        if not model.heads:
            raise ValueError("a model without attention keeps nothing of a session")
        self.model = model
        shape = (2, sessions, capacity, model.heads, model.dim // model.heads)
        self.cache = torch.zeros(shape, dtype=torch.bfloat16, device=model.table.device)
        self.lengths = torch.zeros(sessions, dtype=torch.int64, device=model.table.device)
        self.length = 0  # the same on the host, for the check of the capacity

    def append(self, items: torch.Tensor) -> torch.Tensor:
        """Adds one item to every session; scores [sessions, items] of what may follow."""
        if items.shape != self.lengths.shape:
            raise ValueError("one item for every session")
        if self.length == self.cache.shape[2]:
            raise ValueError("the sessions have reached their capacity")
        self.length += 1
        m, rows = self.model, torch.arange(len(items), device=items.device)
        x = te.token_forward(m.table, items, scale=math.sqrt(m.dim))
        q, k, v = m._projected(x)[3]
        self.cache[0, rows, self.lengths], self.cache[1, rows, self.lengths] = k, v
        self.lengths += 1
        out = wa.window_attention_step(q, self.cache[0], self.cache[1], self.lengths, m.window, m.sinks)
        x = x + out.view(len(items), m.dim).float() @ m.w_out
        return (x + (x @ m.w1).relu() @ m.w2) @ m.table.T / math.sqrt(m.dim)


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


def train(steps: int = 200, items: int = 2000, sessions: int = 64, length: int = 50, seed: int = 0, heads: int = 0,
          window: int = 32, sinks: int = 2, max_norm: float | None = None) -> list[float]:
    model = NextItem(items, seed=seed, heads=heads, window=window, sinks=sinks)
    losses = [model.step(make_sessions(items, sessions, length, seed=1000 + k), max_norm=max_norm) for k in range(steps)]
    return torch.stack(losses).tolist()


def main() -> None:
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--steps", type=int, default=200)
    p.add_argument("--items", type=int, default=2000)
    p.add_argument("--heads", type=int, default=0)
    p.add_argument("--window", type=int, default=32)
    p.add_argument("--sinks", type=int, default=2)
    p.add_argument("--max-norm", type=float, default=None)
    a = p.parse_args()
    losses = train(a.steps, a.items, heads=a.heads, window=a.window, sinks=a.sinks, max_norm=a.max_norm)
    for k in range(0, len(losses), max(1, len(losses) // 10)):
        print(f"step {k:5d}  loss {losses[k]:.4f}")
    print(f"step {len(losses) - 1:5d}  loss {losses[-1]:.4f}  (uniform {math.log(a.items):.4f})")


if __name__ == "__main__":
    main()
