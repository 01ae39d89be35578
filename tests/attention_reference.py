"""Windowed attention over packed sessions in 64 bits, with bounds on what rounding may add to it.

u = 2^-24; h: the half step (eps / 2) to which P, dS and the outputs of 16-bit rows are rounded (outputs of fp32
rows too, P and dS then are not). A sum of D products in fp32, in any order, is off by at most 2 D u of its magnitudes (2 u for
each addition: tensor cores may cut off where others round to nearest), so

  S      es = |scale| (2 D + 4) u sum |q||k|, and 4 u |S| for its scaling and the exponential's argument
  P      relative ep = 2 es (its own, and that of the lse, a mean of the same errors) + 2^-20 (exponentials, their sum) + h
  out    sum_j P |v| ep + 2 u n P |v| over n keys + h |out|
  dP     ed = (2 D + 4) u sum |do||v|;  delta: the same of |do||out|, and h sum |do||out| as out was rounded
  dS     P (ed + edelta) + |dS| (ep + 4 u);  dq, dk, dv: such errors against |k|, |q|, |do|, 2 n u of the sum's magnitudes, h of it
"""

import torch

U = 2.0 ** -24
DEV = "cuda:0"


def half(dtype):
    return torch.finfo(dtype).eps / 2


def tiny(dtype):
    return torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps


def visible(tokens, lens, window, sinks, begin=0):
    """[tokens, tokens] of what each token sees; sessions of `lens` tokens from token `begin` on."""
    session = torch.full((tokens,), -1, device=DEV)
    place = torch.zeros(tokens, dtype=torch.long, device=DEV)
    at = begin
    for i, n in enumerate(lens):
        session[at:at + n] = i
        place[at:at + n] = torch.arange(n, device=DEV)
        at += n
    back = place[:, None] - place[None, :]
    same = (session[:, None] == session[None, :]) & (session >= 0)[:, None]
    return same & (back >= 0) & ((back < window) | (place < sinks)[None, :])


def reference(q, k, v, seen, scale, go=None):
    """({name: (value, bound)}) in 64 bits: out, lse and, with go, dq, dk, dv; rows of one head at a time."""
    heads, kv = q.shape[1], k.shape[1]
    dtype, D = q.dtype, q.shape[2]
    h = half(dtype)
    hp = 0.0 if dtype == torch.float32 else h
    res = {n: [torch.zeros(t.shape, dtype=torch.float64, device=DEV) for _ in range(2)]
           for n, t in (("out", q), ("dq", q), ("dk", k), ("dv", v))}
    lse = torch.full((heads, q.shape[0]), -torch.inf, dtype=torch.float64, device=DEV)
    lse_bound = torch.zeros_like(lse)
    n = seen.sum(1, keepdim=True).double()
    for x in range(heads):
        y = x // (heads // kv)
        a, b, c = q[:, x].double(), k[:, y].double(), v[:, y].double()
        s = (a @ b.T * scale).masked_fill(~seen, -torch.inf)
        es = (abs(scale) * (2 * D + 4) * U * (a.abs() @ b.abs().T) + 4 * U * s.abs().nan_to_num(posinf=0)) * seen
        e = torch.logsumexp(s, 1, keepdim=True)
        p = torch.where(seen, torch.exp(s - e), 0.0).nan_to_num(nan=0.0)
        lse[x] = torch.where(seen.any(1), e.squeeze(1), -torch.inf)
        worst = es.amax(1)
        lse_bound[x] = 2 * worst + 2.0 ** -20 + 4 * U * lse[x].abs().nan_to_num(posinf=0.0)
        ep = (2 * worst.unsqueeze(1) + 2.0 ** -20 + hp) * (1 + 2.0 ** -6)
        o = p @ c
        o_bound = (p * (ep + 2 * U * n)) @ c.abs() + h * o.abs()
        res["out"][0][:, x], res["out"][1][:, x] = o, o_bound
        if go is None:
            continue
        g = go[:, x].double()
        dp = g @ c.T
        delta = (g * o).sum(1, keepdim=True)
        ed = (2 * D + 4) * U * (g.abs() @ c.abs().T)
        edelta = ((2 * D + 4) * U * g.abs() * o.abs() + g.abs() * (o_bound + h * o.abs())).sum(1, keepdim=True)
        ds = p * (dp - delta) * scale
        ds_bound = (p * (ed + edelta) * (1 + 2.0 ** -6)) * abs(scale) + ds.abs() * (ep + 4 * U)
        m = seen.sum(0).amax().double() * (heads // kv) + n.amax()
        res["dq"][0][:, x] = ds @ b
        res["dq"][1][:, x] = ds_bound @ b.abs() + 2 * U * n * (ds.abs() @ b.abs())
        for name, w, wb, z in (("dk", ds, ds_bound, a), ("dv", p, p * ep, g)):
            res[name][0][:, y] += w.T @ z
            res[name][1][:, y] += wb.T @ z.abs() + 2 * U * m * (w.abs().T @ z.abs())
    for name in ("dq", "dk", "dv"):
        res[name][1] += h * res[name][0].abs()
    return {**{n: (a, b * (1 + 2.0 ** -6) + tiny(dtype)) for n, (a, b) in res.items()}, "lse": (lse, lse_bound)}


def check(got, want, what=""):
    value, bound = want
    off = (got.double() - value).abs()
    bad = ~((off <= bound) | (got.double() == value))
    assert not bad.any(), (what, int(bad.sum()), (off / bound.clamp(min=1e-300))[bad].max().item(),
                           torch.nonzero(bad)[:4].tolist())
