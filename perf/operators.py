"""Operators for training sequence models on top of the embedding tables, as measured cases.

Four calls, of two kinds that one training step makes side by side:

* ``lookup``: a row of one table for every token of a batch of sequences, scaled
  (``token_embedding.token_forward``);
* ``grad``: the gradient of that lookup with respect to the table, dense, every row the
  sum over the positions that hold its token (``token_embedding.token_backward``), written
  new or added into the gradient that an output head tied to the table has left;
* ``ortho``: a matrix update replaced by its approximate orthogonal factor, by Newton-Schulz
  products (``muon.newton_schulz``);
* ``step``: the same inside an optimizer step: momentum, orthogonalised update, weight decay
  and the new weights (``muon.muon_step``).

``run`` computes them in plain 32-bit torch operations, or with ``own`` set by the calls
above. ``exact`` states each result in 64 bits, by another route.
"""

from __future__ import annotations

import math
from functools import lru_cache

import numpy as np
import torch

own = False

DEV = torch.device("cuda:0")
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
INDEX = {"i32": torch.int32, "i64": torch.int64}
COEF = (3.4445, -4.7750, 2.0315)
EPS = 1e-7
STEPS = 5
LR, BETA, DECAY = 3e-4, 0.95, 0.1

LOOKUP = {"kind": "lookup", "seqs": 1, "length": 1, "rows": 1000, "dim": 64, "dtype": "f32", "out": "f32",
          "index": "i64", "zipf": 0.0, "pad": 0.0, "shifted": False, "accumulate": False}
MATRIX = {"kind": "ortho", "batch": 1, "m": 128, "n": 128, "dtype": "bf16", "out": "bf16"}


def _tok(name, **kw):
    return {"name": name, **LOOKUP, **kw}


def _mat(name, **kw):
    return {"name": name, **MATRIX, **kw}


def listed():
    return [
        # One new token for each of 64 sequences being generated: latency.
        _tok("lookup_step", seqs=64, length=1, rows=32768, dim=1024, dtype="bf16", out="bf16", zipf=1.0),
        # Three ragged prompts, fp32 master table read into half-precision activations, a
        # width that is no multiple of a warp's.
        _tok("lookup_odd", seqs=3, length=1001, rows=50001, dim=1000, dtype="f32", out="bf16", index="i32",
             zipf=1.05),
        # The inputs of a training step, a slice of sequences that carry their targets too.
        _tok("lookup_train", seqs=16, length=2048, rows=65536, dim=2048, dtype="bf16", out="bf16", zipf=1.0,
             shifted=True),
        # The largest: long sequences, wide rows.
        _tok("lookup_large", seqs=32, length=8192, rows=131072, dim=4096, dtype="bf16", out="bf16", zipf=1.0),
        # The smallest table of the repository's workloads, a small batch.
        _tok("grad_small", kind="grad", seqs=2, length=60, rows=1000, dim=64, dtype="f32", out="f32"),
        # A training step over padded sequences: the padding's row gets no gradient.
        _tok("grad_train", kind="grad", seqs=8, length=2048, rows=65536, dim=1024, dtype="bf16", out="f32",
             zipf=1.0, pad=0.1, shifted=True),
        # Added into the gradient of a head tied to the table.
        _tok("grad_tied", kind="grad", seqs=16, length=4096, rows=131072, dim=2048, dtype="bf16", out="f32",
             zipf=1.0, accumulate=True),
        # The largest: every position of long sequences, gradients in the table's type.
        _tok("grad_large", kind="grad", seqs=32, length=8192, rows=131072, dim=4096, dtype="bf16", out="bf16",
             zipf=1.0),
        # The small projections of a layer per table, stacked: latency of a chain of products.
        _mat("ortho_stack", batch=26, m=64, n=128, dtype="f32"),
        # A tall matrix of odd sizes.
        _mat("ortho_odd", m=1001, n=513, dtype="f32"),
        # The update of four wide layers at once, weights and momentum in fp32.
        _mat("step_wide", kind="step", batch=4, m=1024, n=4096, dtype="bf16", out="f32"),
        # The largest: one square layer.
        _mat("ortho_large", m=4096, n=4096, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["lookup", "lookup", "grad", "grad", "ortho", "ortho", "step"])
    if kind in ("lookup", "grad"):
        dim = _log(rng, 64, 4096)
        if rng.random() < 0.7:
            dim = (dim + 7) // 8 * 8
        dtype = rng.choice(["f32", "f16", "bf16", "bf16"])
        total = min(_log(rng, 1, 262144), 2 ** 30 // dim if dtype != "f32" else 2 ** 29 // dim)
        seqs = min(total, _log(rng, 1, 64))
        c = dict(LOOKUP, kind=kind, seqs=seqs, length=max(1, total // seqs), rows=_log(rng, 1000, 131072), dim=dim,
                 dtype=dtype, out=rng.choice([dtype, dtype, "f32" if kind == "grad" else "bf16"]),
                 index=rng.choice(["i32", "i64"]), zipf=rng.choice([0.0, 1.0, 1.0, 1.1]), shifted=rng.random() < 0.4)
        if kind == "grad":
            c["pad"] = rng.choice([0.0, 0.0, 0.1, 0.3])
            c["accumulate"] = rng.random() < 0.4
        return c
    m, n = _log(rng, 48, 4096), _log(rng, 48, 4096)
    if rng.random() < 0.6:
        m, n = (m + 15) // 16 * 16, (n + 15) // 16 * 16
    c = dict(MATRIX, kind=kind, m=m, n=n, dtype=rng.choice(["bf16", "f32"]),
             out=rng.choice(["bf16", "bf16", "f16"]) if kind == "ortho" else rng.choice(["f32", "bf16"]))
    most = min(64.0, 0.9 * 4096.0 ** 3 / (min(m, n) ** 2 * max(m, n)), 0.9 * 4096.0 ** 2 / (m * n))
    c["batch"] = max(1, _log(rng, 1, max(1.0, most)))
    return c


# ----------------------------------------------------------------------------- inputs

def _gen(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 1_000_003 + case.get("rows", 0) * 31 + case.get("dim", case.get("m", 0)))
    return g


def _tokens(case, g):
    """Tokens with the skew of text or of items: rank k with probability ~ k^-zipf, ranks scattered over the rows."""
    rows, total = case["rows"], case["seqs"] * (case["length"] + 1)
    u = torch.rand(total, generator=g, device=DEV, dtype=torch.float64)
    if case["zipf"]:
        cdf = torch.arange(1, rows + 1, device=DEV, dtype=torch.float64).pow(-case["zipf"]).cumsum(0)
        rank = torch.searchsorted(cdf, u * cdf[-1]).clamp_(max=rows - 1)
        tok = torch.randperm(rows, generator=g, device=DEV)[rank]
    else:
        tok = (u * rows).long().clamp_(max=rows - 1)
    tok = tok.view(case["seqs"], case["length"] + 1)
    if case["pad"]:  # the ends of the sequences hold the padding token 0
        keep = torch.rand(case["seqs"], 1, generator=g, device=DEV) * 2 * case["pad"]
        at = torch.arange(case["length"] + 1, device=DEV)[None, :]
        tok = torch.where(at >= (1 - keep) * (case["length"] + 1), torch.zeros_like(tok), tok)
    tok = tok.to(INDEX[case["index"]])
    return tok[:, :-1] if case["shifted"] else tok[:, :-1].contiguous()


def _updates(case, g):
    """Gradients of weight matrices: a few strong directions over a noise floor, small values."""
    b, m, n = case["batch"], case["m"], case["n"]
    r = max(1, min(m, n) // 8)
    left = torch.randn(b, m, r, generator=g, device=DEV) * torch.linspace(0, -3, r, device=DEV).exp()
    x = left @ torch.randn(b, r, n, generator=g, device=DEV) / r ** 0.5
    x.add_(torch.randn(b, m, n, generator=g, device=DEV), alpha=0.05)
    return (x * 1e-3).to(DTYPES[case["dtype"]])


def prepare(case, seed):
    g = _gen(case, seed)
    s = {"case": case}
    if case["kind"] in ("lookup", "grad"):
        s["tokens"] = _tokens(case, g)
        s["scale"] = math.sqrt(case["dim"])
        shape = (case["seqs"], case["length"], case["dim"])
        if case["kind"] == "lookup":
            s["table"] = (torch.randn(case["rows"], case["dim"], generator=g, device=DEV)
                          .mul_(0.02).to(DTYPES[case["dtype"]]))
        else:
            s["grad_out"] = torch.empty(shape, dtype=DTYPES[case["dtype"]], device=DEV)
            s["grad_out"].normal_(generator=g).mul_(1e-3)
            if case["accumulate"]:
                s["grad"] = torch.empty(case["rows"], case["dim"], dtype=DTYPES[case["out"]], device=DEV)
                s["grad"].normal_(generator=g).mul_(1e-2)
        return s
    s["update"] = _updates(case, g)
    if case["kind"] == "step":
        shape = (case["batch"], case["m"], case["n"])
        s["weight"] = torch.randn(shape, generator=g, device=DEV).mul_(0.02).to(DTYPES[case["out"]])
        s["momentum"] = torch.randn(shape, generator=g, device=DEV).mul_(2e-3)
    return s


# ----------------------------------------------------------------------------- the operators, plain

def _plain_newton_schulz(x, transposed):
    a, b, c = COEF
    x = x.transpose(-1, -2) if transposed else x
    x = x / (x.square().sum(dim=(-2, -1), keepdim=True).sqrt() + EPS)
    for _ in range(STEPS):
        gram = x @ x.transpose(-1, -2)
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return x.transpose(-1, -2) if transposed else x


def _adjust(case):
    """The update's values brought to the size of an Adam step's: 0.2 sqrt(max(m, n))."""
    return 0.2 * math.sqrt(max(case["m"], case["n"]))


def run(state):
    case = state["case"]
    kind, out = case["kind"], DTYPES[case["out"]]
    if own:
        from paper_2609_30656_gb300 import muon, token_embedding as te
        if kind == "lookup":
            return te.token_forward(state["table"], state["tokens"], scale=state["scale"], out_dtype=out)
        if kind == "grad":
            return te.token_backward(state["grad_out"], state["tokens"], case["rows"], scale=state["scale"],
                                     padding_idx=0 if case["pad"] else None, out=state.get("grad"), out_dtype=out,
                                     accumulate=case["accumulate"])
        if kind == "ortho":
            return muon.newton_schulz(state["update"], out_dtype=out, steps=STEPS, coefficients=COEF, eps=EPS)
        muon.muon_step(state["weight"], state["update"], state["momentum"], lr=LR, beta=BETA, nesterov=True,
                       weight_decay=DECAY, adjust="rms", steps=STEPS, coefficients=COEF, eps=EPS)
        return {"weight": state["weight"], "momentum": state["momentum"]}
    if kind == "lookup":
        return (state["table"][state["tokens"].long()].float() * state["scale"]).to(out)
    if kind == "grad":
        tok = state["tokens"].reshape(-1).long()
        go = state["grad_out"].reshape(-1, case["dim"]).float() * state["scale"]
        if case["pad"]:
            go = go * (tok != 0).unsqueeze(1)
        if case["accumulate"] and case["out"] == "f32":
            return state["grad"].index_add_(0, tok, go)
        grad = torch.zeros(case["rows"], case["dim"], device=DEV)
        grad.index_add_(0, tok, go)
        if case["accumulate"]:
            return state["grad"].copy_(state["grad"].float() + grad)
        return grad.to(out)
    tall = case["m"] > case["n"]
    if kind == "ortho":
        return _plain_newton_schulz(state["update"].float(), tall).to(out)
    grad = state["update"].float()
    m = state["momentum"].mul_(BETA).add_(grad)
    o = _plain_newton_schulz(grad + BETA * m, tall)
    w = state["weight"]
    if w.dtype == torch.float32:
        w.mul_(1 - LR * DECAY).add_(o, alpha=-LR * _adjust(case))
    else:
        w.copy_(w.float() * (1 - LR * DECAY) - LR * _adjust(case) * o)
    return {"weight": w, "momentum": m}


# ----------------------------------------------------------------------------- what a pass cannot do without

@lru_cache(maxsize=64)
def _distinct(rows, zipf, total):
    """Expected number of distinct rows among `total` tokens."""
    p = np.arange(1, rows + 1, dtype=np.float64) ** -zipf
    p /= p.sum()
    return float(-np.expm1(total * np.log1p(-np.minimum(p, 1 - 1e-12))).sum())


def work(case):
    if case["kind"] in ("lookup", "grad"):
        total, dim = case["seqs"] * case["length"], case["dim"]
        touched = _distinct(case["rows"], case["zipf"], total)
        src, dst = BYTES[case["dtype"]], BYTES[case["out"]]
        index = total * (4 if case["index"] == "i32" else 8)
        if case["kind"] == "lookup":
            return {"bytes": index + dim * (touched * src + total * dst), "flops": total * dim}
        read = (1 - case["pad"]) * total * dim
        wrote = touched * 2 if case["accumulate"] else case["rows"]
        return {"bytes": index + read * src + wrote * dim * dst, "flops": 2 * read}
    b, m, n = case["batch"], case["m"], case["n"]
    p, q = min(m, n), max(m, n)
    # X X^T and A A are symmetric: half of their products determine them.
    flops = b * STEPS * (p * p * q + p * p * p + 2 * p * p * q)
    values = b * m * n
    if case["kind"] == "ortho":
        return {"bytes": values * (BYTES[case["dtype"]] + BYTES[case["out"]]), "flops": flops}
    return {"bytes": values * (BYTES[case["dtype"]] + 8 + 2 * BYTES[case["out"]]), "flops": flops}


# ----------------------------------------------------------------------------- 64 bits

def _exact_newton_schulz(x):
    """Every matrix on its own, by Horner's rule with the Gram matrix of its shorter side."""
    a, b, c = COEF
    out = torch.empty_like(x)
    for i in range(x.shape[0]):
        y = x[i] / (torch.linalg.vector_norm(x[i]) + EPS)
        eye = torch.eye(min(y.shape), dtype=torch.float64, device=y.device)
        for _ in range(STEPS):
            if y.shape[0] <= y.shape[1]:
                k = y @ y.T
                y = (a * eye + k @ (b * eye + c * k)) @ y
            else:
                k = y.T @ y
                y = y @ (a * eye + k @ (b * eye + c * k))
        out[i] = y
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "lookup":
        return torch.nn.functional.embedding(s["tokens"].long(), s["table"].double()) * s["scale"]
    if case["kind"] == "grad":
        tok = s["tokens"].reshape(-1).long()
        go = s["grad_out"].reshape(-1, case["dim"])
        at = torch.nonzero(tok != 0).squeeze(1) if case["pad"] else torch.arange(tok.numel(), device=DEV)
        at = at[torch.argsort(tok[at], stable=True)]
        rows, counts = torch.unique_consecutive(tok[at], return_counts=True)
        grad = s["grad"].double() if case["accumulate"] else torch.zeros(case["rows"], case["dim"],
                                                                          dtype=torch.float64, device=DEV)
        # running sums of the sorted positions, their differences at the ends of each row's run
        ends = counts.cumsum(0)
        for lo in range(0, case["dim"], 256):
            run_sum = go[:, lo:lo + 256][at].double().cumsum(0)[ends - 1]
            run_sum[1:] -= run_sum[:-1].clone()
            grad[rows, lo:lo + 256] += run_sum * s["scale"]
        return grad
    g = s["update"].double()
    if case["kind"] == "ortho":
        return _exact_newton_schulz(g)
    m = BETA * s["momentum"].double() + g
    o = _exact_newton_schulz(g + BETA * m)
    return {"weight": (1 - LR * DECAY) * s["weight"].double() - LR * _adjust(case) * o, "momentum": m}
