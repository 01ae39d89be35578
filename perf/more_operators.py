"""Operators for a sequence model's blocks and its training step, as measured cases.

What stands between the token lookup and the matrix steps of ``perf/operators.py``:

* ``norm`` / ``normgrad``: layer normalisation of rows, and its backward pass with the
  gradients of weight and bias (``layer_norm.layer_norm``, ``layer_norm.layer_norm_backward``);
* ``attn`` / ``attngrad`` / ``step``: causal attention within the sessions of a packed batch,
  to a window of the last tokens and to the first few of the session, its backward pass, and
  the same for one new token of each session over a cache of keys and values
  (``window_attention.window_attention``, ``..._backward``, ``..._step``);
* ``clip``: the norm over all gradients of a model, and the gradients scaled to at most a
  given norm (``clip.clip_grad_norm``).

``run`` computes them in plain 32-bit torch operations, or with ``own`` set by the calls
above. ``exact`` states each result in 64 bits, by another route.
"""

from __future__ import annotations

import math
import random

import torch

own = False

DEV = torch.device("cuda:0")
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
INDEX = {"i32": torch.int32, "i64": torch.int64}
EPS = 1e-5
CLIP_EPS = 1e-6

NORM = {"kind": "norm", "rows": 64, "dim": 64, "dtype": "bf16", "out": "bf16", "params": "f32", "bias": True}
ATTN = {"kind": "attn", "seqs": 1, "length": 64, "ragged": False, "heads": 4, "kv_heads": 4, "dim": 64, "dtype": "bf16",
        "window": 64, "sinks": 4, "index": "i32", "fused": False}
STEP = {"kind": "step", "seqs": 1, "capacity": 64, "full": True, "heads": 4, "kv_heads": 4, "dim": 64, "dtype": "bf16",
        "window": 64, "sinks": 4, "index": "i32"}
CLIP = {"kind": "clip", "layers": 1, "dim": 64, "hidden": 256, "rows": 1000, "dtype": "f32", "table": "f32",
        "sparse": 0, "clipped": False}


def _case(base, name, **kw):
    return {"name": name, **base, **kw}


def listed():
    return [
        # One new token for each of 64 sessions being served: latency.
        _case(NORM, "norm_step", rows=64, dim=1024),
        # The activations of a large batch.
        _case(NORM, "norm_large", rows=131072, dim=4096),
        # Three ragged sessions of an odd width, fp32 activations, gradients of bf16 products.
        _case(NORM, "normgrad_odd", kind="normgrad", rows=3003, dim=1001, dtype="f32", out="f32"),
        # The backward pass of a training step.
        _case(NORM, "normgrad_large", kind="normgrad", rows=131072, dim=2048),
        # Click sessions: short, ragged, empty ones among them; queries, keys and values slices of one product.
        _case(ATTN, "attn_sessions", seqs=512, length=60, ragged=True, heads=4, kv_heads=4, dim=32, window=50, sinks=2,
              index="i64", fused=True),
        # Long histories, heads that share keys.
        _case(ATTN, "attn_long", seqs=8, length=8192, heads=16, kv_heads=4, dim=128, window=2048, sinks=4),
        # The backward pass of ragged middling sequences, a head of an odd width.
        _case(ATTN, "attngrad_odd", kind="attngrad", seqs=33, length=700, ragged=True, heads=8, kv_heads=2, dim=72,
              dtype="f16", window=301, sinks=3),
        # The backward pass of long histories.
        _case(ATTN, "attngrad_long", kind="attngrad", seqs=8, length=8192, heads=16, kv_heads=4, dim=128, window=2048,
              sinks=4),
        # The next item of a few sessions.
        _case(STEP, "step_few", seqs=5, capacity=1024, full=False, heads=8, kv_heads=8, dim=64, dtype="f16", window=301,
              sinks=4, index="i64"),
        # Of many, with long histories.
        _case(STEP, "step_many", seqs=256, capacity=8192, heads=16, kv_heads=4, dim=128, window=4096, sinks=4),
        # The gradients of a small model, a row-sparse one of pooled tables among them; the usual step, whose norm is
        # below the limit.
        _case(CLIP, "clip_small", layers=2, dim=64, hidden=256, rows=1000, sparse=20000),
        # A large model in bf16 with an fp32 table, clipped into another set of tensors.
        _case(CLIP, "clip_large", layers=24, dim=1024, hidden=4096, rows=131072, dtype="bf16", clipped=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "normgrad", "normgrad", "attn", "attn", "attngrad", "attngrad", "step", "step", "clip",
                       "clip"])
    if kind in ("norm", "normgrad"):
        dim = _log(rng, 32, 16384)
        if rng.random() < 0.7:
            dim = (dim + 7) // 8 * 8
        most = 2 ** 29 if kind == "norm" else 2 ** 28
        dtype = rng.choice(["f32", "f16", "bf16", "bf16"])
        rows = max(1, min(_log(rng, 1, 262144), most // dim // (2 if dtype == "f32" else 1)))
        return dict(NORM, kind=kind, rows=rows, dim=dim, dtype=dtype,
                    out=rng.choice([dtype, dtype, "f32" if kind == "normgrad" else "bf16"]),
                    params=rng.choice(["f32", dtype]), bias=rng.random() < 0.8)
    if kind in ("attn", "attngrad", "step"):
        kv_heads = rng.choice([1, 2, 4, 4, 8])
        group = rng.choice([1, 1, 2, 4])
        c = {"heads": kv_heads * group, "kv_heads": kv_heads, "dim": rng.choice([32, 40, 64, 64, 72, 96, 128, 128]),
             "dtype": rng.choice(["bf16", "bf16", "f16"]), "window": _log(rng, 1, 4096), "sinks": rng.choice([0, 1, 4, 4, 9]),
             "index": rng.choice(["i32", "i64"])}
        if kind == "step":
            capacity = _log(rng, 16, 16384)
            most = 2 ** 31 // (capacity * kv_heads * c["dim"])
            return dict(STEP, kind=kind, **c, seqs=min(_log(rng, 1, 512), max(1, most)), capacity=capacity,
                        full=rng.random() < 0.3)
        length = _log(rng, 1, 8192)
        # Plain scores are of length x length for each head of each sequence: bounded, as the tokens are.
        most = min(65536 * 16 / (length * c["heads"]), 2 ** 33 / (float(length) * length * c["heads"]))
        return dict(ATTN, kind=kind, **c, seqs=_log(rng, 1, max(1.0, min(1024.0, most))), length=length,
                    ragged=rng.random() < 0.6, fused=rng.random() < 0.5)
    dim = _log(rng, 32, 1024)
    return dict(CLIP, layers=_log(rng, 1, 24), dim=dim, hidden=dim * rng.choice([2, 4]) + rng.choice([0, 0, 3]),
                rows=_log(rng, 100, 131072), dtype=rng.choice(["f32", "bf16", "f16"]), table=rng.choice(["f32", "bf16"]),
                sparse=rng.choice([0, 0, _log(rng, 1000, 10 ** 7)]), clipped=rng.random() < 0.5)


# ----------------------------------------------------------------------------- inputs

def _numbers(case):
    """A generator of the case's own shapes (they are the same for every seed)."""
    return random.Random(" ".join(f"{k}={v}" for k, v in sorted(case.items()) if k not in ("name", "kind")))


def _lengths(case):
    """Tokens of each sequence; ragged ones are mostly short, some are empty."""
    if not case["ragged"]:
        return [case["length"]] * case["seqs"]
    rng = _numbers(case)
    lens = [min(int(case["length"] * rng.expovariate(1.0)), 4 * case["length"], 8192) for _ in range(case["seqs"])]
    lens[0] = max(lens[0], 1)
    return lens


def _cached(case):
    """Tokens of each session in its cache."""
    if case["full"]:
        return [case["capacity"] - i % 7 % case["capacity"] for i in range(case["seqs"])]
    rng = _numbers(case)
    return [max(1, case["capacity"] // 2)] + [rng.randint(0, case["capacity"]) for _ in range(case["seqs"] - 1)]


def _shapes(case):
    """Gradients of a model: of each layer four matrices and five vectors, and of its table."""
    d, h = case["dim"], case["hidden"]
    layer = [(d, d), (d, d), (d, h), (h, d), (d,), (d,), (d,), (d,), (h,)]
    return layer * case["layers"] + [(case["rows"], d)]


def _views(flat, table, shapes):
    parts = flat.split([math.prod(shape) for shape in shapes[:-1]])
    return [part.view(shape) for part, shape in zip(parts, shapes)] + [table]


def _gen(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 1_000_003 + _numbers(case).randrange(1_000_000))
    return g


def _normal(g, *shape, std=1.0, dtype="f32"):
    out = torch.empty(shape, dtype=DTYPES[dtype], device=DEV)
    return out.normal_(generator=g).mul_(std)


def _prepare_norm(case, g):
    rows, dim = case["rows"], case["dim"]
    # Activations: a shift for each row, a few strong channels.
    x = torch.empty(rows, dim, dtype=DTYPES[case["dtype"]], device=DEV).normal_(generator=g)
    strong = torch.ones(dim, device=DEV)
    strong[::97] = 8.0
    x.mul_(strong.to(x.dtype)).add_(_normal(g, rows, 1, std=0.5).to(x.dtype))
    s = {"x": x, "weight": (1 + _normal(g, dim, std=0.1)).to(DTYPES[case["params"]])}
    s["bias"] = _normal(g, dim, std=0.1).to(DTYPES[case["params"]]) if case["bias"] else None
    if case["kind"] == "normgrad":
        f = x.float()
        s["mean"] = f.mean(1)
        s["rstd"] = (f.var(1, unbiased=False) + EPS).rsqrt()
        s["grad_out"] = _normal(g, rows, dim, std=1e-3, dtype=case["dtype"])
    return s


def _prepare_attention(case, g):
    heads, kv, dim, dtype = case["heads"], case["kv_heads"], case["dim"], case["dtype"]
    lens = _lengths(case)
    tokens = sum(lens)
    offsets = torch.tensor([0] + lens, device=DEV).cumsum(0)
    all_of = _normal(g, tokens, heads + 2 * kv, dim, dtype=dtype)
    # The first tokens of a session draw attention to them.
    firsts = (offsets[:-1][:, None] + torch.arange(case["sinks"], device=DEV)[None, :])
    firsts = firsts[firsts < offsets[1:][:, None]]
    all_of[firsts, heads:heads + kv] *= 1.5
    parts = all_of.split([heads, kv, kv], dim=1)
    q, k, v = parts if case["fused"] else (t.contiguous() for t in parts)
    s = {"q": q, "k": k, "v": v, "offsets": offsets.to(INDEX[case["index"]]), "lens": lens, "scale": dim ** -0.5}
    if case["kind"] == "attngrad":
        s["grad_out"] = _normal(g, tokens, heads, dim, dtype=dtype)
        s["out"], s["lse"] = _plain_attention(s, case)
    return s


def prepare(case, seed):
    g = _gen(case, seed)
    kind = case["kind"]
    if kind in ("norm", "normgrad"):
        return {"case": case, **_prepare_norm(case, g)}
    if kind in ("attn", "attngrad"):
        return {"case": case, **_prepare_attention(case, g)}
    if kind == "step":
        lens = _cached(case)
        cache = (case["seqs"], case["capacity"], case["kv_heads"], case["dim"])
        s = {"case": case, "q": _normal(g, case["seqs"], case["heads"], case["dim"], dtype=case["dtype"]),
             "k": _normal(g, *cache, dtype=case["dtype"]), "v": _normal(g, *cache, dtype=case["dtype"]),
             "lengths": torch.tensor(lens, device=DEV).to(INDEX[case["index"]]), "lens": lens,
             "scale": case["dim"] ** -0.5}
        s["k"][:, :case["sinks"]] *= 1.5
        return s
    shapes = _shapes(case)
    # The layers' gradients behind one another in one buffer, the table's in its own.
    flat = _normal(g, sum(math.prod(shape) for shape in shapes[:-1]), std=1e-3, dtype=case["dtype"])
    table = _normal(g, *shapes[-1], std=1e-3, dtype=case["table"])
    values = flat.numel() + table.numel() + case["sparse"]
    s = {"case": case, "flat": flat, "table": table, "grads": _views(flat, table, shapes),
         "max_norm": 1e-3 * math.sqrt(values) * (0.7 if case["clipped"] else 2.0)}
    if case["sparse"]:
        # A row-sparse gradient in a buffer that has room for more; how much of it counts is known on the device.
        s["sparse"] = _normal(g, case["sparse"] + case["sparse"] // 4 + 4, std=1e-3)
        s["count"] = torch.tensor([case["sparse"]], device=DEV)
    if case["clipped"]:
        s["clipped_flat"], s["clipped_table"] = torch.empty_like(flat), torch.empty_like(table)
        s["clipped"] = _views(s["clipped_flat"], s["clipped_table"], shapes)
        if case["sparse"]:
            s["clipped_sparse"] = torch.zeros_like(s["sparse"])
    return s


# ----------------------------------------------------------------------------- the operators, plain

def _plain_norm(s):
    x = s["x"].float()
    mean = x.mean(1)
    centred = x - mean[:, None]
    rstd = 1.0 / (centred.square().mean(1) + EPS).sqrt()
    y = centred * rstd[:, None] * s["weight"].float()
    if s["bias"] is not None:
        y = y + s["bias"].float()
    return y.to(DTYPES[s["case"]["out"]]), mean, rstd


def _plain_norm_backward(s):
    x, dy = s["x"].float(), s["grad_out"].float()
    xhat = (x - s["mean"][:, None]) * s["rstd"][:, None]
    dw, db = (dy * xhat).sum(0), dy.sum(0)
    g = dy * s["weight"].float()
    dx = s["rstd"][:, None] * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))
    return dx.to(DTYPES[s["case"]["out"]]), dw, db if s["bias"] is not None else None


def _padded(lens, heads):
    """Sequences of like length together, [batch, length] of token numbers each; how many queries at a time."""
    starts, at = [], 0
    for n in lens:
        starts.append(at)
        at += n
    groups: dict[int, list[int]] = {}
    for i, n in enumerate(lens):
        if n:
            groups.setdefault(max(16, 1 << (n - 1).bit_length()), []).append(i)
    for _, members in sorted(groups.items()):
        longest = max(lens[i] for i in members)
        per = max(1, 2 ** 28 // (heads * longest * longest))
        for lo in range(0, len(members), per):
            part = members[lo:lo + per]
            first = torch.tensor([starts[i] for i in part], device=DEV)
            n = torch.tensor([lens[i] for i in part], device=DEV)
            place = torch.arange(longest, device=DEV)[None, :]
            yield (first[:, None] + torch.minimum(place, n[:, None] - 1)), place < n[:, None], max(
                1, 2 ** 28 // (heads * longest * len(part)))


def _seen(rows, cols, case):
    back = rows[:, None] - cols[None, :]
    return (back >= 0) & ((back < case["window"]) | (cols < case["sinks"])[None, :])


def _plain_attention(s, case):
    """(out, lse); lse is [heads, tokens]."""
    tokens, heads, dim = s["q"].shape
    kv = case["kv_heads"]
    out = torch.zeros(tokens, heads, dim, dtype=s["q"].dtype, device=DEV)
    lse = torch.zeros(heads, tokens, device=DEV)
    for index, real, chunk in _padded(s["lens"], heads):
        b, longest = index.shape
        q = s["q"][index].float().view(b, longest, kv, heads // kv, dim)
        k, v = s["k"][index].float(), s["v"][index].float()
        for lo in range(0, longest, chunk):
            hi = min(lo + chunk, longest)
            seen = _seen(torch.arange(lo, hi, device=DEV), torch.arange(hi, device=DEV), case)
            score = torch.einsum("bqhgd,bkhd->bhgqk", q[:, lo:hi], k[:, :hi]) * s["scale"]
            score = score.masked_fill(~seen, -math.inf)
            top = score.amax(-1, keepdim=True)
            p = (score - top).exp()
            total = p.sum(-1, keepdim=True)
            o = torch.einsum("bhgqk,bkhd->bqhgd", p / total, v[:, :hi]).reshape(b, hi - lo, heads, dim)
            e = (top + total.log()).squeeze(-1).reshape(b, heads, hi - lo).transpose(1, 2)
            keep = real[:, lo:hi]
            out[index[:, lo:hi][keep]] = o[keep].to(out.dtype)
            lse[:, index[:, lo:hi][keep]] = e[keep].T
    return out, lse


def _plain_attention_backward(s, case):
    tokens, heads, dim = s["q"].shape
    kv = case["kv_heads"]
    grads = [torch.zeros(t.shape, dtype=t.dtype, device=DEV) for t in (s["q"], s["k"], s["v"])]
    for index, real, chunk in _padded(s["lens"], heads):
        b, longest = index.shape
        q = s["q"][index].float().view(b, longest, kv, heads // kv, dim)
        do = (s["grad_out"][index].float() * real[..., None, None]).view(q.shape)
        k, v = s["k"][index].float(), s["v"][index].float()
        dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
        lse = s["lse"][:, index].transpose(0, 1).reshape(b, kv, heads // kv, longest, 1)
        for lo in range(0, longest, chunk):
            hi = min(lo + chunk, longest)
            seen = _seen(torch.arange(lo, hi, device=DEV), torch.arange(hi, device=DEV), case)
            score = torch.einsum("bqhgd,bkhd->bhgqk", q[:, lo:hi], k[:, :hi]) * s["scale"]
            # Beside real rows there are none whose lse is not their own; padded ones are cut off at 1.
            p = (score - lse[:, :, :, lo:hi]).clamp_(max=0.0).masked_fill(~seen, -math.inf).exp()
            dv[:, :hi] += torch.einsum("bhgqk,bqhgd->bkhd", p, do[:, lo:hi])
            dp = torch.einsum("bqhgd,bkhd->bhgqk", do[:, lo:hi], v[:, :hi])
            ds = p * (dp - (p * dp).sum(-1, keepdim=True)) * s["scale"]
            dq[:, lo:hi] = torch.einsum("bhgqk,bkhd->bqhgd", ds, k[:, :hi])
            dk[:, :hi] += torch.einsum("bhgqk,bqhgd->bkhd", ds, q[:, lo:hi])
        for whole, part in zip(grads, (dq.reshape(b, longest, heads, dim), dk, dv)):
            whole[index[real]] = part[real].to(whole.dtype)
    return tuple(grads)


def _plain_step(s, case):
    seqs, heads, dim = s["q"].shape
    kv, capacity = case["kv_heads"], case["capacity"]
    out = torch.empty_like(s["q"])
    per = max(1, 2 ** 28 // (capacity * kv * dim))
    for lo in range(0, seqs, per):
        n = s["lengths"][lo:lo + per].long()[:, None]
        cols = torch.arange(capacity, device=DEV)[None, :]
        seen = (cols < n) & ((n - 1 - cols < case["window"]) | (cols < case["sinks"]))
        q = s["q"][lo:lo + per].float().view(-1, kv, heads // kv, dim)
        score = torch.einsum("bhgd,bkhd->bhgk", q, s["k"][lo:lo + per].float()) * s["scale"]
        score = score.masked_fill(~seen[:, None, None, :], -math.inf)
        top = score.amax(-1, keepdim=True).clamp(min=-1e30)  # a session without a token has none
        p = (score - top).exp()
        total = p.sum(-1, keepdim=True)
        p = p / torch.where(total == 0, torch.ones_like(total), total)
        out[lo:lo + per] = torch.einsum("bhgk,bkhd->bhgd", p, s["v"][lo:lo + per].float()).reshape(-1, heads, dim).to(
            out.dtype)
    return out


def _plain_clip(s):
    parts = [t.float().square().sum() for t in s["grads"]]
    counted = None
    if "sparse" in s:
        counted = torch.arange(s["sparse"].numel(), device=DEV) < s["count"]
        parts.append((s["sparse"] * counted).square().sum())
    norm = torch.stack(parts).sum().sqrt()
    factor = (s["max_norm"] / (norm + CLIP_EPS)).clamp(max=1.0)
    targets = s.get("clipped", s["grads"])
    for t, to in zip(s["grads"], targets):
        if t.dtype == torch.float32:
            torch.mul(t, factor, out=to)
        else:
            to.copy_(t.float() * factor)
    if "sparse" in s:
        to = s.get("clipped_sparse", s["sparse"])
        to.copy_(torch.where(counted, s["sparse"] * factor, to))
    return _clipped(s, norm)


def _clipped(s, norm):
    """The norm, and the buffers that the scaled gradients are in."""
    result = {"norm": norm, "flat": s.get("clipped_flat", s["flat"]), "table": s.get("clipped_table", s["table"])}
    if "sparse" in s:
        result["sparse"] = s.get("clipped_sparse", s["sparse"])
    return result


def _own(state):
    case = state["case"]
    kind = case["kind"]
    if kind in ("norm", "normgrad"):
        from paper_2609_30656_gb300 import layer_norm as ln
        out = DTYPES[case["out"]]
        if kind == "norm":
            return ln.layer_norm(state["x"], state["weight"], state["bias"], eps=EPS, out_dtype=out, stats=True)
        return ln.layer_norm_backward(state["grad_out"], state["x"], state["mean"], state["rstd"], state["weight"],
                                      bias=state["bias"] is not None, out_dtype=out)
    if kind in ("attn", "attngrad", "step"):
        from paper_2609_30656_gb300 import window_attention as wa
        shape = {"window": case["window"], "sinks": case["sinks"], "scale": state["scale"]}
        if kind == "attn":
            return wa.window_attention(state["q"], state["k"], state["v"], state["offsets"], **shape, stats=True)
        if kind == "attngrad":
            return wa.window_attention_backward(state["grad_out"], state["q"], state["k"], state["v"], state["out"],
                                                state["lse"], state["offsets"], **shape)
        return wa.window_attention_step(state["q"], state["k"], state["v"], state["lengths"], **shape)
    from paper_2609_30656_gb300 import clip
    grads, to = list(state["grads"]), list(state["clipped"]) if case["clipped"] else None
    if case["sparse"]:
        grads.append((state["sparse"], state["count"]))
        if to is not None:
            to.append((state["clipped_sparse"], state["count"]))
    return _clipped(state, clip.clip_grad_norm(grads, state["max_norm"], eps=CLIP_EPS, out=to))


def run(state):
    case = state["case"]
    if own:
        return _own(state)
    if case["kind"] == "norm":
        return _plain_norm(state)
    if case["kind"] == "normgrad":
        return _plain_norm_backward(state)
    if case["kind"] == "attn":
        return _plain_attention(state, case)
    if case["kind"] == "attngrad":
        return _plain_attention_backward(state, case)
    if case["kind"] == "step":
        return _plain_step(state, case)
    return _plain_clip(state)


# ----------------------------------------------------------------------------- what a pass cannot do without

def _pairs(n, window, sinks):
    """Visible pairs of a sequence of n tokens."""
    w = min(window, n)
    near = n * w - w * (w - 1) // 2
    # Query i sees first token j < sinks beside its window where i - j >= window.
    return near + sum(max(0, n - window - j) for j in range(min(sinks, n)))


def work(case):
    kind = case["kind"]
    if kind in ("norm", "normgrad"):
        values, src, dst = case["rows"] * case["dim"], BYTES[case["dtype"]], BYTES[case["out"]]
        params = case["dim"] * (2 if case["bias"] else 1)
        if kind == "norm":
            return {"bytes": values * (src + dst) + params * BYTES[case["params"]] + 8 * case["rows"], "flops": 8 * values}
        return {"bytes": values * (2 * src + dst) + case["dim"] * BYTES[case["params"]] + params * 4 + 8 * case["rows"],
                "flops": 16 * values}
    if kind in ("attn", "attngrad"):
        lens = _lengths(case)
        pairs = sum(_pairs(n, case["window"], case["sinks"]) for n in lens) * case["heads"]
        rows = sum(lens) * case["dim"] * 2
        own_heads, shared = rows * case["heads"], rows * case["kv_heads"]
        index = (case["seqs"] + 1) * (4 if case["index"] == "i32" else 8) + 4 * sum(lens) * case["heads"]
        if kind == "attn":
            return {"bytes": 2 * own_heads + 2 * shared + index, "flops": 4 * case["dim"] * pairs}
        return {"bytes": 4 * own_heads + 4 * shared + index, "flops": 10 * case["dim"] * pairs}
    if kind == "step":
        seen = sum(min(n, case["window"]) + max(0, min(n - case["window"], case["sinks"])) for n in _cached(case))
        return {"bytes": seen * case["kv_heads"] * case["dim"] * 4 + case["seqs"] * case["heads"] * case["dim"] * 4,
                "flops": 4 * seen * case["heads"] * case["dim"]}
    shapes = _shapes(case)
    sizes = [math.prod(shape) * BYTES[case["dtype"]] for shape in shapes[:-1]]
    sizes.append(math.prod(shapes[-1]) * BYTES[case["table"]])
    total = sum(sizes) + 4 * case["sparse"]
    values = sum(math.prod(shape) for shape in shapes) + case["sparse"]
    return {"bytes": total * (2 if case["clipped"] else 1), "flops": values * (3 if case["clipped"] else 2)}


# ----------------------------------------------------------------------------- 64 bits

def _exact_norm(s, case):
    x = s["x"].double()
    mean = x.sum(1) / case["dim"]
    var = x.square().sum(1) / case["dim"] - mean.square()  # values of order 1 to 10: 64 bits have room for it
    rstd = torch.rsqrt(var + EPS)
    w = s["weight"].double()
    if case["kind"] == "norm":
        y = torch.addcmul(-(mean * rstd)[:, None] * w, x * rstd[:, None], w)
        return (y if s["bias"] is None else y + s["bias"].double()), mean, rstd
    mean, rstd = s["mean"].double(), s["rstd"].double()
    dy = s["grad_out"].double()
    # Sums over rows by products with a vector, x-hat never formed.
    shift = mean * rstd
    db = dy.T @ torch.ones_like(mean)
    dw = (dy * x).T @ rstd - dy.T @ shift
    a = dy @ w / case["dim"]
    b = ((dy * x) @ w * rstd - (dy @ w) * shift) / case["dim"]
    dx = rstd[:, None] * (dy * w - a[:, None] - (x * rstd[:, None] - shift[:, None]) * b[:, None])
    return dx, dw, (db if s["bias"] is not None else None)


def _exact_attention(s, case):
    """Sequence after sequence, 256 queries at a time with the keys that any of them sees."""
    tokens, heads, dim = s["q"].shape
    kv, group = case["kv_heads"], case["heads"] // case["kv_heads"]
    back = case["kind"] == "attngrad"
    out = torch.zeros(tokens, heads, dim, dtype=torch.float64, device=DEV)
    lse = torch.zeros(heads, tokens, dtype=torch.float64, device=DEV)
    dq, dk, dv = (torch.zeros(tokens, h, dim, dtype=torch.float64, device=DEV) for h in (heads, kv, kv))
    at = 0
    for n in s["lens"]:
        for lo in range(0, n, 256):
            hi = min(lo + 256, n)
            first = max(0, lo - case["window"] + 1)
            cols = torch.cat([torch.arange(min(case["sinks"], first), device=DEV), torch.arange(first, hi, device=DEV)])
            rows = torch.arange(lo, hi, device=DEV)
            hidden = (cols > rows[:, None]) | ((cols <= rows[:, None] - case["window"]) & (cols >= case["sinks"]))
            q = s["q"][at + rows].double().view(-1, kv, group, dim).permute(1, 2, 0, 3).reshape(kv, -1, dim)
            k, v = (s[x][at + cols].double().transpose(0, 1) for x in ("k", "v"))
            score = (q * s["scale"]) @ k.mT
            score = score.view(kv, group, len(rows), -1).masked_fill_(hidden, -math.inf).view(kv, -1, len(cols))
            e = torch.logsumexp(score, -1, keepdim=True)
            p = torch.exp(score - e)
            o = p @ v
            if not back:
                out[at + rows] = o.view(heads, -1, dim).transpose(0, 1)
                lse[:, at + rows] = e.view(heads, -1)
                continue
            do = s["grad_out"][at + rows].double().view(-1, kv, group, dim).permute(1, 2, 0, 3).reshape(kv, -1, dim)
            ds = p * (do @ v.mT - (do * o).sum(-1, keepdim=True)) * s["scale"]
            dq[at + rows] = (ds @ k).view(heads, -1, dim).transpose(0, 1)
            dk.index_add_(0, at + cols, (ds.mT @ q).transpose(0, 1))
            dv.index_add_(0, at + cols, (p.mT @ do).transpose(0, 1))
        at += n
    return (dq, dk, dv) if back else (out, lse)


def _exact_step(s, case):
    heads, dim, kv = case["heads"], case["dim"], case["kv_heads"]
    out = torch.zeros(case["seqs"], heads, dim, dtype=torch.float64, device=DEV)
    for i, n in enumerate(s["lens"]):
        if not n:
            continue
        first = max(0, n - case["window"])
        cols = list(range(min(case["sinks"], first))) + list(range(first, n))
        k, v = (s[x][i, cols].double().transpose(0, 1) for x in ("k", "v"))
        q = s["q"][i].double().view(kv, -1, dim)
        out[i] = (torch.softmax(q @ k.mT * s["scale"], -1) @ v).view(heads, dim)
    return out


def _exact_clip(s):
    norm = math.sqrt(math.fsum(torch.linalg.vector_norm(t.double()).item() ** 2 for t in s["grads"]) +
                     (torch.linalg.vector_norm(s["sparse"][:s["case"]["sparse"]].double()).item() ** 2
                      if "sparse" in s else 0.0))
    factor = min(1.0, s["max_norm"] / (norm + CLIP_EPS))
    result = {"norm": torch.tensor(norm, dtype=torch.float64, device=DEV), "flat": s["flat"].double() * factor,
              "table": s["table"].double() * factor}
    if "sparse" in s:
        n = s["case"]["sparse"]
        rest = s.get("clipped_sparse", s["sparse"])
        result["sparse"] = torch.cat([s["sparse"][:n].double() * factor, rest[n:].double()])
    return result


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] in ("norm", "normgrad"):
        return _exact_norm(s, case)
    if case["kind"] in ("attn", "attngrad"):
        return _exact_attention(s, case)
    if case["kind"] == "step":
        return _exact_step(s, case)
    return _exact_clip(s)
