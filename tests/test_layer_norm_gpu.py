"""Layer normalisation and its backward pass against 64 bits (GPU).

Tolerances, with u = 2^-24 and h the output type's half step (eps / 2, relative). A row's sum is taken in at
most S additions one after another: 16 in a thread, 5 in a warp, 5 over warps (D / 1024 + 10 for rows over 16384),
each off by u of the sum of magnitudes.
  mean      S u mean|x|
  rstd      relative: half of the variance's (S + 3) u, two roundings, and mean's error squared, below them
  out       |w| r (mean's error) + (S / 2 + 6) u |w xh| + u (|w xh| + |b|) + h |out|
  xh        2 u |xh| from the mean and rstd given
  grad_x    r (2 u |g| + S u mean|g| + |xh| (S + 4) u mean|g xh| + 4 u |xh mean(g xh)| + 3 u |all|) + h |grad_x|
  grad_weight, grad_bias  N u (sum of magnitudes); N = 300 covers rows of a thread (under 40), the groups of a
            block (4), the blocks' sums of a warp (at most 77), its warps (8), and a term's own roundings (4)
"""

import math

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
TYPES = [torch.float32, torch.float16, torch.bfloat16]


def _ln():
    from paper_2609_30656_gb300 import layer_norm
    return layer_norm


def _half(dtype):
    return torch.finfo(dtype).eps / 2


def _tiny(dtype):  # half a step of the smallest numbers
    return torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps / 2


def _depth(dim):
    return 26 if dim <= 16384 else dim / 1024 + 11


def _rand(g, *shape, dtype=torch.float32, std=1.0, shift=0.0):
    return (torch.randn(shape, generator=g, device=DEV) * std + shift).to(dtype)


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def check_forward(x, w, b, eps, y, mean, rstd):
    xd = x.double()
    S = _depth(x.shape[-1])
    m = xd.mean(-1, keepdim=True)
    r = 1 / ((xd - m).square().mean(-1, keepdim=True) + eps).sqrt()
    wd = torch.ones_like(xd[..., :1]) if w is None else w.double()
    bd = torch.zeros_like(xd[..., :1]) if b is None else b.double()
    scaled = (xd - m) * r * wd
    want = scaled + bd
    m_err = S * U * xd.abs().mean(-1, keepdim=True)
    assert ((mean.double() - m.squeeze(-1)).abs() <= m_err.squeeze(-1) + 1e-44).all()
    r_rel = (S / 2 + 4) * U + 2 * (m_err * r).square()
    assert ((rstd.double() - r.squeeze(-1)).abs() <= (r_rel * r).squeeze(-1)).all()
    tol = wd.abs() * r * m_err + (r_rel + 3 * U) * scaled.abs() + U * (scaled.abs() + bd.abs()) + _half(y.dtype) * want.abs()
    tol = tol * (1 + 2 ** -7) + _tiny(y.dtype)
    assert ((y.double() - want).abs() <= tol).all()


def check_backward(go, x, mean, rstd, w, dx, dw, db):
    D = x.shape[-1]
    S = _depth(D)
    xh = (x.double() - mean.double().unsqueeze(-1)) * rstd.double().unsqueeze(-1)
    d = go.double()
    g = d if w is None else d * w.double()
    r = rstd.double().unsqueeze(-1)
    m0, m1 = g.mean(-1, keepdim=True), (g * xh).mean(-1, keepdim=True)
    want = r * (g - m0 - xh * m1)
    every = g.abs() + m0.abs() + (xh * m1).abs()
    tol = r * U * (2 * g.abs() + S * g.abs().mean(-1, keepdim=True) + xh.abs() * (S + 4) * (g * xh).abs().mean(-1, keepdim=True)
                   + 4 * (xh * m1).abs() + 3 * every) + _half(dx.dtype) * want.abs()
    assert ((dx.double() - want).abs() <= tol * (1 + 2 ** -7) + _tiny(dx.dtype)).all()
    over = tuple(range(x.dim() - 1))
    for got, terms in ((dw, d * xh), (db, d)):
        if got is not None:
            assert got.dtype == torch.float32
            assert ((got.double() - terms.sum(over)).abs() <= 300 * U * terms.abs().sum(over) + 1e-44).all()


DIMS = [1, 2, 7, 8, 31, 32, 64, 100, 505, 512, 513, 1000, 1001, 2048, 4093, 4096, 8192, 8191, 12289, 16384, 16377, 16385, 20008]


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("dim", DIMS)
def test_rows_of_every_length(dim, dtype):
    ln = _ln()
    g = _gen(dim)
    for rows in (1, 9, 67):
        x = _rand(g, rows, dim, dtype=dtype, shift=0.5)
        w, b = _rand(g, dim, dtype=dtype, std=0.2, shift=1.0), _rand(g, dim)
        y, mean, rstd = ln.layer_norm(x, w, b, eps=1e-3, stats=True)
        assert y.dtype == dtype and y.shape == x.shape and mean.shape == rstd.shape == (rows,)
        check_forward(x, w, b, 1e-3, y, mean, rstd)
        go = _rand(g, rows, dim, dtype=dtype)
        check_backward(go, x, mean, rstd, w, *ln.layer_norm_backward(go, x, mean, rstd, w))


@pytest.mark.parametrize("dim", [64, 200, 1001, 4096, 17000])
@pytest.mark.parametrize("out", TYPES, ids=str)
@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_every_pair_of_types_with_and_without_parameters(dtype, out, dim):
    ln = _ln()
    g = _gen(dim + 1)
    x, go = _rand(g, 5, 7, dim, dtype=dtype), _rand(g, 5, 7, dim, dtype=dtype)
    for w, b in ((None, None), (_rand(g, dim, dtype=out), None), (None, _rand(g, dim, dtype=torch.float16))):
        y, mean, rstd = ln.layer_norm(x, w, b, out_dtype=out, stats=True)
        assert y.dtype == out and mean.shape == (5, 7)
        check_forward(x, w, b, 1e-5, y, mean, rstd)
        dx, dw, db = ln.layer_norm_backward(go, x, mean, rstd, w, bias=b is not None, out_dtype=out)
        assert (dw is None) == (w is None) and (db is None) == (b is None) and dx.dtype == out
        check_backward(go, x, mean, rstd, w, dx, dw, db)


@pytest.mark.parametrize("rows,dim", [(5000, 24), (40000, 33), (5000, 1024), (3003, 1001), (2000, 5000)])
def test_many_rows(rows, dim):
    ln = _ln()
    g = _gen(rows)
    for dtype in (torch.float32, torch.bfloat16):
        x, go, w = _rand(g, rows, dim, dtype=dtype), _rand(g, rows, dim, dtype=dtype), _rand(g, dim)
        y, mean, rstd = ln.layer_norm(x, w, stats=True)
        check_forward(x, w, None, 1e-5, y, mean, rstd)
        first = ln.layer_norm_backward(go, x, mean, rstd, w)
        check_backward(go, x, mean, rstd, w, *first)
        for a, b in zip(first, ln.layer_norm_backward(go, x, mean, rstd, w)):
            assert torch.equal(a, b)  # the same bits every time


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("dim", [9, 40, 333, 1024, 3001])
def test_strides_and_alignments(dim, dtype):
    """Slices of wider rows, rows that begin anywhere, results in such places; what lies beside them stays."""
    ln = _ln()
    g = _gen(dim)
    for pad, begin in ((3, 1), (8, 0), (8, 8), (5, 2), (16, 3)):
        flat = _rand(g, 11 * (dim + pad) + 32, dtype=dtype)
        x = flat[begin:begin + 11 * (dim + pad)].view(11, dim + pad)[:, :dim]
        go = _rand(g, 11, dim + 1, dtype=dtype)[:, 1:]
        w, b = _rand(g, dim + 1)[1:], _rand(g, dim, dtype=dtype)
        room = torch.full((11 * (dim + pad) + 32,), 7.0, dtype=dtype, device=DEV)
        for out_begin in (begin, 0):
            y = room[out_begin:out_begin + 11 * (dim + pad)].view(11, dim + pad)[:, :dim]
            room.fill_(7.0)
            got, mean, rstd = ln.layer_norm(x, w, b, out=y, stats=True)
            assert got.data_ptr() == y.data_ptr()
            check_forward(x, w, b, 1e-5, y, mean, rstd)
            beside = torch.ones_like(room, dtype=torch.bool)
            beside[out_begin:out_begin + 11 * (dim + pad)].view(11, dim + pad)[:, :dim] = False
            assert (room[beside] == 7.0).all()
            room.fill_(7.0)
            dx, dw, db = ln.layer_norm_backward(go, x, mean, rstd, w, out=y)
            check_backward(go, x, mean, rstd, w, dx, dw, db)
            assert (room[beside] == 7.0).all()


def test_other_layouts_are_copied_or_refused():
    ln = _ln()
    g = _gen(3)
    x = _rand(g, 6, 10, 40).permute(1, 0, 2)  # rows in two strides that are not one
    y, mean, rstd = ln.layer_norm(x, stats=True)
    check_forward(x, None, None, 1e-5, y, mean, rstd)
    t = _rand(g, 40, 12).T  # columns that are contiguous
    y, mean, rstd = ln.layer_norm(t, stats=True)
    check_forward(t, None, None, 1e-5, y, mean, rstd)
    check_backward(t, t, mean, rstd, None, *ln.layer_norm_backward(t, t, mean, rstd))
    one = _rand(g, 1, 40).expand(9, 40)  # the same row again and again
    y, mean, rstd = ln.layer_norm(one, stats=True)
    check_forward(one, None, None, 1e-5, y, mean, rstd)
    c = _rand(g, 3, 8)
    for bad in (lambda: ln.layer_norm(c, out=torch.empty(8, 3, device=DEV).T),
                lambda: ln.layer_norm(c, out=c[:1].expand(3, 8)), lambda: ln.layer_norm(c, out=c[:2]),
                lambda: ln.layer_norm(c, weight=c), lambda: ln.layer_norm(c, weight=c[0].double()),
                lambda: ln.layer_norm(c, bias=torch.ones(8)), lambda: ln.layer_norm(c.double()),
                lambda: ln.layer_norm(torch.tensor(1.0, device=DEV)),
                lambda: ln.layer_norm(c.half(), out=c.half().float().half()[:, :7]),
                lambda: ln.layer_norm_backward(c.half(), c, c[:, 0], c[:, 0]),
                lambda: ln.layer_norm_backward(c, c, c[:, :1], c[:, 0]),
                lambda: ln.layer_norm_backward(c, c, c[:, 0].half(), c[:, 0])):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(TypeError):
        ln.layer_norm(c, out=torch.empty_like(c), out_dtype=torch.float16)
    with pytest.raises(Exception):
        ln.layer_norm(c, eps=-1.0)


@pytest.mark.parametrize("dim", [40, 41, 1024, 1027, 18000])
def test_in_place(dim):
    ln = _ln()
    g = _gen(dim)
    x, go, w = _rand(g, 33, dim), _rand(g, 33, dim), _rand(g, dim)
    y, mean, rstd = ln.layer_norm(x, w, stats=True)
    copy = x.clone()
    assert torch.equal(ln.layer_norm(copy, w, out=copy), y)
    dx, dw, db = ln.layer_norm_backward(go, x, mean, rstd, w)
    for which in (0, 1):
        a, b = go.clone(), x.clone()
        got = ln.layer_norm_backward(a, b, mean, rstd, w, out=(a, b)[which])
        assert all(torch.equal(s, t) for s, t in zip(got, (dx, dw, db)))
    with pytest.raises(ValueError):
        ln.layer_norm(x, out=x.view(torch.float16)[:, :dim])


def test_empty_tensors():
    ln = _ln()
    x = torch.empty(0, 16, device=DEV)
    y, mean, rstd = ln.layer_norm(x, stats=True)
    assert y.shape == (0, 16) and mean.shape == (0,)
    dx, dw, db = ln.layer_norm_backward(x, x, mean, rstd, torch.ones(16, device=DEV))
    assert dx.shape == (0, 16) and torch.equal(dw, torch.zeros_like(dw)) and torch.equal(db, torch.zeros_like(db))
    x = torch.empty(3, 0, device=DEV)
    assert ln.layer_norm(x).shape == (3, 0)


def test_large_means_small_spreads_and_rows_with_nan():
    ln = _ln()
    g = _gen(5)
    x = _rand(g, 40, 2000, shift=1000.0)  # sum x^2 - mean^2 would lose half of the digits of the variance
    y, mean, rstd = ln.layer_norm(x, stats=True)
    check_forward(x, None, None, 1e-5, y, mean, rstd)
    x = _rand(g, 6, 64)
    x[1, 3], x[2, 5], x[3] = float("nan"), float("inf"), 2.5
    y, mean, rstd = ln.layer_norm(x, stats=True)
    assert y[1].isnan().all() and y[2].isnan().all() and (y[3] == 0).all()
    assert rstd[3].item() == pytest.approx(1e-5 ** -0.5, rel=1e-6)
    for row in (0, 4, 5):
        assert torch.equal(y[row], ln.layer_norm(x[row:row + 1])[0])


def test_gradients_against_differences():
    ln = _ln()
    g = _gen(9)
    x, w, b, go = _rand(g, 4, 24), _rand(g, 24, shift=1.0), _rand(g, 24), _rand(g, 4, 24)
    _, mean, rstd = ln.layer_norm(x, w, b, stats=True)
    grads = ln.layer_norm_backward(go, x, mean, rstd, w)
    def loss(x, w, b):
        x, w, b = x.double(), w.double(), b.double()
        c = x - x.mean(-1, keepdim=True)
        return ((c / (c.square().mean(-1, keepdim=True) + 1e-5).sqrt() * w + b) * go.double()).sum()
    step = 2.0 ** -8
    for k, t in enumerate((x, w, b)):
        for _ in range(4):
            way = _rand(g, *t.shape)
            args = [[s if i != k else s.double() + sign * step * way.double() for i, s in enumerate((x, w, b))]
                    for sign in (1, -1)]
            slope = (loss(*args[0]) - loss(*args[1])) / (2 * step)
            # central differences: off by step^2 / 6 of the third derivative along `way` (a few hundred here)
            assert abs((grads[k].double() * way.double()).sum() - slope) < 1e-4 * 100


def test_streams_and_graphs():
    ln = _ln()
    g = _gen(11)
    x, go, w = _rand(g, 300, 1001), _rand(g, 300, 1001), _rand(g, 1001)
    y, mean, rstd = ln.layer_norm(x, w, stats=True)
    want = (y, mean, rstd, *ln.layer_norm_backward(go, x, mean, rstd, w))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = ln.layer_norm(x, w, stats=True)
        got = (*other, *ln.layer_norm_backward(go, x, other[1], other[2], w))
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        other = ln.layer_norm(x, w, stats=True)
        got = (*other, *ln.layer_norm_backward(go, x, other[1], other[2], w))
    for scale in (1.0, 3.0):
        x.mul_(scale)
        graph.replay()
        y, mean, rstd = ln.layer_norm(x, w, stats=True)
        want = (y, mean, rstd, *ln.layer_norm_backward(go, x, mean, rstd, w))
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_offsets_past_32_bits():
    ln = _ln()
    rows, dim = 70000, 64
    wide = torch.empty(rows * 65536 // 2 + 64, dtype=torch.bfloat16, device=DEV)  # 4.6 GB
    x = wide.as_strided((rows, dim), (32768, 1))
    x.copy_(_rand(_gen(1), rows, dim))
    y, mean, rstd = ln.layer_norm(x, stats=True)
    check_forward(x, None, None, 1e-5, y, mean, rstd)
    assert math.isfinite(y.float().sum().item())


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("gap", [0, 1, 5])
@pytest.mark.parametrize("dim", [1, 7, 33, 1001])
def test_neighbours_at_a_rows_ends_stay_out_of_it(dim, gap, dtype):
    """Odd rows share 16-byte pieces with the rows (or what lies between them) before and behind."""
    from paper_2609_30656_gb300 import layer_norm as ln
    g = torch.Generator(device=DEV)
    g.manual_seed(dim)
    x, dy = (torch.randn(41, dim + gap, generator=g, device=DEV).to(dtype) for _ in range(2))
    w = torch.randn(dim, generator=g, device=DEV)
    clean = [t.clone()[:, :dim] for t in (x, dy)]  # lying alike: a row's sums go by where it begins
    for t in (x, dy):
        t[::2] = float("nan")
        t[:, dim:] = float("inf")
    runs = []
    for a, b in ((x[:, :dim], dy[:, :dim]), clean):
        y, mean, rstd = ln.layer_norm(a, w, w, stats=True)
        runs.append((y, mean, rstd, ln.layer_norm_backward(b, a, mean, rstd, w)[0]))
    for got, want in zip(*runs):
        assert torch.equal(got[1::2], want[1::2]) and got[::2].isnan().all()
