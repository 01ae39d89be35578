"""The norm over all gradients and clipping to it, against 64 bits (GPU).

Tolerances, u = 2^-24. Squares of 8 values are summed in fp32 (at most 8 u of a sum of positive terms); what the
additions of those sums round off is kept, the last ones are in fp64: 8 u of the sum, 4 u of the norm, and one
rounding: 5 u. The factor: 4 u of the norm's and one rounding; a product's rounding to fp32 and one to its type.
"""

import math

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
TYPES = [torch.float32, torch.float16, torch.bfloat16]


def _clip():
    from paper_2609_30656_gb300 import clip
    return clip


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _rand(g, *shape, dtype=torch.float32, std=1.0):
    return (torch.randn(shape, generator=g, device=DEV) * std).to(dtype)


def _norm(grads):
    return math.sqrt(math.fsum(t.double().square().sum().item() for t in grads))


def _check_scaled(got, was, norm, max_norm, eps):
    f = min(1.0, max_norm / (norm + eps))
    want = was.double() * f
    if f == 1.0 and got.dtype == was.dtype:
        assert torch.equal(got, was)
        return
    info = torch.finfo(got.dtype)
    half = info.eps / 2 if got.dtype != torch.float32 else 0.0
    tol = (7 * U + half) * want.abs() * (1 + 2 ** -7) + info.smallest_normal * info.eps
    assert ((got.double() - want).abs() <= tol).all()


SHAPES = [(1,), (7,), (8,), (33, 5), (129, 64), (1, 1000), (4097,), (300, 301), (8192,), (8193,), (70000,)]


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_tensors_of_every_size(dtype):
    clip = _clip()
    g = _gen(1)
    for shape in SHAPES:
        t = _rand(g, *shape, dtype=dtype)
        norm = _norm([t])
        assert abs(clip.grad_norm([t]).item() - norm) <= 5 * U * norm
        for max_norm in (norm * 2, norm * 0.3, 0.0):
            c = t.clone()
            got = clip.clip_grad_norm([c], max_norm)
            assert abs(got.item() - norm) <= 5 * U * norm
            _check_scaled(c, t, norm, max_norm, 1e-6)


@pytest.mark.parametrize("count", [2, 24, 25, 100, 400, 401, 900])
def test_many_tensors_of_mixed_types(count):
    clip = _clip()
    g = _gen(count)
    grads = [_rand(g, 1 + (37 * i) % 511, dtype=TYPES[i % 3], std=10.0 ** (i % 5 - 2)) for i in range(count)]
    norm = _norm(grads)
    was = [t.clone() for t in grads]
    assert abs(clip.grad_norm(grads).item() - norm) <= 5 * U * norm
    got = clip.clip_grad_norm(grads, norm / 3, eps=0.0)
    assert abs(got.item() - norm) <= 5 * U * norm
    for a, b in zip(grads, was):
        _check_scaled(a, b, norm, norm / 3, 0.0)
    again = [t.clone() for t in was]
    assert torch.equal(clip.clip_grad_norm(again, norm / 3, eps=0.0), got)
    assert all(torch.equal(a, b) for a, b in zip(again, grads))  # the same bits every time


@pytest.mark.parametrize("to", TYPES, ids=str)
@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_into_other_tensors_of_other_types(dtype, to):
    clip = _clip()
    g = _gen(4)
    flat, room = _rand(g, 40000, dtype=dtype), torch.full((40064,), 5.0, dtype=to, device=DEV)
    for begin, out_begin, n in ((0, 0, 40000), (1, 1, 9000), (3, 0, 8200), (0, 5, 8190), (5, 13, 17), (2, 2, 0)):
        t = flat[begin:begin + n]
        room.fill_(5.0)
        out = room[out_begin:out_begin + n]
        was = t.clone()
        norm = _norm([t, t])  # reading a tensor twice is allowed where it is not written
        spare = torch.empty(n, dtype=to, device=DEV)
        got = clip.clip_grad_norm([t, t], 0.5 * norm, out=[out, spare])
        assert abs(got.item() - norm) <= 5 * U * norm
        assert torch.equal(t, was) and torch.equal(out, spare)
        _check_scaled(out, t, norm, 0.5 * norm, 1e-6)
        assert (room[:out_begin] == 5.0).all() and (room[out_begin + n:] == 5.0).all()
        clip.clip_grad_norm([t], 10 * norm + 1.0, out=[out])  # not clipped: copied
        assert torch.equal(out, t.to(to))


def test_layouts():
    clip = _clip()
    g = _gen(6)
    whole = _rand(g, 50, 96)
    was = whole.clone()
    left, right = whole[:, :40], whole[:, 41:]
    norm = _norm([left, right])
    assert abs(clip.clip_grad_norm([left, right], 1.0).item() - norm) <= 5 * U * norm
    _check_scaled(left, was[:, :40], norm, 1.0, 1e-6)
    _check_scaled(right, was[:, 41:], norm, 1.0, 1e-6)
    assert torch.equal(whole[:, 40], was[:, 40])
    t = _rand(g, 30, 20, 10)
    p = t.permute(2, 0, 1)
    was = p.clone()
    norm = _norm([p])
    clip.clip_grad_norm(p, 2.0)
    _check_scaled(p, was, norm, 2.0, 1e-6)
    src, dst = _rand(g, 60, 33), torch.zeros(60, 50, device=DEV)[:, 3:36]
    clip.clip_grad_norm([src], 2.0, out=[dst])
    _check_scaled(dst, src, _norm([src]), 2.0, 1e-6)


def test_counted_values_and_sparse_gradients():
    clip = _clip()
    from paper_2609_30656_gb300 import tbe
    g = _gen(8)
    dense = _rand(g, 1000)
    for n in (0, 1, 5000, 8192, 20000):
        values, count = _rand(g, 20000), torch.tensor([n], device=DEV)
        values[n:] = float("nan")
        was = values.clone()
        d = dense.clone()
        norm = _norm([d, values[:n]])
        got = clip.clip_grad_norm([d, (values, count)], 3.0)
        assert abs(got.item() - norm) <= 5 * U * norm
        _check_scaled(values[:n], was[:n], norm, 3.0, 1e-6)
        assert values[n:].isnan().all()
    table = _rand(g, 200, 64)
    m = tbe.TBE([table])
    ind = torch.randint(0, 200, (300,), generator=g, device=DEV)
    off = torch.arange(0, 301, 10, device=DEV)
    sparse = m.backward(ind, off, _rand(g, 30, 64))
    was = sparse.grads.clone()
    n = sparse.num_floats
    norm = _norm([was[:n], dense])
    got = clip.clip_grad_norm([sparse, dense], 0.5)
    assert abs(got.item() - norm) <= 5 * U * norm
    _check_scaled(sparse.grads[:n], was[:n], norm, 0.5, 1e-6)
    m.apply_sparse(sparse, lr=1.0)


def test_all_magnitudes():
    clip = _clip()
    for scale in (1e-44, 1e-38, 1e-30, 1e-20, 1e-10, 1.0, 1e10, 1e19, 1e30):
        t = torch.linspace(0.5, 2.0, 3001, device=DEV) * scale
        norm = _norm([t])
        assert abs(clip.grad_norm([t]).item() - norm) <= 5 * U * norm + 1e-45, scale
    mixed = torch.cat([torch.full((100,), 1e-30, device=DEV), torch.zeros(5000, device=DEV), torch.full((50,), 1e25, device=DEV)])
    norm = _norm([mixed])
    assert abs(clip.grad_norm([mixed]).item() - norm) <= 5 * U * norm
    small = torch.zeros(100000, device=DEV)
    small[::7] = 1e-25
    norm = _norm([small])
    assert abs(clip.grad_norm([small]).item() - norm) <= 5 * U * norm
    c = mixed.clone()
    clip.clip_grad_norm([c], 1.0)
    _check_scaled(c, mixed, _norm([mixed]), 1.0, 1e-6)


def test_zeros_nan_and_infinities():
    clip = _clip()
    z = torch.zeros(100, device=DEV)
    assert clip.clip_grad_norm([z], 1.0).item() == 0.0 and (z == 0).all()
    assert clip.clip_grad_norm([z], 0.0, eps=0.0).item() == 0.0 and (z == 0).all()  # not 0 / 0
    e = torch.empty(0, device=DEV)
    assert clip.grad_norm([e]).item() == 0.0 and clip.clip_grad_norm([e], 1.0).item() == 0.0
    t = torch.ones(50, device=DEV)
    t[7] = float("inf")
    assert clip.clip_grad_norm([t], 1.0).item() == float("inf")
    assert t[7].isnan() and (t[:7] == 0).all()
    t = torch.ones(50, device=DEV, dtype=torch.bfloat16)
    t[7] = float("nan")
    assert math.isnan(clip.clip_grad_norm([t], 1.0).item()) and t.isnan().all()


def test_refusals():
    clip = _clip()
    from paper_2609_30656_gb300 import tbe
    t = torch.ones(6, 8, device=DEV)
    n = torch.tensor([3], device=DEV)
    for bad in (lambda: clip.grad_norm([]), lambda: clip.grad_norm([t.double()]), lambda: clip.grad_norm([t[:, ::2][:, :3]]),
                lambda: clip.grad_norm([(t, n.int())]), lambda: clip.grad_norm([(t.half(), n)]),
                lambda: clip.grad_norm([(t[:, :4], n)]), lambda: clip.clip_grad_norm([t], 1.0, out=[t, t]),
                lambda: clip.clip_grad_norm([t], 1.0, out=[t[:3]]), lambda: clip.clip_grad_norm([(t, n)], 1.0, out=[t]),
                lambda: clip.clip_grad_norm([t], 1.0, out=[torch.ones(8, 6, device=DEV).T])):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(TypeError):
        clip.grad_norm([3.0])
    was = t.clone()
    for bad in (lambda: clip.clip_grad_norm([t, t], 1.0), lambda: clip.clip_grad_norm([t, t[2:]], 1.0),
                lambda: clip.clip_grad_norm([t], -1.0), lambda: clip.clip_grad_norm([t], float("nan")),
                lambda: clip.clip_grad_norm([t[:5]], 1.0, out=[t[1:]])):
        with pytest.raises(tbe.CbTbeError):
            bad()
    assert torch.equal(t, was)


def test_streams_and_graphs():
    clip = _clip()
    g = _gen(13)
    source = [_rand(g, n, dtype=TYPES[n % 3]) for n in (100, 8193, 50000, 7)]
    work = [torch.empty_like(t) for t in source]

    def step():
        for a, b in zip(work, source):
            a.copy_(b)
        return clip.clip_grad_norm(work, 10.0)

    want = step()
    kept = [t.clone() for t in work]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = step()
    side.synchronize()
    assert torch.equal(got, want) and all(torch.equal(a, b) for a, b in zip(work, kept))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for t in work:
        t.zero_()
    graph.replay()
    assert torch.equal(got, want) and all(torch.equal(a, b) for a, b in zip(work, kept))
    source[1].mul_(2.0)
    graph.replay()
    norm = _norm(source)
    assert abs(got.item() - norm) <= 5 * U * norm


def test_values_past_32_bits():
    clip = _clip()
    t = torch.zeros(2 ** 31 + 2 ** 20 + 11, dtype=torch.bfloat16, device=DEV)
    t[-3:] = 2.0
    t[5] = 3.0
    assert clip.clip_grad_norm([t], 1.0).item() == pytest.approx(math.sqrt(21.0), rel=5 * U)
    assert t[-1].item() == pytest.approx(2.0 / math.sqrt(21.0), rel=2 ** -8) and t[5].item() > 0.6


def test_one_place_is_written_once():
    from paper_2609_30656_gb300 import tbe
    clip = _clip()
    g = _gen(12)
    a, b = _rand(g, 40, 16), _rand(g, 40, 16)
    was = a.clone()
    for grads, out in (([a, b, a], None), ([a, a], [b, b]), ([a, b], [b, torch.empty_like(a)]), ([a[:8], a], None)):
        with pytest.raises(tbe.CbTbeError):
            clip.clip_grad_norm(grads, 0.1, out=out)
    assert torch.equal(a, was)
    # The norm of a list reads alone; empty tensors lie nowhere.
    assert abs(clip.grad_norm([a, a]).item() - _norm([a, a])) <= 5 * U * _norm([a, a])
    clip.clip_grad_norm([a[:0], a, a[:0]], 0.1)
    _check_scaled(a, was, _norm([was]), 0.1, 1e-6)
