"""Windowed attention over packed sessions, its backward pass, and the form for one new token, against 64 bits
(GPU). The bounds are derived in attention_reference.py."""

import pytest
import torch

from tests.attention_reference import check, reference, visible

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HALVES = [torch.bfloat16, torch.float16]


def _wa():
    from paper_2609_30656_gb300 import window_attention
    return window_attention


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _rand(g, *shape, dtype, std=1.0):
    return (torch.randn(shape, generator=g, device=DEV) * std).to(dtype)


def _offsets(lens, begin=0, dtype=torch.int32):
    return (torch.tensor([0] + list(lens), device=DEV).cumsum(0) + begin).to(dtype)


def run_and_check(lens, heads, kv, dim, dtype, window, sinks, begin=0, behind=0, seed=0, index=torch.int32, scale=None, std=1.0,
                  fused=False):
    wa = _wa()
    g = _gen(seed)
    tokens = begin + sum(lens) + behind
    if fused:
        whole = _rand(g, tokens, heads + 2 * kv, dim, dtype=dtype, std=std)
        q, k, v = whole.split([heads, kv, kv], dim=1)
    else:
        q, k, v = (_rand(g, tokens, n, dim, dtype=dtype, std=std) for n in (heads, kv, kv))
    go = _rand(g, tokens, heads, dim, dtype=dtype)
    off = _offsets(lens, begin, index)
    error = torch.zeros(1, dtype=torch.int32, device=DEV)
    out, lse = wa.window_attention(q, k, v, off, window, sinks, scale, stats=True, error=error)
    grads = wa.window_attention_backward(go, q, k, v, out, lse, off, window, sinks, scale, error=error)
    assert error.item() == 0
    seen = visible(tokens, lens, window if window is not None else tokens, sinks, begin)
    want = reference(q, k, v, seen, dim ** -0.5 if scale is None else scale, go)
    check(out, want["out"], "out")
    check(lse, want["lse"], "lse")
    for got, name in zip(grads, ("dq", "dk", "dv")):
        assert got.dtype == dtype
        check(got, want[name], name)
    return q, k, v, go, off, out, lse, grads


@pytest.mark.parametrize("dtype", [*HALVES, torch.float32], ids=str)
@pytest.mark.parametrize("lens,window,sinks", [
    ([1], 1, 0), ([1, 1, 1], 5, 2), ([50, 0, 3, 77, 1, 0, 0, 129], 20, 2), ([128], None, 0), ([129], 64, 0),
    ([300], 100, 4), ([127, 1, 128, 256], 128, 1), ([64] * 9, 1, 0), ([5] * 60, 3, 1), ([500, 20], 7, 0), ([513], 600, 9),
    ([40, 700], 130, 140), ([260, 300], 1, 1)], ids=str)
def test_sessions_windows_and_sinks(lens, window, sinks, dtype):
    run_and_check(lens, 2, 2, 64, dtype, window, sinks, seed=len(lens))


@pytest.mark.parametrize("dtype", [*HALVES, torch.float32], ids=str)
@pytest.mark.parametrize("dim", [1, 7, 8, 16, 24, 32, 40, 64, 72, 80, 96, 100, 120, 128, 136, 200, 256])
def test_widths_of_heads(dim, dtype):
    run_and_check([150, 30, 90], 2, 1, dim, dtype, 70, 3, seed=dim)


@pytest.mark.parametrize("heads,kv", [(1, 1), (3, 3), (4, 2), (6, 1), (8, 2), (16, 4), (32, 32)])
def test_shared_heads(heads, kv):
    run_and_check([200, 61], heads, kv, 64, torch.bfloat16, 90, 4, seed=heads, index=torch.int64)


@pytest.mark.parametrize("dtype", HALVES, ids=str)
def test_slices_of_one_product(dtype):
    run_and_check([33, 250], 4, 2, 40, dtype, 50, 2, fused=True)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=str)
@pytest.mark.parametrize("begin,behind", [(5, 0), (0, 9), (130, 140), (1, 300)])
def test_tokens_of_no_session_give_zeros(begin, behind, dtype):
    q, k, v, go, off, out, lse, grads = run_and_check([60, 0, 100], 2, 1, 64, dtype, 40, 2, begin, behind)
    for lo, hi in ((0, begin), (begin + 160, begin + 160 + behind)):
        assert (out[lo:hi] == 0).all() and (lse[:, lo:hi] == -torch.inf).all()
        assert all((t[lo:hi] == 0).all() for t in grads)


@pytest.mark.parametrize("dim", [64, 128])
def test_longer_sequences(dim):
    run_and_check([1500, 700, 2000], 2, 1, dim, torch.bfloat16, 300, 5, seed=3)
    run_and_check([3000], 1, 1, dim, torch.float16, None, 0, seed=4)
    run_and_check([2600, 3], 2, 2, dim, torch.bfloat16, 40, 200, seed=5)


def test_large_scores_and_scales():
    # Scores of up to a few hundred: the running maximum carries them.
    run_and_check([400], 2, 2, 64, torch.bfloat16, 200, 2, std=6.0, seed=6)
    run_and_check([400], 2, 2, 64, torch.float16, 200, 2, scale=0.01, seed=7)
    run_and_check([400], 2, 2, 64, torch.bfloat16, 200, 2, scale=-0.3, seed=8)
    run_and_check([400], 2, 2, 64, torch.bfloat16, 200, 2, scale=0.0, seed=9)


def test_maxima_that_rise_along_the_keys():
    wa = _wa()
    T, D = 640, 64
    g = _gen(2)
    q = torch.ones(T, 1, D, device=DEV).to(torch.bfloat16)
    k = (torch.arange(T, device=DEV)[:, None, None] / 8 * torch.ones(D, device=DEV)).to(torch.bfloat16)
    v = _rand(g, T, 1, D, dtype=torch.bfloat16)
    for kk in (k, k.flip(0)):
        out, lse = wa.window_attention(q, kk, v, _offsets([T]), scale=1 / 32, stats=True)
        want = reference(q, kk, v, visible(T, [T], T, 0), 1 / 32)
        check(out, want["out"])
        check(lse, want["lse"])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=str)
def test_infinities_and_nan_behind_the_mask_stay_there(dtype):
    wa = _wa()
    g = _gen(12)
    lens = [100, 90, 120]
    q, k, v, go = (_rand(g, 310, 2, 64, dtype=dtype) for _ in range(4))
    off = _offsets(lens)
    out, lse = wa.window_attention(q, k, v, off, 30, 0, stats=True)
    grads = wa.window_attention_backward(go, q, k, v, out, lse, off, 30, 0)
    k2, v2, q2, go2 = (t.clone() for t in (k, v, q, go))
    for t in (k2, v2, q2, go2):
        t[100:190] = float("nan")
        t[130] = float("inf")
    out2, lse2 = wa.window_attention(q2, k2, v2, off, 30, 0, stats=True)
    grads2 = wa.window_attention_backward(go2, q2, k2, v2, out2, lse2, off, 30, 0)
    # Rows of the other sessions that share a tile with it may be computed another way (with P and dS unrounded): within the
    # same bounds, not always the same bits.
    want = reference(q, k, v, visible(310, lens, 30, 0), 0.125, go)
    apart = torch.ones(310, dtype=torch.bool, device=DEV)
    apart[100:190] = False
    for name, a, b in zip(("out", "dq", "dk", "dv"), (out, *grads), (out2, *grads2)):
        for got in (a, b):
            check(got[apart], (want[name][0][apart], want[name][1][apart]), name)
    check(lse2[:, apart], (want["lse"][0][:, apart], want["lse"][1][:, apart]))
    assert out2[130:160].isnan().any()


def test_the_same_bits_every_time_and_anywhere_in_the_batch():
    q, k, v, go, off, out, lse, grads = run_and_check([300, 500, 70], 4, 2, 64, torch.bfloat16, 200, 4)
    wa = _wa()
    again = wa.window_attention(q, k, v, off, 200, 4, stats=True)
    assert torch.equal(again[0], out) and torch.equal(again[1], lse)
    for a, b in zip(wa.window_attention_backward(go, q, k, v, out, lse, off, 200, 4), grads):
        assert torch.equal(a, b)


def test_gradients_against_differences():
    wa = _wa()
    g = _gen(21)
    lens, heads, kv, dim, window, sinks = [9, 14], 4, 2, 6, 5, 1
    T = sum(lens)
    q, k, v = (_rand(g, T, n, dim, dtype=torch.float32) for n in (heads, kv, kv))
    go = _rand(g, T, heads, dim, dtype=torch.float32)
    off = _offsets(lens)
    out, lse = wa.window_attention(q, k, v, off, window, sinks, stats=True)
    grads = wa.window_attention_backward(go, q, k, v, out, lse, off, window, sinks)
    seen = visible(T, lens, window, sinks)
    step = 2.0 ** -10
    for i in range(3):
        for _ in range(3):
            way = torch.randn((q, k, v)[i].shape, generator=g, device=DEV, dtype=torch.float64)
            loss = []
            for sign in (1, -1):
                a = [t.double() for t in (q, k, v)]
                a[i] = a[i] + sign * step * way
                loss.append((reference(*a, seen, dim ** -0.5)["out"][0] * go.double()).sum())
            slope = (loss[0] - loss[1]) / (2 * step)
            # central differences: step^2 / 6 of the third derivative (under a few thousand: 4e-4), fp32 gradients 1e-5
            assert abs((grads[i].double() * way).sum() - slope) < 2e-3


def test_outputs_given_and_strided():
    wa = _wa()
    g = _gen(31)
    T, H, KV, D = 200, 4, 2, 64
    q, k, v, go = (_rand(g, T, n, D, dtype=torch.bfloat16) for n in (H, KV, KV, H))
    off = _offsets([T])
    out, lse = wa.window_attention(q, k, v, off, 50, stats=True)
    want = wa.window_attention_backward(go, q, k, v, out, lse, off, 50)
    room = torch.full((T, H + 2 * KV + 1, D + 8), 3.0, dtype=torch.bfloat16, device=DEV)
    wa.window_attention(q, k, v, off, 50, out=room[:, 1:1 + H, 8:])
    assert torch.equal(room[:, 1:1 + H, 8:], out)
    assert (room[:, 0] == 3).all() and (room[:, 1 + H:] == 3).all() and (room[:, :, :8] == 3).all()
    parts = room[:, :H, :D], room[:, H:H + KV, :D], room[:, H + KV:H + 2 * KV, :D]
    wa.window_attention_backward(go, q, k, v, out, lse, off, 50, grads=parts)
    assert all(torch.equal(a, b) for a, b in zip(parts, want))
    assert (room[:, -1] == 3).all()
    # heads before tokens, and rows at odd places, which are copied
    turned = [t.transpose(0, 1).contiguous().transpose(0, 1) for t in (q, k, v)]
    assert torch.equal(wa.window_attention(*turned, off, 50), out)
    odd = torch.empty(T * H * D + 1, dtype=torch.bfloat16, device=DEV)[1:].view(T, H, D)
    odd.copy_(q)
    assert torch.equal(wa.window_attention(odd, k, v, off, 50), out)
    wa.window_attention(q, k, v, off, 50, out=odd)
    assert torch.equal(odd, out)
    one = k[:1].expand(T, KV, D)  # the same key for all
    assert torch.equal(wa.window_attention(q, one, v, off, 50), wa.window_attention(q, one.contiguous(), v, off, 50))


def test_streams_and_graphs():
    wa = _wa()
    g = _gen(41)
    q, k, v, go = (_rand(g, 700, n, 64, dtype=torch.bfloat16) for n in (4, 2, 2, 4))
    off = _offsets([300, 400])

    def both():
        out, lse = wa.window_attention(q, k, v, off, 100, 4, stats=True)
        return (out, lse, *wa.window_attention_backward(go, q, k, v, out, lse, off, 100, 4))

    want = both()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = both()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both()
    for lens in ([300, 400], [10, 650], [700, 0]):
        off.copy_(_offsets(lens))
        q.copy_(_rand(g, 700, 4, 64, dtype=torch.bfloat16))
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(got, both()))


def test_bad_offsets_are_reported_and_stay_in_bounds():
    wa = _wa()
    g = _gen(51)
    q, k, v = (_rand(g, 300, 2, 64, dtype=torch.bfloat16) for _ in range(3))
    for off in ([0, 200, 100, 300], [-5, 300], [0, 301], [0, 10 ** 6, 300], [300, 0]):
        error = torch.zeros(1, dtype=torch.int32, device=DEV)
        out, lse = wa.window_attention(q, k, v, torch.tensor(off, device=DEV), 50, 2, stats=True, error=error)
        assert error.item() == 3
        wa.window_attention_backward(q, q, k, v, out, lse, torch.tensor(off, device=DEV), 50, 2, error=error)
    torch.cuda.synchronize()


def test_no_tokens():
    wa = _wa()
    q = torch.empty(0, 2, 64, dtype=torch.bfloat16, device=DEV)
    off = torch.zeros(1, dtype=torch.int32, device=DEV)
    out, lse = wa.window_attention(q, q, q, off, stats=True)
    assert out.shape == q.shape and lse.shape == (2, 0)
    assert all(t.shape == q.shape for t in wa.window_attention_backward(q, q, q, q, out, lse, off))
    q = torch.ones(5, 2, 64, dtype=torch.bfloat16, device=DEV)
    assert (wa.window_attention(q, q, q, off) == 0).all()  # no session


# ----------------------------------------------------------------------------- one new token

def step_reference(q, k, v, lens, window, sinks, scale):
    out, bound = (torch.zeros(q.shape, dtype=torch.float64, device=DEV) for _ in range(2))
    for b, n in enumerate(lens):
        if n == 0:
            continue
        place = torch.arange(n, device=DEV)
        keep = place[(n - 1 - place < window) | (place < sinks)]
        want = {}
        kk, vv = k[b, keep], v[b, keep]
        rows = torch.zeros(len(keep), *q.shape[1:], dtype=q.dtype, device=DEV)
        rows[-1] = q[b]
        seen = torch.zeros(len(keep), len(keep), dtype=torch.bool, device=DEV)
        seen[-1] = True
        want = reference(rows, kk, vv, seen, scale)["out"]
        out[b], bound[b] = want[0][-1], want[1][-1]
    return out, bound


@pytest.mark.parametrize("dtype", [*HALVES, torch.float32], ids=str)
@pytest.mark.parametrize("heads,kv,dim", [(1, 1, 64), (8, 8, 32), (8, 2, 128), (6, 2, 72), (16, 1, 64), (40, 2, 64), (4, 4, 7),
                                          (2, 1, 200), (3, 1, 128)])
def test_step_heads_and_widths(heads, kv, dim, dtype):
    wa = _wa()
    g = _gen(heads + dim)
    lens = [0, 1, 5, 33, 100, 64, 16]
    q = _rand(g, len(lens), heads, dim, dtype=dtype)
    k, v = (_rand(g, len(lens), 100, kv, dim, dtype=dtype) for _ in range(2))
    for window, sinks in ((None, 0), (16, 0), (20, 4), (1, 0), (3, 50)):
        got = wa.window_attention_step(q, k, v, torch.tensor(lens, device=DEV), window, sinks)
        check(got, step_reference(q, k, v, lens, window or 200, sinks, dim ** -0.5), (window, sinks))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=str)
def test_step_long_caches(dtype):
    wa = _wa()
    g = _gen(61)
    lens = [9000, 3, 4097, 8192, 0]
    q = _rand(g, 5, 4, 64, dtype=dtype)
    k, v = (_rand(g, 5, 9000, 2, 64, dtype=dtype) for _ in range(2))
    n = torch.tensor(lens, device=DEV, dtype=torch.int32)
    for window, sinks in ((None, 0), (4096, 4), (1000, 0), (100, 300)):
        got = wa.window_attention_step(q, k, v, n, window, sinks)
        check(got, step_reference(q, k, v, lens, window or 10000, sinks, 0.125), (window, sinks))
        assert torch.equal(got, wa.window_attention_step(q, k, v, n, window, sinks))


def test_step_layouts_and_unused_places():
    wa = _wa()
    g = _gen(62)
    lens = [50, 7, 64, 0]
    n = torch.tensor(lens, device=DEV)
    q = _rand(g, 4, 4, 64, dtype=torch.bfloat16)
    k, v = (_rand(g, 4, 64, 2, 64, dtype=torch.bfloat16) for _ in range(2))
    want = wa.window_attention_step(q, k, v, n, 20, 2)
    for t in (k, v):
        for b, m in enumerate(lens):
            t[b, m:] = float("nan")         # places not yet filled
            t[b, 2:max(2, m - 20)] = float("inf")  # and tokens out of sight
    assert torch.equal(wa.window_attention_step(q, k, v, n, 20, 2), want)
    turned = [t.transpose(1, 2).contiguous().transpose(1, 2) for t in (k, v)]
    assert torch.equal(wa.window_attention_step(q, *turned, n, 20, 2), want)
    wide = torch.zeros(4, 64, 5, 72, dtype=torch.bfloat16, device=DEV)
    wide[:, :, 1:3, 1:65], wide[:, :, 3:5, 8:] = k, v
    assert torch.equal(wa.window_attention_step(q, wide[:, :, 1:3, 1:65], wide[:, :, 3:5, 8:], n, 20, 2).isnan(), want.isnan())
    room = torch.full((4, 6, 70), 2.0, dtype=torch.bfloat16, device=DEV)
    wa.window_attention_step(q, k, v, n, 20, 2, out=room[:, 1:5, 3:67])
    assert torch.equal(room[:, 1:5, 3:67], want) and (room[:, 0] == 2).all() and (room[:, :, :3] == 2).all()


def test_step_reports_lengths_out_of_range():
    wa = _wa()
    q = torch.ones(3, 2, 64, dtype=torch.bfloat16, device=DEV)
    k = torch.ones(3, 8, 2, 64, dtype=torch.bfloat16, device=DEV)
    error = torch.zeros(1, dtype=torch.int32, device=DEV)
    got = wa.window_attention_step(q, k, k, torch.tensor([9, 8, -1], device=DEV), error=error)
    assert error.item() == 2 and (got[0] == 0).all() and (got[1] == 1).all() and (got[2] == 0).all()


def test_step_continues_the_forward():
    """Tokens one by one over a growing cache give what the packed call gives."""
    wa = _wa()
    g = _gen(63)
    T = 70
    q, k, v = (_rand(g, T, n, 64, dtype=torch.bfloat16) for n in (4, 2, 2))
    whole = wa.window_attention(q, k, v, _offsets([T]), 25, 3)
    caches = torch.zeros(2, 1, 80, 2, 64, dtype=torch.bfloat16, device=DEV)
    want = reference(q, k, v, visible(T, [T], 25, 3), 0.125)["out"]
    n = torch.zeros(1, dtype=torch.int32, device=DEV)
    graph = None
    for t in range(T):
        caches[0, 0, t], caches[1, 0, t] = k[t], v[t]
        n += 1
        got = wa.window_attention_step(q[t:t + 1], caches[0], caches[1], n, 25, 3)
        check(got[0], (want[0][t], want[1][t]))
        check(whole[t], (want[0][t], want[1][t]))
    assert graph is None


def test_step_graphs():
    wa = _wa()
    g = _gen(64)
    q = _rand(g, 3, 8, 128, dtype=torch.bfloat16)
    k, v = (_rand(g, 3, 3000, 2, 128, dtype=torch.bfloat16) for _ in range(2))
    n = torch.tensor([5, 3000, 700], device=DEV)
    wa.window_attention_step(q, k, v, n, 1000, 4)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = wa.window_attention_step(q, k, v, n, 1000, 4)
    for lens in ([5, 3000, 700], [3000, 0, 1]):
        n.copy_(torch.tensor(lens))
        graph.replay()
        assert torch.equal(got, wa.window_attention_step(q, k, v, n, 1000, 4))


def test_refusals():
    wa = _wa()
    q = torch.ones(10, 4, 64, dtype=torch.bfloat16, device=DEV)
    k = q[:, :2]
    off = torch.tensor([0, 10], device=DEV)
    c = torch.ones(10, 6, 2, 64, dtype=torch.bfloat16, device=DEV)
    lse = torch.zeros(4, 10, device=DEV)
    for bad in (lambda: wa.window_attention(q, k, k, off, 0), lambda: wa.window_attention(q, k, k, off, sinks=-1),
                lambda: wa.window_attention(q, k, k, off.float()), lambda: wa.window_attention(q, k, k, off.cpu()),
                lambda: wa.window_attention(q, k.half(), k, off), lambda: wa.window_attention(q, q[:, :3], q[:, :3], off),
                lambda: wa.window_attention(q, k[:5], k, off), lambda: wa.window_attention(q.double(), k.double(), k.double(), off),
                lambda: wa.window_attention(q[0], k[0], k[0], off), lambda: wa.window_attention(q, k, k, off[:0]),
                lambda: wa.window_attention(q, k, k, off, out=q[:, :2]),
                lambda: wa.window_attention_backward(q, q, k, k, q, lse.T, off),
                lambda: wa.window_attention_backward(q, q, k, k, q, lse.half(), off),
                lambda: wa.window_attention_backward(q[:5], q, k, k, q, lse, off),
                lambda: wa.window_attention_backward(q, q, k, k, q, lse, off, grads=(q, k)),
                lambda: wa.window_attention_step(q, c, c, off), lambda: wa.window_attention_step(q, c, c[:, :5], off),
                lambda: wa.window_attention_step(q, c, c, torch.zeros(10, device=DEV)),
                lambda: wa.window_attention_step(q, c[..., ::2], c[..., ::2], torch.zeros(10, device=DEV, dtype=torch.int32))):
        with pytest.raises(ValueError):
            bad()
    wide = torch.ones(10, 4, 257, device=DEV)
    with pytest.raises(ValueError):
        wa.window_attention(wide, wide, wide, off)
    with pytest.raises(Exception):
        wa.window_attention(q, k, k, off, scale=float("nan"))
    with pytest.raises(Exception):
        wa.window_attention(q, k, k, off, out=q[:1].expand(10, 4, 64))


def test_results_in_the_place_of_inputs_are_refused():
    from paper_2609_30656_gb300 import tbe
    wa = _wa()
    g = _gen(40)
    q, k, v, go = (_rand(g, 50, 2, 64, dtype=torch.bfloat16) for _ in range(4))
    off = _offsets([50])
    for t in (q, k, v):
        with pytest.raises(tbe.CbTbeError):
            wa.window_attention(q, k, v, off, 8, out=t)
    out, lse = wa.window_attention(q, k, v, off, 8, stats=True)
    a, b, c = (torch.empty_like(q) for _ in range(3))
    for grads in ((a, b, b), (a, a, c), (q, b, c), (a, b, go), (out, b, c)):
        with pytest.raises(tbe.CbTbeError):
            wa.window_attention_backward(go, q, k, v, out, lse, off, 8, grads=grads)
    with pytest.raises(tbe.CbTbeError):
        wa.window_attention_step(q, k.view(50, 1, 2, 64), v.view(50, 1, 2, 64), off[:0].new_ones(50), 8, out=q)


@pytest.mark.parametrize("dtype", [*HALVES, torch.float32], ids=str)
@pytest.mark.parametrize("where", [0, 3, 100, 149])
def test_keys_of_no_weight(where, dtype):
    """A score of -inf has the weight 0, the first key's too; a row of only such ones is NaN, as the formula's 0 / 0."""
    wa = _wa()
    g = _gen(41)
    q, k, v = (_rand(g, 150, 1, 64, dtype=dtype) for _ in range(3))
    q[..., 0] = q[..., 0].abs() + 0.5
    k[where, 0, 0] = -torch.inf
    off = _offsets([150])
    out, lse = wa.window_attention(q, k, v, off, 40, 2, stats=True)
    seen = visible(150, [150], 40, 2)
    alone = seen.sum(1) == 1
    without = seen.clone()
    without[:, where] = False
    clean = k.clone()
    clean[where] = 0
    want = reference(q, clean, v, without, 0.125)
    some = without.any(1)
    check(out[some], (want["out"][0][some], want["out"][1][some]), "out")
    check(lse[:, some], (want["lse"][0][:, some], want["lse"][1][:, some]), "lse")
    assert (some | alone).all() and out[~some].isnan().all()
    step = wa.window_attention_step(q, k.view(1, 150, 1, 64).expand(150, 150, 1, 64), v.view(1, 150, 1, 64).expand(150, 150, 1, 64),
                                    torch.arange(1, 151, device=DEV), 40, 2)
    check(step[some], (want["out"][0][some], want["out"][1][some]), "step")
    assert step[~some].isnan().all()


@pytest.mark.parametrize("heads,kv,window", [(2, 1, None), (4, 2, 3000)])
def test_a_batch_of_nan_is_computed_in_time(heads, kv, window):
    """Every row is computed again, a key at a time: a row of NaNs is done when its sums are."""
    wa = _wa()
    g = _gen(42)
    T = 60000
    q, k, v, go = (_rand(g, T, n, 64, dtype=torch.float16) for n in (heads, kv, kv, heads))
    q.fill_(float("nan"))
    off = _offsets([T])
    error = torch.zeros(1, dtype=torch.int32, device=DEV)
    out, lse = wa.window_attention(q, k, v, off, window, 40, stats=True, error=error)
    grads = wa.window_attention_backward(go, q, k, v, out, lse, off, window, 40, error=error)
    assert error.item() == 0
    assert all(t.isnan().all() for t in (out, lse, *grads))
