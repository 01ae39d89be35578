"""Newton-Schulz updates and the optimizer step around them against 64 bits (GPU).

Tolerance. The products' operands X, A and B are rounded to fp16, u = 2^-11, whose errors
spread evenly: u / sqrt(3) of a value in the root mean square. A step rounds three matrices; an
error of A or B enters the update times at most |b| = 4.8 (the largest coefficient), and the
errors of the 5 steps are independent, so in the 2-norm the result is off by about
sqrt(3 * 5) * 4.8 * 2^-11 / sqrt(3) = 5.2e-3 at the most (steps after an error's own take
singular values back towards 1). The output's rounding adds u_out / sqrt(3).
"""

import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
UNIT = {F32: 2.0 ** -24, F16: 2.0 ** -11, BF16: 2.0 ** -8}
DEV = "cuda:0"
COEF = (3.4445, -4.7750, 2.0315)


def mu():
    from paper_2609_30656_gb300 import muon
    return muon


def tolerance(dtype, steps=5, b=4.775):
    return math.sqrt(3 * steps) * b * 2.0 ** -11 / math.sqrt(3) + UNIT[dtype]


def _updates(shape, dtype=F32, seed=0, kind="noisy"):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    x = torch.randn(shape, generator=g, device=DEV)
    if kind == "low":  # a few strong directions over a noise floor
        r = max(1, min(shape[-2:]) // 8)
        left = torch.randn(*shape[:-1], r, generator=g, device=DEV) * torch.linspace(0, -3, r, device=DEV).exp()
        x = left @ torch.randn(*shape[:-2], r, shape[-1], generator=g, device=DEV) / r ** 0.5 + 0.05 * x
    return (x * 1e-3).to(dtype)


def reference(g, steps=5, coefficients=COEF, eps=1e-7):
    """The definition in float64 on the CPU, one matrix at a time."""
    x = g.detach().double().cpu().numpy()
    flat = x.reshape(-1, *x.shape[-2:]) if x.ndim == 3 else x[None]
    out = np.empty_like(flat)
    table = [coefficients] * steps if not hasattr(coefficients[0], "__len__") else coefficients
    for i, m in enumerate(flat):
        y = m if m.shape[0] <= m.shape[1] else m.T
        y = y / (np.sqrt((y * y).sum()) + eps)
        for a, b, c in table:
            gram = y @ y.T
            y = a * y + (b * gram + c * (gram @ gram)) @ y
        out[i] = y if m.shape[0] <= m.shape[1] else y.T
    return torch.from_numpy(out.reshape(x.shape))


def check(got, want, tol):
    off = (got.double().cpu() - want).norm() / want.norm()
    assert off.item() <= tol, f"off by {off.item()} of {tol}"


SIZES = [(1, 1), (1, 9), (7, 1), (5, 5), (16, 64), (48, 48), (63, 65), (64, 128), (100, 300), (127, 129), (128, 128),
         (128, 256), (129, 257), (256, 256), (300, 100), (384, 512), (513, 1001), (1001, 513), (640, 640)]


@pytest.mark.parametrize("m,n", SIZES)
@pytest.mark.parametrize("kind", ["noisy", "low"])
def test_factor(m, n, kind):
    g = _updates((m, n), F32, m * 7 + n, kind)
    got = mu().newton_schulz(g)
    assert got.dtype == BF16 and got.shape == g.shape
    check(got, reference(g), tolerance(BF16))


@pytest.mark.parametrize("m,n", [(1536, 2048), (2050, 700), (129, 4000)])
def test_factor_of_larger_matrices(m, n):
    g = _updates((m, n), BF16, 3, "low")
    check(mu().newton_schulz(g, out_dtype=F32), reference(g), tolerance(F32))


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("out", [F32, F16, BF16])
def test_types(dtype, out):
    g = _updates((70, 200), F32, 4).mul(1e3).to(dtype)
    got = mu().newton_schulz(g, out_dtype=out)
    assert got.dtype == out
    check(got, reference(g), tolerance(out))


@pytest.mark.parametrize("batch,m,n", [(0, 8, 8), (3, 0, 8), (1, 20, 30), (5, 64, 128), (7, 33, 90), (3, 200, 130),
                                       (40, 16, 16), (200, 130, 140)])
def test_stacks_are_their_matrices(batch, m, n):
    g = _updates((batch, m, n), F32, 5)
    got = mu().newton_schulz(g)
    assert got.shape == g.shape
    for i in range(0, batch, max(1, batch // 4)):
        if m * n:
            assert torch.equal(got[i], mu().newton_schulz(g[i]))
            check(got[i], reference(g[i]), tolerance(BF16))


@pytest.mark.parametrize("batch,m,n", [(170, 64, 100), (3, 100, 384), (2, 100, 385), (5, 70, 1500), (2, 120, 3000),
                                       (2, 100, 3300)])
def test_narrow_stacks(batch, m, n):
    # One block per matrix (of 256 or 512 threads), clusters of 2, 4 and 8, and beyond them.
    g = _updates((batch, m, n), BF16, 31, "low")
    got = mu().newton_schulz(g)
    for i in (0, batch - 1):
        assert torch.equal(got[i], mu().newton_schulz(g[i]))
        check(got[i], reference(g[i]), tolerance(BF16))
    assert torch.equal(mu().newton_schulz(g.mT.contiguous()).mT, got)


@pytest.mark.parametrize("batch,m,n", [(40, 144, 1600), (9, 300, 3200), (12, 200, 3100)])
def test_long_rows_give_the_same_bits_alone_and_in_a_stack(batch, m, n):
    # The sum over a long side is shared by blocks, or not, by the number of matrices.
    g = _updates((batch, m, n), BF16, 30)
    got = mu().newton_schulz(g)
    for i in (0, batch - 1):
        assert torch.equal(got[i], mu().newton_schulz(g[i]))
        assert torch.equal(got[i].t(), mu().newton_schulz(g[i].t().contiguous()))
    check(got[0], reference(g[0]), tolerance(BF16))


@pytest.mark.parametrize("m,n", [(60, 130), (300, 520)])
def test_transposes_and_strides(m, n):
    g = _updates((m, n), F32, 6)
    want = mu().newton_schulz(g)
    assert torch.equal(mu().newton_schulz(g.t().contiguous()), want.t())
    assert torch.equal(mu().newton_schulz(g.t()), want.t())
    padded = torch.full((m + 3, n + 5), 9.0, device=DEV)
    padded[1:m + 1, 2:n + 2] = g
    assert torch.equal(mu().newton_schulz(padded[1:m + 1, 2:n + 2]), want)
    out = torch.full((m, n + 9), 4.0, dtype=BF16, device=DEV)
    mu().newton_schulz(g, out=out[:, 3:n + 3])
    assert torch.equal(out[:, 3:n + 3], want)
    assert bool((out[:, :3] == 4.0).all()) and bool((out[:, n + 3:] == 4.0).all())
    columns = torch.empty(n, m, dtype=BF16, device=DEV).t()
    assert torch.equal(mu().newton_schulz(g, out=columns), want)
    assert torch.equal(mu().newton_schulz(g[:, ::2]), mu().newton_schulz(g[:, ::2].contiguous()))
    three = g.expand(3, m, n)
    assert torch.equal(mu().newton_schulz(three)[2], want)
    inplace = g.clone()
    mu().newton_schulz(inplace, out=inplace)
    assert torch.equal(inplace.to(BF16), want)


@pytest.mark.parametrize("scale", [1e-42, 1e-30, 1e-12, 1.0, 1e15, 1e36])
@pytest.mark.parametrize("m", [96, 300])
def test_any_magnitude(scale, m):
    g = _updates((m, 140), F32, 7).mul(1e3).double().mul(scale).float()
    eps = 0.0 if scale < 1e-6 else 1e-7
    got = mu().newton_schulz(g, eps=eps, out_dtype=F32)
    check(got, reference(g, eps=eps), tolerance(F32))


@pytest.mark.parametrize("m,n", [(64, 100), (200, 150)])
def test_zeros_stay_zeros_and_nan_spreads(m, n):
    z = torch.zeros(m, n, device=DEV)
    for eps in (1e-7, 0.0):
        assert not mu().newton_schulz(z, eps=eps).any()
    for bad in (float("nan"), float("inf")):
        g = torch.stack([_updates((m, n), F32, 8), _updates((m, n), F32, 9)])
        g[0, 3, 5] = bad
        got = mu().newton_schulz(g)
        assert bool(got[0].isnan().all())
        check(got[1], reference(g[1]), tolerance(BF16))


def test_rank_deficient_and_orthogonal_inputs():
    g = torch.zeros(150, 220, device=DEV)
    g[10] = _updates((220,) * 2, F32, 10)[0]  # one row: the rest of the factor is zero
    got = mu().newton_schulz(g, out_dtype=F32)
    assert not got[:10].any() and not got[11:].any()
    check(got, reference(g), tolerance(F32))
    eye = torch.eye(160, device=DEV)
    got = mu().newton_schulz(eye, out_dtype=F32)
    check(got, reference(eye), tolerance(F32))
    assert not (got - torch.diag(got.diagonal())).any()


@pytest.mark.parametrize("steps", [1, 2, 3, 6])
@pytest.mark.parametrize("m", [100, 260])
def test_steps_and_their_own_coefficients(steps, m):
    g = _updates((m, 300), F32, 11)
    check(mu().newton_schulz(g, steps=steps, out_dtype=F32), reference(g, steps=steps), tolerance(F32, steps))
    table = [(3.9, -8.0, 5.0), (3.5, -6.0, 3.0), (3.0, -4.0, 2.0), (1.875, -1.25, 0.375), (1.875, -1.25, 0.375),
             (0.0, 2.0, -1.0)][:steps]
    got = mu().newton_schulz(g, steps=steps, coefficients=table, out_dtype=F32)
    check(got, reference(g, steps=steps, coefficients=table), tolerance(F32, steps, 8.0))


def test_singular_values_come_near_one():
    g = _updates((256, 384), F32, 12)
    s = torch.linalg.svdvals(mu().newton_schulz(g, out_dtype=F32).double().cpu())
    # five steps of the polynomial take (0.01, 1] into about [0.68, 1.21]
    assert 0.6 < s.min() and s.max() < 1.25


@pytest.mark.parametrize("shape", [(64, 128), (200, 72), (3, 130, 260), (2, 300, 128), (513, 257)])
@pytest.mark.parametrize("weight_dtype,grad_dtype", [(F32, F32), (F32, BF16), (BF16, BF16)])
@pytest.mark.parametrize("nesterov", [True, False])
def test_step(shape, weight_dtype, grad_dtype, nesterov):
    g = torch.Generator(device=DEV)
    g.manual_seed(13)
    w = torch.randn(shape, generator=g, device=DEV).mul(0.02).to(weight_dtype)
    grad = _updates(shape, grad_dtype, 14)
    mom = torch.randn(shape, generator=g, device=DEV).mul(1e-3)
    m64 = 0.95 * mom.double().cpu() + grad.double().cpu()
    u64 = grad.double().cpu() + 0.95 * m64 if nesterov else m64
    rows, cols = shape[-2:]
    move = 0.02 * 0.2 * math.sqrt(max(rows, cols)) * reference(u64)
    want = (1 - 0.02 * 0.1) * w.double().cpu() - move
    mu().muon_step(w, grad, mom, lr=0.02, nesterov=nesterov, weight_decay=0.1)
    # beta in fp32 and two roundings of the sum
    assert bool(((mom.double().cpu() - m64).abs() <= 2.0 ** -23 * (m64.abs() + grad.double().cpu().abs())).all())
    off = (w.double().cpu() - want).norm()
    # the factor's error on the step, fp32 arithmetic and the weight's rounding on the weight
    limit = tolerance(F32) * move.norm() + (4 * 2.0 ** -24 + UNIT[weight_dtype]) * want.norm()
    assert off <= limit, f"{off} over {limit}"


@pytest.mark.parametrize("adjust,scale", [("spectral", math.sqrt(300 / 100)), (None, 1.0)])
def test_step_adjustments_and_strided_weights(adjust, scale):
    big = torch.zeros(300, 160, device=DEV)
    w = big[:, 30:130]
    mom = torch.zeros(300, 100, device=DEV)
    grad = _updates((100, 300), F32, 15).t()
    mu().muon_step(w, grad, mom, lr=1.0, adjust=adjust)
    check(-w / scale, reference(grad), tolerance(F32))
    assert not big[:, :30].any() and not big[:, 130:].any()
    assert torch.equal(mom, grad)


@pytest.mark.parametrize("skip", [1, 2, 4, 8, 16])
@pytest.mark.parametrize("pad", [0, 4, 8, 16])
@pytest.mark.parametrize("m,n", [(160, 272), (272, 160), (150, 424)])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_weights_of_every_alignment_get_the_same_bits(skip, pad, m, n, dtype):
    """How a row may be read and written is no part of what is computed: the weights of an
    aligned stack and those at any other base and stride are equal, and nothing around them moves."""
    grad = _updates((2, m, n), BF16, 50)
    start = _updates((2, m, n), F32, 51).mul(1e3).to(dtype)
    plain, momentum = start.clone(), torch.zeros(2, m, n, device=DEV)
    mu().muon_step(plain, grad, momentum, lr=0.02, weight_decay=0.1)
    flat = torch.full((skip + 2 * m * (n + pad),), 7.0, device=DEV).to(dtype)
    weight = flat[skip:].view(2, m, n + pad)[..., :n]
    weight.copy_(start)
    momentum.zero_()
    mu().muon_step(weight, grad, momentum, lr=0.02, weight_decay=0.1)
    assert torch.equal(weight, plain) and not torch.equal(plain, start)
    weight.fill_(7.0)
    assert bool((flat == 7.0).all())


@pytest.mark.parametrize("m,n", [(96, 120), (700, 400)])
def test_deterministic_on_any_stream_and_in_a_graph(m, n):
    g = _updates((4, m, n), BF16, 16)
    first = mu().newton_schulz(g)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(3):
        with torch.cuda.stream(side):
            again = mu().newton_schulz(g)
        side.synchronize()
        assert torch.equal(first, again)
    out = torch.empty_like(first)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mu().newton_schulz(g, out=out)
    g.copy_(_updates((4, m, n), BF16, 17))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, mu().newton_schulz(g))


def test_no_wait_runs_out():
    error = torch.zeros(1, dtype=torch.int32, device=DEV)
    for m, n in ((64, 64), (300, 700), (1500, 1200)):
        mu().newton_schulz(_updates((m, n), F32, 18), error=error)
    assert error.item() == 0


def test_refusals_of_the_binding():
    t = mu()
    g = torch.zeros(8, 16, device=DEV)
    bad = [
        lambda: t.newton_schulz(g.cpu()),
        lambda: t.newton_schulz(g[0]),
        lambda: t.newton_schulz(g.double()),
        lambda: t.newton_schulz(g, out=torch.zeros(16, 8, device=DEV)),
        lambda: t.newton_schulz(g, out=torch.zeros(8, 32, device=DEV)[:, ::2]),
        lambda: t.newton_schulz(g.expand(2, 8, 16), out=torch.zeros(8, 16, device=DEV).expand(2, 8, 16)),
        lambda: t.newton_schulz(g, steps=0),
        lambda: t.newton_schulz(g, coefficients=(1.0, 2.0)),
        lambda: t.newton_schulz(g, steps=2, coefficients=[(1, 2, 3)]),
        lambda: t.muon_step(g, g, g.half(), lr=0.1),
        lambda: t.muon_step(g, g[:, :8], g, lr=0.1),
        lambda: t.muon_step(g.t(), g.t(), torch.zeros(16, 8, device=DEV), lr=0.1),
        lambda: t.muon_step(g, g, torch.zeros(8, 16, device=DEV), lr=0.1, adjust="other"),
    ]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    from paper_2609_30656_gb300 import tbe
    for kw in ({"eps": -1.0}, {"eps": float("nan")}, {"steps": 65}, {"coefficients": (1.0, float("inf"), 0.0)}):
        with pytest.raises(tbe.CbTbeError):
            t.newton_schulz(g, **kw)
    with pytest.raises(tbe.CbTbeError):
        t.muon_step(g, g, torch.zeros(8, 16, device=DEV), lr=float("nan"))
