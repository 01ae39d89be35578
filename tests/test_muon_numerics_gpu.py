"""Accuracy of Newton-Schulz updates over the spectra that training gives them, over
magnitudes, and at the limits of fp16 (GPU), against 64 bits.

Limit. u = 2^-11 is fp16's rounding unit, u / sqrt(3) the root mean square of a rounding. With
B(s) = b s^2 + c s^4 and singular values s of at most 1.2, a step adds, relative to X,
  * from X's second fp16 value, which the products leave out: |B| <= b^2 / 4c = 2.81 of a rounding;
  * from B's rounding: at most |B| of a rounding;
  * from A's: s^2 |b + 2 c s^2| <= 1.55 of a rounding.
Steps after take what a step adds along with the singular values (the polynomial's slope is at most
about 1 in size on what has grown; what is still small has nothing added to it in proportion, since B
vanishes there). Five steps: LIMIT = sqrt(5 (2.81^2 + 2.81^2 + 1.55^2)) u / sqrt(3) = 2.7e-3. Losing X's second
value from the third step on costs 1e-2 on the low-rank spectra here, from the fourth on 2.9e-3. Single
elements: 8 times that of the elements' root mean square (8 deviations).
"""

import math

import pytest
import torch

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
UNIT = {F32: 2.0 ** -24, F16: 2.0 ** -11, BF16: 2.0 ** -8}
DEV = "cuda:0"
COEF = (3.4445, -4.7750, 2.0315)
LIMIT = math.sqrt(5 * (2.81 ** 2 + 2.81 ** 2 + 1.55 ** 2)) * 2.0 ** -11 / math.sqrt(3)


def mu():
    from paper_2609_30656_gb300 import muon
    return muon


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def reference(g, coefficients=(COEF,) * 5, eps=1e-7):
    """The definition in float64, one matrix."""
    y = g.double()
    y = y.T if y.shape[0] > y.shape[1] else y
    y = y / (torch.linalg.vector_norm(y) + eps)
    for a, b, c in coefficients:
        gram = y @ y.T
        y = a * y + (b * gram + c * (gram @ gram)) @ y
    return y.T if g.shape[0] > g.shape[1] else y


def check(got, want, limit=LIMIT, dtype=F32):
    off = got.double() - want
    rms = (off.norm() / want.norm()).item()
    assert rms <= limit + UNIT[dtype], f"off by {rms} of {limit}"
    worst = (off.abs().max() / want.square().mean().sqrt()).item()
    assert worst <= 8 * (limit + UNIT[dtype]), f"an element off by {worst}"


def with_singular_values(s, n, seed):
    """[len(s), n] with these singular values, in fp32."""
    g = _gen(seed)
    left = torch.linalg.qr(torch.randn(len(s), len(s), generator=g, device=DEV, dtype=torch.float64))[0]
    right = torch.linalg.qr(torch.randn(n, len(s), generator=g, device=DEV, dtype=torch.float64))[0]
    return (left * s @ right.T).float()


# ----------------------------------------------------------------------------- spectra

# One block, a cluster of four, and products: by single blocks, by clusters over K, square.
@pytest.mark.parametrize("m,n", [(96, 200), (100, 1500), (256, 512), (300, 1600), (1024, 1024)])
@pytest.mark.parametrize("floor", [1e-2, 1e-3, 1e-4, 1e-5])
@pytest.mark.parametrize("strong", ["one", "an eighth"])
def test_strong_directions_over_a_floor(m, n, floor, strong):
    s = torch.full((m,), floor, dtype=torch.float64, device=DEV)
    s[:1 if strong == "one" else m // 8] = 1.0
    g = with_singular_values(s, n, m + n)
    check(mu().newton_schulz(g, out_dtype=F32), reference(g))


@pytest.mark.parametrize("m,n", [(128, 256), (384, 384)])
@pytest.mark.parametrize("power", [0.0, 1.0, 2.0])
def test_decaying_singular_values(m, n, power):
    s = torch.arange(1, m + 1, dtype=torch.float64, device=DEV) ** -power
    g = with_singular_values(s, n, 5)
    check(mu().newton_schulz(g, out_dtype=F32), reference(g))


# ----------------------------------------------------------------------------- magnitudes

def _plain_norm_matters(g, eps=0.0):
    check(mu().newton_schulz(g, eps=eps, out_dtype=F32), reference(g, eps=eps))


@pytest.mark.parametrize("std", [2e-12, 1e-12, 6e-13, 3e-13])
@pytest.mark.parametrize("shape", [(2048, 2048), (128, 3000)])
def test_values_about_two_to_the_minus_40(std, shape):
    """Where the norm's classes of magnitude meet, each with a good part of the sum."""
    _plain_norm_matters(torch.randn(shape, generator=_gen(7), device=DEV).mul(std))


@pytest.mark.parametrize("shape", [(4096, 4096), (120, 3000)])
@pytest.mark.parametrize("floor,spike", [(2.0 ** -41, 2.0 ** -30), (2.0 ** -45, 2.0 ** -36), (2.0 ** -60, 2.0 ** -39)])
def test_a_power_of_two_times_a_matrix_has_its_factor(shape, floor, spike):
    """One value of the middle class above many of the small one, and the same in the middle class alone."""
    g = torch.full(shape, floor, device=DEV)
    g[3, 70] = spike
    want = mu().newton_schulz(g.mul(2.0 ** 38), eps=0.0, out_dtype=F32).double()
    got = mu().newton_schulz(g, eps=0.0, out_dtype=F32).double()
    assert ((got - want).norm() / want.norm()).item() <= LIMIT


@pytest.mark.parametrize("shape", [(1024, 1024), (100, 600)])
def test_values_about_two_to_the_40(shape):
    _plain_norm_matters(torch.randn(shape, generator=_gen(8), device=DEV).mul(2.0 ** 40))


# ----------------------------------------------------------------------------- range

def _one_value(m, n):
    g = torch.zeros(m, n, device=DEV)
    g[5, 7] = 1.0
    return g


@pytest.mark.parametrize("m,n", [(60, 100), (150, 220)])
def test_singular_values_up_to_the_limit_of_a(m, n):
    """A = s^2 up to 255.9: a step that takes s to 15.9 and one that takes it back."""
    g = _one_value(m, n)
    for top in (15.9, 16.1):
        table = ((top, 0.0, 0.0), (0.05, 0.0, 0.0))
        got = mu().newton_schulz(g, steps=2, coefficients=table, out_dtype=F32)
        if top < 16:
            # one value: hi + lo to 2^-22, three products in fp32
            want = reference(g, table)
            assert (got.double() - want).abs().max().item() <= 2.0 ** -20
        else:
            assert not bool(got.isfinite().all())  # and no plausible number


@pytest.mark.parametrize("m,n", [(60, 100), (150, 220)])
def test_polynomials_up_to_the_limit_of_b(m, n):
    """b s^2 + d of -254 and of -258 (s = 3, d = 16), with an `a` that takes most of it off again."""
    g = _one_value(m, n)
    for b in (-30.0, -30.5):
        table = ((3.0, 0.0, 0.0), (-9.0 * b + 0.25, b, 0.0))
        got = mu().newton_schulz(g, steps=2, coefficients=table, out_dtype=F32)
        if b == -30.0:
            # B's rounding, half of fp16's spacing of 32 of 2^8 B, times s; A = 9 and X = 3 have few bits
            assert (got.double() - reference(g, table)).abs().max().item() <= 3 * 16 / 256 + 2.0 ** -10
        else:
            assert not bool(got.isfinite().all())
