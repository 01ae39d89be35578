"""Steps of stacks whose matrices' rows lie in turn, or between one another's (GPU)."""

import pytest
import torch

from test_muon_numerics_gpu import BF16, DEV, F32, _gen, mu

pytestmark = pytest.mark.gpu


def _randn(shape, seed):
    return torch.randn(shape, generator=_gen(seed), device=DEV)


@pytest.mark.parametrize("m,n", [(60, 100), (144, 200), (300, 136)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_in_turn(m, n, dtype):
    start, grad = _randn((3, m, n), 1).to(dtype), _randn((3, m, n), 2).mul(1e-3)
    plain, plain_m = start.clone(), _randn((3, m, n), 3).mul(1e-3)
    turn = torch.full((m, 3, n + 8), 7.0, dtype=dtype, device=DEV)
    turn_m = torch.empty(m, 3, n, device=DEV)
    w, mom = turn[..., :n].transpose(0, 1), turn_m.transpose(0, 1)
    w.copy_(start)
    mom.copy_(plain_m)
    mu().muon_step(plain, grad, plain_m, lr=0.02)
    mu().muon_step(w, grad, mom, lr=0.02)
    assert torch.equal(w, plain) and torch.equal(mom, plain_m) and bool((turn[..., n:] == 7.0).all())
    out = torch.empty(m, 3, n, dtype=BF16, device=DEV)
    mu().newton_schulz(grad, out=out.transpose(0, 1))
    assert torch.equal(out.transpose(0, 1), mu().newton_schulz(grad))


def test_rows_between_rows():
    m, n = 100, 64
    flat = torch.full((4000 * n,), 7.0, device=DEV)
    w = flat.as_strided((2, m, n), ((2 * m + 1) * n, 4 * n, 1))  # ends inside the first matrix, a row on
    start, grad = _randn((2, m, n), 1), _randn((2, m, n), 2)
    w.copy_(start)
    plain, mom = start.clone(), torch.zeros(2, m, n, device=DEV)
    mu().muon_step(plain, grad, mom, lr=0.02)
    mu().muon_step(w, grad, mom.zero_(), lr=0.02)
    assert torch.equal(w, plain)
    w.fill_(7.0)
    assert bool((flat == 7.0).all())


def test_rows_in_one_place_are_refused():
    g = torch.zeros(2, 2, 4, device=DEV)
    w = torch.zeros(32, device=DEV).as_strided((2, 2, 4), (8, 8, 1))
    with pytest.raises(ValueError):
        mu().muon_step(w, g, g.clone(), lr=0.1)
    with pytest.raises(ValueError):
        mu().muon_step(g.clone(), g, w, lr=0.1)
    with pytest.raises(ValueError):
        mu().newton_schulz(g, out=w)
