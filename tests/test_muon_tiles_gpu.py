"""Newton-Schulz updates and steps through every kind of tile that the sizes choose between (GPU).

Stacks bring the tiles of large matrices to small ones: on 152 SMs the three products (X X^T, A A, B X)
of these are taken by one block in tiles 64 or 128 wide, by a cluster over K, or by pairs of blocks 160, 192,
224 and 256 wide. The limits are those of test_muon_numerics_gpu.
"""

import math

import pytest
import torch

from test_muon_numerics_gpu import BF16, DEV, F32, LIMIT, UNIT, _gen, check, mu, reference

pytestmark = pytest.mark.gpu


def _noise(shape, seed):
    return torch.randn(shape, generator=_gen(seed), device=DEV).mul(1e-3)


SHAPES = [(1, 1001, 1400),   # tiles of 64 for the symmetric products, 128 for the update
          (40, 130, 263),    # 128 for X X^T, 64
          (8, 700, 700),     # pairs of 192 for the symmetric products, 128
          (4, 1050, 1050),   # pairs of 224 for them, 160
          (200, 130, 263),   # pairs of 160 for X X^T and the update, 128
          (6, 900, 1803),    # pairs of 256 for X X^T, 128, 160
          (2, 900, 1803),    # 64, pairs of 224 for the update
          (5, 1050, 1471),   # 128, pairs of 256 for the update
          (1, 2050, 2900),   # pairs for all three: 160, 160, 192
          (1, 2600, 3300)]   # and 256


@pytest.mark.parametrize("batch,m,n", SHAPES)
@pytest.mark.parametrize("tall", [False, True])
def test_factor_by_every_tile(batch, m, n, tall):
    g = _noise((batch, n, m) if tall else (batch, m, n), m + n)
    got = mu().newton_schulz(g, out_dtype=F32)
    for i in sorted({0, batch // 2, batch - 1}):
        check(got[i], reference(g[i]))


@pytest.mark.parametrize("batch,m,n", [(40, 130, 263), (2, 900, 1803), (5, 1050, 1471), (5, 1050, 1472), (8, 700, 700),
                                       (4, 1024, 4096), (1, 2600, 3300)])
@pytest.mark.parametrize("tall", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_step_by_every_tile(batch, m, n, tall, dtype):
    shape = (batch, n, m) if tall else (batch, m, n)
    start = torch.randn(shape, generator=_gen(1), device=DEV).mul(0.02).to(dtype)
    grad, mom = _noise(shape, 2), _noise(shape, 3)
    w, before = start.clone(), mom.clone()
    mu().muon_step(w, grad, mom, lr=0.02, weight_decay=0.1)
    for i in sorted({0, batch // 2, batch - 1}):
        m64 = 0.95 * before[i].double() + grad[i].double()
        move = 0.02 * 0.2 * math.sqrt(max(m, n)) * reference(grad[i].double() + 0.95 * m64)
        want = (1 - 0.02 * 0.1) * start[i].double() - move
        off = (w[i].double() - want).abs()
        # the factor's error, the weight's rounding, four operations in fp32
        own = (UNIT[dtype] + 4 * 2.0 ** -24) * want.abs()
        worst = ((off - own) / move.square().mean().sqrt()).max().item()
        assert worst <= 8 * LIMIT, f"an element off by {worst} of the step"
        assert ((off - own).clamp_min(0).norm() / move.norm()).item() <= LIMIT
