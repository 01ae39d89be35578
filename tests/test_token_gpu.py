"""Token lookup and its gradient against plain 64-bit statements of them (GPU).

Tolerances. The lookup is one fp32 product rounded once: bit-equal to the same two
roundings in torch. A gradient row of k positions is a sum in fp32 in any order, one product
with the scale, at most one addition of the value that was there, and one rounding to the
output's type, so it is off by at most
    (k + 1) 2^-24 scale sum |grad_out|  +  2^-24 |result| (the addition)  +  u |result| (+ u_min),
u = 2^-24, 2^-11, 2^-8 for fp32, fp16, bf16, and u_min = 2^-25, half of fp16's least value.
"""

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
UNIT = {F32: 2.0 ** -24, F16: 2.0 ** -11, BF16: 2.0 ** -8}
DEV = "cuda:0"


def te():
    from paper_2609_30656_gb300 import token_embedding
    return token_embedding


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _randn(shape, dtype, seed):
    return torch.randn(shape, generator=_gen(seed), device=DEV).to(dtype)


def _randint(hi, shape, seed, dtype=torch.int64):
    return torch.randint(0, hi, shape, generator=_gen(seed), device=DEV).to(dtype)


def reference_backward(go, tokens, rows, scale, padding=None, base=None):
    """(value, bound without the output's rounding) in float64, by a plain scatter-add."""
    go = go.detach().reshape(-1, go.shape[-1]).double().cpu()
    tok = tokens.reshape(-1).long().cpu()
    keep = (tok >= 0) & (tok < rows)
    if padding is not None:
        keep &= tok != padding
    go, tok = go[keep], tok[keep]
    value = torch.zeros(rows, go.shape[1], dtype=torch.float64).index_add_(0, tok, go) * scale
    size = torch.zeros(rows, go.shape[1], dtype=torch.float64).index_add_(0, tok, go.abs()) * abs(scale)
    count = torch.bincount(tok, minlength=rows).double().unsqueeze(1)
    bound = (count + 1) * 2.0 ** -24 * size
    if base is not None:
        value = value + base.double().cpu()
        bound = bound + 2.0 ** -24 * value.abs()
    return value, bound


def check_backward(got, go, tokens, rows, scale, padding=None, base=None):
    value, bound = reference_backward(go, tokens, rows, scale, padding, base)
    u = UNIT[got.dtype]
    bound = bound * (1 + u) + u * value.abs() + (2.0 ** -25 if got.dtype == F16 else 0.0)
    off = (got.double().cpu() - value).abs()
    assert bool((off <= bound + 1e-300).all()), f"off by {off.max().item()} at {int((off - bound).argmax())}"


# ----------------------------------------------------------------------------- lookup

@pytest.mark.parametrize("dim", [1, 3, 8, 63, 64, 100, 257, 1000, 1024, 4096])
@pytest.mark.parametrize("dtype,out", [(F32, F32), (F32, BF16), (F16, F16), (F16, F32), (BF16, BF16), (BF16, F16)])
def test_lookup_matches_the_same_roundings(dim, dtype, out):
    table = _randn((301, dim), dtype, 1)
    tokens = _randint(301, (5, 67), 2)
    got = te().token_forward(table, tokens, scale=dim ** 0.5, out_dtype=out)
    assert got.dtype == out and got.shape == (5, 67, dim)
    want = (table[tokens].float() * torch.tensor(dim ** 0.5, dtype=F32)).to(out)
    assert torch.equal(got, want)


@pytest.mark.parametrize("shape", [(), (1,), (0,), (1, 1), (7, 0), (3, 1, 5), (2, 3, 4, 5), (5000,)])
@pytest.mark.parametrize("index", [torch.int32, torch.int64])
def test_lookup_shapes(shape, index):
    table = _randn((50, 24), BF16, 3)
    tokens = _randint(50, shape, 4, index)
    got = te().token_forward(table, tokens)
    assert torch.equal(got, table[tokens.long()])


def test_lookup_strided_operands():
    big = _randn((100, 80), F32, 5)
    table = big[:, 8:72]                      # row stride 80, 16-byte aligned
    odd = big[:, 3:66]                        # unaligned rows of 63
    tokens = _randint(100, (6, 33), 6)
    for t in (table, odd):
        for tok in (tokens[:, :-1], tokens[:, 1:], tokens[::2], tokens.t(), tokens[:, 5], tokens[2],
                    tokens[:1].expand(4, 33)):
            assert torch.equal(te().token_forward(t, tok, scale=2.0), t[tok] * 2.0)
    out = torch.zeros(6, 40, 64, device=DEV)
    te().token_forward(table, tokens, out=out[:, 4:37])
    assert torch.equal(out[:, 4:37], table[tokens])
    assert not out[:, :4].any() and not out[:, 37:].any()
    swapped = torch.zeros(33, 6, 64, device=DEV)
    te().token_forward(table, tokens, out=swapped.transpose(0, 1))
    assert torch.equal(swapped.transpose(0, 1), table[tokens])


def _rows_at(values, dtype, skip, stride):
    """`values` in rows `stride` apart, the first `skip` values into an allocation."""
    n, dim = values.shape
    flat = torch.zeros(skip + n * stride, dtype=dtype, device=DEV)
    assert flat.data_ptr() % 256 == 0
    view = flat[skip:].view(n, stride)[:, :dim]
    view.copy_(values)
    return view


@pytest.mark.parametrize("skip", [1, 2, 4, 8, 16])
@pytest.mark.parametrize("pad", [0, 4, 8, 16])
@pytest.mark.parametrize("dtype,out", [(F32, F32), (F32, BF16), (BF16, F32), (F16, F16), (BF16, BF16)])
def test_bases_and_strides_of_every_alignment(skip, pad, dtype, out):
    """Each width of piece that the base address or the stride of one operand rules out."""
    rows, dim, n = 90, 96, 70
    tokens = _randint(rows, (n,), 60)
    plain = _randn((rows, dim), dtype, 61)
    want = (plain[tokens].float() * 1.5).to(out)
    room = torch.zeros(n, dim, dtype=out, device=DEV)
    for table, into in [(_rows_at(plain, dtype, skip, dim + pad), room), (plain, _rows_at(room, out, skip, dim + pad))]:
        into.fill_(7)
        te().token_forward(table, tokens, scale=1.5, out=into)
        assert torch.equal(into, want)
    go = _randn((n, dim), dtype, 62)
    grad = torch.zeros(rows, dim, dtype=out, device=DEV)
    for g, into in [(_rows_at(go, dtype, skip, dim + pad), grad), (go, _rows_at(grad, out, skip, dim + pad))]:
        into.fill_(7)
        te().token_backward(g, tokens, rows, scale=1.5, out=into)
        check_backward(into, go, tokens, rows, 1.5)


@pytest.mark.parametrize("n", [0, 5, 3000])
@pytest.mark.parametrize("dim", [1, 3, 16, 63, 64, 1001])
@pytest.mark.parametrize("skip,pad", [(0, 0), (1, 0), (3, 1), (8, 0), (0, 8), (16, 5)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_zeros_stay_within_their_rows(n, dim, skip, pad, dtype):
    """Rows without a token become zeros, alone and as neighbours, and what lies between, before
    and behind the rows stays; in 16 and 32 bits at any alignment."""
    rows = 1003
    tokens = _randint(rows, (n,), 70)
    go = _randn((n, dim), dtype, 71)
    flat = torch.full((skip + rows * (dim + pad) + 40,), 7.0, dtype=dtype, device=DEV)
    grad = flat[skip:skip + rows * (dim + pad)].view(rows, dim + pad)[:, :dim]
    te().token_backward(go, tokens, rows, out=grad)
    check_backward(grad, go, tokens, rows, 1.0)
    empty = torch.ones(rows, dtype=torch.bool, device=DEV)
    empty[tokens] = False
    assert not grad[empty].any()
    grad.fill_(7.0)
    assert bool((flat == 7.0).all())


@pytest.mark.parametrize("dim", [2, 6, 62, 66, 258, 514, 1030])
@pytest.mark.parametrize("dtype,out", [(F32, F32), (BF16, BF16), (F16, F32), (F32, F16)])
def test_rows_of_twice_an_odd_number(dim, dtype, out):
    table = _randn((120, dim), dtype, 40)
    for n in (70, 3000):
        tokens = _randint(120, (n,), 41)
        got = te().token_forward(table, tokens, scale=3.0, out_dtype=out)
        assert torch.equal(got, (table[tokens].float() * 3.0).to(out))
        go = _randn((n, dim), dtype, 42)
        check_backward(te().token_backward(go, tokens, 120, scale=0.5, out_dtype=out), go, tokens, 120, 0.5)


@pytest.mark.parametrize("dim", [64, 63])
def test_lookup_out_of_range_tokens_give_zeros_and_an_error(dim):
    table = _randn((20, dim), F32, 7)
    tokens = torch.tensor([3, -1, 19, 20, 2 ** 40, -2 ** 40, 0], device=DEV)
    error = torch.zeros(1, dtype=torch.int32, device=DEV)
    got = te().token_forward(table, tokens, error=error)
    assert error.item() == 2
    good = (tokens >= 0) & (tokens < 20)
    assert torch.equal(got[good], table[tokens[good]])
    assert not got[~good].any()
    error.zero_()
    te().token_forward(table, tokens[good], error=error)
    assert error.item() == 0


def test_lookup_keeps_infinities_and_nan():
    table = _randn((10, 16), BF16, 8)
    table[3, 2], table[3, 5], table[4, 0] = float("inf"), float("nan"), float("-inf")
    tokens = torch.tensor([3, 4, 5], device=DEV)
    want = table[tokens].float() * 4.0
    got = te().token_forward(table, tokens, scale=4.0, out_dtype=F32)
    assert torch.equal(torch.nan_to_num(got, 7.0), torch.nan_to_num(want, 7.0))


def test_lookup_past_2_to_the_31_values():
    rows, dim = 600_000, 4096  # 2.46e9 values of the table
    table = torch.zeros(rows, dim, dtype=F16, device=DEV)
    tokens = torch.tensor([0, rows - 1, 524_288, 524_287], device=DEV)
    table[tokens] = _randn((4, dim), F16, 9)
    assert torch.equal(te().token_forward(table, tokens), table[tokens])


# ----------------------------------------------------------------------------- gradient

# 2048 tokens are the most that are matched, longer calls are sorted.
COUNTS = [1, 2, 31, 128, 2047, 2048, 2049, 4096, 4097, 20000]


@pytest.mark.parametrize("n", COUNTS)
@pytest.mark.parametrize("dim", [8, 65, 264])
@pytest.mark.parametrize("dtype,out", [(F32, F32), (BF16, F32), (BF16, BF16), (F16, F16)])
def test_gradient(n, dim, dtype, out):
    rows = 997
    tokens = _randint(rows, (n,), n)
    go = _randn((n, dim), dtype, n + 1)
    got = te().token_backward(go, tokens, rows, scale=1.5, out_dtype=out)
    assert got.dtype == out
    check_backward(got, go, tokens, rows, 1.5)


@pytest.mark.parametrize("n", [100, 2048, 5000, 70000])
@pytest.mark.parametrize("rows", [1, 2, 255, 256, 65535, 65536, 70001])
def test_gradient_key_widths_and_empty_rows(n, rows):
    tokens = _randint(rows, (n,), rows + n, torch.int32)
    go = _randn((n, 16), F32, 3)
    check_backward(te().token_backward(go, tokens, rows), go, tokens, rows, 1.0)


@pytest.mark.parametrize("n", [1500, 2048, 9000, 40000])
@pytest.mark.parametrize("dim", [24, 513])
def test_gradient_of_hot_tokens(n, dim):
    # Long runs over many chunks, beside rows of one position, and one run of everything.
    rows = 500
    tokens = _randint(rows, (n,), 11)
    hot = torch.rand(n, generator=_gen(12), device=DEV)
    tokens = torch.where(hot < 0.6, torch.full_like(tokens, 17), tokens)
    tokens = torch.where((hot >= 0.6) & (hot < 0.8), torch.full_like(tokens, 499), tokens)
    go = _randn((n, dim), BF16, 13)
    check_backward(te().token_backward(go, tokens, rows), go, tokens, rows, 1.0)
    same = torch.full((n,), 3, device=DEV)
    check_backward(te().token_backward(go, same, rows), go, same, rows, 1.0)


@pytest.mark.parametrize("n", [64, 3000])
def test_gradient_runs_of_every_length_at_every_chunk_position(n):
    # Sorted tokens whose runs end at, just before and just after multiples of 32.
    lengths = [1, 31, 32, 33, 63, 64, 65, 1, 30, 2, 95, 97, 128, 3]
    tokens = torch.repeat_interleave(torch.arange(len(lengths)), torch.tensor(lengths))
    tokens = tokens.repeat(n // tokens.numel() + 1)[:n].sort().values.to(DEV)
    go = _randn((n, 40), F32, 14)
    check_backward(te().token_backward(go, tokens, 20), go, tokens, 20, 1.0)


@pytest.mark.parametrize("n", [700, 6000])
@pytest.mark.parametrize("out", [F32, BF16, F16])
@pytest.mark.parametrize("dim", [32, 33])
def test_gradient_accumulates_into_the_rows_of_its_tokens_only(n, out, dim):
    rows = 3001
    tokens = _randint(rows // 2, (n,), 15)
    go = _randn((n, dim), BF16, 16)
    base = _randn((rows, dim), out, 17)
    base[rows - 1, 0] = float("nan")  # a row without a token is not touched
    got = base.clone()
    r = te().token_backward(go, tokens, rows, scale=0.5, out=got, accumulate=True)
    assert r is got
    check_backward(got[:rows // 2], go, tokens, rows // 2, 0.5, base=base[:rows // 2])
    assert torch.equal(torch.nan_to_num(got[rows // 2:], 9.0), torch.nan_to_num(base[rows // 2:], 9.0))


@pytest.mark.parametrize("n", [900, 5000])
def test_gradient_of_padding_and_out_of_range_tokens(n):
    rows = 300
    tokens = _randint(rows, (n,), 18)
    tokens[::3] = 5
    tokens[1::7] = -1
    tokens[2::11] = rows
    tokens[3::13] = 2 ** 33 + 1
    go = _randn((n, 48), F32, 19)
    go[0] = float("nan")  # tokens[0] is padding
    error = torch.zeros(1, dtype=torch.int32, device=DEV)
    got = te().token_backward(go, tokens, rows, padding_idx=5, error=error)
    assert error.item() == 2
    assert not got[5].any()
    check_backward(got, go, tokens, rows, 1.0, padding=5)
    everything = torch.full((n,), 5, device=DEV)
    got = te().token_backward(go, everything, rows, padding_idx=5, out=torch.full((rows, 48), 7.0, device=DEV))
    assert not got.any()


@pytest.mark.parametrize("length", [40, 900])
def test_gradient_strided_operands(length):
    rows = 200
    tokens = _randint(rows, (6, length + 1), 20)
    go = _randn((6, length + 1, 72), BF16, 21)
    for t, g in ((tokens[:, :-1], go[:, 1:]), (tokens[:, 1:], go[:, 1:, :64]), (tokens.t(), go.transpose(0, 1)),
                 (tokens[:, ::2], go[:, ::2, 3:60]), (tokens, go[:1].expand(6, length + 1, 72)),
                 (tokens, go[:, :, :1].expand(6, length + 1, 16)), (tokens, go.flip(0)[..., 8:])):
        buffer = torch.full((rows, g.shape[-1] + 5), 3.0, device=DEV)
        got = te().token_backward(g, t, rows, out=buffer[:, :g.shape[-1]])
        check_backward(got, g, t, rows, 1.0)
        assert bool((buffer[:, g.shape[-1]:] == 3.0).all())


def test_gradient_without_tokens():
    go = torch.empty(0, 16, device=DEV)
    tokens = torch.empty(0, dtype=torch.int64, device=DEV)
    out = torch.full((37, 16), 5.0, device=DEV)
    te().token_backward(go, tokens, 37, out=out, accumulate=True)
    assert bool((out == 5.0).all())
    te().token_backward(go, tokens, 37, out=out)
    assert not out.any()
    assert te().token_backward(go, tokens, 0).shape == (0, 16)


@pytest.mark.parametrize("n", [10, 3000])
def test_gradient_and_lookup_of_a_table_without_rows(n):
    tokens = torch.zeros(n, dtype=torch.int64, device=DEV)
    error = torch.zeros(1, dtype=torch.int32, device=DEV)
    assert te().token_backward(torch.ones(n, 16, device=DEV), tokens, 0, error=error).shape == (0, 16)
    assert error.item() == 2
    assert not te().token_forward(torch.empty(0, 16, device=DEV), tokens).any()


def test_gradient_with_many_sort_tiles():
    # More tiles than the one-kernel radix pass takes.
    n, rows = 2_200_000, 100_003
    tokens = _randint(rows, (n,), 22, torch.int32)
    go = _randn((n, 4), F32, 23)
    check_backward(te().token_backward(go, tokens, rows), go, tokens, rows, 1.0)


@pytest.mark.parametrize("n", [1000, 30000])
def test_gradient_is_deterministic_on_any_stream(n):
    tokens = (torch.rand(n, generator=_gen(24), device=DEV) ** 4 * 800).long()
    go = _randn((n, 128), BF16, 25)
    first = te().token_backward(go, tokens, 800)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(3):
        with torch.cuda.stream(side):
            again = te().token_backward(go, tokens, 800)
        side.synchronize()
        assert torch.equal(first, again)


def test_lookup_and_gradient_in_a_graph():
    table = _randn((400, 64), BF16, 26)
    tokens = _randint(400, (4, 700), 27)
    go = _randn((4, 700, 64), BF16, 28)
    out = torch.empty(4, 700, 64, dtype=BF16, device=DEV)
    grad = torch.empty(400, 64, device=DEV)

    def call():
        te().token_forward(table, tokens, scale=8.0, out=out)
        te().token_backward(go, tokens, 400, scale=8.0, out=grad)

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    tokens.copy_(_randint(400, (4, 700), 29))
    go.copy_(_randn((4, 700, 64), BF16, 30))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, (table[tokens].float() * 8.0).to(BF16))
    check_backward(grad, go, tokens, 400, 8.0)


def test_gradient_is_the_derivative_of_the_lookup():
    # The lookup is linear in the table, so differences along any direction are exact up to
    # rounding: <go, f(E + D) - f(E)> = <dE, D>, with small whole numbers without any rounding.
    table = torch.randint(-8, 8, (50, 24), generator=_gen(31), device=DEV).float()
    step = torch.randint(-4, 4, (50, 24), generator=_gen(32), device=DEV).float()
    for n in (300, 4000):
        tokens = _randint(50, (n,), 33)
        go = torch.randint(-3, 3, (n, 24), generator=_gen(34), device=DEV).float()
        grad = te().token_backward(go, tokens, 50, scale=2.0)
        change = te().token_forward(table + step, tokens, scale=2.0) - te().token_forward(table, tokens, scale=2.0)
        assert (go.double() * change.double()).sum().item() == (grad.double() * step.double()).sum().item()


def test_agrees_with_the_pooled_lookup_of_single_tokens():
    from paper_2609_30656_gb300 import tbe
    table = _randn((500, 64), F32, 35)
    tokens = _randint(500, (600,), 36)
    m = tbe.TBE([table])
    offsets = torch.arange(601, device=DEV)
    assert torch.equal(m.forward(tokens, offsets), te().token_forward(table, tokens))
    m.close()


# ----------------------------------------------------------------------------- refusals

def test_refusals_of_the_binding():
    t = te()
    table = torch.zeros(10, 8, device=DEV)
    tokens = torch.zeros(4, dtype=torch.int64, device=DEV)
    go = torch.zeros(4, 8, device=DEV)
    bad = [
        lambda: t.token_forward(table.cpu(), tokens),
        lambda: t.token_forward(table[0], tokens),
        lambda: t.token_forward(table.double(), tokens),
        lambda: t.token_forward(table.t(), tokens),
        lambda: t.token_forward(table, tokens.cpu()),
        lambda: t.token_forward(table, tokens.short()),
        lambda: t.token_forward(table, tokens, out=torch.zeros(5, 8, device=DEV)),
        lambda: t.token_forward(table, tokens, out=torch.zeros(4, 8, device=DEV, dtype=torch.float64)),
        lambda: t.token_forward(table, tokens, error=torch.zeros(2, dtype=torch.int32, device=DEV)),
        lambda: t.token_backward(go.cpu(), tokens, 10),
        lambda: t.token_backward(go[:3], tokens, 10),
        lambda: t.token_backward(go, tokens.float(), 10),
        lambda: t.token_backward(go, tokens, -1),
        lambda: t.token_backward(go, tokens, 10, padding_idx=10),
        lambda: t.token_backward(go, tokens, 10, accumulate=True),
        lambda: t.token_backward(go, tokens, 10, out=torch.zeros(9, 8, device=DEV)),
        lambda: t.token_backward(go, tokens, 10, out=torch.zeros(8, 10, device=DEV).t()),
        lambda: t.token_backward(go, tokens, 10, out_dtype=torch.float64),
    ]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    with pytest.raises(TypeError):
        t.token_forward(table, tokens, out=go, out_dtype=BF16)
    from paper_2609_30656_gb300 import tbe
    with pytest.raises(tbe.CbTbeError):
        t.token_forward(table, tokens, scale=float("nan"))
