"""How many bits linear attention keeps: of a weighted value that enters the state all 24, of the
state and of a chunk's products, where they are operands for o, 16."""
import pytest
import torch

from tests.test_gpu_linear import DTYPES, F64, L, gpu, make, recurrence  # noqa: F401

U = 2.0 ** -24
LOSS = 2.0 ** -16  # of a value as two bfloat16: each leaves at most 2^-8 of what it stands for
# One weighted value, as test_weighted_values has it: the exponential's argument, at most 3, is
# rounded once (3 ln 2 u), the exponential is 2 u off, the product 1, three values leave less
# than 1 of it, and their three additions up to 2 u each (they need not round to nearest).
ONE = (3 + 2 + 1 + 1 + 6) * U


def parts(x, n):
    """Sum of the first n bfloat16 values that stand for x."""
    y = torch.zeros_like(x, dtype=F64)
    for _ in range(n):
        y += (x.to(F64) - y).to(torch.bfloat16).to(F64)
    return y


def test_two_values_would_be_noticed():
    """What tells three values from two: of as many weighted values as the test below has, some are
    further off as two than all its other roundings together (so that the sum is, in either sign)."""
    gen = torch.Generator().manual_seed(51)
    x = (torch.randn(64, generator=gen).bfloat16().float() * torch.rand(64, generator=gen)).abs()
    assert ((parts(x, 3) - x.to(F64)).abs() <= U * x).all()
    assert ((parts(x, 2) - x.to(F64)).abs() / x).max() > 2 * ONE


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("dk", [64, 128, 256])
@pytest.mark.parametrize("dv", [64, 128, 512])
@pytest.mark.parametrize("T,at", [(1, 0), (40, 5), (64, 0), (64, 62)])
def test_weighted_values(L, dtype, dk, dv, T, at):  # noqa: F811
    """One token's k is 1 in one place: that row of the state is v, decayed since."""
    c, _ = make([T], 2, dk, dv, dtype, h0=False, seed=52 + T + at, dense=True)
    c["k"].zero_()
    c["k"][0, at, 0, 7], c["k"][0, at, 1, dk - 1] = 1, 1
    c["log_alpha"] *= 2 / max(2.0, float(-c["log_alpha"].sum(1).min()))
    for f in (L.gdn_linear_chunk_fwd, L.gdn_linear_recurrent_fwd):
        _, ht = f(**gpu(c))
        for h, row in ((0, 7), (1, dk - 1)):
            want = c["log_alpha"][0, at + 1:, h].to(F64).sum().exp() * c["v"][0, at, h].to(F64)
            # (token by token: each step's exponential and product)
            slack = ONE if f is L.gdn_linear_chunk_fwd else 4 * T * U
            err = (ht[0, h, row].cpu().to(F64) - want).abs() / want.abs()
            assert err.max() <= slack, float(err.max() / U)


@pytest.mark.gpu
@pytest.mark.parametrize("dk,dv", [(64, 64), (64, 128), (128, 64), (128, 128), (256, 64), (256, 512)])
@pytest.mark.parametrize("lens", [[1], [130], [50, 400, 64], [1500]])
@pytest.mark.parametrize("decay", ["token", "none"])
def test_outputs(L, dk, dv, lens, decay):  # noqa: F811
    """In bfloat16 o is its 64-bit value rounded once, but for LOSS (and fp32 sums as in bounds) of the
    sum of its terms' absolute values."""
    c, cu = make(lens, 2, dk, dv, torch.bfloat16, decay, seed=53)
    o, _, mo, _ = recurrence(c, lens)
    got = L.gdn_linear_chunk_fwd(**gpu(c), **cu)[0].cpu().to(F64)
    extra = (LOSS + (max(lens) + dk + 128) * U) * mo
    err = (got - o).abs()
    assert (err <= extra + 2.0 ** -8 * (o.abs() + extra)).all(), \
        float((err / (extra + 2.0 ** -8 * o.abs())).max())


@pytest.mark.gpu
@pytest.mark.parametrize("dk,dv", [(64, 64), (64, 128), (128, 64), (128, 128), (256, 64), (256, 512)])
@pytest.mark.parametrize("lens", [[130], [70, 200], [1500]])
@pytest.mark.parametrize("decay", ["head", "none"])
@pytest.mark.parametrize("where", ["h0", "q", "k"])
def test_outputs_beside_infinities(L, dk, dv, lens, decay, where):  # noqa: F811
    """An infinity in the state, in q or in k takes no bits from what it does not reach, and in the
    state it is the infinity that the recurrence has."""
    c, cu = make(lens, 2, dk, dv, torch.bfloat16, decay, seed=55)
    at = lens[0] - 40
    hit = torch.zeros(c["v"].shape, dtype=torch.bool)
    if where == "h0":
        c["h0"][0, 1, 3, 5] = float("inf")
        hit[0, :lens[0], 1, 5] = True
    elif where == "q":
        c["q"][0, at, 1, 3] = float("inf")
        hit[0, at, 1] = True
    else:
        c["k"][0, at, 1, 3] = float("-inf")
        hit[0, at:lens[0], 1] = True
    o, ht, mo, mt = recurrence(c, lens)
    got, gt = (x.cpu().to(F64) for x in L.gdn_linear_chunk_fwd(**gpu(c), **cu))
    assert torch.equal(~torch.isfinite(o), hit) and torch.equal(~torch.isfinite(got), hit)
    if where != "q":
        # (decays of a head at most 0.1 a token: 1500 leave more than float32's least)
        assert torch.equal(got[hit], o[hit])
    odd = torch.isinf(ht)
    assert torch.equal(gt[odd], ht[odd]) and torch.isfinite(gt[~odd]).all()
    extra = (LOSS + (max(lens) + dk + 128) * U) * mo
    err = (got - o).abs()
    assert (err <= extra + 2.0 ** -8 * (o.abs() + extra))[~hit].all(), \
        float((err / (extra + 2.0 ** -8 * o.abs()))[~hit].max())
