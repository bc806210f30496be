"""Choice of the next token where the range of a row, or of its weights, passes what a float holds:
infinite and enormous temperatures beside masks, logits at both ends of the type."""
import math

import pytest
import torch

from tests.test_gpu_sample import DTYPES, S, check  # noqa: F401  (S: the fixture)

pytestmark = pytest.mark.gpu
KS = [1, 5, 300, 512, 700, 0]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("t", [math.inf, 1e38, 3e38, 2e37, 1e36])
@pytest.mark.parametrize("mask", [-math.inf, "lowest"])
@pytest.mark.parametrize("vocab", [40, 999, 9000])
def test_hot_and_masked(S, dtype, t, mask, vocab):  # noqa: F811
    """All that is not masked weighs alike (or nearly)."""
    gen = torch.Generator().manual_seed(31)
    logits = torch.randn(6, vocab, generator=gen)
    logits[:, ::2] = torch.finfo(dtype).min if mask == "lowest" else mask
    for u in (0.0, 0.4, 0.99):
        check(S, logits.to(dtype).cuda(), [u] * 6, t=[t] * 6, k=KS)
        check(S, logits.to(dtype).cuda(), [u] * 6, t=[t] * 6, k=KS, p=[0.5] * 6, m=[0.1] * 6)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("t", [math.inf, 1e38, 1.0])
def test_both_ends_of_the_type(S, dtype, t):  # noqa: F811
    """A spread that passes the type's largest value."""
    gen = torch.Generator().manual_seed(32)
    most = torch.finfo(dtype).max
    logits = torch.empty(6, 3000)
    logits[0] = (torch.rand(3000, generator=gen) * 2 - 1) * most
    logits[1] = -most
    logits[1, 5::700] = most
    logits[2] = -most
    logits[3] = -most
    logits[3, 9] = -math.inf
    logits[4] = most
    logits[4, 3] = -most
    logits[5] = -math.inf
    logits[5, 100:104] = torch.tensor([-most, most, 0.0, -most])
    for u in (0.0, 0.4, 0.9999):
        for k in (1, 5, 300):
            check(S, logits.to(dtype).cuda(), [u] * 6, t=[t] * 6, k=[k] * 6)
