"""The bound from which a small top-k gathers its tokens: rows whose lowest logits are among the k
largest, and rows whose range, or range over temperature, has no float."""
import math

import numpy as np
import pytest
import torch

from tests.test_gpu_sample import S, check  # noqa: F401  (S: the fixture)

pytestmark = pytest.mark.gpu
US = [0.0, 0.03, 0.3, 0.6, 0.97, 1 - 2.0 ** -24]


@pytest.mark.parametrize("vocab", [51, 400, 3001])
@pytest.mark.parametrize("top,low", [(1.0, 0.3), (10.0, 0.1), (3.3, -0.7), (14.9, -4.9),
                                     (1e6, 1e6 - 1.0), (0.1, 1e-3)])
def test_ties_at_the_lowest(S, vocab, top, low):  # noqa: F811
    """One larger logit, or 30, over many alike: the k-th is one of these."""
    logits = torch.full((6, vocab), low)
    logits[:, 7] = top
    logits[3:, 20:50] = torch.linspace(low, top, 32)[1:-1]
    for k in (2, 50):
        check(S, logits.cuda(), US, k=[k] * 6)
        check(S, logits.cuda(), US, t=[0.5, 1, 2, 0.5, 1, 2], k=[k] * 6, p=[0.99] * 6)


def test_lowest_is_kept(S):  # noqa: F811
    """Random rows and every k up to the vocabulary: the last of the kept, drawn by the largest
    random number, is the k-th, also where that is the row's last."""
    gen = torch.Generator().manual_seed(21)
    rows = 255
    logits = (torch.rand(rows, rows + 1, generator=gen) * 0.5 + torch.rand(rows, 1, generator=gen) * 9)
    check(S, logits.cuda(), [1 - 2.0 ** -24] * rows, k=list(range(1, rows + 1)))
    wide = torch.randn(rows, 5000, generator=gen) * 0.01 + torch.rand(rows, 1, generator=gen) * 9
    check(S, wide.cuda(), [1 - 2.0 ** -24] * rows, k=[1 + 2 * i for i in range(rows)])


@pytest.mark.parametrize("low", np.random.default_rng(22).uniform(-5, 0, 6).astype(np.float32).tolist())
@pytest.mark.parametrize("top", np.random.default_rng(23).uniform(0, 15, 6).astype(np.float32).tolist())
def test_two_values(S, top, low):  # noqa: F811
    logits = torch.full((6, 64), low)
    logits[:, 33] = top
    check(S, logits.cuda(), US, t=[15.0] * 6, k=[50] * 6)
