"""Sequences of few rows keep the accuracy that gdn_cache_attn gives them when they share a prefix:
their outputs are the exact ones but for 32-bit evaluation and one rounding."""
import math

import pytest
import torch

from tests.test_gpu_paged_shared import F64, P, Shared  # noqa: F401  (P: the fixture)
from tests.test_gpu_paged_weights import bound

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.mark.parametrize("d,Hq,Hk", [(64, 4, 4), (64, 16, 1), (128, 8, 2), (128, 3, 1), (256, 6, 2)])
@pytest.mark.parametrize("new,prefix,own,window", [
    ([1] * 6, 200, 40, 0),                    # 32 rows of a cache head and less
    ([1] * 40, 333, 120, 0),                  # a block of rows of many sequences, and several
    ([1, 0] * 35, 1500, 3, 0),                # the prefix's keys split
    ([2, 1, 0, 2] * 11, 400, 60, 300),        # two tokens, a window; up to 32 rows a sequence
    ([1] * 70, 64, 500, 0)])                  # own keys split
def test_one_rounding(P, d, Hq, Hk, new, prefix, own, window):  # noqa: F811
    kv = [prefix + max(m, (i * 37) % (own + 1)) for i, m in enumerate(new)]
    c = Shared(new, kv, prefix, Hq, Hk, d, 32, BF, window, seed=d + len(new))
    print("[gpu-case] shared weights", d, Hq, Hk, len(new), prefix, own, window, flush=True)
    o, _ = c.call(P, max_kv=max(kv))
    ro, lse, rel, mass = c.attend()
    assert (lse > -math.inf).all()
    bad = ~((o.to(F64) - ro).abs() <= bound(ro, rel, mass))
    assert not bad.any(), (int(bad.sum()), torch.nonzero(bad)[:3])
