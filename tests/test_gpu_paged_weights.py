"""The weights of a softmax keep more than a bfloat16's bits in the kernel of few rows: its outputs
are the exact ones but for 32-bit evaluation and one rounding."""
import math

import pytest
import torch

from tests.paged_ref import Case

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.fixture(scope="module")
def P():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2412_06464_amd import paged
    paged.load_library()
    return paged


def bound(o, rel, mass):
    """32-bit evaluation; a weight as the sum of two bfloat16 values, each off by 2^-8 of what it
    stands for (2^-16 of the weight in all); the output rounded once (2^-8 of itself, and of what
    it is off by before)."""
    before = (rel[..., None] + 2.0 ** -16) * mass
    return before * (1 + 2.0 ** -8) + 2.0 ** -8 * o.abs() + 1e-30


@pytest.mark.parametrize("d,Hq,Hk", [(64, 4, 4), (64, 16, 1), (128, 8, 2), (128, 3, 1), (256, 6, 2)])
@pytest.mark.parametrize("new,kv,window", [
    ([1] * 6, [1, 2, 17, 65, 130, 511], 0),   # single tokens
    ([1, 0, 1], [2999, 5, 1200], 0),          # keys split over workgroups
    ([2, 1, 0, 2], [33, 700, 4, 90], 20)])    # two tokens, a window; up to 32 rows
def test_one_rounding(P, d, Hq, Hk, new, kv, window):
    c = Case(new, kv, Hq, Hk, d, 32, BF, window, seed=d + len(new))
    print("[gpu-case] weights", d, Hq, Hk, new, kv, window, flush=True)
    o = P.gdn_cache_attn(c.q[None].cuda(), c.k_pages.cuda(), c.v_pages.cuda(), c.table.cuda(),
                         c.kv_lens.cuda(), window=window, max_kv=max(kv), cu_seqlens=c.cu.cuda(),
                         cu_seqlens_host=c.cu)[0].cpu()
    ro, lse, rel, mass = c.attend()
    assert (lse > -math.inf).all()
    bad = ~((o.double() - ro).abs() <= bound(ro, rel, mass))
    assert not bad.any(), (int(bad.sum()), torch.nonzero(bad)[:3])
