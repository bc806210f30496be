"""Infinities in k of linear attention: chunks give the infinities that the recurrence has, as
single tokens do."""
import math

import pytest
import torch

from tests.test_gpu_linear import DTYPES, F64, L, bounds, gpu, make, recurrence  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("dk,dv", [(64, 64), (128, 128), (256, 128), (64, 512)])
@pytest.mark.parametrize("decay", ["none", "head"])
@pytest.mark.parametrize("lens", [[70], [20, 200], [1300]])
def test_infinite_k(L, dtype, dk, dv, decay, lens):  # noqa: F811
    """Weighted values that a bfloat16 holds (no decay), and others."""
    c, cu = make(lens, 2, dk, dv, dtype, decay, seed=41)
    at = lens[0] - 9
    c["k"][0, at, 1, 3], c["k"][0, at, 1, 21] = math.inf, -math.inf
    c["k"][0, at + 2, 0, 5] = -math.inf
    # (no zeros where an infinity meets them, and one sign for what two of them make together)
    c["q"][..., 21] = -c["q"][..., 3]
    c["h0"][:, :, :, 2] = 0
    o, ht, mo, mt = recurrence(c, lens)
    for f in (L.gdn_linear_chunk_fwd, L.gdn_linear_recurrent_fwd):
        go, gt = (x.cpu().to(F64) for x in f(**gpu(c), **cu))
        odd, odd_t = torch.isinf(o), torch.isinf(ht)
        assert odd[0, at:lens[0], 1].all() and odd_t[0, 1, 3].all()
        assert torch.equal(go[odd], o[odd]) and torch.equal(gt[odd_t], ht[odd_t])
        o0, ht0, mo0, mt0 = (torch.where(w, 0.0, x) for w, x in
                             ((odd, o), (odd_t, ht), (odd, mo), (odd_t, mt)))
        bo, bt = bounds(c, lens, o0, mo0, mt0)
        assert ((torch.where(odd, 0.0, go) - o0).abs() <= bo).all()
        assert ((torch.where(odd_t, 0.0, gt) - ht0).abs() <= bt).all()
