"""Rotary positions of more tokens than one direction of a launch holds workgroups for."""
import pytest
import torch

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def test_rotation_of_many_tokens():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2412_06464_amd import paged as P
    T = (1 << 26) + 11  # 2^24 workgroups of 4 tokens, and three more
    at = torch.tensor([0, 5, (1 << 24) - 1, 1 << 24, (1 << 25) + 7, (1 << 26) - 1, 1 << 26,
                       T - 4, T - 3, T - 1]).cuda()
    q = torch.zeros(1, T, 1, 64, dtype=BF, device="cuda")
    x = torch.randn(1, len(at), 1, 64, generator=torch.Generator().manual_seed(1)).to(BF).cuda()
    q[:, at] = x
    r = P.gdn_rotary(64)
    want = P.gdn_rotary_fwd(x, None, r, positions=at.to(torch.int32)[None])[0]
    P.gdn_rotary_fwd(q, None, r, q_out=q)
    torch.cuda.synchronize()
    assert torch.equal(q[:, at], want)
    q[:, at] = 0
    assert not any(part.any() for part in q.split(1 << 22, dim=1))
