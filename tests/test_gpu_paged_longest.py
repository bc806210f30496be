"""Attention over a cache of the greatest length: positions up to 2^31 - 2^18, nearly all of them
holes, with the visible keys in a few ranges of the split."""
import pytest
import torch

from tests.paged_ref import Case

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
PAGE = 1024
BLOCKS = (2 ** 31 - 2 ** 18) // PAGE


@pytest.fixture(scope="module")
def P():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2412_06464_amd import paged
    paged.load_library()
    return paged


@pytest.mark.parametrize("window,blocks", [
    (0, [BLOCKS - 1]),                      # the last range alone
    (0, [0, BLOCKS // 2, BLOCKS - 1]),
    (2 ** 30, [BLOCKS // 4, BLOCKS - 2 ** 19, BLOCKS - 1])])  # the first: behind the window
def test_keys_at_the_end(P, window, blocks):
    seen = blocks[1:] if window else blocks
    # the same keys in a short cache
    c = Case([1], [PAGE * len(seen)], 2, 1, 64, PAGE, BF, seed=len(blocks), spare=1)
    spare = (set(range(c.k_pages.shape[0])) - set(c.table[0].tolist())).pop()
    table = torch.full((1, BLOCKS), -1, dtype=torch.int32)
    for i, b in enumerate(seen):
        table[0, b] = c.table[0, i]
    if window:
        table[0, blocks[0]] = spare  # holds NaN
    print("[gpu-case] longest", window, blocks, flush=True)
    q, kp, vp = c.q[None].cuda(), c.k_pages.cuda(), c.v_pages.cuda()
    lens = torch.tensor([BLOCKS * PAGE], dtype=torch.int32, device="cuda")
    lse = torch.zeros(1, 1, 2, device="cuda")
    o = P.gdn_cache_attn(q, kp, vp, table.cuda(), lens, window=window, lse=lse)
    torch.cuda.synchronize()
    ro, rl, rel, mass = c.attend()
    assert ((o[0].cpu().double() - ro).abs() <= c.bound(rel, mass)).all()
    tol = rel + rl.abs() * 2.0 ** -22 + 2.0 ** -20
    assert ((lse[0].cpu().double() - rl).abs() <= tol).all()
