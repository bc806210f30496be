"""How attention over a shared prefix is cut (no GPU): its workspace holds the partial sums of every
range of keys, so its size tells how many there are."""
import os

import pytest

from paper_2412_06464_amd import gdn, paged
from tests.test_paged_abi import attn, cache, ref, tokens


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(gdn.LIB_PATH):
        from paper_2412_06464_amd import build
        build.build()
    return paged.load_library()


def ranges(lib, N, prefix, room, max_kv, dtype, d=128, Hq=16, Hk=4, page=64):
    """Ranges of the prefix, by the size that the call has beside that of the own keys (one range
    of these for each sequence where the sequences fill the GPU)."""
    t = tokens(B=N, T=1, Hq=Hq, Hk=Hk, d=d, dtype=dtype)
    c = cache(page_size=page, num_pages=1 << 20, max_blocks=room // page, token_stride=Hk * d,
              head_stride=d, page_stride=page * Hk * d)
    size = lib.gdn_cache_attn_shared_workspace_size(ref(t), ref(c), ref(attn(max_kv=max_kv)), prefix)
    assert size > 0
    return size // (N * Hq * (d + 2) * 4) - 1


@pytest.mark.parametrize("dtype", [gdn.GDN_BF16, gdn.GDN_F32])
@pytest.mark.parametrize("N", [256, 512])
@pytest.mark.parametrize("room", [1 << 15, 1 << 17, 1 << 20])
def test_unused_room_leaves_the_prefix_its_share(lib, dtype, N, room):
    """Without max_kv the tables' room says nothing of what the sequences hold: the prefix is still
    cut, into about a quarter of the workgroups that run at once (512)."""
    prefix = 8192
    told = ranges(lib, N, prefix, room, prefix + 64, dtype)
    untold = ranges(lib, N, prefix, room, 0, dtype)
    least = 512 // 4 // (-(-N * 4 // 128) * 4)  # of row blocks of 128, for four cache heads
    assert told >= least >= 2 and untold >= least
