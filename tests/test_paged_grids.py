"""Calls whose grids would pass what one launch holds are refused before any launch."""
import pytest

from tests.test_paged_abi import SHAPE, attn, cache, lib, ref, rows, tokens  # noqa: F401


@pytest.mark.parametrize("kw,keys", [
    (dict(B=1 << 22, T=1, Hq=4, Hk=4), 4000),        # few rows: 2^24 workgroups
    (dict(B=1 << 22, T=1, Hq=4, Hk=4), 100),         # the other kernel
    (dict(B=1 << 21, T=40, Hq=8, Hk=8), 4000)])
def test_too_many_workgroups(lib, kw, keys):  # noqa: F811
    t, r, c, a = tokens(**kw), rows(), cache(max_blocks=1 << 10), attn(max_kv=keys)
    assert lib.gdn_cache_attn(ref(t), ref(a), ref(r), ref(c), ref(r), None, None, 0, None) == SHAPE
    assert lib.gdn_cache_attn_workspace_size(ref(t), ref(c), ref(a)) == 0
