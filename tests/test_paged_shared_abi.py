"""Refusals of attention over a shared prefix, made on the host before any launch (no GPU)."""
import ctypes
import os

import pytest
import torch

from paper_2412_06464_amd import gdn, paged
from tests.test_paged_abi import (ALIGN, BAD_TOKENS, CU, FAKE, NULL, ODD, SHAPE, VALUE, WS, attn,
                                  cache, ref, rows, tokens)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(gdn.LIB_PATH):
        from paper_2412_06464_amd import build
        build.build()
    return paged.load_library()


def call(lib, t=None, a=None, q=None, c=None, table=FAKE, prefix=100, o=None, lse=None, ws=FAKE,
         size=1 << 40, without=()):
    t, a, c, q, o = t or tokens(), a or attn(), c or cache(), q or rows(), o or rows()
    t, a, c, q, o = (None if n in without else ref(x)
                     for n, x in (("t", t), ("a", a), ("c", c), ("q", q), ("o", o)))
    return lib.gdn_cache_attn_shared(t, a, q, c, table, prefix, o, lse, ws, size, None)


def need(lib, t=None, c=None, a=None, prefix=100):
    return lib.gdn_cache_attn_shared_workspace_size(ref(t or tokens()), ref(c or cache()),
                                                    ref(a or attn()), prefix)


@pytest.mark.parametrize("kw,code", BAD_TOKENS)
def test_bad_tokens(lib, kw, code):
    assert call(lib, t=tokens(**kw)) == code
    assert need(lib, t=tokens(**kw)) == 0


def test_boundaries(lib):
    cu = (ctypes.c_int32 * 3)(0, 7, 6)
    t = tokens(B=1, T=10, num_seqs=2, cu_seqlens=FAKE, cu_seqlens_host=ctypes.addressof(cu))
    assert call(lib, t=t) == CU and need(lib, t=t) == 0


@pytest.mark.parametrize("kw,code", [
    (dict(page_size=48), SHAPE), (dict(num_pages=0), SHAPE), (dict(table=None), NULL),
    (dict(kv_lens=None), NULL), (dict(v=ODD), ALIGN), (dict(token_stride=-128), SHAPE)])
def test_bad_cache(lib, kw, code):
    assert call(lib, c=cache(**kw)) == code


def test_refusals(lib):
    for name in "tacqo":
        assert call(lib, without=(name,)) == NULL, name
    assert call(lib, table=None) == NULL
    assert call(lib, table=FAKE + 2) == ALIGN
    assert call(lib, lse=FAKE + 2) == ALIGN
    assert call(lib, q=rows(ODD)) == ALIGN and call(lib, o=rows(hs=132)) == ALIGN
    for kw in (dict(scale=0.0), dict(window=-1), dict(max_kv=-1), dict(window=4, causal=0)):
        assert call(lib, a=attn(**kw)) == VALUE, kw
    assert call(lib, t=tokens(Hk=3)) == SHAPE
    for prefix, code in ((-1, VALUE), (257, SHAPE), (2 ** 31 - 1, SHAPE)):  # room: 4 x 64 tokens
        assert call(lib, prefix=prefix) == code and need(lib, prefix=prefix) == 0


def test_workspace(lib):
    """Sums of the prefix and of the own keys, at least one of each, for each row."""
    for prefix in (1, 100, 256):
        n = need(lib, prefix=prefix)
        assert n >= 2 * 20 * 4 * (128 + 2) * 4
        assert call(lib, prefix=prefix, ws=None) == WS
        assert call(lib, prefix=prefix, size=n - 1) == WS
        assert call(lib, prefix=prefix, ws=ODD, size=n) == ALIGN
    # without a prefix it is the attention over the cache: what that needs, and refuses
    long = cache(max_blocks=4096)
    n = need(lib, c=long, prefix=0)
    assert n == lib.gdn_cache_attn_workspace_size(ref(tokens()), ref(long), ref(attn())) > 0
    assert call(lib, c=long, prefix=0, size=n - 1) == WS


def test_no_more_splits_than_the_join_takes(lib):
    """The sums of a row, over sizes from a few rows to many and short keys to the longest."""
    for Hq, Hk in ((1, 1), (8, 8), (16, 2)):
        for B, T in ((1, 1), (1, 33), (2, 17), (64, 1), (3, 500), (257, 1)):
            for blocks in (2, 100, 5000, 1 << 20):
                for prefix in (1, 64 * blocks // 2, 64 * blocks - 1):
                    for dt in (gdn.GDN_F32, gdn.GDN_BF16):
                        t = tokens(B=B, T=T, Hq=Hq, Hk=Hk, d=64, dtype=dt)
                        c = cache(max_blocks=blocks, head_stride=4096, token_stride=64)
                        n = need(lib, t=t, c=c, prefix=prefix)
                        row = B * T * Hq * (64 + 2) * 4
                        assert 2 * row <= n <= 512 * row + 512, (B, T, Hq, Hk, blocks, prefix)


def test_binding_refuses():
    q, k = torch.zeros(1, 4, 2, 64), torch.zeros(5, 1, 16, 64)
    i = torch.zeros(1, 3, dtype=torch.int32)
    with pytest.raises(TypeError, match="prefix_table"):
        paged.gdn_cache_attn_shared(q, k, k, i, i[0, :1], [0], 4)
    for bad in (-1, 1 << 31):
        with pytest.raises(ValueError, match="prefix"):
            paged.gdn_cache_attn_shared(q, k, k, i, i[0, :1], i[0], bad)
    with pytest.raises(ValueError, match="GPU"):
        paged.gdn_cache_attn_shared(q, k, k, i, i[0, :1], i[0], 4)
