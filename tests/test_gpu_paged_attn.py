"""Attention over the paged cache against a plain 64-bit evaluation."""
import math

import pytest
import torch

from tests.paged_ref import Case

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def say(*a):
    print("[gpu-case]", *a, flush=True)


@pytest.fixture(scope="module")
def P():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2412_06464_amd import paged
    paged.load_library()
    return paged


def call(P, c, dense=False, scale=None, max_kv=None, **kw):
    q = c.q.cuda()
    q = q.reshape(len(c.new), -1, c.Hq, c.d) if dense else q[None]
    cu = {} if dense else dict(cu_seqlens=c.cu.cuda(), cu_seqlens_host=c.cu)
    lse = torch.full(q.shape[:3], math.nan, device="cuda")
    o = torch.full_like(q, math.nan)
    P.gdn_cache_attn(q, c.k_pages.cuda(), c.v_pages.cuda(), c.table.cuda(), c.kv_lens.cuda(),
                     scale=scale, causal=c.causal, window=c.window,
                     max_kv=max(c.kv) if max_kv is None else max_kv, o=o, lse=lse, **cu, **kw)
    torch.cuda.synchronize()
    return o.reshape(c.q.shape).cpu(), lse.reshape(c.q.shape[:2]).cpu()


def check(c, o, lse, scale=None):
    ro, rl, rel, mass = c.attend(scale)
    err = (o.double() - ro).abs()
    bad = ~(err <= c.bound(rel, mass))
    assert not bad.any(), (int(bad.sum()), err[bad].max(), torch.nonzero(bad)[:3])
    empty = rl == -math.inf
    assert (lse[empty] == -math.inf).all()
    # log of the sum: its relative error, and the rounding of the result
    tol = rel[~empty] + rl[~empty].abs() * 2.0 ** -22 + 2.0 ** -20
    assert ((lse[~empty].double() - rl[~empty]).abs() <= tol).all()


HEADS = [(BF, 64, 4, 4), (BF, 64, 16, 1), (BF, 128, 8, 2), (BF, 128, 3, 1), (BF, 256, 6, 2),
         (F32, 64, 4, 2), (F32, 128, 2, 2), (F32, 256, 3, 1)]


@pytest.mark.parametrize("dtype,d,Hq,Hk", HEADS)
@pytest.mark.parametrize("page,window", [(16, 0), (64, 0), (32, 33), (128, 1)])
def test_decode(P, dtype, d, Hq, Hk, page, window):
    """One token a sequence, caches of 1 to several hundred keys, ends inside tiles and pages."""
    kv = [1, 2, 15, 16, 17, 63, 64, 65, 127, 130, 511]
    c = Case([1] * len(kv), kv, Hq, Hk, d, page, dtype, window, seed=d + page)
    say("decode", dtype, d, Hq, Hk, page, window)
    check(c, *call(P, c, dense=True))


@pytest.mark.parametrize("dtype,d,Hq,Hk", HEADS)
@pytest.mark.parametrize("window", [0, 1, 20, 200])
def test_chunks(P, dtype, d, Hq, Hk, window):
    """Packed chunks of 0 to a few hundred tokens over prefixes of any length, both kernels in
    one call."""
    new, old = [5, 0, 1, 70, 33, 0, 16, 129, 2], [0, 40, 100, 0, 31, 0, 300, 65, 1]
    kv = [a + b for a, b in zip(new, old)]
    c = Case(new, kv, Hq, Hk, d, 32, dtype, window, seed=d + window)
    say("chunks", dtype, d, Hq, Hk, window)
    check(c, *call(P, c))


@pytest.mark.parametrize("dtype,d,Hq,Hk", HEADS)
def test_split_keys(P, dtype, d, Hq, Hk):
    """Few sequences with long caches: the keys are split over workgroups."""
    for new, old in (([1], [2999]), ([3, 1], [1800, 700]), ([40], [2500])):
        c = Case(new, [a + b for a, b in zip(new, old)], Hq, Hk, d, 64, dtype, seed=7)
        say("split", dtype, d, new, old)
        check(c, *call(P, c))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_not_causal(P, dtype):
    new, kv = [7, 1, 90], [200, 64, 33]
    c = Case(new, kv, 8, 2, 128, 16, dtype, causal=False, seed=3)
    check(c, *call(P, c))


@pytest.mark.parametrize("dtype,d", [(BF, 128), (F32, 64)])
@pytest.mark.parametrize("new,kv", [([1, 4, 60], [0, 0, 0]),       # nothing cached
                                    ([5, 80], [2, 33])])           # more tokens than cached ones
def test_rows_without_keys(P, dtype, d, new, kv):
    c = Case(new, kv, 4, 2, d, 16, dtype, seed=5)
    o, lse = call(P, c, max_kv=64)
    check(c, o, lse)
    assert (o[0] == 0).all() and (lse[0] == -math.inf).all()


@pytest.mark.parametrize("dtype,d", [(BF, 64), (BF, 256), (F32, 128)])
def test_holes(P, dtype, d):
    """Blocks without a page anywhere, whole windows of them, and table entries out of range."""
    new, kv = [1, 3, 50], [100, 70, 150]
    holes = {(0, 0), (0, 6), (1, 2), (2, 1), (2, 4), (2, 9)}
    for window in (0, 18):
        c = Case(new, kv, 4, 2, d, 16, dtype, window, holes=holes, seed=9)
        c.table[0, 6] = c.k_pages.shape[0]  # one past the last page
        o, lse = call(P, c)
        c.table[0, 6] = -1
        check(c, o, lse)


def test_only_holes(P):
    c = Case([1, 40], [64, 64], 4, 4, 128, 64, BF, holes={(0, 0), (1, 0)}, seed=1)
    o, lse = call(P, c)
    assert (o == 0).all() and (lse == -math.inf).all()


@pytest.mark.parametrize("dtype,d,Hq,Hk", HEADS)
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
def test_later_tokens_do_not_reach_earlier_ones(P, dtype, d, Hq, Hk, value):
    """A non-finite k or v of a token: the rows before it (and, in a window, those far behind it)
    are what they are without it; with it in v, rows that see it are not finite in that channel."""
    for new, old in (([6], [30]), ([100], [20])):
        c = Case(new, [new[0] + old[0]], Hq, Hk, d, 16, dtype, window=40, seed=11)
        at = old[0] + 3  # position of the token, new token 3
        p, s = int(c.table[0, at // 16]), at % 16
        ro, rl, rel, mass = c.attend()
        c.v_pages[p, :, s, 5] = value
        o, lse = call(P, c)
        sees = torch.tensor([at in c.visible(0, i) for i in range(new[0])])
        assert sees.any() and not sees.all()
        ok = (o.double() - ro).abs() <= c.bound(rel, mass)
        assert ok[~sees].all()
        ok[:, :, 5] = True
        assert ok[sees].all()
        assert not torch.isfinite(o[sees][:, :, 5].float()).any()
        c.k_pages[p, :, s, 2] = math.nan
        o, lse = call(P, c)
        assert ((o.double() - ro).abs() <= c.bound(rel, mass))[~sees].all()
        assert torch.isnan(o[sees].float()).all()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_strides(P, dtype):
    """q and o as slices of wider rows, a cache with its tokens' heads side by side, and k and v
    of several layers in one allocation."""
    c = Case([3, 60, 1], [50, 90, 200], 4, 2, 128, 16, dtype, seed=13)
    ro, rl, rel, mass = c.attend()
    T = c.q.shape[0]
    wide = torch.full((1, T, 9, 128), math.nan, dtype=dtype, device="cuda")
    wide[0, :, 2:6] = c.q.cuda()
    out = torch.full((1, T, 7, 128), -1.0, dtype=dtype, device="cuda")
    pool = torch.full((2, 2, c.k_pages.shape[0], 16, 2, 128), math.nan, dtype=dtype, device="cuda")
    pool[1, 0] = c.k_pages.cuda().transpose(1, 2)
    pool[1, 1] = c.v_pages.cuda().transpose(1, 2)
    P.gdn_cache_attn(wide[:, :, 2:6], pool[1, 0].transpose(1, 2), pool[1, 1].transpose(1, 2),
                     c.table.cuda(), c.kv_lens.cuda(), cu_seqlens=c.cu.cuda(),
                     cu_seqlens_host=c.cu, o=out[:, :, 1:5])
    o = out[0].cpu()
    assert ((o[:, 1:5].double() - ro).abs() <= c.bound(rel, mass)).all()
    assert (o[:, [0, 5, 6]] == -1).all()


def test_lengths_bound_costs_time_not_results(P):
    """max_kv below the lengths, above them, and left out; lengths past the table's room."""
    c = Case([1, 40], [700, 500], 4, 1, 128, 16, BF, seed=15)
    for max_kv in (1, 64, 700, 100000, 0):
        check(c, *call(P, c, max_kv=max_kv))
    c.table = c.table[:, :44].contiguous()  # room for 704 tokens
    c.kv_lens[0] = 9000
    o, lse = call(P, c)
    c.kv[0], c.kv_lens[0] = 704, 704
    # slots 700..703 are visible then; they hold NaN
    assert torch.isnan(o[0].float()).all()
    c.kv_lens[0] = -5
    o, lse = call(P, c)
    assert (o[0] == 0).all() and (lse[0] == -math.inf).all()


@pytest.mark.parametrize("dtype,scale", [(BF, 0.03), (BF, 2.0), (F32, 1.0), (F32, 8.0)])
def test_scale_and_extreme_scores(P, dtype, scale):
    """Scores far apart: the softmax is all but one key's, sums span the range of exp."""
    c = Case([1, 5, 50], [300, 200, 100], 4, 2, 64, 16, dtype, seed=17, std=3.0)
    check(c, *call(P, c, scale=scale), scale=scale)


def test_offsets_past_32_bits(P):
    """A pool of more than 2^32 bytes whose pages lie at its end."""
    Hk, d, page = 2, 256, 64
    num = (1 << 32) // (Hk * d * page * 2) + 40
    c = Case([1, 30], [300, 170], 4, Hk, d, page, BF, seed=19)
    n = c.k_pages.shape[0]
    kp = torch.empty(num, Hk, page, d, dtype=BF, device="cuda")
    vp = torch.empty(num, Hk, page, d, dtype=BF, device="cuda")
    kp[num - n:] = c.k_pages.cuda()
    vp[num - n:] = c.v_pages.cuda()
    table = torch.where(c.table >= 0, c.table + num - n, -1).to(torch.int32)
    o = P.gdn_cache_attn(c.q.cuda()[None], kp, vp, table.cuda(), c.kv_lens.cuda(),
                         cu_seqlens=c.cu.cuda(), cu_seqlens_host=c.cu)
    ro, rl, rel, mass = c.attend()
    assert ((o[0].cpu().double() - ro).abs() <= c.bound(rel, mass)).all()


def test_same_bits_and_streams(P):
    """Twice the same bits, on another stream too, with the workspace handed in."""
    c = Case([1, 2, 64], [2000, 900, 300], 8, 2, 128, 64, BF, seed=21)
    o1, l1 = call(P, c)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        q, cu = c.q.cuda()[None], c.cu.cuda()
        table = c.table.cuda()
        need = P.gdn_cache_attn_workspace_size(q, c.k_pages.cuda(), table, max_kv=2000,
                                               cu_seqlens=cu, cu_seqlens_host=c.cu)
        assert need > 0
        ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
        o2, l2 = call(P, c, workspace=ws)
    assert torch.equal(o1, o2) and torch.equal(l1, l2)


def test_graph(P):
    """A decode step captured once and replayed on new tokens and lengths."""
    c = Case([1] * 5, [40, 800, 3, 129, 500], 8, 2, 128, 16, BF, seed=23)
    q, kp, vp = c.q.cuda()[:, None], c.k_pages.cuda(), c.v_pages.cuda()
    table, lens = c.table.cuda(), c.kv_lens.cuda()
    o = torch.zeros_like(q)
    kw = dict(max_kv=1000)
    ws = torch.empty(P.gdn_cache_attn_workspace_size(q, kp, table, **kw), dtype=torch.uint8,
                     device="cuda")
    P.gdn_cache_attn(q, kp, vp, table, lens, o=o, workspace=ws, **kw)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        P.gdn_cache_attn(q, kp, vp, table, lens, o=o, workspace=ws, **kw)
    for step in range(4):
        q.copy_(torch.randn(q.shape, device="cuda"))
        lens.copy_(torch.tensor([40 - step, 800, 3, 129 - step, 400 + 20 * step]))
        want = P.gdn_cache_attn(q, kp, vp, table, lens, **kw)
        torch.cuda.synchronize()
        o.fill_(0)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, want), step
