"""Attention over the paged cache: batches of many row blocks, drawn problems and the binding's
own checks, against 64 bits."""
import math
import random

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


def plain(c):
    """Case.attend with a sequence's tokens together, in 64 bits on the GPU: (o, lse, rel, mass)."""
    G, d = c.Hq // c.Hk, c.d
    o = torch.zeros(c.q.shape, dtype=torch.float64, device="cuda")
    mass, row = torch.zeros_like(o), 0
    lse = torch.full(c.q.shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    rel = torch.zeros_like(lse)
    for n, (m, kv) in enumerate(zip(c.new, c.kv)):
        if m and kv:
            j = torch.arange(kv)
            page = c.table[n].long()[j // c.page]
            there = (page >= 0).cuda()
            at = page.clamp(min=0), j % c.page
            # [Hq, keys, d]; a hole's slots hold anything
            k, v = (torch.where(there[:, None, None], x[at[0], :, at[1]].cuda().double(), 0.0)
                    .nan_to_num(0.0, 0.0, 0.0)
                    .repeat_interleave(G, 1).transpose(0, 1).contiguous()
                    for x in (c.k_pages, c.v_pages))
            q = c.q[row:row + m].cuda().double().transpose(0, 1).contiguous()
            pos = torch.arange(kv - m, kv, device="cuda")[:, None]
            key = torch.arange(kv, device="cuda")[None]
            sees = (key <= pos if c.causal else key < kv) & there
            if c.window:
                sees = sees & (key > pos - c.window)
            kt = k.transpose(1, 2).contiguous()
            x = torch.where(sees, torch.matmul(q, kt) * d ** -0.5, -math.inf)
            big = torch.where(sees, torch.matmul(q.abs(), kt.abs()) * d ** -0.5, 0.0).amax(-1)
            some = sees.any(-1)
            w = torch.where(some[:, None], torch.softmax(x, -1), 0.0)
            sl = slice(row, row + m)
            o[sl] = torch.matmul(w, v).transpose(0, 1)
            mass[sl] = torch.matmul(w, v.abs()).transpose(0, 1)
            lse[sl] = torch.logsumexp(x, -1).T
            rel[sl] = torch.where(some, 2 * (d + 8) * 2.0 ** -24 * (big + 1)
                                  + (sees.sum(-1) + 16) * 2.0 ** -24, 0.0).T
        row += m
    return o.cpu(), lse.cpu(), rel.cpu(), mass.cpu()


def run(P, c, **kw):
    q = c.q.cuda()[None]
    lse = torch.full(q.shape[:3], math.nan, device="cuda")
    o = torch.full_like(q, math.nan)
    args = dict(cu_seqlens=c.cu.cuda(), cu_seqlens_host=c.cu, max_kv=max(c.kv), **kw)
    P.gdn_cache_attn(q, c.k_pages.cuda(), c.v_pages.cuda(), c.table.cuda(), c.kv_lens.cuda(),
                     causal=c.causal, window=c.window, o=o, lse=lse, **args)
    torch.cuda.synchronize()
    return o[0].cpu(), lse[0].cpu()


def check(c, o, lse):
    ro, rl, rel, mass = plain(c)
    bad = ~((o.double() - ro).abs() <= c.bound(rel, mass))
    assert not bad.any(), (int(bad.sum()), torch.nonzero(bad)[:3])
    empty = rl == -math.inf
    assert (lse[empty] == -math.inf).all()
    tol = rel[~empty] + rl[~empty].abs() * 2.0 ** -22 + 2.0 ** -20
    assert ((lse[~empty].double() - rl[~empty]).abs() <= tol).all()


def test_the_two_references_agree():
    """The vectorised reference is the token-by-token one."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    c = Case([3, 0, 20, 1], [40, 9, 15, 64], 4, 2, 64, 16, F32, 7, holes={(0, 1), (3, 3)}, seed=4)
    for x, y in zip(plain(c), c.attend()):
        assert torch.allclose(x, y, rtol=1e-12, atol=1e-14)


@pytest.mark.parametrize("dtype,d,Hq,Hk", [(BF, 128, 64, 32), (BF, 256, 36, 18), (BF, 64, 64, 64),
                                           (F32, 64, 32, 32), (F32, 256, 24, 24)])
@pytest.mark.parametrize("N,window", [(2, 0), (17, 0), (17, 50), (64, 100), (65, 0)])
def test_many_blocks(P, dtype, d, Hq, Hk, N, window):
    """More row blocks than run at once: sequences of very different lengths, some without new
    tokens, one whose cache holds fewer tokens than it is said to add."""
    rng = random.Random(N + d)
    most = 700 if N == 2 else 150
    new = [rng.choice([0, 1, rng.randint(2, most)]) for _ in range(N)]
    new[0], new[-1] = most, most - 13
    kv = [m + rng.choice([0, 3, rng.randint(0, 400)]) for m in new]
    kv[N // 2] = new[N // 2] // 2
    kv[0] = new[0]
    c = Case(new, kv, Hq, Hk, d, 32, dtype, window, seed=N + d)
    say("many blocks", dtype, d, Hq, Hk, N, window)
    check(c, *run(P, c))


@pytest.mark.parametrize("seed", range(24))
def test_drawn(P, seed):
    """Problems drawn over the whole range: a long cache beside short ones, chunks beside single
    tokens, holes, windows, both kinds of rows."""
    rng = random.Random(100 + seed)
    dtype, d = rng.choice([BF, BF, F32]), rng.choice([64, 128, 256])
    Hk = rng.choice([1, 2, 3, 8])
    Hq = Hk * rng.choice([1, 2, 3, 4, 8])
    N = rng.choice([1, 2, 5, 20])
    page = rng.choice([16, 32, 64, 128])
    new = [rng.choice([0, 1, 1, rng.randint(1, 9), rng.randint(10, 300)]) for _ in range(N)]
    new[rng.randrange(N)] = rng.choice([1, 4, 77, 301])
    kv = [m + rng.choice([0, 1, rng.randint(0, 60), rng.randint(0, 800)]) for m in new]
    kv[rng.randrange(N)] += rng.choice([0, 3000])
    causal = rng.random() < 0.8
    window = rng.choice([0, 0, 1, 17, 129, 1000]) if causal else 0
    holes = {(n, b) for n in range(N) for b in range(-(-kv[n] // page)) if rng.random() < 0.05}
    c = Case(new, kv, Hq, Hk, d, page, dtype, window, causal, holes, seed=seed)
    say("drawn", seed, dtype, d, Hq, Hk, page, window, causal, new, kv)
    check(c, *run(P, c))


def test_boundaries_of_other_types(P):
    """64-bit boundaries, and boundaries without a host copy, give the same bits."""
    c = Case([5, 0, 70], [50, 3, 70], 8, 2, 128, 16, BF, seed=2)
    want, _ = run(P, c)
    args = [x.cuda() for x in (c.q[None], c.k_pages, c.v_pages, c.table, c.kv_lens)]
    for cu, host in ((c.cu.cuda(), None), (c.cu.long().cuda(), None),
                     (c.cu.long().cuda(), c.cu.long())):
        o = P.gdn_cache_attn(*args, max_kv=70, cu_seqlens=cu, cu_seqlens_host=host)
        torch.cuda.synchronize()
        assert torch.equal(o[0].cpu(), want)


def test_binding_refusals(P):
    """Tensors of other types, shapes, devices and strides are refused before anything runs."""
    c = Case([2], [20], 4, 2, 64, 16, BF, seed=3)
    good = dict(q=c.q[None].cuda(), k_pages=c.k_pages.cuda(), v_pages=c.v_pages.cuda(),
                table=c.table.cuda(), kv_lens=c.kv_lens.cuda())
    P.gdn_cache_attn(**good)
    q = good["q"]
    for bad in (dict(q=q.float()), dict(q=q[0]), dict(q=q.cpu()), dict(q=q[..., ::2]),
                dict(k_pages=good["k_pages"].float()), dict(k_pages=c.k_pages),
                dict(v_pages=good["v_pages"][:-1]), dict(v_pages=good["v_pages"][:, :1]),
                dict(table=good["table"].long()), dict(table=c.table), dict(table=good["table"][0]),
                dict(kv_lens=good["kv_lens"].long()), dict(kv_lens=good["kv_lens"][:0]),
                dict(o=torch.empty_like(q, dtype=F32)), dict(o=q[:, :1].clone()),
                dict(lse=torch.empty(1, 2, 3, device="cuda")), dict(lse=torch.empty(1, 2, 4)),
                dict(scale=0.0), dict(scale=math.nan), dict(window=-1),
                dict(window=4, causal=False), dict(max_kv=-1),
                dict(cu_seqlens_host=c.cu)):
        with pytest.raises((ValueError, TypeError, RuntimeError)):
            P.gdn_cache_attn(**{**good, **bad})
    k = torch.zeros(1, 2, 2, 64, dtype=BF, device="cuda")
    r = P.gdn_rotary(64)
    ok = dict(q=q, k=k, v=k, k_pages=good["k_pages"], v_pages=good["v_pages"],
              table=good["table"], kv_lens=good["kv_lens"], rotary=r)
    for bad in (dict(k=k.float()), dict(v=k[:, :1]), dict(v=k.cpu()), dict(k=k[:, :, :1]),
                dict(rotary=r.turns), dict(rotary=r._replace(turns=r.turns.float())),
                dict(rotary=r._replace(turns=r.turns.cpu())), dict(rotary=r._replace(layout="both")),
                dict(table=c.table), dict(q=q[:, :1])):
        with pytest.raises((ValueError, TypeError, RuntimeError)):
            P.gdn_cache_append(**{**ok, **bad})
    for bad in (dict(positions=torch.zeros(1, 2, device="cuda")),
                dict(positions=torch.zeros(2, 1, dtype=torch.int32, device="cuda")),
                dict(positions=torch.zeros(1, 2, dtype=torch.int32)),
                dict(q_out=torch.empty_like(q)[:, :1]), dict(k_out=k.float())):
        with pytest.raises((ValueError, TypeError, RuntimeError)):
            P.gdn_rotary_fwd(q, k, r, **bad)


@pytest.mark.parametrize("new,kv", [([40, 3], [25, 90]), ([200], [150])])
def test_widest_window(P, new, kv):
    """A window that no cache reaches is no window, also for tokens before the cache's first."""
    c = Case(new, kv, 4, 2, 128, 16, BF, 0, seed=5)
    want, lse = run(P, c)
    check(c, want, lse)
    c.window = 2 ** 31 - 1
    got, again = run(P, c)
    check(c, got, again)
