"""Attention over a prefix that all sequences share, against its definition in 64 bits (the cache
of gdn_cache_attn whose first pages are the prefix's): types, head layouts, rows from one to many
blocks, prefixes that end anywhere, windows, holes, infinities, short sequences, graphs."""
import math

import pytest
import torch

from tests.paged_ref import F64, Case

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float32]


@pytest.fixture(scope="module")
def P():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2412_06464_amd import paged
    paged.load_library()
    return paged


class Shared(Case):
    """A Case whose sequences begin with the same prefix: their rows of the table name the prefix's
    pages, so that Case.attend gives the result; `own` is the table that the call gets, with
    other entries there."""

    def __init__(self, new, kv, prefix, Hq, Hk, d, page, dtype, window=0, causal=True, holes=(),
                 seed=0, bad=-7):
        super().__init__(new, kv, Hq, Hk, d, page, dtype, 0, causal, [], seed)
        self.window, self.prefix = window, prefix
        gen = torch.Generator().manual_seed(seed + 1)
        blocks, full = -(-prefix // page), prefix // page
        lead = torch.arange(blocks) + self.k_pages.shape[0]
        more = [torch.randn(blocks, Hk, page, d, generator=gen).to(dtype) for _ in range(2)]
        self.k_pages, self.v_pages = (torch.cat([x, y]) for x, y in
                                      zip((self.k_pages, self.v_pages), more))
        width = max(self.table.shape[1], blocks)
        self.table = torch.cat([self.table, torch.full((len(new), width - self.table.shape[1]), -1)], 1)
        self.own = self.table.to(torch.int32).clone()
        self.lead = lead.to(torch.int32)
        self.lead[list(holes)] = -1
        # what the definition sees: the prefix's pages in place of the full blocks, and in the block
        # that it ends in its slots
        for n, c in enumerate(kv):
            self.table[n, :full] = self.lead[:full]
            self.own[n, :full] = bad
            if prefix % page:
                p = int(self.own[n, full])
                if p >= 0 and int(self.lead[full]) >= 0:
                    cut = prefix % page
                    for x, y in zip((self.k_pages, self.v_pages), more):
                        x[p, :, :cut] = float("nan")  # the call does not look there
                elif p < 0 and c > full * page:
                    self.table[n, full] = self.lead[full]
        self.more = more

    def visible(self, n, i):
        pos = self.kv[n] - self.new[n] + i
        hi = min(self.kv[n], pos + 1) if self.causal else self.kv[n]
        lo = max(0, pos - self.window + 1) if self.window else 0
        t = self.lead, self.own[n]
        return [j for j in range(lo, hi)
                if 0 <= t[j >= self.prefix][j // self.page] < self.k_pages.shape[0]]

    def attend(self, scale=None):
        """Case.attend, keys from both tables."""
        scale = self.d ** -0.5 if scale is None else scale
        G = self.Hq // self.Hk
        o = torch.zeros(self.q.shape, dtype=F64)
        lse = torch.full(self.q.shape[:2], -math.inf, dtype=F64)
        mass, rel = torch.zeros(self.q.shape, dtype=F64), torch.zeros(self.q.shape[:2], dtype=F64)
        row = 0
        for n, m in enumerate(self.new):
            for i in range(m):
                j = torch.tensor(self.visible(n, i), dtype=torch.long)
                if len(j):
                    block = j // self.page
                    p = torch.where(j < self.prefix, self.lead.long()[block.clamp(max=len(self.lead) - 1)],
                                    self.own[n].long()[block])
                    s = j % self.page
                    k = self.k_pages[p, :, s].to(F64).repeat_interleave(G, 1)
                    v = self.v_pages[p, :, s].to(F64).repeat_interleave(G, 1)
                    q = self.q[row].to(F64)
                    x = (q * k).sum(-1) * scale
                    lse[row] = torch.logsumexp(x, 0)
                    w = torch.softmax(x, 0)
                    o[row] = (w[..., None] * v).sum(0)
                    mass[row] = (w[..., None] * v.abs()).sum(0)
                    big = ((q * k).abs().sum(-1) * scale).amax(0)
                    rel[row] = 2 * (self.d + 8) * 2.0 ** -24 * (big + 1) + (len(j) + 16) * 2.0 ** -24
                row += 1
        return o, lse, rel, mass

    def call(self, P, dense=False, **kw):
        q = self.q.reshape(len(self.new), -1, self.Hq, self.d) if dense else self.q[None]
        cu = {} if dense else dict(cu_seqlens=self.cu.cuda(), cu_seqlens_host=self.cu)
        q = q.cuda()
        lse = torch.empty(q.shape[:3], device="cuda")
        o = P.gdn_cache_attn_shared(q, self.k_pages.cuda(), self.v_pages.cuda(), self.own.cuda(),
                                    self.kv_lens.cuda(), self.lead.cuda(), self.prefix,
                                    causal=self.causal, window=self.window, lse=lse, **cu, **kw)
        return o.reshape(self.q.shape).cpu(), lse.reshape(self.q.shape[:2]).cpu()

    def check(self, got):
        o, lse, rel, mass = self.attend()
        err = (got[0].to(F64) - o).abs()
        bound = self.bound(rel, mass)
        assert (err <= bound).all(), float((err / bound).max())
        seen = lse > -math.inf
        assert torch.equal(seen, got[1] > -math.inf)
        # the sum's relative error, its logarithm's rounding and that of the maximum beside it
        slack = rel + 4 * 2.0 ** -24 * (1 + lse.abs().nan_to_num(posinf=0))
        assert ((got[1].to(F64) - lse).abs()[seen] <= slack[seen]).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("Hq,Hk", [(4, 4), (4, 1), (6, 2)])
def test_heads(P, dtype, d, Hq, Hk):
    """One token a sequence (few rows), several (a block), many (blocks)."""
    for new, kv in (([1, 1, 1], [150, 131, 140]), ([1, 7, 3, 0], [150, 135, 133, 140]),
                    ([40, 1, 60], [190, 131, 200])):
        c = Shared(new, kv, 130, Hq, Hk, d, 16, dtype, seed=d + Hq)
        c.check(c.call(P))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("prefix", [1, 15, 16, 17, 63, 64, 100, 128, 400])
@pytest.mark.parametrize("page", [16, 64])
def test_prefixes(P, dtype, prefix, page):
    """Ends inside a page, a tile, a group of 16; prefixes of one token; new tokens right behind."""
    new = [1, 5, 20, 1]
    kv = [prefix + n + x for n, x in zip(new, (0, 3, 40, 90))]
    c = Shared(new, kv, prefix, 4, 2, 64, page, dtype, seed=prefix)
    c.check(c.call(P))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("window", [1, 8, 50, 130, 1000])
def test_windows(P, dtype, window):
    """Windows that leave the prefix, that reach into it from some sequences, that hold all of it."""
    c = Shared([1, 9, 30, 1, 1], [205, 300, 231, 201, 460], 200, 4, 2, 64, 16, dtype, window=window,
               seed=window)
    c.check(c.call(P))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("causal", [True, False])
def test_short_sequences(P, dtype, causal):
    """Sequences that hold less than the prefix, or nothing, or end with it: they see what they hold."""
    c = Shared([1, 5, 1, 4, 40], [20, 5, 100, 98, 70], 100, 4, 2, 64, 16, dtype, causal=causal, seed=3)
    c.check(c.call(P))
    c.kv[0], c.kv_lens[0] = 0, 0
    o, lse = c.call(P)
    assert not o[0].any() and (lse[0] == -math.inf).all()
    c.check((o, lse))


@pytest.mark.parametrize("dtype", DTYPES)
def test_holes_and_bad_pages(P, dtype):
    """Blocks of the prefix that are not there; free entries of either kind in the own table."""
    for bad in (-1, -2 ** 31, 2 ** 31 - 1):
        c = Shared([1, 20, 1], [210, 240, 220], 200, 4, 2, 64, 16, dtype, holes=[0, 3, 4, 12], seed=4,
                   bad=bad)
        c.own[1, 13] = bad
        c.check(c.call(P))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("new", [[1, 1], [30, 12]])
@pytest.mark.parametrize("odd", [math.inf, -math.inf, math.nan])
def test_odd_values(P, dtype, new, odd):
    """An infinity or NaN in a v of the prefix reaches the rows that see it and no others."""
    kv = [30 + n for n in new]
    kv[1] = 14 + new[1]
    c = Shared(new, kv, 30, 4, 2, 64, 16, dtype, seed=5)
    clean = c.attend()
    at = 20  # sequence 1 sees it from its token 6 on, if it has that many
    page, slot = int(c.lead[at // 16]), at % 16
    c.v_pages[page, 1, slot, 9] = odd
    o, _ = c.call(P)
    hit = torch.zeros(c.q.shape, dtype=torch.bool)
    row = 0
    for n, m in enumerate(new):
        for i in range(m):
            hit[row, 2:, 9] = at in c.visible(n, i)
            row += 1
    bound = c.bound(clean[2], clean[3])
    assert ((o.to(F64) - clean[0]).abs() <= bound)[~hit].all()
    assert not torch.isfinite(o[hit].float()).any()
    if odd == odd and hit.any():
        assert (o[hit].float() == odd).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T", [1, 3])
def test_dense_and_split(P, dtype, T):
    """Dense rows; a prefix long enough to be split over many workgroups."""
    c = Shared([T] * 9, [2100 + T + i for i in range(9)], 2100, 8, 2, 64, 64, dtype, seed=6)
    c.check(c.call(P, dense=True))


def test_as_the_plain_call(P):
    """The same keys through gdn_cache_attn, whose own sums differ in their order alone."""
    c = Shared([1] * 70, [330 + i for i in range(70)], 320, 8, 2, 128, 32, torch.float32, seed=7)
    o, lse = c.call(P)
    table = c.own.clone()
    table[:, :10] = c.lead
    q, cu = c.q[None].cuda(), dict(cu_seqlens=c.cu.cuda(), cu_seqlens_host=c.cu)
    l2 = torch.empty(q.shape[:3], device="cuda")
    o2 = P.gdn_cache_attn(q, c.k_pages.cuda(), c.v_pages.cuda(), table.cuda(), c.kv_lens.cuda(),
                          lse=l2, **cu)
    _, _, rel, mass = c.attend()
    assert ((o - o2[0].cpu()).abs().to(F64) <= 2 * c.bound(rel, mass)).all()
    assert torch.equal(P.gdn_cache_attn_shared(q, c.k_pages.cuda(), c.v_pages.cuda(), table.cuda(),
                                               c.kv_lens.cuda(), c.lead.cuda(), 0, **cu), o2)


def test_skipped_and_replayed(P):
    """In a graph, with sequences left out and lengths that grow between replays; rows behind the
    last sequence stay as they were."""
    c = Shared([1, 2, 1, 30], [110, 120, 130, 140], 96, 4, 2, 64, 16, torch.float32, seed=8)
    cu = c.cu.cuda()
    q = torch.cat([c.q, torch.randn(6, 4, 64)])[None].cuda()
    host = c.cu.clone()
    host[-1] = 40
    skip = torch.zeros(4, dtype=torch.int32, device="cuda")
    lens = c.kv_lens.cuda()
    o, lse = torch.empty_like(q), torch.empty(q.shape[:3], device="cuda")
    kw = dict(o=o, lse=lse, skip=skip, cu_seqlens=cu, cu_seqlens_host=host, max_kv=200)
    args = (q, c.k_pages.cuda(), c.v_pages.cuda(), c.own.cuda(), lens, c.lead.cuda(), 96)
    kw["workspace"] = torch.empty(P.gdn_cache_attn_shared_workspace_size(
        q, args[1], args[3], 96, max_kv=200, cu_seqlens=cu, cu_seqlens_host=host), dtype=torch.uint8,
        device="cuda")
    P.gdn_cache_attn_shared(*args, **kw)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.gdn_cache_attn_shared(*args, **kw)
    for step in range(4):
        c.kv = [x + (step > 0) * (n != 3) for n, x in enumerate(c.kv)]
        c.kv[3] = 140 - step
        c.kv_lens = torch.tensor(c.kv, dtype=torch.int32)
        for n in range(4):  # pages for the tokens that came
            for b in range(6, -(-c.kv[n] // 16)):
                if c.own[n, b] < 0:
                    c.own[n, b] = 0
        c.k_pages, c.v_pages = (x.nan_to_num(0.5) for x in (c.k_pages, c.v_pages))
        args[1].copy_(c.k_pages), args[2].copy_(c.v_pages), args[3].copy_(c.own)
        lens.copy_(c.kv_lens)
        skip[2] = step % 2
        o.fill_(7), lse.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        full = list(c.kv)
        if step % 2:
            c.kv[2] = 0
        c.check((o[0, :34].cpu(), lse[0, :34].cpu()))
        c.kv = full
        assert (o[0, 34:] == 7).all() and (lse[0, 34:] == 7).all()


def test_same_bits(P):
    c = Shared([1, 40, 1], [500, 600, 700], 450, 4, 1, 128, 16, torch.bfloat16, seed=9)
    first = c.call(P)
    for _ in range(3):
        assert all(torch.equal(x, y) for x, y in zip(first, c.call(P)))
