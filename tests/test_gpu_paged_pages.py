"""Management of the pages against a plain sequential model; whole numbers, exact."""
import random

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2412_06464_amd import paged
    paged.load_library()
    return paged


def blocks(n, page):
    return -(-n // page)


class Model:
    """The book as Python lists, and its rules one page at a time."""

    def __init__(self, S, width, num, page, seed, fill=0.5, shared=0.3):
        rng = random.Random(seed)
        self.S, self.width, self.num, self.page = S, width, num, page
        free = list(range(num))
        rng.shuffle(free)
        self.table, self.lens, self.refs = [], [], [0] * num
        for s in range(S):
            n, row = rng.randint(0, int(width * page * fill)), []
            if s and rng.random() < shared:
                o = rng.randrange(s)
                row = self.table[o][:min(self.lens[o], n) // page]
            while len(row) < blocks(n, page) and free:
                row = row + [free.pop()]
            n = min(n, len(row) * page)
            row = row[:blocks(n, page)]
            for p in row:
                self.refs[p] += 1
            self.table.append(row)
            self.lens.append(n)

    def tensors(self):
        pad = [r + [-1] * (self.width - len(r)) for r in self.table]
        return [torch.tensor(x, dtype=torch.int32).cuda() for x in (pad, self.lens, self.refs)]

    def free(self):
        return [p for p in range(self.num) if self.refs[p] <= 0]

    def extend(self, add):
        free, short, left, stop = self.free(), [], 0, False
        left = len(free)
        for s in range(self.S):
            n = self.lens[s] + max(0, add[s])
            need = blocks(n, self.page) - len(self.table[s])
            if blocks(n, self.page) > self.width:
                short.append(need)
                continue
            stop = stop or need > left
            if stop and need > 0:
                short.append(need)
                continue
            new = [free.pop(0) for _ in range(need)]
            left -= need
            for p in new:
                self.refs[p] = 1
            self.table[s] = self.table[s] + new
            self.lens[s] = n
            short.append(0)
        return short

    def select(self, parents):
        """Returns short and the copies (src, dst)."""
        free, heirs, copies, short = self.free(), {}, [], []
        table, lens, refs = [], [], list(self.refs)
        for row in self.table:
            for p in row:
                refs[p] -= 1
        for i, p in enumerate(parents):
            row, n, s = [], 0, 0
            if 0 <= p < self.S:
                row, n = list(self.table[p]), self.lens[p]
                if n % self.page and heirs.setdefault(p, i) != i:
                    if free:
                        copies.append((row[-1], free[0]))
                        row[-1] = free.pop(0)
                    else:
                        row, n, s = [], 0, 1
            for x in row:
                refs[x] += 1
            table.append(row)
            lens.append(n)
            short.append(s)
        self.table, self.lens, self.refs = table, lens, refs
        return short, copies

    def compact(self):
        live = [p for p in range(self.num) if self.refs[p] > 0]
        holes = [p for p in range(len(live)) if self.refs[p] <= 0]
        to = {p: p for p in live if p < len(live)}
        moves = list(zip([p for p in live if p >= len(live)], holes))
        to.update(moves)
        self.table = [[to[p] for p in r] for r in self.table]
        refs = [0] * self.num
        for p in live:
            refs[to[p]] = self.refs[p]
        self.refs = refs
        return [to.get(p, -1) for p in range(self.num)], moves


def same(m, got, lens=None):
    table, ln, refs = m.tensors()
    used = torch.tensor([[j < len(r) for j in range(m.width)] for r in m.table]).cuda()
    assert torch.equal(got["table"][used], table[used])
    assert torch.equal(got["refs"], refs)
    assert torch.equal(got["lens"] if lens is None else lens, ln)


SIZES = [(1, 3, 2, 16), (5, 9, 40, 16), (64, 20, 900, 32), (300, 6, 700, 64), (1500, 3, 2600, 16),
         (40, 300, 20000, 16)]


@pytest.mark.parametrize("S,width,num,page", SIZES)
@pytest.mark.parametrize("in_place", [False, True])
def test_extend(P, S, width, num, page, in_place):
    for seed, most in ((0, 1), (1, page), (2, 3 * page), (3, width * page)):
        m = Model(S, width, num, page, seed)
        rng = random.Random(seed + 50)
        add = [rng.choice([0, 1, rng.randint(-3, most)]) for _ in range(S)]
        t, ln, r = m.tensors()
        before = t.clone()
        out = dict(table=t, lens=ln, refs=r) if in_place else None
        got = P.gdn_pages_extend(t, ln, r, torch.tensor(add, dtype=torch.int32).cuda(), page,
                                 out=out)
        assert in_place or torch.equal(t, before)
        short = m.extend(add)
        assert got["short"].tolist() == short
        same(m, got)


def test_extend_without_free_pages(P):
    m = Model(30, 8, 200, 16, 5)
    for p in range(200):
        m.refs[p] = max(m.refs[p], 1)  # held by someone outside the table
    add = [0 if s % 3 else 16 for s in range(30)]
    got = P.gdn_pages_extend(*m.tensors(), torch.tensor(add, dtype=torch.int32).cuda(), 16)
    assert got["short"].tolist() == m.extend(add)
    same(m, got)


@pytest.mark.parametrize("S,width,num,page", SIZES)
@pytest.mark.parametrize("in_place", [False, True])
def test_select(P, S, width, num, page, in_place):
    for seed, kind in ((0, "any"), (1, "one"), (2, "keep"), (3, "end"), (4, "any")):
        m = Model(S, width, num, page, seed, fill=0.9 if seed == 4 else 0.4)
        rng = random.Random(seed + 70)
        parents = {"any": [rng.randint(-2, S + 1) for _ in range(S)], "one": [S // 2] * S,
                   "keep": list(range(S)), "end": [-1] * S}[kind]
        t, ln, r = m.tensors()
        pool = torch.randint(0, 1 << 30, (3, num, 2, 12), dtype=torch.int32, device="cuda")
        want = pool.clone()
        out = dict(table=t, lens=ln, refs=r) if in_place else None
        got = P.gdn_pages_select(t, ln, r, torch.tensor(parents, dtype=torch.int32).cuda(), page,
                                 pool=pool, out=out)
        short, copies = m.select(parents)
        assert got["short"].tolist() == short
        same(m, got)
        past = torch.tensor([[j >= len(r) for j in range(width)] for r in m.table]).cuda()
        assert (got["table"][past] == -1).all()
        if copies:
            src, dst = (torch.tensor(x).cuda() for x in zip(*copies))
            want[:, dst] = want[:, src]
        assert torch.equal(pool, want)


@pytest.mark.parametrize("S,width,num,page", SIZES)
@pytest.mark.parametrize("in_place", [False, True])
def test_compact(P, S, width, num, page, in_place):
    for seed in range(3):
        m = Model(S, width, num, page, seed)
        if seed == 2:
            m.refs[num - 1] += 1  # held outside the table
        t, ln, r = m.tensors()
        pool = torch.randint(0, 1 << 30, (2, num, 40), dtype=torch.int32, device="cuda")
        want = pool.clone()
        out = dict(table=t, refs=r) if in_place else None
        got = P.gdn_pages_compact(t, ln, r, page, pool=pool, out=out)
        to, moves = m.compact()
        assert got["map"].tolist() == to
        same(m, got, lens=ln)
        if moves:
            src, dst = (torch.tensor(x).cuda() for x in zip(*moves))
            want[:, dst] = want[:, src]
        assert torch.equal(pool, want)


@pytest.mark.parametrize("shape,dtype", [((2, 9, 4, 16, 128), torch.bfloat16),
                                         ((1, 30, 2, 64, 64), torch.float32),
                                         ((4, 7, 4), torch.float32), ((3, 12, 5, 1028), torch.float32)])
def test_copy(P, shape, dtype):
    """Pages of 16 bytes to several units, pairs out of range, strided parts and pages."""
    big = torch.randn(shape[0], shape[1] + 1, 2, *shape[2:]).to(dtype).cuda()
    pool = big[:, 1:, 1]
    src = torch.tensor([0, 2, -1, 4, shape[1], 1], dtype=torch.int32).cuda()
    dst = torch.tensor([3, 5, 6, shape[1], 6, -7], dtype=torch.int32).cuda()
    want = big.clone()
    want[:, 4, 1], want[:, 6, 1] = want[:, 1, 1], want[:, 3, 1]
    P.gdn_pages_copy(pool, src, dst)
    assert torch.equal(big, want)
    P.gdn_pages_copy(pool, src[:0], dst[:0])
    assert torch.equal(big, want)


def test_graph(P):
    """Growing in place inside a captured graph, replayed until pages run out."""
    m = Model(9, 12, 60, 16, 3)
    t, ln, r = m.tensors()
    add = torch.full((9,), 5, dtype=torch.int32, device="cuda")
    out = dict(table=t, lens=ln, refs=r, short=torch.zeros_like(ln))
    ws = torch.empty(P.gdn_pages_workspace_size(t, r), dtype=torch.uint8, device="cuda")
    keep = [x.clone() for x in (t, ln, r)]
    P.gdn_pages_extend(t, ln, r, add, 16, out=out, workspace=ws)
    for x, y in zip((t, ln, r), keep):
        x.copy_(y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.gdn_pages_extend(t, ln, r, add, 16, out=out, workspace=ws)
    for _ in range(12):
        graph.replay()
        torch.cuda.synchronize()
        assert out["short"].tolist() == m.extend([5] * 9)
        same(m, out)
    assert any(out["short"].tolist())
