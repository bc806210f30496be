"""The choice of the next token against its definition in 64 bits, row by row: every rule and their
mixtures, flat and peaked distributions, ties, infinities, strides, graphs."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float32]


@pytest.fixture(scope="module")
def S():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2412_06464_amd import sample
    sample.load_library()
    return sample


def choose(x, t, k, p, m, u):
    """({tokens that may be drawn}, logprob of each): the definition in 64 bits.  Weights are within
    2^-42 of theirs and there are fewer than 2^20, so a border nearer than 2^-22 to u times
    the sum may fall to either side (and so may a top_p border: its token changes the sum by its
    own weight, which has to be as small for that)."""
    x = np.where(np.isnan(x), -np.inf, np.asarray(x, np.float64))
    order = np.lexsort((np.arange(len(x)), -x))
    x = x[order]
    if x[0] == -np.inf:
        return {-1: -math.inf}
    if not t > 0:
        return {int(order[0]): 0.0}
    with np.errstate(invalid="ignore", over="ignore"):
        y = np.where(x == x[0], 0.0, (x - x[0]) / np.float64(t))
    if x[0] == np.inf:
        y = np.where(x == np.inf, 0.0, -np.inf)
    y = np.where(np.isnan(y), -np.inf, y)  # (-infinity at an infinite temperature)
    y = y[y >= -43 * math.log(2)]
    if k > 0:
        y = y[:k]
    w = np.exp(y)
    if p < 1:
        run = np.cumsum(w)
        y = y[:max(1, 1 + int((run[:-1] < p * run[-1]).sum()))]
    if m > 0:
        y = y[:max(1, int((np.exp(y) >= m).sum()))]
    w = np.exp(y)
    run = np.cumsum(w)
    u = min(max(u, 0.0), 1 - 2.0 ** -24) if u == u else 0.0
    slack = 2.0 ** -22
    first = int((run <= u * run[-1] - slack).sum())
    last = min(int((run <= u * run[-1] + slack).sum()), len(y) - 1)
    return {int(order[i]): float(y[i] - math.log(run[-1])) for i in range(first, last + 1)}


def check(S, logits, u, t=None, k=None, p=None, m=None):
    rows = logits.shape[0]

    def dev(x, dtype):
        return None if x is None else torch.tensor(x, dtype=dtype).cuda()

    args = [dev(x, d) for x, d in ((u, torch.float32), (t, torch.float32), (k, torch.int32),
                                   (p, torch.float32), (m, torch.float32))]
    tokens, logprob = S.gdn_sample(logits, *args)
    tokens, logprob, x = tokens.tolist(), logprob.tolist(), logits.float().cpu().numpy()
    u, t, k, p, m = (([d] * rows if a is None else a.tolist())
                     for a, d in zip(args, (0.0, 1.0, 0, 1.0, 0.0)))
    for r in range(rows):
        want = choose(x[r], t[r], k[r], p[r], m[r], u[r])
        assert tokens[r] in want, (r, tokens[r], want, t[r], k[r], p[r], m[r], u[r])
        # rounded once from 64 bits, and a sum that is 2^-22 off at most
        assert logprob[r] == pytest.approx(want[tokens[r]], rel=2.0 ** -23, abs=2.0 ** -22)


RULES = {"plain": {}, "top_k": dict(k=50), "top_1": dict(k=1), "top_many": dict(k=1500),
         "top_p": dict(p=0.9), "top_k_p": dict(k=40, p=0.8), "min_p": dict(m=0.05),
         "all": dict(k=300, p=0.95, m=0.01), "many_all": dict(k=3000, p=0.99, m=1e-4)}


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rule", RULES)
@pytest.mark.parametrize("vocab", [1, 2, 7, 64, 1000, 2049, 8200, 50001])
def test_rules(S, dtype, rule, vocab):
    gen = torch.Generator().manual_seed(vocab)
    rows = 6
    logits = (torch.randn(rows, vocab, generator=gen) * 2.5).to(dtype).cuda()
    u = torch.rand(rows, generator=gen).tolist()
    kw = {x: [v] * rows for x, v in RULES[rule].items()}
    check(S, logits, u, t=[0.3, 0.7, 1.0, 1.5, 4.0, 0.0], **kw)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vocab", [5000, 100003])
@pytest.mark.parametrize("kw", [{}, dict(k=2100), dict(p=0.5), dict(k=4000, p=0.25, m=0.3)])
def test_all_alike(S, dtype, vocab, kw):
    """Equal logits: the order is the indexes', every border lies among thousands of ties."""
    u = [0.0, 0.25, 0.333, 0.5, 0.9999999, 0.7]
    logits = torch.full((6, vocab), -3.5, dtype=dtype, device="cuda")
    check(S, logits, u, **{x: [v] * 6 for x, v in kw.items()})
    tokens, logprob = S.gdn_sample(logits, torch.tensor(u).cuda())
    assert tokens.tolist() == [int(float(np.float32(x)) * vocab) for x in u]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("spread", [1e-3, 0.03, 30.0, 1000.0])
def test_spreads(S, dtype, spread):
    """From nearly flat (a bin holds all, or thousands of neighbours) to a single token."""
    gen = torch.Generator().manual_seed(3)
    logits = (torch.randn(8, 20000, generator=gen) * spread).to(dtype).cuda()
    u = torch.rand(8, generator=gen).tolist()
    for kw in RULES.values():
        check(S, logits, u, **{x: [v] * 8 for x, v in kw.items()})


def test_few_values(S):
    gen = torch.Generator().manual_seed(4)
    logits = torch.randint(-2, 3, (8, 30000), generator=gen).float().cuda()
    logits[:, ::3] *= -0.0  # zeros of either sign are one value
    for kw in RULES.values():
        check(S, logits, torch.rand(8, generator=gen).tolist(), **{x: [v] * 8 for x, v in kw.items()})


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("kw", [{}, dict(k=3), dict(p=0.5), dict(m=0.5), dict(t=0.0)])
def test_odd_logits(S, dtype, kw):
    gen = torch.Generator().manual_seed(5)
    logits = torch.randn(7, 999, generator=gen).to(dtype)
    logits[0] = -math.inf
    logits[1] = math.nan
    logits[2, ::2] = math.nan
    logits[3, ::2] = -math.inf
    logits[4, 100::300] = math.inf
    logits[5, :] = -math.inf
    logits[5, 998] = -5
    logits[6, 3], logits[6, 4] = math.nan, math.inf
    check(S, logits.cuda(), torch.rand(7, generator=gen).tolist(), **{x: [v] * 7 for x, v in kw.items()})


def test_odd_settings(S):
    nan, inf = math.nan, math.inf
    t = [nan, inf, 1e-30, 1e-45, 1e30, -1.0, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1]
    k = [0, 0, 0, 0, 0, 5, -3, 2 ** 31 - 1, 700, 0, 0, 0, 0, 0, 0, 0, 5]
    p = [1, 1, 1, 1, 1, 1, 1, 1, 1, 0, -1, nan, 2, 1, 1, 1, 0]
    m = [0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 1, 2, nan, -1]
    gen = torch.Generator().manual_seed(6)
    logits = torch.randn(len(t), 700, generator=gen).cuda()
    for u in (0.0, 1.0, 1.5, -1.0, nan, 0.4, 1 - 2.0 ** -24):
        check(S, logits, [u] * len(t), t, k, p, m)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("off,stride", [(0, 1003), (1, 1003), (5, 1009), (3, 2048), (7, 1024)])
def test_rows_anywhere(S, dtype, off, stride):
    """Rows that begin and end at any element; what lies beside them is never drawn."""
    gen = torch.Generator().manual_seed(7)
    store = torch.full((6 * stride + 64,), 1e4, dtype=dtype)
    logits = store[off:].as_strided((6, 1000), (stride, 1), off)
    logits.copy_(torch.randn(6, 1000, generator=gen))
    wide = store.cuda()
    view = wide.as_strided((6, 1000), (stride, 1), off)
    check(S, view, torch.rand(6, generator=gen).tolist())
    check(S, view, torch.rand(6, generator=gen).tolist(), k=[9] * 6, p=[0.9] * 6)


def test_one_row_for_many(S):
    """Rows of stride 0: many draws from one distribution, in the shares of its probabilities."""
    gen = torch.Generator().manual_seed(8)
    row = torch.randn(300, generator=gen).cuda()
    n = 4096
    u = (torch.arange(n) + 0.5) / n  # evenly: each token's count is its share to within one
    tokens, logprob = S.gdn_sample(row.expand(n, 300), u.cuda())
    counts = torch.bincount(tokens.long(), minlength=300).cpu()
    share = torch.softmax(row.double().cpu(), 0) * n
    assert ((counts - share).abs() <= 1).all()
    torch.testing.assert_close(logprob.cpu().double(),
                               torch.log_softmax(row.double().cpu(), 0)[tokens.cpu().long()],
                               rtol=2.0 ** -23, atol=2.0 ** -22)


def test_greedy_without_random_numbers(S):
    logits = torch.randn(5, 100).cuda()
    tokens, _ = S.gdn_sample(logits, None, temperature=torch.zeros(5, device="cuda"))
    assert torch.equal(tokens.long(), logits.argmax(-1))
    out = S.gdn_sample(logits, None, temperature=torch.zeros(5, device="cuda"), output_logprob=False)
    assert out[1] is None and torch.equal(out[0], tokens)


def test_replayed(S):
    gen = torch.Generator().manual_seed(9)
    logits, u = torch.empty(40, 9000, device="cuda"), torch.empty(40, device="cuda")
    t = torch.rand(40, generator=gen).cuda()
    k = torch.randint(0, 60, (40,), generator=gen, dtype=torch.int32).cuda()
    p = (0.5 + torch.rand(40, generator=gen)).cuda()
    tokens, lp = torch.empty(40, dtype=torch.int32, device="cuda"), torch.empty(40, device="cuda")
    logits.normal_()
    u.uniform_()
    S.gdn_sample(logits, u, t, k, p, tokens=tokens, logprob=lp)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        S.gdn_sample(logits, u, t, k, p, tokens=tokens, logprob=lp)
    for _ in range(4):
        logits.copy_(torch.randn(40, 9000, generator=gen))
        u.copy_(torch.rand(40, generator=gen))
        want = S.gdn_sample(logits, u, t, k, p)
        tokens.fill_(-7)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(tokens, want[0]) and torch.equal(lp, want[1])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads", [1, 40])
def test_draws_from_the_tail(S, dtype, heads):
    """A few likely tokens and tens of thousands far below, which are drawn from at times: all alike,
    nearly so, or spread; and the tokens at the end of the order."""
    gen = torch.Generator().manual_seed(11)
    logits = torch.empty(6, 60000)
    logits[0] = -13.0
    logits[1] = -13.0 + 1e-3 * torch.randn(60000, generator=gen)
    logits[2] = -13.0 + 2 * torch.randn(60000, generator=gen)
    logits[3] = -20.0 - 0.1 * torch.arange(60000) / 60000
    logits[4] = torch.linspace(-29, -1, 60000)
    logits[5] = -29.0
    logits[:, torch.randperm(60000, generator=gen)[:heads]] = 0.0
    logits = logits.to(dtype).cuda()
    for u in (0.5, 0.97, 0.999, 0.99999, 1 - 2.0 ** -20, 1 - 2.0 ** -24):
        check(S, logits, [u] * 6)
        check(S, logits, [u] * 6, k=[50000] * 6, p=[0.99999] * 6)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("kw", [{}, dict(k=700), dict(p=0.9), dict(p=0.5, m=0.2), dict(k=3)])
def test_masked_and_zeros(S, dtype, kw):
    """Rows most of which is the type's lowest value, or -infinity, or zeros of both signs: more of
    one value than 16 bits count, too."""
    vocab, gen = 150001, torch.Generator().manual_seed(12)
    low = torch.finfo(dtype).min
    logits = torch.full((6, vocab), low)
    logits[1] = -math.inf
    some = torch.randperm(vocab, generator=gen)[:900]
    for r in (0, 1):
        logits[r, some] = torch.randn(900, generator=gen) * 2
    logits[3] = 0.0
    logits[3, ::2] = -0.0
    logits[4] = torch.where(torch.rand(vocab, generator=gen) < 0.5, 0.0, -0.0)
    logits[4, some] = torch.randn(900, generator=gen)
    logits[5] = -math.inf
    logits[5, 700:1400] = 1.0
    logits = logits.to(dtype).cuda()
    rows = {x: [v] * 6 for x, v in kw.items()}
    check(S, logits, [0.3, 0.6, 0.99999, 0.5, 0.7, 0.25], **rows)
