"""Serving steps in which pages run out: growing, storing and attending in one captured graph.
Sequences that were refused room are left alone, and so are the pages they share."""
import math

import pytest
import torch

from tests.paged_ref import Case
from tests.test_gpu_paged_pages import Model

pytestmark = pytest.mark.gpu
PAGE, HQ, HK, D = 16, 4, 2, 64


@pytest.fixture(scope="module")
def P():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2412_06464_amd import paged
    paged.load_library()
    return paged


def book(rows, lens, num):
    """A Model with these rows."""
    m = Model(1, 1, 1, PAGE, 0)
    m.S, m.width, m.num, m.page = len(rows), 6, num, PAGE
    m.table, m.lens, m.refs = [list(r) for r in rows], list(lens), [0] * num
    for r in rows:
        for p in r:
            m.refs[p] += 1
    return m


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T", [1, 5, 40])
@pytest.mark.parametrize("num", [14, 10])
def test_step_until_pages_run_out(P, dtype, T, num):
    """Rows 0 and 1 are forks that share two full pages; each step brings T tokens a row.  Of 14
    pages 8 are free: both go on for a while.  Of 10 pages one is free (three are held elsewhere):
    row 1 is refused where its last token, and so the place that its length gives the new one,
    lies in a shared page."""
    m = book([[3, 8], [3, 8], [0], [5, 1, 9]], [32, 32, 5, 37], num)
    if num == 10:
        for p in (2, 4, 6):
            m.refs[p] = 1
    table, lens, refs = m.tensors()
    short = torch.zeros_like(lens)
    add = torch.full_like(lens, T)
    gen = torch.Generator().manual_seed(T)
    kp, vp = (torch.randn(m.num, HK, PAGE, D, generator=gen).to(dtype) for _ in range(2))
    want_k, want_v = kp.clone(), vp.clone()
    kp, vp = kp.cuda(), vp.cuda()
    q = torch.zeros(m.S, T, HQ, D, dtype=dtype, device="cuda")
    k, v = (torch.zeros(m.S, T, HK, D, dtype=dtype, device="cuda") for _ in range(2))
    qo, o = torch.empty_like(q), torch.empty_like(q)
    lse = torch.empty(q.shape[:3], device="cuda")
    ws = torch.empty(max(P.gdn_pages_workspace_size(table, refs),
                         P.gdn_cache_attn_workspace_size(q, kp, table)) + 16,
                     dtype=torch.uint8, device="cuda")

    def step():
        P.gdn_pages_extend(table, lens, refs, add, PAGE, workspace=ws,
                           out=dict(table=table, lens=lens, refs=refs, short=short))
        P.gdn_cache_append(q, k, v, kp, vp, table, lens, q_out=qo, skip=short)
        P.gdn_cache_attn(qo, kp, vp, table, lens, o=o, lse=lse, workspace=ws, skip=short)

    keep = [x.clone() for x in (table, lens, refs, kp, vp)]
    step()
    for x, y in zip((table, lens, refs, kp, vp), keep):
        x.copy_(y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    refused = 0
    for i in range({1: 40, 5: 12, 40: 4}[T]):
        new = [torch.randn(x.shape, generator=gen).to(dtype) for x in (q, k, v)]
        for x, y in zip((q, k, v), new):
            x.copy_(y)
        o.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        gone = m.extend([T] * m.S)
        assert short.tolist() == gone and lens.tolist() == m.lens
        for s in range(m.S):
            for j in range(T if not gone[s] else 0):
                at = m.lens[s] - T + j
                want_k[m.table[s][at // PAGE], :, at % PAGE] = new[1][s, j]
                want_v[m.table[s][at // PAGE], :, at % PAGE] = new[2][s, j]
        assert torch.equal(kp.cpu(), want_k) and torch.equal(vp.cpu(), want_v), i
        c = Case([T] * m.S, m.lens, HQ, HK, D, PAGE, dtype)
        c.q, c.k_pages, c.v_pages = new[0].reshape(-1, HQ, D), want_k, want_v
        c.table = table.cpu()
        ro, rl, rel, mass = c.attend()
        ok = (o.cpu().double().reshape(ro.shape) - ro).abs() <= c.bound(rel, mass)
        for s in range(m.S):
            sl = slice(s * T, (s + 1) * T)
            if gone[s]:
                refused += 1
                assert not o[s].any() and (lse[s] == -math.inf).all()
                assert torch.equal(qo[s], q[s])
            else:
                assert ok[sl].all(), (i, s)
    assert refused and (num == 14 or m.lens[1] == 32 and (T == 40 or m.lens[0] > 32))


def test_one_sequence_left_out(P):
    """Packed input, rotated: the sequence's tokens turn as those before position 0."""
    c = Case([3, 20, 1], [40, 50, 7], HQ, HK, D, PAGE, torch.float32, seed=2)
    gen = torch.Generator().manual_seed(3)
    k, v = (torch.randn(1, 24, HK, D, generator=gen).cuda() for _ in range(2))
    q, cu = c.q[None].cuda(), dict(cu_seqlens=c.cu.cuda(), cu_seqlens_host=c.cu)
    r = P.gdn_rotary(D)
    got = []
    skip = torch.tensor([0, 2, 0], dtype=torch.int32).cuda()
    lens = c.kv_lens.clone()
    for n, s in ((lens, skip), (torch.tensor([40, 0, 7], dtype=torch.int32), None)):
        kp, vp = c.k_pages.cuda(), c.v_pages.cuda()
        args = (kp, vp, c.table.cuda(), n.cuda())
        qo = P.gdn_cache_append(q, k, v, *args, rotary=r, skip=s, **cu)
        o = P.gdn_cache_attn(qo, *args, skip=s, **cu)
        got.append((qo, kp.nan_to_num(9.0), vp.nan_to_num(9.0), o))
    assert all(torch.equal(x, y) for x, y in zip(*got))
    pos = torch.arange(-20, 0, dtype=torch.int32)[None].cuda()
    want = P.gdn_rotary_fwd(q[:, 3:23], None, r, positions=pos)[0]
    assert torch.equal(got[0][0][:, 3:23], want)


def test_refusals(P):
    c = Case([2], [20], HQ, HK, D, PAGE, torch.float32, seed=3)
    q = c.q[None].cuda()
    args = (c.k_pages.cuda(), c.v_pages.cuda(), c.table.cuda(), c.kv_lens.cuda())
    k = torch.zeros(1, 2, HK, D, device="cuda")
    for skip in (torch.zeros(1, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda"),
                 torch.zeros(1, dtype=torch.int32), [0]):
        with pytest.raises((ValueError, TypeError)):
            P.gdn_cache_append(q, k, k, *args, skip=skip)
        with pytest.raises((ValueError, TypeError)):
            P.gdn_cache_attn(q, *args, skip=skip)
