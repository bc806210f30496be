"""Many answers to one prompt: linear attention, attention over the shared prompt and the choice of
tokens together, as the serving example runs them and in a captured step; and each of them where
offsets pass 32 bits."""
import math

import pytest
import torch

from tests.test_gpu_hybrid_serving import ex  # noqa: F401
from tests.test_gpu_linear import check as check_linear, make, recurrence
from tests.test_gpu_paged_shared import Shared
from tests.test_gpu_sample import check as check_sample, choose

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("n", [150, 9])
def test_answers(ex, n):  # noqa: F811
    """Every token is one that its logits and random number allow, and the last logits are those
    of a prompt of the same tokens (in bfloat16, over six layers: as over the four of the
    example's other tests, 4 roundings of 2^-8 each, against the largest logit)."""
    g = torch.Generator().manual_seed(n)
    model = ex.HybridModel(window=0, linear=True)
    prompt = torch.randint(0, 211, (n,), generator=g).tolist()
    S, count = 5, 14
    server = ex.Server(model, S=S)
    seen, shared = [], []
    decode = server.decode

    def record(ids):
        shared.append(server.prefix)
        seen.append(decode(ids))
        return seen[-1]

    server.decode = record
    gen = torch.Generator(device="cuda").manual_seed(3)
    tokens, logprobs = server.answers(prompt, count, temperature=0.7, top_k=20, top_p=0.9,
                                      generator=gen)
    assert tokens.shape == logprobs.shape == (S, count) and len(seen) == count - 1
    assert shared == [n // 16 * 16] * len(shared) and server.prefix == 0
    gen.manual_seed(3)
    temperature, top_p = (float(torch.tensor(x)) for x in (0.7, 0.9))  # as the call gets them
    for step in range(count):
        u = torch.rand(S, device="cuda", generator=gen).tolist()
        if step:
            x = seen[step - 1].float().cpu().numpy()
            for r in range(S):
                want = choose(x[r], temperature, 20, top_p, 0.0, u[r])
                assert int(tokens[r, step]) in want
                assert float(logprobs[r, step]) == pytest.approx(want[int(tokens[r, step])],
                                                                 rel=2.0 ** -23, abs=2.0 ** -22)
    assert len({tuple(t) for t in tokens.tolist()}) > 1  # forks differ
    whole = ex.Server(model, S=S, num_pages=96)
    want = whole.prefill([prompt + t[:-1] for t in tokens.tolist()]).float()
    assert (seen[-1].float() - want).abs().max() <= 24 * 2.0 ** -8 * want.abs().max()


def test_answers_of_a_window(ex):  # noqa: F811
    """Where pages leave a window nothing is shared, and the same call works."""
    server = ex.Server(ex.HybridModel(), S=4)
    tokens, _ = server.answers(list(range(120)), 40)
    assert tokens.shape == (4, 40) and ((tokens >= 0) & (tokens < 211)).all()
    assert server.lens.tolist() == [159] * 4


def test_main_shows_them(ex, capsys):  # noqa: F811
    ex.main()
    assert "answers (8, 12)" in capsys.readouterr().out


def test_captured_step():
    """One token of each kind for every sequence in a graph, replayed with the program's own work
    between the replays: what the calls give one by one."""
    from paper_2412_06464_amd import linear, paged, sample
    N, H, Hk, d, page, prefix, vocab = 6, 4, 2, 64, 16, 70, 500
    gen = torch.Generator().manual_seed(5)

    def randn(*shape, dtype=BF16):
        return torch.randn(*shape, generator=gen).to("cuda", dtype)

    blocks = 10
    k_pages, v_pages = (randn(blocks * N, Hk, page, d) for _ in range(2))
    table = torch.randperm(blocks * N, generator=gen).reshape(N, blocks).to("cuda", torch.int32)
    table[:, :prefix // page] = table[0, :prefix // page]
    lead = table[0].clone()
    lens = torch.tensor([71, 80, 97, 70, 120, 75], dtype=torch.int32, device="cuda")
    q, k, v = (randn(N, 1, H, d) for _ in range(3))
    la = -torch.rand(N, 1, H, generator=gen).cuda()
    state, u = torch.zeros(N, H, d, d, device="cuda"), torch.zeros(N, device="cuda")
    head = randn(2 * H * d, vocab) * 0.1
    top_p = torch.full((N,), 0.9, device="cuda")
    ws = torch.empty(paged.gdn_cache_attn_shared_workspace_size(q, k_pages, table, prefix),
                     dtype=torch.uint8, device="cuda")
    out = dict(o=torch.empty_like(q), a=torch.empty_like(q),
               t=torch.empty(N, dtype=torch.int32, device="cuda"),
               lp=torch.empty(N, device="cuda"))

    def step(state, out):
        linear.gdn_linear_recurrent_fwd(q, k, v, la, h0=state, ht=state, o=out["o"])
        paged.gdn_cache_attn_shared(q, k_pages, v_pages, table, lens, lead, prefix, o=out["a"],
                                    workspace=ws)
        logits = torch.cat([out["o"], out["a"]], 2).reshape(N, -1) @ head
        sample.gdn_sample(logits, u, top_p=top_p, tokens=out["t"], logprob=out["lp"])

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(state.clone(), {x: y.clone() for x, y in out.items()})
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(state, out)
    state.zero_()
    mine = state.clone()
    drawn = set()
    for i in range(4):
        u.copy_(torch.rand(N, generator=gen))
        lens += 1
        q.copy_(torch.randn(q.shape, generator=gen))
        want = {x: torch.zeros_like(y) for x, y in out.items()}
        step(mine, want)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for x in out:
            assert torch.equal(out[x], want[x]), (i, x)
        assert torch.equal(state, mine)
        drawn.add(tuple(out["t"].tolist()))
    assert len(drawn) > 1


def test_linear_rows_past_32_bits():
    """q and k of over 2^31 elements; the last 200 tokens see none of those before them."""
    from paper_2412_06464_amd import linear
    T, H, dk, dv, tail = 140000, 64, 256, 64, 200
    torch.manual_seed(1)
    q, k = (torch.empty(1, T, H, dk, dtype=BF16, device="cuda").normal_() for _ in range(2))
    v = torch.empty(1, T, H, dv, dtype=BF16, device="cuda").normal_()
    q *= dk ** -0.5
    la = -torch.rand(1, T, H, device="cuda") * 0.2
    la[:, T - tail] = -math.inf
    assert q.numel() > 2 ** 31
    o, ht = linear.gdn_linear_chunk_fwd(q, k, v, la)
    heads = [0, H - 1]
    c = {x: y[:, T - tail:][:, :, heads].cpu() for x, y in
         dict(q=q, k=k, v=v, log_alpha=la).items()}
    c["h0"] = None
    check_linear((o[:, T - tail:][:, :, heads], ht[:, heads]), c, [tail], recurrence(c, [tail]))


def test_prefix_pages_past_32_bits():
    from paper_2412_06464_amd import paged as P
    c = Shared([1, 2], [70, 90], 50, 4, 2, 64, 16, BF16, seed=4)
    pages = c.k_pages.shape[0]
    stride = (2 ** 31 // (pages - 1) + 8192) // 64 * 64

    def spread(x):
        store = torch.empty(stride * (pages - 1) + x[0].numel(), dtype=BF16, device="cuda")
        view = store.as_strided(x.shape, (stride,) + x.stride()[1:])
        view.copy_(x.cuda())
        return view

    k, v = spread(c.k_pages), spread(c.v_pages)
    assert int(c.lead.max()) == pages - 1 and stride * (pages - 1) > 2 ** 31
    q = c.q[None].cuda()
    lse = torch.empty(q.shape[:3], device="cuda")
    o = P.gdn_cache_attn_shared(q, k, v, c.own.cuda(), c.kv_lens.cuda(), c.lead.cuda(), c.prefix,
                                lse=lse, cu_seqlens=c.cu.cuda(), cu_seqlens_host=c.cu)
    c.check((o.reshape(c.q.shape).cpu(), lse.reshape(c.q.shape[:2]).cpu()))


def test_logits_past_32_bits():
    from paper_2412_06464_amd import sample
    stride, vocab = 2 ** 30 + 8, 1000
    store = torch.zeros(2 * stride + vocab, dtype=BF16, device="cuda")
    logits = store.as_strided((3, vocab), (stride, 1))
    logits.copy_(torch.randn(3, vocab, generator=torch.Generator().manual_seed(6)))
    check_sample(sample, logits, [0.2, 0.5, 0.9], k=[0, 30, 30], p=[1.0, 0.9, 0.8])


def test_tensors_that_do_not_belong():
    """Refused on the host: memory of another kind or device as workspace or settings."""
    from paper_2412_06464_amd import linear, sample
    c, _ = make([2000], 2, 64, 64, BF16, dense=True)
    d = {x: None if y is None else y.cuda() for x, y in c.items()}
    need = linear.gdn_linear_chunk_fwd_workspace_size(d["q"], d["v"])
    assert need > 0
    for bad in (torch.empty(need, dtype=torch.uint8), torch.empty(need, dtype=F32, device="cuda"),
                torch.empty(2 * need, dtype=torch.uint8, device="cuda")[::2]):
        with pytest.raises(ValueError, match="workspace"):
            linear.gdn_linear_chunk_fwd(**d, workspace=bad)
    with pytest.raises(ValueError):
        linear.gdn_linear_chunk_fwd(**dict(d, h0=c["h0"]))
    with pytest.raises(ValueError):
        linear.gdn_linear_chunk_fwd(**dict(d, k=d["k"][:, :, :, :32]))
    x, u = torch.zeros(4, 10, device="cuda"), torch.zeros(4, device="cuda")
    for kw in (dict(u=u.cpu()), dict(u=u[:3]), dict(u=u.double()),
               dict(u=torch.zeros(8, device="cuda")[::2]),
               dict(top_k=torch.zeros(4, dtype=torch.int64, device="cuda")),
               dict(tokens=torch.zeros(4, dtype=torch.int64, device="cuda")),
               dict(temperature=torch.ones(4))):
        with pytest.raises(ValueError):
            sample.gdn_sample(x, **{**dict(u=u), **kw})
    with pytest.raises(ValueError, match="contiguous in a row"):
        sample.gdn_sample(x.t().contiguous().t(), u)
    with pytest.raises(TypeError):
        sample.gdn_sample(x, u, temperature=1.0)
