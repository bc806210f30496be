"""Linear attention with a decay against its recurrence in 64 bits: chunks and single tokens, all
head dims, lengths from none to many segments, decays of every kind, infinities, graphs."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
F64 = torch.float64


@pytest.fixture(scope="module")
def L():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2412_06464_amd import linear
    linear.load_library()
    return linear


def make(lens, H, dk, dv, dtype, decay="token", h0=True, seed=0, dense=False):
    """CPU tensors of sequences with these lengths (dense: all alike, [N, T, ...])."""
    gen = torch.Generator().manual_seed(seed)
    lead = (len(lens), lens[0]) if dense else (1, sum(lens))
    c = dict(q=(torch.randn(*lead, H, dk, generator=gen) * dk ** -0.5).to(dtype),
             k=torch.randn(*lead, H, dk, generator=gen).to(dtype),
             v=torch.randn(*lead, H, dv, generator=gen).to(dtype), log_alpha=None, h0=None)
    if decay == "token":
        c["log_alpha"] = -torch.nn.functional.softplus(torch.randn(*lead, H, generator=gen)) * 0.4
    if decay == "head":
        c["log_alpha"] = -torch.rand(H, generator=gen) * 0.1
    if h0:
        c["h0"] = torch.randn(len(lens), H, dk, dv, generator=gen)
    cu = torch.tensor([0] + list(lens)).cumsum(0).to(torch.int32)
    return c, {} if dense else dict(cu_seqlens=cu.cuda(), cu_seqlens_host=cu)


def recurrence(c, lens):
    """o, ht and the same sums of absolute values, which the errors are measured by; a token's
    outputs also with the state's and the chunk's rounding (see bounds)."""
    q, k, v = (c[x].flatten(0, 1).to(F64) for x in "qkv")
    H, dk, dv = q.shape[1], q.shape[2], v.shape[2]
    la = torch.zeros(q.shape[:2], dtype=F64)
    if c["log_alpha"] is not None:
        la = c["log_alpha"].to(F64).expand(*c["q"].shape[:3]).flatten(0, 1)
    o, mo = torch.zeros_like(v), torch.zeros_like(v)
    ht, mt = [], []
    row = 0
    for n, m in enumerate(lens):
        S = torch.zeros(H, dk, dv, dtype=F64) if c["h0"] is None else c["h0"][n].to(F64).clone()
        A = S.abs()
        for i in range(row, row + m):
            al = torch.exp(la[i])[:, None, None]
            S = al * S + k[i][:, :, None] * v[i][:, None, :]
            A = al * A + k[i].abs()[:, :, None] * v[i].abs()[:, None, :]
            o[i] = (S * q[i][:, :, None]).sum(1)
            mo[i] = (A * q[i].abs()[:, :, None]).sum(1)
        ht.append(S)
        mt.append(A)
        row += m
    return (o.reshape(c["v"].shape), torch.stack(ht), mo.reshape(c["v"].shape), torch.stack(mt))


def bounds(c, lens, o, mo, mt):
    """Errors allowed, with u = 2^-24 and sums of absolute values mo, mt.

    In fp32 a value is a sum of at most max(lens) + dk terms (each sum's order is free), each a
    product of four factors, one of them an exponential (its argument is a difference that
    carries at most 3 u of itself, at most 30 for a weight that counts, the exponential 2 u):
    (lens + dk + 128) u.  From bf16 input v is weighted in three values, 2^-24 relative together; o's
    terms pass once through the state or the chunk's products as a bf16 operand (2^-8), and o is
    rounded once (2^-8 of itself)."""
    u = 2.0 ** -24
    base = (max(lens) + c["q"].shape[3] + 128) * u
    if c["q"].dtype is torch.float32:
        return base * mo + 1e-30, base * mt + 1e-30
    return ((base + u + 2.0 ** -8) * mo + 2.0 ** -8 * o.abs() * (1 + 2.0 ** -7) + 1e-30,
            (base + u) * mt + 1e-30)


def gpu(c):
    return {x: None if y is None else y.cuda() for x, y in c.items()}


def check(got, c, lens, ref=None):
    o, ht, mo, mt = ref or recurrence(c, lens)
    bo, bt = bounds(c, lens, o, mo, mt)
    eo, et = (got[0].cpu().to(F64) - o).abs(), (got[1].cpu().to(F64) - ht).abs()
    assert (eo <= bo).all(), ("o", float((eo / bo).max()))
    assert (et <= bt).all(), ("ht", float((et / bt).max()))


DTYPES = [torch.bfloat16, torch.float32]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("dk", [64, 128, 256])
@pytest.mark.parametrize("dv", [64, 128, 256, 512])
def test_head_dims(L, dtype, dk, dv):
    lens = [70, 0, 1, 129]
    c, cu = make(lens, 2, dk, dv, dtype, seed=dk + dv)
    d, ref = gpu(c), recurrence(c, lens)
    check(L.gdn_linear_chunk_fwd(**d, **cu), c, lens, ref)
    check(L.gdn_linear_recurrent_fwd(**d, **cu), c, lens, ref)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("decay", ["token", "head", "none"])
@pytest.mark.parametrize("lens,H,dense", [([1], 1, True), ([63, 63], 3, True), ([64], 5, True),
                                          ([65, 0, 0, 64, 1, 200], 3, False), ([0, 5], 1, False)])
@pytest.mark.parametrize("h0", [True, False])
def test_lengths(L, dtype, decay, lens, H, dense, h0):
    c, cu = make(lens, H, 64, 128, dtype, decay, h0, seed=sum(lens), dense=dense)
    d, ref = gpu(c), recurrence(c, lens)
    check(L.gdn_linear_chunk_fwd(**d, **cu), c, lens, ref)
    check(L.gdn_linear_recurrent_fwd(**d, **cu), c, lens, ref)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("decay", ["token", "head", "none"])
@pytest.mark.parametrize("lens,dense", [([1300], True), ([700, 0, 3, 1025, 512], False),
                                        ([769, 769], True)])
def test_segments(L, dtype, decay, lens, dense):
    """Few heads and long sequences: walked in pieces, whose entry states are joined."""
    c, cu = make(lens, 2, 64, 64, dtype, decay, seed=3, dense=dense)
    assert L.gdn_linear_chunk_fwd_workspace_size(c["q"], c["v"], **(
        {x: y.cpu() for x, y in cu.items()})) > 0
    d, ref = gpu(c), recurrence(c, lens)
    check(L.gdn_linear_chunk_fwd(**d, **cu), c, lens, ref)
    d["h0"] = d["h0"].clone()  # and in place
    o, ht = L.gdn_linear_chunk_fwd(**d, ht=d["h0"], **cu)
    assert ht is d["h0"]
    check((o, ht), c, lens, ref)


@pytest.mark.parametrize("dtype", DTYPES)
def test_states_in_place(L, dtype):
    lens = [130, 0, 7]
    c, cu = make(lens, 2, 128, 128, dtype, seed=5)
    ref = recurrence(c, lens)
    for f in (L.gdn_linear_chunk_fwd, L.gdn_linear_recurrent_fwd):
        d = gpu(c)
        check(f(**d, ht=d["h0"], **cu), c, lens, ref)


def test_step_after_prompt(L):
    """A prompt in chunks, then single tokens from its state, as one sequence."""
    c, _ = make([90, 90], 3, 128, 256, torch.float32, seed=6, dense=True)
    d, ref = gpu(c), recurrence(c, [90, 90])

    def part(lo, hi, h0):
        return dict(q=d["q"][:, lo:hi].contiguous(), k=d["k"][:, lo:hi].contiguous(),
                    v=d["v"][:, lo:hi].contiguous(),
                    log_alpha=d["log_alpha"][:, lo:hi].contiguous(), h0=h0)

    o, h = L.gdn_linear_chunk_fwd(**part(0, 86, d["h0"]))
    outs = [o]
    for t in range(86, 90):
        o, h = L.gdn_linear_recurrent_fwd(**part(t, t + 1, h), ht=h)
        outs.append(o)
    check((torch.cat(outs, 1), h), c, [90, 90], ref)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("lens", [[150], [1300]])
def test_forgetting(L, dtype, lens):
    """Decays from none to all: log alpha of -infinity, -200, -1e-6, 0, -3e38."""
    c, cu = make(lens, 2, 64, 64, dtype, seed=7)
    la = c["log_alpha"]
    la[:, ::5] = -1e-6
    la[:, 1::7] = 0.0
    la[:, 40], la[:, 41, 0], la[:, 100], la[:, 63], la[:, 64] = -math.inf, -200.0, -3e38, -90.0, -1e3
    d, ref = gpu(c), recurrence(c, lens)
    check(L.gdn_linear_chunk_fwd(**d, **cu), c, lens, ref)
    check(L.gdn_linear_recurrent_fwd(**d, **cu), c, lens, ref)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("bad", [math.inf, math.nan])
@pytest.mark.parametrize("lens", [[70, 130], [1300]])
def test_odd_values_stay_behind(L, dtype, bad, lens):
    """An infinity or NaN in v reaches its column, from its token on; one in k or q (or the gate) no
    earlier token, no other sequence or head."""
    at = lens[0] - 30
    for name in ("v", "k", "q", "log_alpha"):
        c, cu = make(lens, 2, 64, 128, dtype, seed=8)
        ref = recurrence(c, lens)
        if name == "log_alpha":
            if bad == math.inf:
                continue
            c[name][0, at, 1] = bad
        else:
            c[name][0, at, 1, 5] = bad
        o, ht = L.gdn_linear_chunk_fwd(**gpu(c), **cu)
        bo, bt = bounds(c, lens, ref[0], ref[2], ref[3])
        hit = torch.zeros_like(ref[0], dtype=torch.bool)
        hit_t = torch.zeros_like(ref[1], dtype=torch.bool)
        if name == "v":
            hit[0, at:lens[0], 1, 5] = True
            hit_t[0, 1, :, 5] = True
        elif name == "q":
            hit[0, at, 1] = True
        else:
            hit[0, at:lens[0], 1] = True
            hit_t[0, 1] = True
        o, ht = o.cpu().to(F64), ht.cpu().to(F64)
        assert ((o - ref[0]).abs() <= bo)[~hit].all(), name
        assert ((ht - ref[1]).abs() <= bt)[~hit_t].all(), name
        assert not torch.isfinite(o[0, at, 1, 5]), name


def test_infinite_v_keeps_its_sign(L):
    c, cu = make([20], 1, 64, 64, torch.bfloat16, "none", False, seed=9)
    c["v"][0, 10, 0, 3] = -math.inf
    o, _ = L.gdn_linear_chunk_fwd(**gpu(c), **cu)
    sign = (c["k"][0, 10, 0].double() @ c["q"][0, 10:, 0].double().T).sign()
    assert torch.equal(o[0, 10:, 0, 3].cpu().double(), -sign * math.inf)


def test_same_bits(L):
    c, cu = make([700, 30, 900], 2, 128, 128, torch.bfloat16, seed=10)
    d = gpu(c)
    first = L.gdn_linear_chunk_fwd(**d, **cu)
    for _ in range(3):
        assert all(torch.equal(x, y) for x, y in zip(first, L.gdn_linear_chunk_fwd(**d, **cu)))


@pytest.mark.parametrize("T", [1, 900])
def test_replayed_on_another_stream(L, T):
    """Captured with its own workspace, replayed beside eager calls, inputs changed in between."""
    c, _ = make([T, T], 2, 64, 64, torch.float32, seed=11, dense=True)
    d = gpu(c)
    f = L.gdn_linear_recurrent_fwd if T == 1 else L.gdn_linear_chunk_fwd
    o, ht = torch.empty_like(d["v"]), torch.empty_like(d["h0"])
    kw = dict(o=o, ht=ht)
    if T > 1:
        kw["workspace"] = torch.empty(L.gdn_linear_chunk_fwd_workspace_size(d["q"], d["v"]),
                                      dtype=torch.uint8, device="cuda")
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        f(**d, **kw)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        f(**d, **kw)
    for i in range(4):
        new, _ = make([T, T], 2, 64, 64, torch.float32, seed=20 + i, dense=True)
        for x in d:
            d[x].copy_(new[x])
        eager = f(**d)
        o.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, eager[0]) and torch.equal(ht, eager[1]), i
    check((o, ht), new, [T, T])


def test_boundaries_changed_on_the_device(L):
    """A captured call follows cu_seqlens' device values; rows behind the last sequence are left as
    they were."""
    c, cu = make([300, 500], 1, 64, 64, torch.float32, seed=12)
    d = gpu(c)
    o, ht = torch.empty_like(d["v"]), torch.empty_like(d["h0"])
    ws = torch.empty(L.gdn_linear_chunk_fwd_workspace_size(d["q"], d["v"], **cu) + 16,
                     dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    L.gdn_linear_chunk_fwd(**d, o=o, ht=ht, workspace=ws, **cu)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        L.gdn_linear_chunk_fwd(**d, o=o, ht=ht, workspace=ws, **cu)
    lens = [640, 33]
    cu["cu_seqlens"].copy_(torch.tensor([0, 640, 673], dtype=torch.int32))
    o.fill_(7)
    graph.replay()
    torch.cuda.synchronize()
    short = {x: y if x in ("h0",) else y[:, :673] for x, y in c.items()}
    check((o[:, :673], ht), short, lens)
    assert (o[:, 673:] == 7).all()
