"""Serving many answers to one prompt, as measurable cases.

Beside the gated delta rule a hybrid model has layers of linear attention with a
decay, and a program that draws several answers to a prompt attends from all of
them over the prompt's pages and chooses their tokens.  Kinds of a case:

  chunk   linear attention with a decay for each head over prompts
          (gdn_linear_chunk_fwd)
  step    the same, token by token (gdn_linear_recurrent_fwd)
  shared  attention of a batch's new tokens over a prefix that all of them share
          and over their own pages (gdn_cache_attn_shared)
  sample  the next tokens from logits and given random numbers: temperature,
          top-k, top-p, min-p (gdn_sample)

``listed()`` holds the fixed cases, ``draw()`` makes more of the same ranges.
With ``own`` false, ``run`` computes them with elementary torch operations; with
``own`` true it calls ``paper_2412_06464_amd``.
"""
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
NEG = -math.inf
CHUNK = 64
# a weight below this share of the largest counts as none
LEAST = 2.0 ** -43


def _chunk(dtype, N, T, H, dk, dv, decay="token", h0=True, style="even"):
    """N sequences of T tokens (ragged: packed, of 1 to T); ``decay`` of each "token" and head, of
    each "head", or "none"."""
    return dict(kind="chunk", dtype=dtype, N=N, T=T, H=H, dk=dk, dv=dv, decay=decay, h0=h0,
                style=style)


def _step(dtype, N, T, H, dk, dv, decay="token"):
    return dict(kind="step", dtype=dtype, N=N, T=T, H=H, dk=dk, dv=dv, decay=decay, h0=True,
                style="even")


def _shared(dtype, N, T, prefix, after, Hq, Hk, d, page, window=0, style="even"):
    """N sequences that share ``prefix`` tokens and hold up to ``after`` of their own before the T
    (ragged: 1 to T) new ones."""
    return dict(kind="shared", dtype=dtype, N=N, T=T, prefix=prefix, after=after, Hq=Hq, Hk=Hk,
                d=d, page=page, window=window, style=style)


def _sample(dtype, rows, vocab, rule):
    """``rule``: how the rows choose, "top_k", "top_p", "top_k_p", "min_p", "plain" or "mixed"."""
    return dict(kind="sample", dtype=dtype, rows=rows, vocab=vocab, rule=rule)


def listed():
    named = {
        # a batch's prompts of mixed lengths, packed, through one layer
        "linear_prompts_packed": _chunk("bf16", 16, 8192, 16, 128, 128, style="ragged"),
        # prompts of one length at the wide heads that the rule is benchmarked at
        "linear_prompts_wide": _chunk("bf16", 8, 4096, 6, 256, 512),
        # one long prompt: few heads side by side, a long axis
        "linear_prompt_long": _chunk("bf16", 1, 16384, 16, 128, 64, "head", False),
        # two short prompts in full precision, an odd length
        "linear_prompts_f32": _chunk("f32", 2, 1001, 4, 64, 64),
        # one token for each of a serving batch
        "linear_step": _step("bf16", 256, 1, 6, 256, 512),
        # one token for a handful of sequences: latency
        "linear_step_small": _step("bf16", 4, 1, 16, 128, 128, "head"),
        # 256 answers to a prompt of 8K tokens, a token each
        "shared_decode": _shared("bf16", 256, 1, 8192, 1000, 16, 4, 128, 64, style="ragged"),
        # a few answers about a long document
        "shared_decode_long": _shared("bf16", 16, 1, 131072, 300, 16, 4, 128, 64, style="ragged"),
        # a handful of answers to a short prompt, their proposed tokens verified in full precision
        "shared_verify_f32": _shared("f32", 6, 5, 700, 60, 8, 2, 64, 16, style="ragged"),
        # the next tokens of a handful of sequences: latency
        "sample_small": _sample("bf16", 4, 32000, "top_k_p"),
        # the next tokens of a serving batch, each request with its own settings
        "sample_batch": _sample("bf16", 256, 128000, "mixed"),
        # draws from nearly the whole of an odd vocabulary, in full precision
        "sample_wide_f32": _sample("f32", 64, 100003, "top_p"),
    }
    return [dict(c, name=n) for n, c in named.items()]


def draw(rng):
    def logint(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))

    kind = rng.choice(["chunk", "chunk", "step", "shared", "shared", "sample", "sample"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    e = 2 if dtype == "f32" else 1
    if kind == "sample":
        vocab = logint(50, 262144)
        return _sample(dtype, logint(1, max(1, min(256, 33554432 // (vocab * e)))), vocab,
                       rng.choice(["top_k", "top_p", "top_k_p", "min_p", "plain", "mixed"]))
    if kind in ("chunk", "step"):
        dk, dv = rng.choice([64, 128, 256]), rng.choice([64, 128, 256, 512])
        H, decay = rng.choice([1, 2, 4, 6, 8, 16]), rng.choice(["token", "token", "head", "none"])
        state = H * dk * dv
        if kind == "step":
            N = logint(1, min(512, 201326592 // state))
            return _step(dtype, N, rng.choice([1, 1, 2, 5]), H, dk, dv, decay)
        T = logint(1, 16384)
        most = min(100663296 // (H * (dk + dv) * e), 402653184 // (dk * dv * H) * CHUNK)
        T = min(T, most)
        return _chunk(dtype, logint(1, max(1, min(64, most // T))), T, H, dk, dv, decay,
                      rng.random() < 0.5, rng.choice(["even", "ragged", "ragged"]))
    d, Hk = rng.choice([64, 128, 128, 256]), rng.choice([1, 2, 4, 8])
    Hq = Hk * rng.choice([1, 2, 3, 4, 8] if Hk < 4 else [1, 2, 4])
    T = rng.choice([1, 1, 1, logint(2, 8), logint(9, 64)])
    prefix, after = logint(1, 131072), logint(1, 2000) - 1
    side = Hk * d * e  # a token's k, in bf16 elements
    prefix = min(prefix, 134217728 // side)
    most = (1 if dtype == "f32" else 4) * 4294967296 // (Hq * d * (prefix + after + T))
    N = max(1, min(256, most // T, 134217728 // (side * (after + T))))
    return _shared(dtype, logint(1, N), min(T, max(1, most)), prefix, after, Hq, Hk, d,
                   rng.choice([16, 32, 64, 128]), rng.choice([0, 0, 0, logint(16, 8192)]),
                   rng.choice(["even", "ragged", "ragged"]))


# ------------------------------------------------------------------ what a case fixes


def _lengths(case):
    """New tokens of each sequence, and tokens of its own before them."""
    rng = random.Random("%d %d %d" % (case["N"], case["T"], case.get("after", 0)))
    N, T, after = case["N"], case["T"], case.get("after", 0)
    if case["style"] == "even":
        return [T] * N, [after] * N
    return [rng.randint(1, T) for _ in range(N)], [rng.randint(0, after) for _ in range(N)]


def _rules(case):
    """temperature, top_k, top_p, min_p of each row (None: off for all)."""
    R, V, rule = case["rows"], case["vocab"], case["rule"]
    k = max(1, min(50, V // 2))
    if rule == "mixed":
        kinds = ["greedy", "top_k", "top_p", "top_k_p", "min_p", "plain"]
        rows = [kinds[i % len(kinds)] for i in range(R)]
        return ([0.0 if x == "greedy" else 0.7 + 0.1 * (i % 5) for i, x in enumerate(rows)],
                [(k, 1, 200)[i % 3] if x in ("top_k", "top_k_p") else 0 for i, x in enumerate(rows)],
                [0.9 if x in ("top_p", "top_k_p") else 1.0 for x in rows],
                [0.05 if x == "min_p" else 0.0 for x in rows])
    return ([0.8 if rule != "plain" else 1.0] * R, [k] * R if "top_k" in rule else None,
            [0.95 if rule == "top_p" else 0.9] * R if rule in ("top_p", "top_k_p") else None,
            [0.05] * R if rule == "min_p" else None)


# ------------------------------------------------------------------ inputs


def _inputs(case, seed):
    dev, dt = "cuda", DTYPES[case["dtype"]]
    gen = torch.Generator(device=dev).manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device=dev, dtype=torch.float32)

    def ints(x):
        return torch.tensor(x, dtype=torch.int32, device=dev)

    s = dict(case=case)
    if case["kind"] == "sample":
        R, V = case["rows"], case["vocab"]
        s["logits"] = (normal(R, V) * 2.5).to(dt)
        s["u"] = torch.rand(R, generator=gen, device=dev)
        t, k, p, m = _rules(case)
        s["temperature"] = torch.tensor(t, device=dev)
        s["top_k"] = None if k is None else ints(k)
        s["top_p"] = None if p is None else torch.tensor(p, device=dev)
        s["min_p"] = None if m is None else torch.tensor(m, device=dev)
        return s
    new, before = _lengths(case)
    s["new"], N = new, case["N"]
    if case["style"] == "even":  # [N, T, ...]
        lead, s["cu"] = (N, case["T"]), {}
    else:  # packed
        lead = (1, sum(new))
        host = torch.tensor([0] + new).cumsum(0).to(torch.int32)
        s["cu"] = dict(cu_seqlens=host.to(dev), cu_seqlens_host=host)
    if case["kind"] in ("chunk", "step"):
        H, dk, dv = case["H"], case["dk"], case["dv"]
        s["q"] = (normal(*lead, H, dk) * dk ** -0.5).to(dt)
        s["k"] = normal(*lead, H, dk).to(dt)
        s["v"] = normal(*lead, H, dv).to(dt)
        if case["decay"] == "token":  # a rate a head, a step a token and head
            rate = torch.rand(H, generator=gen, device=dev)
            s["log_alpha"] = -torch.exp(-rate) * torch.nn.functional.softplus(normal(*lead, H))
        elif case["decay"] == "head":
            s["log_alpha"] = torch.log1p(-torch.exp2(-3 - 4 * torch.rand(H, generator=gen,
                                                                         device=dev)))
        else:
            s["log_alpha"] = None
        s["h0"] = normal(N, H, dk, dv) * 0.2 if case["h0"] else None
        return s
    # The prefix's pages, then each sequence's own from the block on in which the prefix ends,
    # in random order; entries before that are not the sequence's.
    Hk, d, page, prefix = case["Hk"], case["d"], case["page"], case["prefix"]
    kv = [prefix + a + n for a, n in zip(before, new)]
    s["kv"] = kv
    head, first = -(-prefix // page), prefix // page
    num = head + sum(-(-c // page) - first for c in kv)
    order = list(range(num))
    random.Random(seed).shuffle(order)
    s["prefix_table"] = ints([order.pop() for _ in range(head)])
    width = max(-(-c // page) for c in kv)
    s["table"] = ints([[-1] * first + [order.pop() for _ in range(-(-c // page) - first)]
                       + [-1] * (width + first - first - -(-c // page)) for c in kv])
    s["kv_lens"] = ints(kv)
    pool = normal(2, num, Hk, page, d).to(dt)
    s["k_pages"], s["v_pages"] = pool[0], pool[1]
    s["q"] = normal(*lead, case["Hq"], d).to(dt)
    return s


def prepare(case, seed):
    """The inputs, and what a program keeps: the outputs and the workspace."""
    s = _inputs(case, seed)
    if not own:
        return s
    if case["kind"] in ("chunk", "step"):
        s["o"] = torch.empty_like(s["v"])
        s["ht"] = torch.empty(case["N"], case["H"], case["dk"], case["dv"], device="cuda")
    if case["kind"] == "chunk":
        from paper_2412_06464_amd import linear
        need = linear.gdn_linear_chunk_fwd_workspace_size(s["q"], s["v"], **s["cu"])
        s["ws"] = torch.empty(max(need, 1), dtype=torch.uint8, device="cuda")
    if case["kind"] == "shared":
        from paper_2412_06464_amd import paged
        s["max_kv"] = max(s["kv"])
        s["o"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty(s["q"].shape[:3], device="cuda")
        need = paged.gdn_cache_attn_shared_workspace_size(
            s["q"], s["k_pages"], s["table"], case["prefix"], window=case["window"],
            max_kv=s["max_kv"], **s["cu"])
        s["ws"] = torch.empty(max(need, 1), dtype=torch.uint8, device="cuda")
    if case["kind"] == "sample":
        s["tokens"] = torch.empty(case["rows"], dtype=torch.int32, device="cuda")
        s["logprob"] = torch.empty(case["rows"], device="cuda")
    return s


# ------------------------------------------------------------------ the framework's calls


def _run_own(s):
    case = s["case"]
    if case["kind"] == "chunk":
        from paper_2412_06464_amd import linear
        o, ht = linear.gdn_linear_chunk_fwd(s["q"], s["k"], s["v"], s["log_alpha"], h0=s["h0"],
                                            o=s["o"], ht=s["ht"], workspace=s["ws"], **s["cu"])
        return dict(o=o, ht=ht)
    if case["kind"] == "step":
        from paper_2412_06464_amd import linear
        o, ht = linear.gdn_linear_recurrent_fwd(s["q"], s["k"], s["v"], s["log_alpha"],
                                                h0=s["h0"], o=s["o"], ht=s["ht"], **s["cu"])
        return dict(o=o, ht=ht)
    if case["kind"] == "shared":
        from paper_2412_06464_amd import paged
        o = paged.gdn_cache_attn_shared(s["q"], s["k_pages"], s["v_pages"], s["table"],
                                        s["kv_lens"], s["prefix_table"], case["prefix"],
                                        window=case["window"], max_kv=s["max_kv"], o=s["o"],
                                        lse=s["lse"], workspace=s["ws"], **s["cu"])
        return dict(o=o, lse=s["lse"])
    from paper_2412_06464_amd import sample
    tokens, logprob = sample.gdn_sample(s["logits"], s["u"], s["temperature"], s["top_k"],
                                        s["top_p"], s["min_p"], tokens=s["tokens"],
                                        logprob=s["logprob"])
    return dict(tokens=tokens, logprob=logprob)


# ------------------------------------------------------------------ the plain form


def _chunk_plain(s):
    """All chunks of 64 tokens at once: what each adds to its sequence's state, each chunk's entry
    state as a weighted sum of those before it, and the output from the entry state and the chunk
    itself.  Sums of log decays in 64 bits, or their differences lose what they weigh."""
    case, dev = s["case"], s["q"].device
    H, dk, dv, new = case["H"], case["dk"], case["dv"], s["new"]
    n = torch.tensor(new, device=dev)
    per = (n + CHUNK - 1) // CHUNK
    seq = torch.repeat_interleave(torch.arange(len(new), device=dev), per)  # of a chunk
    nc, at = len(seq), torch.cumsum(per, 0) - per
    pos = (torch.arange(nc, device=dev) - at[seq])[:, None] * CHUNK + torch.arange(CHUNK, device=dev)
    real = pos < n[seq][:, None]  # [chunk, 64]
    row = torch.where(real, (torch.cumsum(n, 0) - n)[seq][:, None] + pos, 0)

    def tiles(x):  # [chunk, H, 64, d]
        x = x.flatten(0, 1)[row].float() * real[..., None, None]
        return x.transpose(1, 2).contiguous()

    q, k, v = tiles(s["q"]), tiles(s["k"]), tiles(s["v"])
    la = s["log_alpha"]
    if la is None:
        la = torch.zeros(H, device=dev)
    la = la.expand(*s["q"].shape[:3]).flatten(0, 1)[row].double() * real[..., None]
    g = torch.cumsum(la.transpose(1, 2), -1)  # [chunk, H, 64]
    low = torch.tril(torch.ones(CHUNK, CHUNK, dtype=torch.bool, device=dev))
    gamma = torch.where(low, torch.exp((g[..., :, None] - g[..., None, :]).float()), 0.0)
    o = ((q @ k.transpose(-1, -2).contiguous()) * gamma) @ v
    add = (k * torch.exp((g[..., -1:] - g).float())[..., None]).transpose(-1, -2).contiguous() @ v
    total = g[..., -1]  # [chunk, H]
    # log decay from the sequence's start to each chunk's start; then the ends of the sequences
    run = torch.cumsum(total, 0)
    start = run - total
    none = torch.zeros(1, H, dtype=torch.float64, device=dev)
    base = torch.cat([none, run])[at]  # [N, H]
    end = torch.cat([none, run])[at + per]
    to = torch.cat([start, end])  # rows: chunks, then ends
    of = torch.cat([seq, torch.arange(len(new), device=dev)])
    before = torch.cat([torch.arange(nc, device=dev), at + per])
    c = torch.arange(nc, device=dev)
    see = (c < before[:, None]) & (seq == of[:, None])
    w = torch.where(see, torch.exp((to.T[:, :, None] - run.T[:, None, :]).float()), 0.0)
    state = (w @ add.transpose(0, 1).reshape(H, nc, dk * dv)).reshape(H, nc + len(new), dk, dv)
    if s["h0"] is not None:
        fade = torch.exp((to - base[of]).float())
        state = state + (s["h0"][of] * fade[..., None, None]).transpose(0, 1)
    entry = state[:, :nc].transpose(0, 1)
    o = o + torch.exp(g.float())[..., None] * (q @ entry)
    out = torch.empty_like(s["v"])
    out.flatten(0, 1)[row[real]] = o.transpose(1, 2)[real].to(out.dtype)
    return dict(o=out, ht=state[:, nc:].transpose(0, 1).contiguous())


def _step_plain(s):
    case = s["case"]
    state, outs = s["h0"], []
    la = s["log_alpha"]
    if la is None:
        la = torch.zeros(case["H"], device=state.device)
    alpha = torch.exp(la.expand(s["q"].shape[:3]))
    for t in range(case["T"]):
        q, k, v = (s[x][:, t].float() for x in "qkv")
        state = state * alpha[:, t, :, None, None] + k[..., None] * v[..., None, :]
        outs.append((state * q[..., None]).sum(-2))
    return dict(o=torch.stack(outs, 1).to(s["v"].dtype), ht=state)


def _shared_plain(s):
    """Scores of all rows with the prefix as one product, those with a sequence's own keys padded
    to the longest, one softmax over both."""
    case, dev = s["case"], s["q"].device
    Hq, Hk, d, page = case["Hq"], case["Hk"], case["d"], case["page"]
    prefix, window, G, N = case["prefix"], case["window"], Hq // Hk, case["N"]
    new = torch.tensor(s["new"], device=dev)
    kv, T = s["kv_lens"].long(), max(s["new"])
    i = torch.arange(T, device=dev)
    real = i < new[:, None]
    row = torch.where(real, (torch.cumsum(new, 0) - new)[:, None] + i, 0)
    x = s["q"].flatten(0, 1)[row].float().reshape(N, T, Hk, G, d)
    x = x.permute(2, 0, 3, 1, 4).contiguous()  # [Hk, N, G, T, d]
    at = (kv - new)[:, None] + i  # positions [N, T]

    def keys(pages, upto):  # [..., blocks] -> [..., Hk, upto, d]
        got = []
        for pool in (s["k_pages"], s["v_pages"]):
            y = pool[pages.clamp(min=0).long()].float()  # [..., blocks, Hk, page, d]
            y = y.movedim(-3, -4).flatten(-3, -2)
            got.append(y[..., upto, :])
        return got

    def seen(pos):  # [N, 1 or T, keys]
        see = pos <= at[..., None]
        return see & (pos > at[..., None] - window) if window else see

    pos_p = torch.arange(prefix, device=dev)
    kp, vp = keys(s["prefix_table"], slice(0, prefix))  # [Hk, prefix, d]
    first = prefix // page
    skip = prefix - first * page
    ko, vo = keys(s["table"][:, first:], slice(skip, None))  # [N, Hk, own, d]
    pos_o = torch.arange(prefix, prefix + ko.shape[2], device=dev)
    scale = d ** -0.5
    sp = (x.reshape(Hk, -1, d) @ kp.transpose(1, 2).contiguous()).reshape(Hk, N, G, T, prefix)
    sp = torch.where(seen(pos_p)[None, :, None], sp * scale, NEG)
    y = x.transpose(0, 1).reshape(N, Hk, G * T, d)
    so = (y @ ko.transpose(2, 3).contiguous()).reshape(N, Hk, G, T, -1).transpose(0, 1)
    so = torch.where(seen(pos_o)[None, :, None], so * scale, NEG)
    top = torch.maximum(sp.amax(-1, keepdim=True), so.amax(-1, keepdim=True))
    sp, so = torch.exp(sp - top), torch.exp(so - top)
    total = sp.sum(-1, keepdim=True) + so.sum(-1, keepdim=True)
    o = (sp.reshape(Hk, -1, prefix) @ vp).reshape(Hk, N, G, T, d)
    own_part = so.transpose(0, 1).reshape(N, Hk, G * T, -1) @ vo
    o = (o + own_part.reshape(N, Hk, G, T, d).transpose(0, 1)) / total
    lse = (top + torch.log(total))[..., 0]
    out, out_lse = torch.empty_like(s["q"]), torch.empty(s["q"].shape[:3], device=dev)
    out.flatten(0, 1)[row[real]] = o.permute(1, 3, 0, 2, 4).reshape(N, T, Hq, d)[real].to(out.dtype)
    out_lse.flatten(0, 1)[row[real]] = lse.permute(1, 3, 0, 2).reshape(N, T, Hq)[real]
    return dict(o=out, lse=out_lse)


def _sample_plain(s):
    """Tokens from the most to the least likely, the lowest index first among equals; the kept ones
    are the first of them, and the drawn one is where their running sum passes u times its end.
    In 64 bits: a draw lies as near to a border as the random number has it."""
    logits, u = s["logits"], s["u"].double()
    R, V = logits.shape
    t = s["temperature"].double()
    greedy = t <= 0
    x, token = torch.sort(logits.float(), dim=1, descending=True, stable=True)
    w = torch.exp((x.double() - x[:, :1].double()) / torch.where(greedy, 1.0, t)[:, None])
    w = torch.where(w < LEAST, 0.0, w)
    place = torch.arange(V, device=x.device)
    keep = w > 0
    if s["top_k"] is not None:
        k = s["top_k"][:, None]
        keep &= (k <= 0) | (place < k)
    sums = torch.cumsum(torch.where(keep, w, 0.0), 1)
    if s["top_p"] is not None:
        p = s["top_p"].double()[:, None]
        keep &= (p >= 1) | (sums - w < p * sums[:, -1:]) | (place == 0)
    if s["min_p"] is not None:
        keep &= w >= s["min_p"].double()[:, None]
    keep &= ~greedy[:, None] | (place == 0)
    kept = keep.sum(1)
    total = sums.gather(1, kept[:, None] - 1)
    at = torch.searchsorted(sums, u[:, None] * total, right=True)
    at = torch.minimum(at, kept[:, None] - 1)
    logprob = torch.log(w.gather(1, at) / total)[:, 0]
    return dict(tokens=token.gather(1, at)[:, 0].to(torch.int32), logprob=logprob.float())


def run(state):
    if own:
        return _run_own(state)
    plain = dict(chunk=_chunk_plain, step=_step_plain, shared=_shared_plain, sample=_sample_plain)
    return plain[state["case"]["kind"]](state)


# ------------------------------------------------------------------ work


def work(case):
    """Bytes and FLOP of one pass: each input read once, each output written once (of the cache:
    the prefix once, and each sequence's own keys that some new token sees).  Linear attention:
    its two products with the state for each token, the form with the fewest."""
    e = 4 if case["dtype"] == "f32" else 2
    if case["kind"] == "sample":
        return dict(bytes=case["rows"] * (case["vocab"] * e + 12),
                    flops=2 * case["rows"] * case["vocab"])
    new, before = _lengths(case)
    n = sum(new)
    if case["kind"] in ("chunk", "step"):
        H, dk, dv = case["H"], case["dk"], case["dv"]
        states = (2 if case["h0"] else 1) * case["N"] * H * dk * dv * 4
        gates = 4 * n * H if case["decay"] == "token" else 0
        return dict(bytes=n * H * (2 * dk + 2 * dv) * e + gates + states,
                    flops=4 * n * H * dk * dv)
    Hq, Hk, d, w, prefix = (case[x] for x in ("Hq", "Hk", "d", "window", "prefix"))
    own_keys, pairs, low = 0, 0, prefix
    for m, a in zip(new, before):
        first = max(0, prefix + a + 1 - w) if w else 0  # the first key that its first token sees
        low = min(low, first)
        own_keys += prefix + a + m - max(prefix, first)
        for j in range(m):
            pairs += prefix + a + j + 1 - (max(0, prefix + a + j + 1 - w) if w else 0)
    return dict(bytes=n * Hq * (2 * d * e + 4) + 2 * (prefix - low + own_keys) * Hk * d * e,
                flops=4 * pairs * Hq * d)


# ------------------------------------------------------------------ 64 bits


def _exact_linear(case, s):
    """The recurrence, a token at a time, sequences side by side."""
    dev, new, N, H = s["q"].device, s["new"], case["N"], case["H"]
    T = max(new)
    dk, dv = case["dk"], case["dv"]
    state = torch.zeros(N, H, dk, dv, dtype=torch.float64, device=dev)
    if s["h0"] is not None:
        state += s["h0"].double()
    first = [sum(new[:i]) for i in range(N)]
    row = torch.tensor([[first[i] + min(t, new[i] - 1) for i in range(N)] for t in range(T)],
                       device=dev)
    live = torch.tensor([[float(t < n) for n in new] for t in range(T)], dtype=torch.float64,
                        device=dev)
    q, k, v = (s[x].flatten(0, 1) for x in "qkv")
    la = None if s["log_alpha"] is None else s["log_alpha"].expand(s["q"].shape[:3]).flatten(0, 1)
    o = torch.zeros(q.shape[0], H, dv, dtype=torch.float64, device=dev)
    for t in range(T):
        r, on = row[t], live[t][:, None, None, None]
        if la is not None:
            state *= torch.exp(la[r].double() * on[..., 0, 0])[..., None, None]
        state.addcmul_(k[r].double()[..., None] * on, v[r].double()[:, :, None, :])
        # a sequence that has ended gives its last row again, unchanged
        o[r] = torch.matmul(q[r].double()[:, :, None, :], state)[:, :, 0]
    return dict(o=o.reshape(s["v"].shape), ht=state)


def _exact_shared(case, s):
    """Sequence by sequence over its keys gathered from both tables."""
    page, prefix, Hk, G = case["page"], case["prefix"], case["Hk"], case["Hq"] // case["Hk"]
    q, o, lse, row = s["q"].flatten(0, 1), [], [], 0
    cut = -(-prefix // page)
    slots = torch.arange(page, device=q.device)
    where = (s["prefix_table"].long()[:, None] * page + slots).flatten()[:prefix]
    kp, vp = s["k_pages"].transpose(1, 2).flatten(0, 1), s["v_pages"].transpose(1, 2).flatten(0, 1)
    assert len(where) == prefix and cut * page >= prefix
    for n, (m, c) in enumerate(zip(s["new"], s["kv"])):
        j = torch.arange(prefix, c, device=q.device)
        mine = s["table"][n].long()[j // page] * page + j % page
        full = torch.cat([where, mine])
        k, v = kp[full].double(), vp[full].double()  # [keys, Hk, d]
        at = torch.arange(c - m, c, device=q.device)[:, None]
        key = torch.arange(c, device=q.device)
        hide = key > at
        if case["window"]:
            hide |= key <= at - case["window"]
        for h in range(Hk * G):
            x = q[row:row + m, h].double() @ k[:, h // G].T / math.sqrt(case["d"])
            x = x.masked_fill(hide, NEG)
            o.append(torch.softmax(x, -1) @ v[:, h // G])
            lse.append(torch.logsumexp(x, -1))
        row += m
    heads = Hk * G
    o = [torch.stack(o[i:i + heads], 1) for i in range(0, len(o), heads)]
    lse = [torch.stack(lse[i:i + heads], 1) for i in range(0, len(lse), heads)]
    return dict(o=torch.cat(o).reshape(s["q"].shape), lse=torch.cat(lse).reshape(s["q"].shape[:3]))


def _exact_sample(case, s):
    """Row by row on the CPU, the kept tokens counted from their order.  The tokens themselves are
    whole numbers and have no such value."""
    logits, u = s["logits"].double().cpu(), s["u"].double().cpu()
    t, k, p, m = _rules(case)
    out = []
    for r in range(case["rows"]):
        x, _ = torch.sort(logits[r], descending=True)
        temp = float(torch.tensor(t[r]))
        if temp <= 0:
            out.append(0.0)
            continue
        x = (x - x[0]) / temp
        x = x[x > math.log(LEAST)]
        if k is not None and k[r] > 0:
            x = x[:k[r]]
        w = torch.exp(x)
        if p is not None and p[r] < 1:
            run = torch.cumsum(w, 0)
            keep = 1 + int((run[:-1] < float(torch.tensor(p[r])) * run[-1]).sum())
            x, w = x[:keep], w[:keep]
        if m is not None:
            keep = max(1, int((w >= float(torch.tensor(m[r]))).sum()))
            x, w = x[:keep], w[:keep]
        run = torch.cumsum(w, 0)
        at = min(int((run <= float(u[r]) * run[-1]).sum()), len(x) - 1)
        out.append(float(x[at] - torch.logsumexp(x, 0)))
    return dict(tokens=None, logprob=torch.tensor(out, dtype=torch.float64).cuda())


def exact(case, seed):
    """What run returns, in 64 bits."""
    s = _inputs(case, seed)
    if case["kind"] in ("chunk", "step"):
        steps = max(s["new"]) * (1 + case["N"] * case["H"] * case["dk"] * case["dv"] / 2e6)
        return None if steps > 150000 else _exact_linear(case, s)
    if case["kind"] == "shared":
        heavy = case["N"] * case["Hq"] * (case["prefix"] + 5e4)
        return None if heavy > 1e9 else _exact_shared(case, s)
    return _exact_sample(case, s)
