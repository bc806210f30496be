"""The attention layer beside the gated delta rule, as measurable cases.

A model that alternates the rule with (window) attention also has to place
tokens by rotary positions, keep keys and values in pages, attend over them and
manage the pages.  Kinds of a case:

  rotate  rotary positions of q and k: forward, backward, or both as a training
          step runs them (gdn_rotary_fwd, gdn_rotary_bwd)
  append  a call's new tokens: q and k rotated, k and v stored in their
          sequences' pages (gdn_cache_append)
  attend  attention of the new tokens over the pages (gdn_cache_attn)
  pages   growing, selecting (fork, free, reorder) or compacting the pages of a
          cache (gdn_pages_extend, gdn_pages_select, gdn_pages_compact)

``listed()`` holds the fixed cases, ``draw()`` makes more of the same ranges.
With ``own`` false, ``run`` computes them with elementary torch operations in
32 bits; with ``own`` true it calls ``paper_2412_06464_amd.paged``.
"""
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
NEG = -math.inf


def _rotate(way, dtype, N, T, Hq, Hk, d, rot, layout="halves", scaling="none", first=0,
            style="even"):
    """N sequences of T tokens (``style``: all alike, or packed and ragged up to T), the first
    token of a sequence at position ``first``."""
    return dict(kind="rotate", way=way, dtype=dtype, N=N, T=T, Hq=Hq, Hk=Hk, d=d, rot=rot,
                layout=layout, scaling=scaling, first=first, style=style)


def _append(dtype, N, T, prefix, Hq, Hk, d, rot, page, layout="halves", scaling="none",
            style="even"):
    """N sequences with up to ``prefix`` tokens in the cache, T (ragged: up to T) new ones each."""
    return dict(kind="append", dtype=dtype, N=N, T=T, prefix=prefix, Hq=Hq, Hk=Hk, d=d, rot=rot,
                page=page, layout=layout, scaling=scaling, style=style)


def _attend(dtype, N, T, prefix, Hq, Hk, d, page, window=0, style="even"):
    """As _append; ``style`` "mixed": the first sequence has T new tokens, the others one."""
    return dict(kind="attend", dtype=dtype, N=N, T=T, prefix=prefix, Hq=Hq, Hk=Hk, d=d,
                page=page, window=window, style=style)


def _pages(op, S, tokens, parts, page, Hk, d, spare, dtype="bf16"):
    """S sequences of up to ``tokens`` tokens in a pool of ``parts`` tensors (k and v of each
    layer); ``spare``: free pages beyond those in use, as a share of them."""
    return dict(kind="pages", op=op, S=S, tokens=tokens, parts=parts, page=page, Hk=Hk, d=d,
                spare=spare, dtype=dtype)


def listed():
    named = {
        # q and k of a training step on packed documents, both directions
        "rotate_train_packed": _rotate("both", "bf16", 24, 4096, 16, 4, 128, 128, style="ragged"),
        # full-precision gradient of a quarter of each head, interleaved, long-context scaling
        "rotate_bwd_partial_f32": _rotate("bwd", "f32", 2, 1000, 6, 2, 256, 64, "interleaved",
                                          "parts", 30000),
        # one new token for each of a serving batch: latency
        "append_decode": _append("bf16", 256, 1, 4095, 16, 4, 128, 128, 64, style="ragged"),
        # prompts of mixed lengths entering the cache
        "append_prompts": _append("bf16", 8, 4096, 2000, 16, 4, 128, 64, 64, "interleaved",
                                  "linear", "ragged"),
        # one token for a handful of sequences: latency
        "attend_decode_small": _attend("bf16", 4, 1, 999, 16, 4, 128, 16),
        # one token for each of a serving batch, within a 2K window
        "attend_decode_window": _attend("bf16", 256, 1, 4095, 16, 4, 128, 64, 2048, "ragged"),
        # two users deep into a long document: few rows, a long axis
        "attend_decode_long": _attend("bf16", 2, 1, 131071, 16, 4, 128, 64),
        # a long prompt in one piece
        "attend_prompt": _attend("bf16", 1, 8192, 0, 16, 4, 128, 64),
        # a batch's prompts, packed, window attention, three query heads to a cache head
        "attend_prompts_window": _attend("bf16", 8, 4096, 1000, 6, 2, 256, 64, 2048, "ragged"),
        # a few proposed tokens a sequence verified in full precision, a head each
        "attend_verify_f32": _attend("f32", 12, 5, 3000, 8, 8, 64, 32, 0, "ragged"),
        # a step of a beam search: each sequence's best four continuations
        "pages_select": _pages("select", 256, 1200, 4, 64, 4, 128, 0.2),
        # a fragmented cache packed into its lowest pages
        "pages_compact": _pages("compact", 96, 1200, 8, 64, 4, 128, 0.6),
    }
    return [dict(c, name=n) for n, c in named.items()]


def draw(rng):
    def logint(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))

    kind = rng.choice(["rotate", "append", "attend", "attend", "attend", "pages"])
    if kind == "pages":
        op, dtype = rng.choice(["select", "select", "compact", "extend"]), rng.choice(list(DTYPES))
        parts, Hk, d = rng.choice([2, 4, 8]), rng.choice([1, 2, 4]), rng.choice([64, 128])
        tokens = logint(20, 2500)
        S = 314572800 // (tokens * parts * Hk * d * (2 if dtype == "f32" else 1))
        return _pages(op, logint(1, min(256, S)), tokens, parts, rng.choice([16, 32, 64]), Hk, d,
                      round(rng.uniform(0.05, 0.6), 2), dtype)
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    d = rng.choice([64, 128, 128, 256])
    Hk = rng.choice([1, 2, 4, 8])
    Hq = Hk * rng.choice([1, 2, 3, 4, 6, 8] if Hk < 4 else [1, 2, 4])
    layout = rng.choice(["halves", "interleaved"])
    scaling = rng.choice(["none", "linear", "base", "parts"])
    rot = rng.choice([d, d, d // 2, d // 4, 2 * rng.randint(1, d // 2)])
    wide = Hq * d * (2 if dtype == "f32" else 1)
    if kind == "rotate":
        style = rng.choice(["even", "ragged"])
        T = logint(1, 4096)
        N = logint(1, max(1, min(256, 134217728 // (wide * T))))
        return _rotate(rng.choice(["fwd", "bwd", "both"]), dtype, N, T, Hq, Hk, d, rot, layout,
                       scaling, logint(1, 100000) - 1, style)
    page = rng.choice([16, 32, 64, 128])
    if kind == "append":
        T = rng.choice([1, logint(1, 4096)])
        N = logint(1, max(1, min(256, 33554432 // (wide * T))))
        return _append(dtype, N, T, logint(1, 4096) - 1, Hq, Hk, d, rot, page, layout, scaling,
                       rng.choice(["even", "ragged"]))
    style = rng.choice(["even", "ragged", "ragged", "mixed"])
    T = rng.choice([1, 1, logint(2, 8), logint(9, 4096)])
    window = rng.choice([0, 0, logint(16, 4096)])
    side = Hk * d * (2 if dtype == "f32" else 1)  # a token's k, in bf16 elements
    long = rng.choice([2000, 8000, 100000])
    prefix = logint(1, min(long, 134217728 // side)) - 1
    most = (4 if dtype == "bf16" else 1) * 8589934592 // wide  # rows x keys of all heads
    keys = min(T + prefix, T + window) if window else T + prefix
    T = max(1, min(T, most // keys))
    rows = 1 if style == "mixed" else T
    N = min(256, 134217728 // (side * (T + prefix)), most // (rows * keys))
    return _attend(dtype, logint(1, max(1, N)), T, prefix, Hq, Hk, d, page, window, style)


# ------------------------------------------------------------------ what a case fixes


def _lengths(case):
    """(new tokens, tokens in the cache with them) of each sequence."""
    rng = random.Random("%d %d %d" % (case["N"], case["T"], case.get("prefix", 0)))
    N, T, prefix, style = case["N"], case["T"], case.get("prefix", 0), case["style"]
    if style == "even":
        new, old = [T] * N, [prefix] * N
    else:
        new = [rng.randint(1, T) for _ in range(N)] if style == "ragged" else [T] + [1] * (N - 1)
        old = [rng.randint(0, prefix) for _ in range(N)]
    return new, [a + b for a, b in zip(new, old)]


def _theta(case):
    """Radians a position of each pair, in 64 bits, and the factor of cos and sin."""
    rot, base, factor, original = case["rot"], 10000.0, 8.0, 4096
    if case["scaling"] == "base" and rot > 2:
        base *= factor ** (rot / (rot - 2))
    th = base ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    if case["scaling"] == "linear":
        th = th / factor
    if case["scaling"] == "parts":
        turns = original * th / (2 * math.pi)
        keep = ((turns - 1.0) / (32.0 - 1.0)).clamp(0.0, 1.0)
        return th / factor * (1 - keep) + th * keep, 0.1 * math.log(factor) + 1.0
    return th, 1.0


def _first_key(case, new, kv):
    """The first key that a sequence's first new token sees."""
    return max(0, kv - new + 1 - case["window"]) if case.get("window") else 0


def _fragmented(case, seed):
    """Rows of pages, lengths and reference counts of a cache some way into its life (full pages
    shared by forks, pages in no order, free ones between them), and for a selection the row each
    row goes on from: a quarter survive, in four rows each.  The seed gives the pages' order."""
    rng = random.Random("%(op)s %(S)d %(tokens)d %(page)d %(spare)g" % case)
    S, page = case["S"], case["page"]
    lens = [rng.randint(1, case["tokens"]) for _ in range(S)]
    if case["op"] == "extend":
        lens[S // 2] = 0
    rows, pages = [], 0
    for s, n in enumerate(lens):
        row = []
        if s and rng.random() < 0.3:  # forked from an earlier one: full pages of it
            other = rng.randrange(s)
            row = rows[other][:min(n, lens[other], rng.randint(0, 1000)) // page]
        fresh = -(-n // page) - len(row)
        rows.append(row + list(range(pages, pages + fresh)))
        pages += fresh
    best = [rng.randrange(S) for _ in range(-(-S // 4))]
    num = max(pages + 2, int(pages * (1 + case["spare"])))
    order = list(range(num))
    random.Random(seed).shuffle(order)
    rows = [[order[i] for i in row] for row in rows]
    refs = [0] * num
    for row in rows:
        for i in row:
            refs[i] += 1
    return rows, lens, refs, [best[i // 4] for i in range(S)]


# ------------------------------------------------------------------ inputs


def _inputs(case, seed):
    dev, dt = "cuda", DTYPES[case["dtype"]]
    gen = torch.Generator(device=dev).manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device=dev, dtype=torch.float32).to(dt)

    def ints(x):
        return torch.tensor(x, dtype=torch.int32, device=dev)

    s = dict(case=case)
    if case["kind"] == "pages":
        rows, lens, refs, parents = _fragmented(case, seed)
        width = max(len(r) for r in rows) + 2
        s["table"] = ints([r + [-1] * (width - len(r)) for r in rows])
        s["lens"], s["refs"] = ints(lens), ints(refs)
        if case["op"] == "select":
            s["parents"] = ints(parents)
        if case["op"] == "extend":
            rng = random.Random(seed)
            s["add"] = ints([rng.choice([1, 1, 1, rng.randint(0, 2 * case["page"])])
                             for _ in lens])
        s["pool"] = normal(case["parts"], len(refs), case["Hk"], case["page"], case["d"])
        return s
    new, kv = _lengths(case)
    N, Hq, Hk, d = case["N"], case["Hq"], case["Hk"], case["d"]
    s["new"], s["kv"] = new, kv
    if case["style"] == "even":  # [N, T, ...]
        lead, s["cu"] = (N, case["T"]), {}
    else:  # packed
        lead = (1, sum(new))
        host = torch.tensor([0] + new).cumsum(0).to(torch.int32)
        s["cu"] = dict(cu_seqlens=host.to(dev), cu_seqlens_host=host)
    s["q"] = normal(*lead, Hq, d)
    if case["kind"] == "rotate":
        s["k"] = normal(*lead, Hk, d)
        pos = torch.cat([torch.arange(n) for n in new]) + case["first"]
        s["positions"] = pos.to(torch.int32).reshape(lead).to(dev)
        if case["way"] != "fwd":
            s["dq"], s["dk"] = normal(*lead, Hq, d), normal(*lead, Hk, d)
        return s
    # pages in random order; those that no new token sees are no longer held
    page = case["page"]
    blocks = [(_first_key(case, n, c) // page, -(-c // page)) for n, c in zip(new, kv)]
    num = sum(b - a for a, b in blocks)
    order = list(range(num))
    random.Random(seed).shuffle(order)
    width, rows = max(b for _, b in blocks), []
    for a, b in blocks:
        rows.append([-1] * a + [order.pop() for _ in range(b - a)] + [-1] * (width - b))
    s["table"], s["kv_lens"] = ints(rows), ints(kv)
    if case["kind"] == "append":
        s["k"], s["v"] = normal(*lead, Hk, d), normal(*lead, Hk, d)
        pool = torch.zeros(2, num, Hk, page, d, dtype=dt, device=dev)
    else:
        pool = normal(2, num, Hk, page, d)
    s["k_pages"], s["v_pages"] = pool[0], pool[1]
    return s


def prepare(case, seed):
    """The inputs, and what a program keeps: the rotation's handle, the outputs, the workspace."""
    s = _inputs(case, seed)
    if "rot" in case:
        if own:
            from paper_2412_06464_amd import paged
            s["rotary"] = paged.gdn_rotary(case["rot"], base=10000.0, layout=case["layout"],
                                           scaling=case["scaling"], factor=8.0, original=4096,
                                           device="cuda")
        else:
            s["theta"], s["factor"] = _theta(case)
            s["theta"] = s["theta"].cuda()
    if own and case["kind"] == "attend":
        from paper_2412_06464_amd import paged
        s["max_kv"] = max(s["kv"])
        s["o"] = torch.empty_like(s["q"])
        need = paged.gdn_cache_attn_workspace_size(
            s["q"], s["k_pages"], s["table"], window=case["window"], max_kv=s["max_kv"], **s["cu"])
        s["ws"] = torch.empty(max(need, 1), dtype=torch.uint8, device="cuda")
    if own and case["kind"] == "pages":
        from paper_2412_06464_amd import paged
        s["ws"] = torch.empty(paged.gdn_pages_workspace_size(s["table"], s["refs"]),
                              dtype=torch.uint8, device="cuda")
    return s


# ------------------------------------------------------------------ the framework's calls


def _run_own(s):
    from paper_2412_06464_amd import paged
    case = s["case"]
    kind = case["kind"]
    if kind == "rotate":
        out = {}
        if case["way"] != "bwd":
            out["q"], out["k"] = paged.gdn_rotary_fwd(s["q"], s["k"], s["rotary"],
                                                      positions=s["positions"])
        if case["way"] != "fwd":
            out["dq"], out["dk"] = paged.gdn_rotary_bwd(s["dq"], s["dk"], s["rotary"],
                                                        positions=s["positions"])
        return out
    if kind == "append":
        q = paged.gdn_cache_append(s["q"], s["k"], s["v"], s["k_pages"], s["v_pages"], s["table"],
                                   s["kv_lens"], rotary=s["rotary"], **s["cu"])
        return dict(q=q, k_pages=s["k_pages"], v_pages=s["v_pages"])
    if kind == "attend":
        return dict(o=paged.gdn_cache_attn(s["q"], s["k_pages"], s["v_pages"], s["table"],
                                           s["kv_lens"], window=case["window"],
                                           max_kv=s["max_kv"], o=s["o"], workspace=s["ws"],
                                           **s["cu"]))
    book = (s["table"], s["lens"], s["refs"])
    if case["op"] == "extend":
        return paged.gdn_pages_extend(*book, s["add"], page_size=case["page"], workspace=s["ws"])
    if case["op"] == "select":
        out = paged.gdn_pages_select(*book, s["parents"], page_size=case["page"], pool=s["pool"],
                                     workspace=s["ws"])
    else:
        out = paged.gdn_pages_compact(*book, page_size=case["page"], pool=s["pool"],
                                      workspace=s["ws"])
    return dict(out, pool=s["pool"])


# ------------------------------------------------------------------ the plain form


def _turn(x, positions, theta, factor, layout, sign=1.0):
    """Rotation of the first 2 len(theta) channels of x [..., H, d].  The angle is formed in 64
    bits: in 32, a position of 100000 times a frequency is off by 0.004."""
    rot = 2 * theta.numel()
    a = torch.remainder(positions.double()[..., None] * theta, 2 * math.pi).float()
    cos, sin = (torch.cos(a) * factor)[..., None, :], (torch.sin(a) * (factor * sign))[..., None, :]
    y = x.float().clone()
    if layout == "halves":
        i, j = slice(0, rot // 2), slice(rot // 2, rot)
    else:
        i, j = slice(0, rot, 2), slice(1, rot, 2)
    x1, x2 = x[..., i].float(), x[..., j].float()
    y[..., i] = x1 * cos - x2 * sin
    y[..., j] = x2 * cos + x1 * sin
    return y.to(x.dtype)


def _places(s):
    """(sequence, position) of each new token, in row order, on the GPU."""
    seq = torch.cat([torch.full((n,), i, dtype=torch.long) for i, n in enumerate(s["new"])])
    pos = torch.cat([torch.arange(c - n, c) for n, c in zip(s["new"], s["kv"])])
    return seq.cuda(), pos.cuda()


def _append_plain(s):
    case = s["case"]
    seq, pos = _places(s)
    at = pos.reshape(s["q"].shape[:2])
    q = _turn(s["q"], at, s["theta"], s["factor"], case["layout"])
    k = _turn(s["k"], at, s["theta"], s["factor"], case["layout"])
    page, slot = s["table"][seq, pos // case["page"]].long(), pos % case["page"]
    s["k_pages"][page, :, slot] = k.reshape(-1, *k.shape[2:])
    s["v_pages"][page, :, slot] = s["v"].reshape(-1, *k.shape[2:])
    return dict(q=q, k_pages=s["k_pages"], v_pages=s["v_pages"])


def _pieces(case, new, kv):
    """Bunches of (sequence, first row, rows, last position + 1): at most 512 new tokens of a
    sequence each, those of like size together while their scores fit 2^28 values."""
    items, row = [], 0
    for n, (m, c) in enumerate(zip(new, kv)):
        for i in range(0, m, 512):
            t = min(512, m - i)
            items.append((t, c - m + i + t, n, row + i))
        row += m
    items.sort(reverse=True)
    bunches, most = [], 0
    for t, end, n, r in items:
        most = max(most, end - _first_key(case, t, end) + 2 * case["page"])
        if (not bunches or 4 * t < bunches[-1][0][2]
                or (len(bunches[-1]) + 1) * bunches[-1][0][2] * most * case["Hq"] > 1 << 28):
            bunches.append([])
            most = end - _first_key(case, t, end) + 2 * case["page"]
        bunches[-1].append((n, r, t, end))
    return bunches


def _attend_plain(s):
    case = s["case"]
    Hq, Hk, d, page, window = (case[x] for x in ("Hq", "Hk", "d", "page", "window"))
    G, dev = Hq // Hk, s["q"].device
    q = s["q"].reshape(-1, Hq, d)
    o = torch.empty_like(q)
    width = s["table"].shape[1]
    for bunch in _pieces(case, s["new"], s["kv"]):
        n, r, t, end = (torch.tensor(x, device=dev) for x in zip(*bunch))
        T = max(b[2] for b in bunch)
        lo = [_first_key(case, b[2], b[3]) // page for b in bunch]
        blocks = max(-(-b[3] // page) - a for b, a in zip(bunch, lo))
        block = torch.tensor(lo, device=dev)[:, None] + torch.arange(blocks, device=dev)
        pages = s["table"][n[:, None], block.clamp(max=width - 1)].long()
        kpos = (block[..., None] * page + torch.arange(page, device=dev)).reshape(len(bunch), -1)
        held = (pages >= 0).repeat_interleave(page, 1) & (kpos < end[:, None])
        k, v = (x[pages.clamp(min=0)].float().transpose(2, 3).reshape(len(bunch), -1, Hk, d)
                for x in (s["k_pages"], s["v_pages"]))  # [sequence, key, Hk, d]
        v = torch.where(held[..., None, None], v, 0.0)
        i = torch.arange(T, device=dev)
        rows = (r[:, None] + i.clamp(max=T - 1)).clamp(max=q.shape[0] - 1)
        qpos = (end - t)[:, None] + i
        see = held[:, None] & (kpos[:, None] <= qpos[..., None])
        if window:
            see &= kpos[:, None] > qpos[..., None] - window
        see = see[:, None, None]  # [sequence, 1, 1, T, keys]
        x = q[rows].float().reshape(len(bunch), T, Hk, G, d).permute(0, 2, 3, 1, 4)
        x = x.reshape(len(bunch), Hk, G * T, d).contiguous()
        score = (x @ k.permute(0, 2, 3, 1).contiguous()) * d ** -0.5
        score = torch.where(see, score.reshape(len(bunch), Hk, G, T, -1), NEG)
        top = score.amax(-1, keepdim=True)
        p = torch.exp(score - torch.where(top == NEG, 0.0, top))
        total = p.sum(-1, keepdim=True)
        y = p.reshape(len(bunch), Hk, G * T, -1) @ v.transpose(1, 2).contiguous()
        y = y.reshape(len(bunch), Hk, G, T, d) / torch.where(total == 0, 1.0, total)
        y = y.permute(0, 3, 1, 2, 4).reshape(len(bunch), T, Hq, d).to(o.dtype)
        real = i < t[:, None]
        o[rows[real]] = y[real]
    return dict(o=o.reshape(s["q"].shape))


def _counts(table, lens, page, num):
    """References to each page from the rows of a table."""
    used = torch.arange(table.shape[1], device=table.device) * page < lens[:, None]
    return torch.bincount(table[used].long(), minlength=num).to(torch.int32)


def _extend_plain(s):
    table, lens, refs, page = s["table"], s["lens"], s["refs"], s["case"]["page"]
    add = s["add"].clamp(min=0)
    old = (lens + page - 1) // page
    need = (lens + add + page - 1) // page - old
    fits = old + need <= table.shape[1]
    free = torch.nonzero(refs == 0)[:, 0]
    wanted = torch.where(fits, need, 0)
    last = torch.cumsum(wanted, 0)
    served = fits & ((need == 0) | (last <= free.numel()))
    block = torch.arange(table.shape[1], device=table.device)
    fresh = served[:, None] & (block >= old[:, None]) & (block < (old + need)[:, None])
    order = (last - wanted)[:, None] + block - old[:, None]
    page_of = free[order[fresh].long()].to(torch.int32)
    table, refs = table.clone(), refs.clone()
    table[fresh] = page_of
    refs[page_of.long()] = 1
    return dict(table=table, lens=torch.where(served, lens + add, lens).to(torch.int32),
                refs=refs, short=torch.where(served, 0, need).to(torch.int32))


def _select_plain(s):
    table, lens, refs, page = s["table"], s["lens"], s["refs"], s["case"]["page"]
    S, num, parents = table.shape[0], refs.numel(), s["parents"].long()
    rows = torch.arange(S, device=table.device)
    real = (parents >= 0) & (parents < S)
    parent = torch.where(real, parents, 0)
    heir = torch.full((S,), S, device=table.device).scatter_reduce(
        0, parent[real], rows[real], "amin")  # the lowest child keeps the partial page
    n = torch.where(real, lens[parent], 0)
    copies = real & (n % page != 0) & (heir[parent] != rows)
    free = torch.nonzero(refs == 0)[:, 0]
    rank = torch.cumsum(copies, 0) - 1
    short = copies & (rank >= free.numel())
    copies, n = copies & ~short, torch.where(short, 0, n)
    used = torch.arange(table.shape[1], device=table.device) * page < n[:, None]
    out = torch.where(used, table[parent], -1)
    dst, block = free[rank[copies]], (n[copies] // page).long()
    src = out[copies, block].long()
    out[copies, block] = dst.to(torch.int32)
    s["pool"][:, dst] = s["pool"][:, src]
    n = n.to(torch.int32)
    refs = refs - _counts(table, lens, page, num) + _counts(out, n, page, num)
    return dict(table=out.to(torch.int32), lens=n, refs=refs, short=short.to(torch.int32),
                pool=s["pool"])


def _compact_plain(s):
    table, refs = s["table"], s["refs"]
    live = refs > 0
    count = int(live.sum())
    holes = torch.nonzero(~live[:count])[:, 0]
    late = torch.nonzero(live[count:])[:, 0] + count
    to = torch.where(live, torch.arange(refs.numel(), device=refs.device), -1)
    to[late] = holes
    used = (torch.arange(table.shape[1], device=table.device) * s["case"]["page"]
            < s["lens"][:, None])
    table = torch.where(used, to[table.clamp(min=0).long()], -1).to(torch.int32)
    moved = torch.zeros_like(refs)
    moved[to[live]] = refs[live]
    s["pool"][:, holes] = s["pool"][:, late]
    return dict(table=table, refs=moved, map=to.to(torch.int32), pool=s["pool"])


def run(state):
    s, case = state, state["case"]
    if own:
        return _run_own(s)
    if case["kind"] == "rotate":
        out, how = {}, (s["positions"], s["theta"], s["factor"], case["layout"])
        if case["way"] != "bwd":
            out["q"], out["k"] = _turn(s["q"], *how), _turn(s["k"], *how)
        if case["way"] != "fwd":
            out["dq"], out["dk"] = _turn(s["dq"], *how, -1.0), _turn(s["dk"], *how, -1.0)
        return out
    if case["kind"] == "append":
        return _append_plain(s)
    if case["kind"] == "attend":
        return _attend_plain(s)
    return dict(extend=_extend_plain, select=_select_plain, compact=_compact_plain)[case["op"]](s)


# ------------------------------------------------------------------ work


def work(case):
    """Bytes and FLOP of one pass: each input read once, each output written once (of the cache:
    the keys that some new token sees; of the pool: the pages that move)."""
    e = 4 if case["dtype"] == "f32" else 2
    if case["kind"] == "pages":
        rows, lens, refs, parents = _fragmented(case, 0)
        S, book = case["S"], 4 * (sum(len(r) for r in rows) + 2 * case["S"] + len(refs))
        page_bytes = case["parts"] * case["page"] * case["Hk"] * case["d"] * e
        moves = 0
        if case["op"] == "select":
            kept = [n for n in parents if lens[n] % case["page"]]
            moves = len(kept) - len(set(kept))
        if case["op"] == "compact":
            moves = sum(1 for r in refs[:sum(1 for r in refs if r)] if not r)
        return dict(bytes=2 * book + 2 * moves * page_bytes, flops=S)
    new, kv = _lengths(case)
    Hq, Hk, d, n = case["Hq"], case["Hk"], case["d"], sum(new)
    if case["kind"] == "rotate":
        ways = 2 if case["way"] == "both" else 1
        return dict(bytes=ways * n * (2 * (Hq + Hk) * d * e + 4),
                    flops=ways * n * (Hq + Hk) * 3 * case["rot"])
    if case["kind"] == "append":
        return dict(bytes=n * (2 * (Hq + 2 * Hk) * d * e + 4),
                    flops=n * (Hq + Hk) * 3 * case["rot"])
    w, keys, pairs = case["window"], 0, 0
    for m, c in zip(new, kv):
        keys += c - _first_key(case, m, c)
        if not w:
            pairs += m * (c - m) + m * (m + 1) // 2
        else:
            short = max(0, min(m, w - (c - m)))  # tokens that see fewer than w keys
            pairs += short * (c - m) + short * (short + 1) // 2 + (m - short) * w
    return dict(bytes=2 * n * Hq * d * e + 2 * keys * Hk * d * e, flops=4 * pairs * Hq * d)


# ------------------------------------------------------------------ 64 bits


def _exact_turn(x, positions, case, sign):
    theta, factor = _theta(case)
    angle = positions.double().reshape(-1, 1, 1) * theta.to(x.device)
    unit = torch.polar(torch.full_like(angle, factor), sign * angle)
    rot, y = case["rot"], x.double().reshape(-1, *x.shape[2:]).clone()
    part = y[..., :rot]
    pair = (part.reshape(*y.shape[:2], 2, rot // 2).transpose(2, 3)
            if case["layout"] == "halves" else part.reshape(*y.shape[:2], rot // 2, 2))
    z = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * unit)
    y[..., :rot] = (z.transpose(2, 3) if case["layout"] == "halves" else z).reshape(part.shape)
    return y.reshape(x.shape)


def exact(case, seed):
    """What run returns, in 64 bits: the rotation as a complex product, attention sequence by
    sequence and head by head.  The pages' whole numbers and copies have no such value."""
    if case["kind"] == "pages":
        return None
    s = _inputs(case, seed)
    if case["kind"] == "rotate":
        out = {}
        if case["way"] != "bwd":
            out.update({x: _exact_turn(s[x], s["positions"], case, 1.0) for x in ("q", "k")})
        if case["way"] != "fwd":
            out.update({x: _exact_turn(s[x], s["positions"], case, -1.0) for x in ("dq", "dk")})
        return out
    page, Hk, G = case["page"], case["Hk"], case["Hq"] // case["Hk"]
    if case["kind"] == "append":
        _, at = _places(s)
        q, k = _exact_turn(s["q"], at, case, 1.0), _exact_turn(s["k"], at, case, 1.0)
        kp, vp = s["k_pages"].double(), s["v_pages"].double()
        k, v, row = k.flatten(0, 1), s["v"].double().flatten(0, 1), 0
        for n, (m, c) in enumerate(zip(s["new"], s["kv"])):
            j = torch.arange(c - m, c, device=q.device)
            p = s["table"][n].long()[j // page]
            kp[p, :, j % page], vp[p, :, j % page] = k[row:row + m], v[row:row + m]
            row += m
        return dict(q=q, k_pages=kp, v_pages=vp)
    if work(case)["flops"] > 2e12:
        return None
    q, outs, row = s["q"].flatten(0, 1), [], 0
    for n, (m, c) in enumerate(zip(s["new"], s["kv"])):
        j = torch.arange(_first_key(case, m, c), c, device=q.device)
        p = s["table"][n].long()[j // page]
        k = s["k_pages"][p, :, j % page].double().transpose(0, 1)  # [Hk, keys, d]
        v = s["v_pages"][p, :, j % page].double().transpose(0, 1)
        for i in range(0, m, 1024):
            t = min(1024, m - i)
            at = torch.arange(c - m + i, c - m + i + t, device=q.device)[:, None]
            hide = j > at
            if case["window"]:
                hide |= j <= at - case["window"]
            x = q[row + i:row + i + t].double().reshape(t, Hk, G, -1)
            out = torch.empty_like(x)
            for h in range(Hk):
                for g in range(G):
                    score = (x[:, h, g] @ k[h].T / math.sqrt(case["d"])).masked_fill(hide, NEG)
                    out[:, h, g] = torch.softmax(score, -1) @ v[h]
            outs.append(out.reshape(t, Hk * G, -1))
        row += m
    return dict(o=torch.cat(outs).reshape(s["q"].shape))
