"""Plain 64-bit references of the attention layer, token by token, and the
cache layouts the tests build."""
import math
import random

import torch

F64 = torch.float64


def turn(x, positions, theta, layout, scale=1.0, sign=1.0):
    """Rotation of x [rows, H, d] (64 bits) at positions [rows]; theta [rot / 2] radians."""
    x = x.to(F64)
    y = x.clone()
    half = theta.numel()
    a = positions.to(F64)[:, None] * theta
    c, s = (torch.cos(a) * scale)[:, None], (torch.sin(a) * scale * sign)[:, None]
    i = torch.arange(half)
    p, q = (i, i + half) if layout == "halves" else (2 * i, 2 * i + 1)
    y[..., p] = x[..., p] * c - x[..., q] * s
    y[..., q] = x[..., q] * c + x[..., p] * s
    return y


class Case:
    """N sequences in pages: CPU tensors q [tokens, Hq, d], k_pages, v_pages [pages, Hk, page, d],
    table, kv_lens, cu.  What no token may see (free pages, slots past a sequence's end, blocks
    before its window) holds ``dead``; ``holes``: blocks whose table entry is -1."""

    def __init__(self, new, kv, Hq, Hk, d, page, dtype, window=0, causal=True, holes=(), seed=0,
                 dead=float("nan"), spare=3, std=1.0):
        self.__dict__.update(new=new, kv=kv, Hq=Hq, Hk=Hk, d=d, page=page, dtype=dtype,
                             window=window, causal=causal)
        gen = torch.Generator().manual_seed(seed)
        rng = random.Random(seed)
        N = len(new)
        self.q = (torch.randn(sum(new), Hq, d, generator=gen) * std).to(dtype)
        width = max(1, max(-(-c // page) for c in kv)) + 1
        table = torch.full((N, width), -1, dtype=torch.int32)
        want = []
        for n in range(N):
            first = max(0, kv[n] - new[n] + 1 - window) // page if window else 0
            for b in range(first, -(-kv[n] // page)):
                if (n, b) not in holes:
                    want.append((n, b))
        order = list(range(len(want) + spare))
        rng.shuffle(order)
        self.k_pages = torch.full((len(order), Hk, page, d), dead, dtype=dtype)
        self.v_pages = torch.full((len(order), Hk, page, d), dead, dtype=dtype)
        for (n, b), p in zip(want, order):
            table[n, b] = p
            m = min(page, kv[n] - b * page)
            self.k_pages[p, :, :m] = torch.randn(Hk, m, d, generator=gen).to(dtype)
            self.v_pages[p, :, :m] = torch.randn(Hk, m, d, generator=gen).to(dtype)
        self.table, self.kv_lens = table, torch.tensor(kv, dtype=torch.int32)
        self.cu = torch.tensor([0] + new).cumsum(0).to(torch.int32)

    def visible(self, n, i):
        """Keys that new token i of sequence n sees."""
        pos = self.kv[n] - self.new[n] + i
        hi = min(self.kv[n], pos + 1) if self.causal else self.kv[n]
        lo = max(0, pos - self.window + 1) if self.window else 0
        return [j for j in range(lo, hi) if 0 <= self.table[n, j // self.page]]

    def attend(self, scale=None):
        """(o [tokens, Hq, d], lse [tokens, Hq], bound on the error of a 32-bit evaluation per
        output, of its sum of p |v|) in 64 bits."""
        scale = self.d ** -0.5 if scale is None else scale
        G, d = self.Hq // self.Hk, self.d
        o = torch.zeros(self.q.shape, dtype=F64)
        lse = torch.full(self.q.shape[:2], -math.inf, dtype=F64)
        mass = torch.zeros(self.q.shape, dtype=F64)
        rel = torch.zeros(self.q.shape[:2], dtype=F64)
        row = 0
        for n, m in enumerate(self.new):
            for i in range(m):
                j = torch.tensor(self.visible(n, i), dtype=torch.long)
                if len(j):
                    p, s = self.table[n].long()[j // self.page], j % self.page
                    k = self.k_pages[p, :, s].to(F64).repeat_interleave(G, 1)  # [keys, Hq, d]
                    v = self.v_pages[p, :, s].to(F64).repeat_interleave(G, 1)
                    q = self.q[row].to(F64)
                    x = (q * k).sum(-1) * scale  # [keys, Hq]
                    lse[row] = torch.logsumexp(x, 0)
                    w = torch.softmax(x, 0)
                    o[row] = (w[..., None] * v).sum(0)
                    mass[row] = (w[..., None] * v.abs()).sum(0)
                    # a score's error: d products and sums, its scaling and the rounding of the
                    # exponent's argument; it enters a weight twice (itself and the sum)
                    big = ((q * k).abs().sum(-1) * scale).amax(0)
                    rel[row] = 2 * (d + 8) * 2.0 ** -24 * (big + 1) + (len(j) + 16) * 2.0 ** -24
                row += 1
        return o, lse, rel, mass

    def bound(self, rel, mass):
        """Error allowed to each output: 32-bit evaluation; in bfloat16 also p and o rounded (8
        significant bits: 2^-8 relative each), and an absolute floor of a denormal."""
        out = rel[..., None] * mass
        if self.dtype is torch.bfloat16:
            out = out + 2 * 2.0 ** -8 * mass * 1.01
        return out + 1e-30
