"""Serving a small hybrid model: gated delta rule layers beside window attention.

    python examples/hybrid_serving.py

A stack of random weights that alternates the rule (gdn_chunk_fwd for prompts,
gdn_recurrent_fwd for single tokens) with sliding-window attention over a paged
cache (gdn_cache_append, gdn_cache_attn).  ``Server`` keeps, for each of S rows, a
sequence's pages and recurrent states, and shows the calls in the order in which a
serving program makes them: pages for a prompt, the prompt in one packed call,
single tokens, rows that go on from other rows (gdn_pages_select, and
gdn_pages_copy for the states), pages that left the window, and a compacted cache.
``Server.answers`` draws many answers to one prompt: its tokens in one call, a fork for every
row, single tokens whose attention computes the prompt's part once for all rows
(gdn_cache_attn_shared), and gdn_sample for the next ones.  With ``linear`` each pair is led
by a layer of linear attention with a decay (gdn_linear_chunk_fwd,
gdn_linear_recurrent_fwd).  Projections and normalisations are plain torch.
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2412_06464_amd import gdn, linear, paged, sample  # noqa: E402


class HybridModel:
    """Weights and sizes: ``layers`` pairs of a rule layer and an attention layer (``window`` 0:
    over all earlier tokens), with ``linear`` a layer of linear attention before each."""

    def __init__(self, vocab=211, width=256, layers=2, heads=4, d=64, q_heads=4, kv_heads=2,
                 window=96, seed=0, device="cuda", dtype=torch.bfloat16, linear=False):
        g = torch.Generator().manual_seed(seed)
        self.__dict__.update(vocab=vocab, width=width, layers=layers, heads=heads, d=d,
                             q_heads=q_heads, kv_heads=kv_heads, window=window, device=device,
                             dtype=dtype)

        def weight(n, m):
            return (torch.randn(n, m, generator=g) / n ** 0.5).to(device, dtype)

        self.embed = torch.randn(vocab, width, generator=g).to(device, dtype)
        self.rule = [dict(qkv=weight(width, 3 * heads * d), gates=weight(width, 2 * heads).float(),
                          out=weight(heads * d, width)) for _ in range(layers)]
        self.attn = [dict(qkv=weight(width, (q_heads + 2 * kv_heads) * d),
                          out=weight(q_heads * d, width)) for _ in range(layers)]
        self.head = weight(width, vocab)
        self.linear = [dict(qkv=weight(width, 3 * heads * d),
                            gates=weight(width, 2 * heads).float(), out=weight(heads * d, width))
                       for _ in range(layers if linear else 0)]
        self.rotary = paged.gdn_rotary(d, base=10000.0, device=device)

    @staticmethod
    def norm(x):
        x = x.float()
        return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6)

    def rule_inputs(self, w, x):
        """q, k (unit length), v and the gates of rows x [B, T, width]."""
        B, T, _ = x.shape
        y = self.norm(x)
        qkv = (y.to(self.dtype) @ w["qkv"]).reshape(B, T, 3, self.heads, self.d)
        q, k = (torch.nn.functional.normalize(qkv[:, :, i].float(), dim=-1).to(self.dtype)
                for i in (0, 1))
        gates = (y @ w["gates"]).reshape(B, T, 2, self.heads)
        return (q, k, qkv[:, :, 2].contiguous(), torch.sigmoid(gates[:, :, 0]).contiguous(),
                -torch.nn.functional.softplus(gates[:, :, 1]).contiguous())


class Server:
    """S rows of sequences, their pages, and the recurrent states (two sets of S: rows move
    from one to the other when they are selected)."""

    def __init__(self, model, S=8, page_size=16, num_pages=96, max_tokens=512):
        m, dev = model, model.device
        self.m, self.S, self.page = m, S, page_size
        self.blocks = -(-max_tokens // page_size)
        self.cache = torch.zeros(m.layers, 2, num_pages, m.kv_heads, page_size, m.d, dtype=m.dtype,
                                 device=dev)
        # the rules' first, then those of linear attention
        self.states = torch.zeros(m.layers + len(m.linear), 2 * S, m.heads, m.d, m.d, device=dev)
        self.side = self.prefix = 0  # (prefix: tokens that all rows begin with)
        self.table = torch.full((S, self.blocks), -1, dtype=torch.int32, device=dev)
        self.lens = torch.zeros(S, dtype=torch.int32, device=dev)
        self.refs = torch.zeros(num_pages, dtype=torch.int32, device=dev)

    def _book(self, out):
        self.table, self.refs = out["table"], out["refs"]
        self.lens = out.get("lens", self.lens)

    def _grow(self, add):
        """Pages for add[s] more tokens a row; if they do not last, nothing has changed."""
        out = paged.gdn_pages_extend(self.table, self.lens, self.refs, add, page_size=self.page)
        short = torch.nonzero(out["short"])[:, 0].tolist()
        if short:
            raise RuntimeError("no pages left for rows %s" % short)
        self._book(out)

    def _release(self):
        """Drops the pages that lie whole before every later token's window: their entries become
        holes, which later calls neither read nor store to.  On the device, with no copy back."""
        if not self.m.window:
            return
        first = self.lens + 1 - self.m.window  # the first key that a row's next token sees
        end = torch.arange(1, self.blocks + 1, dtype=torch.int32, device=first.device) * self.page
        gone = (self.table >= 0) & (end <= first[:, None])
        page = self.table.clamp(min=0).flatten().long()
        self.refs = self.refs.scatter_add(0, page, -gone.flatten().to(torch.int32))
        self.table = torch.where(gone, -1, self.table)

    def _state(self, layer):
        return self.states[layer, self.side * self.S:(self.side + 1) * self.S]

    def _attend(self, q, k_pages, v_pages, cu):
        window = self.m.window
        if self.prefix:
            return paged.gdn_cache_attn_shared(q, k_pages, v_pages, self.table, self.lens,
                                               self.table[0], self.prefix, window=window, **cu)
        return paged.gdn_cache_attn(q, k_pages, v_pages, self.table, self.lens, window=window, **cu)

    def _layers(self, x, rule, cu, decayed):
        """x [B, T, width] (in 32 bits, as the sum of what the layers add: where a head's output
        nearly cancels, its normalisation magnifies what x is off by) through the stack;
        ``rule(layer, inputs)`` applies the rule,
        ``decayed(layer, q, k, v, log_alpha)`` linear attention."""
        m = self.m
        for i in range(m.layers):
            if m.linear:
                w = m.linear[i]
                q, k, v, _, log_alpha = m.rule_inputs(w, x)
                o = decayed(m.layers + i, q, k, v, log_alpha)
                x = x + m.norm(o).to(m.dtype).flatten(2) @ w["out"]
            w = m.rule[i]
            o = rule(i, m.rule_inputs(w, x))
            x = x + m.norm(o).to(m.dtype).flatten(2) @ w["out"]
            w = m.attn[i]
            qkv = (m.norm(x).to(m.dtype) @ w["qkv"]).unflatten(-1, (-1, m.d))
            q, k, v = qkv.split((m.q_heads, m.kv_heads, m.kv_heads), dim=2)  # slices, as they are
            k_pages, v_pages = self.cache[i, 0], self.cache[i, 1]
            q = paged.gdn_cache_append(q, k, v, k_pages, v_pages, self.table, self.lens, m.rotary,
                                       **cu)
            o = self._attend(q, k_pages, v_pages, cu)
            x = x + o.flatten(2) @ w["out"]
        self._release()
        return m.norm(x).to(m.dtype) @ m.head

    def prefill(self, prompts):
        """Takes a list of S token lists (empty: the row is left alone) in one packed call; the
        rows' logits after their last tokens.  Rows that had tokens go on from them."""
        m = self.m
        n = torch.tensor([len(p) for p in prompts], dtype=torch.int32)
        self._grow(n.to(m.device))
        host = torch.cat([torch.zeros(1, dtype=torch.int32), n.cumsum(0).to(torch.int32)])
        cu = dict(cu_seqlens=host.to(m.device), cu_seqlens_host=host)
        ids = torch.tensor([t for p in prompts for t in p], device=m.device)

        def rule(i, x):
            state = self._state(i)
            return gdn.gdn_chunk_fwd(*x, h0=state, ht=state, **cu)[0]

        def decayed(i, *x):
            state = self._state(i)
            return linear.gdn_linear_chunk_fwd(*x, h0=state, ht=state, **cu)[0]

        logits = self._layers(m.embed[ids][None].float(), rule, cu, decayed)[0]
        last = (host[1:] - 1).clamp(min=0).long()
        return logits[last.to(m.device)]

    def decode(self, ids):
        """One token a row (ids [S], a row without a sequence takes one too); logits [S, vocab]."""
        m = self.m
        self._grow(torch.ones_like(self.lens))

        def rule(i, x):
            state = self._state(i)
            return gdn.gdn_recurrent_fwd(*x, h0=state, ht=state)[0]

        def decayed(i, *x):
            state = self._state(i)
            return linear.gdn_linear_recurrent_fwd(*x, h0=state, ht=state)[0]

        return self._layers(m.embed[ids][:, None].float(), rule, {}, decayed)[:, 0]

    def answers(self, prompt, count, temperature=0.8, top_k=50, top_p=0.95, generator=None):
        """S answers of ``count`` tokens to a prompt (a list), on a server without sequences:
        their tokens [S, count] and log probabilities."""
        S, dev = self.S, self.m.device
        rows = dict(temperature=torch.full((S,), temperature, device=dev),
                    top_k=torch.full((S,), top_k, dtype=torch.int32, device=dev),
                    top_p=torch.full((S,), top_p, device=dev))
        logits = self.prefill([prompt] + [[]] * (S - 1))[:1].expand(S, -1)
        if self.select([0] * S).any():  # every row a fork of the first, on the same full pages
            raise RuntimeError("no pages left for the answers")
        # the prompt's full pages are the same in every row
        self.prefix = 0 if self.m.window else len(prompt) // self.page * self.page
        tokens, logprobs = [], []
        try:
            for step in range(count):
                if step:
                    logits = self.decode(tokens[-1])
                u = torch.rand(S, device=dev, generator=generator)
                token, logprob = sample.gdn_sample(logits, u, **rows)
                tokens.append(token)
                logprobs.append(logprob)
        finally:
            self.prefix = 0  # (rows may go their own ways from here)
        return torch.stack(tokens, 1), torch.stack(logprobs, 1)

    def select(self, parents):
        """Row i goes on from row parents[i] (-1: it ends)."""
        parents = torch.tensor(parents, dtype=torch.int32, device=self.m.device)
        out = paged.gdn_pages_select(self.table, self.lens, self.refs, parents,
                                     page_size=self.page, pool=self.cache.flatten(0, 1))
        self._book(out)
        src = torch.where(parents >= 0, parents + self.side * self.S, -1).to(torch.int32)
        self.side ^= 1
        rows = torch.arange(self.S, dtype=torch.int32, device=self.m.device) + self.side * self.S
        paged.gdn_pages_copy(self.states, src, rows)
        self.states[:, self.side * self.S:(self.side + 1) * self.S][:, parents < 0] = 0
        return out["short"]

    def compact(self):
        """The pages in use into the lowest indexes; how many they are."""
        self._book(paged.gdn_pages_compact(self.table, self.lens, self.refs, page_size=self.page,
                                           pool=self.cache.flatten(0, 1)))
        return int((self.refs > 0).sum())


def main():
    torch.manual_seed(0)
    server = Server(HybridModel())
    prompts = [torch.randint(0, 211, (n,)).tolist() for n in (70, 1, 33, 150)] + [[]] * 4
    ids = server.prefill(prompts).argmax(-1)
    server.select([0, 0, 1, 2, 3, 3, 3, -1])  # forks of rows 0 and 3, the last row stays empty
    ids = ids[torch.tensor([0, 0, 1, 2, 3, 3, 3, 0], device="cuda")]
    for step in range(24):
        logits = server.decode(ids)
        ids = logits.topk(2).indices[torch.arange(8), torch.arange(8) % 2]  # forks differ
    print("lengths", server.lens.tolist())
    print("pages in use", int((server.refs > 0).sum()))
    server.select([4, -1, -1, 3, -1, -1, -1, -1])
    print("after ending six rows", server.compact())
    print("next", server.decode(ids)[[0, 3]].argmax(-1).tolist())

    server = Server(HybridModel(window=0, linear=True))
    tokens, logprobs = server.answers(prompts[3], 12)
    print("answers", tuple(tokens.shape), "of log probability", logprobs.sum(1).tolist())


if __name__ == "__main__":
    main()
