"""Decoding of a batch over a cache in pages with a budget, the calls of this library around a model of random weights.

    python -m paper_2604_02047_b200.paged_prompt [--sequences 8] [--prompt 3000] [--tokens 64] [--draft 8] [--budget 1024]

Prompts go through in chunks of any length, drafts as chains behind the last token (the continuation that context_match finds), and a
cache that has grown beyond its budget loses its lightest rows:

    append_kv_paged    norm and rotation of the chunk's queries and keys, its K / V rows into pages, weights and positions of the new rows
    chunk_attn         attention over the sequence's rows and causally over the chunk's own                            (every layer)
    node_topk, accept  greedy token of every draft token, how many of them it confirms
    kv_weights         what the confirmed tokens looked at, added to the rows' weights                                 (every layer)
    evict_kv           back to the budget: first rows, latest rows, heaviest others; the pages behind it are free again  (every layer)

Sequences take pages from a pool when they grow.  All layers use one page table; rows that are evicted differ by layer and head.
"""
from __future__ import annotations

import argparse
import time

import numpy as np
import torch

from . import binding
from .shared_prompt import D, Model


class Batch:
    """``prompts``: a token at least each, as many as the model has positions for, the last one is the first chunk's anchor.  ``rows``: rows of the pool, of all sequences together.
    ``budget``: rows that a sequence keeps when it has ``slack`` more than that (None: no eviction)."""

    def __init__(self, goose: binding.Goose, model: Model, prompts, rows: int, page: int = 16, chunk: int = 512, draft: int = 8,
                 budget=None, sink: int = 4, recent: int = 64, slack: int = 64):
        if not prompts or not all(len(p) for p in prompts):
            raise ValueError("a batch has sequences, and each of them a token")
        if max(len(p) for p in prompts) - 1 > len(model.rope):
            raise ValueError("a prompt of %d tokens: positions up to %d" % (max(len(p) for p in prompts), len(model.rope)))
        if draft + 1 > goose.max_B:
            raise ValueError("a draft of %d tokens and its anchor: a context of %d nodes" % (draft, goose.max_B))
        if budget is not None and sink + recent > budget:
            raise ValueError("%d first and %d latest rows in a budget of %d" % (sink, recent, budget))
        self.g, self.m, self.S, self.page, self.B = goose, model, len(prompts), page, draft + 1
        self.budget, self.sink, self.recent, self.slack = budget, sink, recent, slack
        self.free = list(range(-(-rows // page)))[::-1]
        pages = len(self.free)
        # entries of a sequence's part of the table: the whole pool, or what a budget, what it may be beyond that and a chunk need
        most = pages if budget is None else -(-(budget + slack + max(chunk, self.B)) // page)
        self.width = min(pages, most, binding.MAX_PAGED_ROWS // page)
        self.table = np.full((self.S, self.width), -1, np.int32)
        self.owned = [0] * self.S                              # pages of a sequence
        shape = (pages, page, model.kv_heads, D)
        self.caches = [(torch.zeros(shape, dtype=torch.bfloat16, device="cuda"), torch.zeros(shape, dtype=torch.bfloat16, device="cuda"))
                       for _ in range(model.layers)]
        # weights and positions of the rows, which eviction goes by
        room, layers = (self.S, model.kv_heads, self.width * page), range(model.layers)
        self.weight = [None if budget is None else torch.zeros(room, device="cuda") for _ in layers]
        self.pos = [None if budget is None else torch.zeros(room, dtype=torch.int32, device="cuda") for _ in layers]
        self.ctx = np.zeros(self.S, np.int32)                  # rows of a sequence, and what has left it
        self.off = np.zeros(self.S, np.int32)
        self.tokens = [list(p) for p in prompts]               # the last one of each has no row yet
        self.chains = torch.arange(-1, draft, dtype=torch.int32, device="cuda").expand(self.S, self.B).contiguous()
        lens = np.array([len(p) - 1 for p in prompts])
        for at in range(0, int(lens.max()), chunk):
            n = np.clip(lens - at, 0, chunk).astype(np.int32)
            part = np.zeros((self.S, int(n.max())), np.int32)
            for s, p in enumerate(prompts):
                part[s, :n[s]] = p[at:at + n[s]]
            _, seen = self._forward(part, n)
            self._keep(seen, n)

    def _dev(self, a):
        return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()

    def _pages(self, n):
        """Pages for n more rows of every sequence."""
        for s in range(self.S):
            need = -(-(int(self.ctx[s]) + int(n[s])) // self.page) if n[s] else self.owned[s]
            if need > self.width or need - self.owned[s] > len(self.free):
                raise ValueError("no room for %d more tokens of sequence %d" % (n[s], s))
            while self.owned[s] < need:
                self.table[s, self.owned[s]] = self.free.pop()
                self.owned[s] += 1
        return self._dev(self.table)

    def _forward(self, tokens, n_new):
        """Logits of a chunk, and what kv_weights needs of its layers."""
        most = int((np.where(n_new > 0, self.off + self.ctx, 0) + n_new).max())
        if most > len(self.m.rope):
            raise ValueError("%d tokens of a sequence: positions up to %d" % (most, len(self.m.rope)))
        table, ctx, off, n = self._pages(n_new), self._dev(self.ctx), self._dev(self.off), self._dev(n_new)
        seen = []

        def attention(i, q, k, v):
            kc, vc = self.caches[i]
            q = self.g.append_kv_paged(q, k, v, kc, vc, table, ctx, rope=self.m.rope, n_new=n, pos_off=off, q_weight=self.m.norms[i][0],
                                       k_weight=self.m.norms[i][1], row_weight=self.weight[i], row_pos=self.pos[i])
            # (rows of tokens that do not exist stay as they are: zeros for the layers behind)
            out, lse = self.g.chunk_attn(q, kc, vc, table, ctx, self.m.scale, out=torch.zeros_like(q), want_lse=True, n_new=n)
            seen.append((q, lse))
            return out

        return self.m.forward(self._dev(tokens), attention), (table, ctx, seen)

    def _keep(self, state, kept):
        """The first ``kept`` tokens of the chunk stay; back to the budget where a sequence is beyond it."""
        table, ctx, seen = state
        if self.budget is not None:
            for i, (q, lse) in enumerate(seen):
                self.g.kv_weights(q, lse, self.caches[i][0], table, ctx, self.m.scale, self.weight[i], n_new=self._dev(kept))
        self.ctx = self.ctx + kept.astype(np.int32)
        if self.budget is None or int(self.ctx.max()) <= self.budget + self.slack:
            return
        ctx, off = self._dev(self.ctx), self._dev(self.off)
        for i, (kc, vc) in enumerate(self.caches):
            new = self.g.evict_kv(kc, vc, table, ctx, self.weight[i], self.pos[i], self.budget, self.sink, self.recent, pos_off=off)
            self.weight[i], self.pos[i] = new[2], new[3]
        self.off = self.off + np.maximum(self.ctx - self.budget, 0)
        self.ctx = np.minimum(self.ctx, self.budget)
        for s in range(self.S):
            need = -(-int(self.ctx[s]) // self.page)
            self.free.extend(self.table[s, need:self.owned[s]][::-1].tolist())
            self.table[s, need:self.owned[s]] = -1
            self.owned[s] = min(self.owned[s], need)

    def step(self, live):
        """A chain behind the last token of every sequence that is ``live``; what the model confirms of it, and its own next token."""
        draft, n = np.full((self.S, self.B), -1, np.int32), np.zeros(self.S, np.int32)
        for s in range(self.S):
            if live[s]:
                left = len(self.m.rope) - int(self.off[s] + self.ctx[s]) - 1   # positions behind the last token's
                chain, _ = binding.context_match(self.tokens[s], max(min(self.B - 1, left), 0))
                n[s] = 1 + len(chain)
                draft[s, :n[s]] = [self.tokens[s][-1]] + list(chain)
        logits, state = self._forward(draft, n)
        n_new, tok = self._dev(n), self._dev(draft)
        argmax, _, _ = self.g.node_topk(logits, 1, n_nodes=n_new, B=self.B)
        _, accepted, bonus = self.g.accept(tok, self.chains, argmax, n_nodes=n_new)
        accepted, bonus = accepted.cpu().numpy(), bonus.cpu().numpy()
        kept = np.where(n > 0, accepted + 1, 0)
        self._keep(state, kept)
        for s in range(self.S):
            if live[s]:
                self.tokens[s].extend(draft[s, 1:kept[s]].tolist() + [int(bonus[s])])


def decode(batch: Batch, tokens: int):
    """``tokens`` more tokens a sequence (ValueError where there are no positions for them).  Returns (the sequences, steps)."""
    most = max(len(t) for t in batch.tokens) + tokens - 1      # rows of the longest, when its last token is chosen
    if most > len(batch.m.rope):
        raise ValueError("%d more tokens: positions up to %d" % (tokens, len(batch.m.rope)))
    want, steps = [len(t) + tokens for t in batch.tokens], 0
    while True:
        live = [len(t) < w for t, w in zip(batch.tokens, want)]
        if not any(live):
            return [t[:w] for t, w in zip(batch.tokens, want)], steps
        batch.step(live)
        steps += 1


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--sequences", type=int, default=8)
    ap.add_argument("--prompt", type=int, default=3000, help="tokens of the longest prompt")
    ap.add_argument("--tokens", type=int, default=64, help="tokens to decode for every sequence")
    ap.add_argument("--draft", type=int, default=8, help="drafted tokens of a step, at most")
    ap.add_argument("--budget", type=int, default=1024, help="rows that a sequence keeps; 0: all")
    a = ap.parse_args()
    rng = np.random.default_rng(0)
    model = Model()
    goose = binding.Goose(max_S=a.sequences, max_B=a.draft + 1, max_H=model.heads)
    prompts = [rng.integers(0, model.vocab, int(n)).tolist() for n in rng.integers(max(a.prompt // 4, 1), a.prompt + 1, a.sequences)]
    rows = a.sequences * (a.prompt + a.tokens + 1024 if a.budget == 0 else a.budget + 1024)
    torch.cuda.synchronize()
    began = time.perf_counter()
    batch = Batch(goose, model, prompts, rows, draft=a.draft, budget=a.budget or None)
    torch.cuda.synchronize()
    ready = time.perf_counter()
    out, steps = decode(batch, a.tokens)
    torch.cuda.synchronize()
    print("%d prompts of up to %d tokens in %.1f ms; %d tokens each in %d steps, %.2f ms a step (drafting on the host included); %d rows a sequence at most" %
          (a.sequences, a.prompt, 1e3 * (ready - began), a.tokens, steps, 1e3 * (time.perf_counter() - ready) / max(steps, 1), int(batch.ctx.max())))
    assert not goose.last_status(a.sequences).any()
    goose.close()


if __name__ == "__main__":
    main()
