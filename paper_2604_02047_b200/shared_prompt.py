"""Decoding of a batch under a shared system prompt, the calls of this library around a model of random weights.

    python -m paper_2604_02047_b200.shared_prompt [--sequences 8] [--prompt 1000] [--tokens 64] [--nodes 32]

A step of the loop (Algorithm 2 for a batch whose sequences share their first rows of the cache):

    append_kv          norm and rotation of the tree nodes' queries and keys, their K / V rows behind each sequence's own
    tree_attn_shared   attention over the shared rows, the sequence's own and the node's ancestors      (every layer)
    adjust_logits      penalties over the sequence's tokens and the node's path, a mask of reserved tokens
    node_topk, accept  greedy token of every node, longest accepted path
    kv_compact         accepted rows behind the sequence's own                                          (every layer)
    append_tokens      accepted tokens behind the sequence's history

The drafts come from the host routines (context match, spine tree) and from what node_topk harvested.  The model (embeddings, projections)
is plain torch: it stands for whatever model a program has.
"""
from __future__ import annotations

import argparse
import time

import numpy as np
import torch

from . import binding, synth

D = binding.HEAD_DIM
CHUNK = 128                                            # nodes of a tree: a prompt goes through in chains of that many


class Model:
    """Attention layers of random weights: x += Wo attention(norm, rotation of Wqkv x); logits = x E^T."""

    def __init__(self, vocab: int = 4096, width: int = 512, layers: int = 2, heads: int = 8, kv_heads: int = 2, positions: int = 8192, seed: int = 0):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def weight(*shape, scale=1.0):
            return (torch.randn(shape, generator=g, device="cuda") * scale).bfloat16()

        self.vocab, self.heads, self.kv_heads, self.layers = vocab, heads, kv_heads, layers
        self.embed = weight(vocab, width)
        self.qkv = [weight(width, (heads + 2 * kv_heads) * D, scale=width ** -0.5) for _ in range(layers)]
        self.out = [weight(heads * D, width, scale=(heads * D) ** -0.5) for _ in range(layers)]
        self.norms = [(1 + weight(D, scale=0.1), 1 + weight(D, scale=0.1)) for _ in range(layers)]
        angle = torch.arange(positions, device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (
            -torch.arange(0, D, 2, device="cuda", dtype=torch.float64) / D)
        self.rope = torch.cat([torch.cos(angle), torch.sin(angle)], 1).float().contiguous()
        self.scale = D ** -0.5

    def forward(self, tokens, layer_attention):
        """Logits [S*B][V] of tokens [S][B]; layer_attention(layer, q, k, v) does the cache and the attention."""
        S, B = tokens.shape
        x = self.embed[tokens.long().clamp(min=0)]
        for i in range(self.layers):
            qkv = (x @ self.qkv[i]).view(S, B, self.heads + 2 * self.kv_heads, D)
            q, k, v = qkv.split([self.heads, self.kv_heads, self.kv_heads], 2)
            x = x + layer_attention(i, q, k, v).reshape(S, B, -1) @ self.out[i]
        return (x.view(S * B, -1) @ self.embed.T) * (x.shape[-1] ** -0.5)


class Batch:
    """The caches of all layers (the shared rows first, then every sequence's own), the sequences' lengths and tokens.  ``sequences``: each one's own
    prompt, a token at least (its last is the first tree's anchor); ``room``: tokens of its own that a sequence may have."""

    def __init__(self, goose: binding.Goose, model: Model, prompt, sequences, room: int, nodes: int, reserved: int = 16):
        if not sequences or not all(len(own) for own in sequences):
            raise ValueError("a batch has sequences, and each of them a token of its own")
        self.g, self.m, self.S, self.B, self.room = goose, model, len(sequences), nodes, room
        self.shared = len(prompt)
        rows = self.shared + self.S * (room + CHUNK)
        shape = (rows, model.kv_heads, D)
        self.caches = [(torch.zeros(shape, dtype=torch.bfloat16, device="cuda"), torch.zeros(shape, dtype=torch.bfloat16, device="cuda"))
                       for _ in range(model.layers)]
        dev = lambda a, t=torch.int32: torch.tensor(np.asarray(a), dtype=t, device="cuda")  # noqa: E731
        self.row_off = dev(self.shared + np.arange(self.S) * (room + CHUNK), torch.int64)
        self.ctx_len = dev(np.zeros(self.S))
        self.pos_off = dev(np.full(self.S, self.shared))
        # a sequence's tokens: the shared prompt's, its own prompt's, what was accepted
        self.hist = dev(np.zeros((self.S, self.shared + room + nodes)))
        self.hist_len = dev([self.shared + len(s) - 1 for s in sequences])
        self.n_prompt = dev([self.shared + len(s) for s in sequences])
        for s, own in enumerate(sequences):
            self.hist[s, :self.shared + len(own)] = dev(list(prompt) + list(own))
        words = (model.vocab + 31) // 32
        mask = np.zeros(words * 32, np.uint8)
        mask[:model.vocab - reserved] = 1
        self.mask = torch.from_numpy(np.packbits(mask, bitorder="little").view(np.int32)).cuda().expand(self.S * nodes, words).contiguous()
        one = lambda v: torch.full((self.S,), v, dtype=torch.float32, device="cuda")  # noqa: E731
        self.penalties = dict(repetition=one(1.1), frequency=one(0.05), presence=one(0.1))
        self._shared_prompt(prompt, dev)
        self._own_prompts(sequences, dev)

    def _shared_prompt(self, prompt, dev):
        zero = dev([0], torch.int64)
        for at in range(0, self.shared, CHUNK):
            part = dev([prompt[at:at + CHUNK]])
            chain = dev([synth.chain_tree(part.shape[1])])
            ctx = dev([at])

            def attention(i, q, k, v):
                kc, vc = self.caches[i]
                q = self.g.append_kv(q, k, v, kc, vc, zero, ctx, rope=self.m.rope, q_weight=self.m.norms[i][0], k_weight=self.m.norms[i][1])
                return self.g.tree_attn_gqa(q, kc, vc, zero, ctx, chain, self.m.scale)[0]

            self.m.forward(part, attention)

    def _own_prompts(self, sequences, dev):
        """All tokens of a sequence's own prompt but the last, which is the first tree's anchor."""
        lens = np.array([len(s) - 1 for s in sequences])
        for at in range(0, int(lens.max()), CHUNK):
            n = np.clip(lens - at, 0, CHUNK)
            part = np.zeros((self.S, int(n.max())), np.int32)
            for s, own in enumerate(sequences):
                part[s, :n[s]] = own[at:at + n[s]]
            chains = dev(np.tile(synth.chain_tree(part.shape[1]), (self.S, 1)))
            self.m.forward(dev(part), self._attention(chains, dev(n)))
            self.ctx_len = self.ctx_len + dev(n)

    def _attention(self, parent, n_nodes):
        def attention(i, q, k, v):
            kc, vc = self.caches[i]
            q = self.g.append_kv(q, k, v, kc, vc, self.row_off, self.ctx_len, rope=self.m.rope, parent=parent, n_nodes=n_nodes,
                                 pos_off=self.pos_off, q_weight=self.m.norms[i][0], k_weight=self.m.norms[i][1])
            return self.g.tree_attn_shared(q, kc, vc, 0, self.shared, self.row_off, self.ctx_len, parent, self.m.scale, n_nodes=n_nodes)
        return attention

    def step(self, draft_tok, parent, n_nodes, k: int = 8):
        """One verified tree a sequence.  Returns (argmax, top-k ids, path, accepted nodes, bonus token); no host round trip."""
        logits = self.m.forward(draft_tok, self._attention(parent, n_nodes))
        self.g.adjust_logits(logits, self.hist, self.hist_len, draft_tok, parent, n_nodes=n_nodes, n_prompt=self.n_prompt, mask=self.mask,
                             out=logits, **self.penalties)
        argmax, ids, _ = self.g.node_topk(logits, k, n_nodes=n_nodes, B=self.B)
        path, accepted, bonus = self.g.accept(draft_tok, parent, argmax, n_nodes=n_nodes)
        for kc, vc in self.caches:
            new_ctx = self.g.kv_compact(kc, vc, self.row_off, self.ctx_len, path, accepted, n_nodes=n_nodes)
        self.hist_len = self.g.append_tokens(draft_tok, path, accepted, self.hist, self.hist_len, n_nodes=n_nodes)
        self.ctx_len = new_ctx
        return argmax, ids, path, accepted, bonus


def decode(batch: Batch, tokens: int, k: int = 8):
    """``tokens`` more tokens a sequence (ValueError where they do not fit).  Returns (the sequences' tokens behind the shared prompt, steps)."""
    S, B, V = batch.S, batch.B, batch.m.vocab
    table = np.full((V, k), -1, np.int32)                    # successors seen in earlier steps
    start = batch.hist_len.cpu().numpy()
    # in front of the last step a sequence has tokens - 1 new ones, and a tree of B nodes behind them
    most = int(start.max()) + tokens - 1
    if most - batch.shared > batch.room or most + B > len(batch.m.rope):
        raise ValueError("%d more tokens: room for %d of a sequence's own, positions up to %d" % (tokens, batch.room, len(batch.m.rope)))
    anchor = batch.hist[torch.arange(S), batch.hist_len.long()].cpu().numpy()
    steps = 0
    while True:
        hist, length = batch.hist.cpu().numpy(), batch.hist_len.cpu().numpy()
        done = length - start >= tokens
        if done.all():
            return [np.append(hist[s, batch.shared:length[s]], anchor[s])[:start[s] - batch.shared + 1 + tokens] for s in range(S)], steps
        draft, parent, nodes = np.full((S, B), -1, np.int32), np.zeros((S, B), np.int32), np.zeros(S, np.int32)
        for s in range(S):
            if not done[s]:
                chain, _ = binding.context_match(np.append(hist[s, :length[s]], anchor[s]), B)
                tok, par, _, n, _ = binding.build_spine_tree(int(anchor[s]), chain, table, B, 6, 0.5, 0.5)
                draft[s, :n], parent[s, :n], nodes[s] = tok, par, n
        dev = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
        argmax, ids, path, accepted, bonus = batch.step(dev(draft), dev(parent), dev(nodes), k)
        ids, bonus = ids.cpu().numpy().reshape(S, B, k), bonus.cpu().numpy()
        for s in range(S):
            if nodes[s]:
                table[draft[s, :nodes[s]]] = ids[s, :nodes[s]]
                anchor[s] = bonus[s]
        steps += 1


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--sequences", type=int, default=8)
    ap.add_argument("--prompt", type=int, default=1000, help="tokens of the shared prompt")
    ap.add_argument("--tokens", type=int, default=64, help="tokens to decode for every sequence")
    ap.add_argument("--nodes", type=int, default=32, help="nodes of a tree, at most")
    a = ap.parse_args()
    rng = np.random.default_rng(0)
    model = Model()
    goose = binding.Goose(max_S=a.sequences, max_B=CHUNK, max_H=model.heads)
    prompt = rng.integers(0, model.vocab - 16, a.prompt).tolist()
    own = [rng.integers(0, model.vocab - 16, int(n)).tolist() for n in rng.integers(5, 200, a.sequences)]
    batch = Batch(goose, model, prompt, own, room=200 + a.tokens + a.nodes, nodes=a.nodes)
    torch.cuda.synchronize()
    began = time.perf_counter()
    out, steps = decode(batch, a.tokens)
    torch.cuda.synchronize()
    print("%d sequences under %d shared tokens: %d tokens each in %d steps, %.2f ms a step (drafting on the host included)" %
          (a.sequences, a.prompt, a.tokens, steps, 1e3 * (time.perf_counter() - began) / steps))
    assert not goose.last_status(a.sequences).any()
    goose.close()


if __name__ == "__main__":
    main()
