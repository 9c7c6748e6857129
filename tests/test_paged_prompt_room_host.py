"""The bounds of the decoding example over a cache in pages, looked at without a GPU: a model and calls that stand for real ones, on the CPU."""
import os
import re
import types

import pytest
import torch

from paper_2604_02047_b200 import binding, build, paged_prompt


@pytest.fixture(autouse=True)
def no_gpu(monkeypatch):
    monkeypatch.setattr(torch.Tensor, "cuda", lambda self, *a, **k: self)
    for name in ("zeros", "arange"):
        real = getattr(torch, name)
        monkeypatch.setattr(torch, name, lambda *a, real=real, **k: real(*a, **{x: y for x, y in k.items() if x != "device"}))


class Goose:
    """Every draft token is what the model would have said; rows that the calls get are counted."""

    max_B = 16

    def __init__(self):
        self.furthest = 0                                      # position behind the last one that was appended

    def append_kv_paged(self, q, k, v, kc, vc, table, ctx, rope=None, n_new=None, pos_off=None, **kw):
        for s, n in enumerate(n_new.tolist()):
            rows = int(ctx[s]) + n
            if n:
                assert rows <= table.shape[1] * kc.shape[1] and (table[s, :-(-rows // kc.shape[1])] >= 0).all()
                self.furthest = max(self.furthest, int(pos_off[s]) + rows)
        return q

    def chunk_attn(self, q, *a, out=None, **kw):
        return out, None

    def kv_weights(self, *a, **kw):
        pass

    def evict_kv(self, kc, vc, table, ctx, weight, pos, *a, **kw):
        return None, None, weight, pos

    def node_topk(self, logits, k, n_nodes=None, B=None):
        return logits, None, None

    def accept(self, tok, chains, argmax, n_nodes=None):
        return None, (n_nodes - 1).clamp(min=0), torch.full_like(n_nodes, 7)


def _model(positions):
    def forward(tokens, layer_attention):
        q = torch.zeros(*tokens.shape, 1, 128)
        layer_attention(0, q, q, q)
        return tokens
    return types.SimpleNamespace(layers=1, heads=1, kv_heads=1, rope=torch.zeros(positions, 128), norms=[(None, None)], scale=1.0, forward=forward)


def _batch(prompts, rows, positions=100000, **kw):
    goose = Goose()
    return goose, paged_prompt.Batch(goose, _model(positions), [[1 + i % 5 for i in range(n)] for n in prompts], rows=rows, **kw)


@pytest.mark.parametrize("prompts,tokens,rows,draft", [([300, 20], 2000, 2400 + 2100, 8), ([30], 1500, 1536, 0), ([1, 1, 1], 1200, 3 * 1216, 4)])
def test_without_a_budget_a_sequence_has_what_the_pool_has(prompts, tokens, rows, draft):
    _, batch = _batch(prompts, rows, draft=draft)
    out, _ = paged_prompt.decode(batch, tokens)
    assert [len(t) for t in out] == [n + tokens for n in prompts]


def test_no_table_is_longer_than_the_calls_take():
    with open(os.path.join(build.INCLUDE, "goose.h")) as f:
        assert int(re.search(r"GOOSE_MAX_PAGED_ROWS (\d+)", f.read()).group(1)) == binding.MAX_PAGED_ROWS == 524288
    _, batch = _batch([5], rows=600000, page=64)
    assert batch.table.shape[1] == 524288 // 64
    _, batch = _batch([5], rows=600000, page=64, budget=524000, slack=64)
    assert batch.table.shape[1] <= 524288 // 64


def test_with_a_budget_a_table_has_room_for_the_budget_and_a_chunk():
    goose, batch = _batch([3000, 10], rows=3000, budget=500, slack=30, chunk=256, draft=8)
    assert batch.table.shape[1] * batch.page >= 500 + 30 + 256
    out, _ = paged_prompt.decode(batch, 1500)
    assert [len(t) for t in out] == [4500, 1510] and goose.furthest >= 4499
    assert int(batch.ctx.max()) <= 530


@pytest.mark.parametrize("budget", [None, 60])
def test_positions_end_with_the_rotation_table(budget):
    """As many tokens as it has positions for, drafts cut where it ends; one more is an error, ahead of the first step."""
    kw = dict(rows=1000, budget=budget, slack=16, recent=20, chunk=32)
    goose, batch = _batch([100, 7], positions=300, **kw)
    out, _ = paged_prompt.decode(batch, 201)
    assert [len(t) for t in out] == [301, 208] and goose.furthest == 300
    goose, batch = _batch([100, 7], positions=300, **kw)
    at = goose.furthest
    with pytest.raises(ValueError):
        paged_prompt.decode(batch, 202)
    assert goose.furthest == at
    with pytest.raises(ValueError):
        _batch([302], positions=300, **kw)
    goose, batch = _batch([301], positions=300, **kw)
    with pytest.raises(ValueError):
        batch.step([True])
    assert goose.furthest == 300
