"""The calls on a paged cache together (paper_2604_02047_b200/paged_prompt.py).  Without a budget every token is the greedy choice of the same model
computed densely in 64 bits; with one, the rows that are left are what the definition leaves: the first, the latest and as many others, every head its
own choice, each with the key that its token had.

Tolerance of the choice: test_gpu_shared_prompt's.  Of a key: bf16 products of the projection are summed in fp32 and rounded, normed, turned and
rounded again: three roundings of 2^-8 of elements of at most about 5, and the size of the head they are normed by: 0.06."""
import numpy as np
import pytest
import torch

from test_gpu_shared_prompt import _dense_logits

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def model():
    from paper_2604_02047_b200 import build, shared_prompt
    build.build()
    return shared_prompt.Model()


@pytest.mark.parametrize("draft,chunk,page", [(0, 100, 16), (7, 333, 32)])
def test_every_token_is_the_greedy_choice(model, draft, chunk, page):
    from paper_2604_02047_b200 import binding, paged_prompt
    rng = np.random.default_rng(5)
    goose = binding.Goose(max_S=3, max_B=16, max_H=model.heads)
    prompts = [rng.integers(0, model.vocab, n).tolist() for n in (1, 130, 700)]
    prompts[1] += prompts[1]                                   # something for the drafts to find
    batch = paged_prompt.Batch(goose, model, [list(p) for p in prompts], rows=2000, page=page, chunk=chunk, draft=draft)
    out, steps = paged_prompt.decode(batch, 30)
    assert not goose.last_status(3).any() and steps <= 30
    for p, got in zip(prompts, out):
        assert got[:len(p)] == p and len(got) == len(p) + 30
        x = _dense_logits(model, got[:-1]).cpu().numpy()
        for i in range(len(p) - 1, len(got) - 1):
            assert x[i, got[i + 1]] >= x[i].max() - 0.06, i
    goose.close()


def test_a_budget(model):
    from paper_2604_02047_b200 import binding, paged_prompt
    rng = np.random.default_rng(6)
    goose = binding.Goose(max_S=3, max_B=16, max_H=model.heads)
    prompts = [rng.integers(0, model.vocab, n).tolist() for n in (90, 400, 1000)]
    budget, sink, recent = 200, 4, 40
    batch = paged_prompt.Batch(goose, model, prompts, rows=3000, chunk=150, draft=4, budget=budget, sink=sink, recent=recent, slack=30)
    pages = len(batch.free) + sum(batch.owned)
    out, _ = paged_prompt.decode(batch, 60)
    assert not goose.last_status(3).any()
    used = [p for s in range(3) for p in batch.table[s, :batch.owned[s]].tolist()]
    assert len(used) == len(set(used)) and sorted(used + batch.free) == list(range(pages))
    w = batch.m.qkv[0].double()
    half = model.rope.shape[1] // 2
    for s in range(3):
        n, total = int(batch.ctx[s]), int(batch.ctx[s] + batch.off[s])
        assert n <= budget + 30 and total == len(batch.tokens[s]) - 1 and (batch.off[s] > 0) == (s > 0)
        rows = [int(batch.table[s, j // 16]) * 16 + j % 16 for j in range(n)]
        x = model.embed[torch.tensor(batch.tokens[s][:total], device="cuda")].double()
        keys = (x @ w).view(total, -1, 128)[:, model.heads:model.heads + model.kv_heads]
        keys = keys / torch.sqrt((keys * keys).mean(-1, keepdim=True) + 1e-6) * model.norms[0][1].double()
        c, sn = model.rope[:total, None, :half].double(), model.rope[:total, None, half:].double()
        keys = torch.cat([keys[..., :half] * c - keys[..., half:] * sn, keys[..., half:] * c + keys[..., :half] * sn], -1)
        for i in range(model.layers):
            for h in range(model.kv_heads):
                at = batch.pos[i][s, h, :n].tolist()
                assert len(set(at)) == n and set(range(min(sink, n))) | set(range(total - min(recent, total), total)) <= set(at)
                assert torch.isfinite(batch.weight[i][s, h, :n]).all() and (batch.weight[i][s, h, :n] >= 0).all()
                if i == 0:
                    off = (batch.caches[0][0].flatten(0, 1)[rows, h].double() - keys[at, h]).abs().max().item()
                    assert off < 0.06, off
    goose.close()


def test_what_does_not_fit_is_an_error(model):
    from paper_2604_02047_b200 import binding, paged_prompt
    goose = binding.Goose(max_S=2, max_B=4, max_H=model.heads)
    for kw in (dict(prompts=[]), dict(prompts=[[1], []]), dict(prompts=[[1, 2]], draft=4), dict(prompts=[[1] * 100], rows=64),
               dict(prompts=[[1] * 10], budget=20, sink=10, recent=11)):
        with pytest.raises(ValueError):
            paged_prompt.Batch(goose, model, **{**dict(rows=256, draft=3), **kw})
    batch = paged_prompt.Batch(goose, model, [[1] * 60], rows=64, draft=0)
    with pytest.raises(ValueError):
        paged_prompt.decode(batch, 10)
    goose.close()
