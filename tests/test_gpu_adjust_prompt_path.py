"""Penalties where the prompt reaches into the tree: hist_len[s] < n_prompt[s] <= hist_len[s] + B.  The node at depth d stands at position
hist_len + d of its sequence, and where that is below n_prompt it is a token of the prompt: it counts for the repetition penalty, not for frequency and
presence.  The first tree of every sequence is such a case (its root is the prompt's last token), and so is the end of a prompt that goes
through as a chain.  Reference in 64 bits, tolerance as in test_gpu_adjust_logits.py."""
import numpy as np
import pytest
import torch

from paper_2604_02047_b200 import synth
from test_gpu_adjust_logits import _f32, _i32, _path

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def goose():
    from paper_2604_02047_b200 import binding, build
    build.build()
    g = binding.Goose(max_S=8, max_B=128, max_H=64)
    yield g
    g.close()


def _check(goose, parents, lens, prompts, V=2100, few=30, nodes=None, seed=0):
    rng = np.random.default_rng(seed)
    S, B = len(parents), len(parents[0])
    g = torch.Generator(device="cuda").manual_seed(seed)
    logits = (3 * torch.randn(S * B, (V + 7) // 8 * 8, generator=g, device="cuda")).bfloat16()
    hist, tok = rng.integers(0, few, (S, max(max(lens), 1) + 3)), rng.integers(0, few, (S, B))
    rep, freq, pres = (np.float32(rng.uniform(lo, hi, S)) for lo, hi in ((1, 2), (.1, 1), (.1, 1)))
    out = goose.adjust_logits(logits, _i32(hist), _i32(lens), _i32(tok), _i32(parents), V=V, n_prompt=_i32(prompts),
                              n_nodes=None if nodes is None else _i32(nodes), repetition=_f32(rep), frequency=_f32(freq), presence=_f32(pres))
    torch.cuda.synchronize()
    assert not goose.last_status(S).any()
    got, x0 = out.double().cpu().numpy(), logits.double().cpu().numpy()
    for s in range(S):
        for i in range(B if nodes is None else nodes[s]):
            tokens = np.concatenate([hist[s, :lens[s]], tok[s, _path(parents[s], i)[::-1]]])       # in order of position
            n = np.bincount(tokens[prompts[s]:], minlength=V)
            x = x0[s * B + i, :V]
            y = np.where(np.bincount(tokens, minlength=V) > 0, np.where(x > 0, x / rep[s], x * rep[s]), x)
            size = np.abs(y) + freq[s] * n + pres[s]
            y = y - freq[s] * np.float64(n) - pres[s] * (n > 0)
            assert (np.abs(got[s * B + i, :V] - y) <= 2.0 ** -8 * np.abs(y) + 2.0 ** -21 * size).all(), (s, i)


@pytest.mark.parametrize("into", [0, 1, 2, 5, 127, 128])
def test_chains_and_trees(goose, into):
    B = 128
    rng = np.random.default_rng(into)
    parents = [synth.chain_tree(B), synth.kary_tree(B, 3), synth.random_tree(rng, B)]
    _check(goose, parents, [50, 0, 1000], [50 + into, into, 1000 + into], seed=into)


def test_node_counts_and_small_trees(goose):
    parents = [[-1, 0, 1, 1, 0]] * 4
    _check(goose, parents, [7, 7, 0, 3], [8, 9, 1, 8], nodes=[5, 1, 4, 0], few=3)
    _check(goose, [[-1]] * 3, [5, 5, 0], [6, 5, 1], few=2)


def test_the_first_step_under_a_prompt():
    """The decoding example's first step: the prompt's last token, the root of the tree, is best by less than the penalties that it must not get."""
    from paper_2604_02047_b200 import binding, shared_prompt
    anchor, other = 77, 1234

    class Scripted(shared_prompt.Model):
        def forward(self, tokens, layer_attention):
            logits = torch.zeros_like(super().forward(tokens, layer_attention))
            logits[:, anchor], logits[:, other] = 11.0, 9.9375  # 11 / 1.1 = 10 is the larger, 10 - 0.05 - 0.1 is not
            return logits

    model = Scripted()
    goose = binding.Goose(max_S=2, max_B=128, max_H=model.heads)
    batch = shared_prompt.Batch(goose, model, list(range(100, 150)), [[anchor], [5, 6, anchor]], room=64, nodes=1)
    dev = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    argmax, ids, path, accepted, bonus = batch.step(dev([[anchor]] * 2), dev([[-1]] * 2), dev([1, 1]))
    assert bonus.tolist() == [anchor] * 2
    # its second occurrence is a generated token
    argmax, ids, path, accepted, bonus = batch.step(dev([[anchor]] * 2), dev([[-1]] * 2), dev([1, 1]))
    assert bonus.tolist() == [other] * 2
    goose.close()
