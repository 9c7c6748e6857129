"""The calls together: a batch decoded under a shared prompt (paper_2604_02047_b200/shared_prompt.py).  Whatever trees were drafted, every token that
came out is the greedy choice of the same model computed densely in 64 bits over its own sequence, penalties and mask applied.

Tolerance: the model's activations are bf16 (rounded some ten times between the embedding and the logits, 2^-9 each on average, of logits
of size about 1 whose sums over 512 random terms average those out): a token whose dense score is within 0.06 of the best counts as the choice;
the gap between the best two of 4080 random scores is larger than that for four tokens in five."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def _dense_logits(m, tokens):
    """Logits [n][V] of one sequence, in 64 bits."""
    D, H, Hkv, n = 128, m.heads, m.kv_heads, len(tokens)
    x = m.embed[torch.tensor(tokens, device="cuda")].double()
    half = m.rope.shape[1] // 2
    c, s = m.rope[:n, None, :half].double(), m.rope[:n, None, half:].double()

    def turn(y, w):
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + 1e-6) * w.double()
        a, b = y[..., :half], y[..., half:]
        return torch.cat([a * c - b * s, b * c + a * s], -1)

    causal = torch.ones(n, n, dtype=torch.bool, device="cuda").tril()
    for i in range(m.layers):
        qkv = (x @ m.qkv[i].double()).view(n, H + 2 * Hkv, D)
        q, k, v = turn(qkv[:, :H], m.norms[i][0]), turn(qkv[:, H:H + Hkv], m.norms[i][1]), qkv[:, H + Hkv:]
        k, v = k.repeat_interleave(H // Hkv, 1), v.repeat_interleave(H // Hkv, 1)
        p = torch.softmax((m.scale * torch.einsum("nhd,khd->hnk", q, k)).masked_fill(~causal, -torch.inf), -1)
        x = x + torch.einsum("hnk,khd->nhd", p, v).reshape(n, -1) @ m.out[i].double()
    return x @ m.embed.double().T * x.shape[-1] ** -0.5


@pytest.mark.parametrize("nodes", [1, 24])
def test_every_token_is_the_greedy_choice(nodes):
    from paper_2604_02047_b200 import binding, build, shared_prompt
    build.build()
    rng = np.random.default_rng(4)
    model = shared_prompt.Model()
    V, reserved, tokens = model.vocab, 16, 40
    goose = binding.Goose(max_S=3, max_B=128, max_H=model.heads)
    prompt = rng.integers(0, V - reserved, 300).tolist()
    own = [rng.integers(0, V - reserved, n).tolist() for n in (1, 40, 150)]
    batch = shared_prompt.Batch(goose, model, prompt, own, room=300, nodes=nodes)
    out, steps = shared_prompt.decode(batch, tokens)
    assert not goose.last_status(3).any()
    assert steps <= tokens and (nodes == 1) == (steps == tokens)
    for s, got in enumerate(out):
        assert len(got) == len(own[s]) + tokens and list(got[:len(own[s])]) == own[s]
        full = prompt + [int(t) for t in got]
        logits = _dense_logits(model, full[:-1]).cpu().numpy()
        for i in range(len(prompt) + len(own[s]) - 1, len(full) - 1):
            x = logits[i].copy()
            count = np.bincount(full[len(prompt) + len(own[s]):i + 1], minlength=V)
            seen = np.bincount(full[:i + 1], minlength=V) > 0
            x = np.where(seen, np.where(x > 0, x / 1.1, x * 1.1), x) - 0.05 * count - 0.1 * (count > 0)
            x[V - reserved:] = -np.inf
            assert x[full[i + 1]] >= x.max() - 0.06, (s, i)
    goose.close()
