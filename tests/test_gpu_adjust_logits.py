"""goose_adjust_logits and goose_append_tokens against the formulas in 64 bits, token by token.

Tolerance of the logits: one fp32 result rounded to bf16, half a unit of its last place, at most 2^-8 of it; the fp32 part has at most six roundings of 2^-24 (a reciprocal and a
product, a product and two sums, a sum with the bias) of intermediate sizes up to |x| * rep + freq * n + pres + |bias|: 2^-21 of that sum."""
import numpy as np
import pytest
import torch

from paper_2604_02047_b200 import synth

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def goose():
    from paper_2604_02047_b200 import binding, build
    build.build()
    g = binding.Goose(max_S=40, max_B=128, max_H=64)
    yield g
    g.close()


def _i32(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


def _f32(a):
    return torch.tensor(np.asarray(a), dtype=torch.float32, device="cuda")


def _path(parent, i):
    p = []
    while i >= 0:
        p.append(i)
        i = parent[i]
    return p


def _reference(x, hist, prompt, tokens, rep, freq, pres, bias, allowed):
    """(result, sum of the sizes) of one row in 64 bits."""
    V = len(x)
    inside = lambda t: t[(t >= 0) & (t < V)]  # noqa: E731
    n = np.bincount(inside(np.concatenate([hist[prompt:], tokens])), minlength=V)
    seen = (np.bincount(inside(hist), minlength=V) + n) > 0
    with np.errstate(invalid="ignore", over="ignore"):
        y = np.where(seen, np.where(x > 0, x / rep, x * rep), x)
        size = np.abs(y) + freq * n + pres * (n > 0) + np.abs(bias)
        y = y - freq * n - pres * (n > 0) + bias
    return np.where(allowed, y, -np.inf), size


def _case(goose, S, B, V, lens, *, seed=0, parents=None, nodes=None, prompts=None, mask="random", bias="one", pen=True, extra=0, in_place=False,
          few=None, x=None):
    rng = np.random.default_rng(seed)
    ldl = (V + 7) // 8 * 8 + extra
    g = torch.Generator(device="cuda").manual_seed(seed)
    logits = (3 * torch.randn(S * B, ldl, generator=g, device="cuda")).bfloat16()
    if x is not None:
        logits[:, :V] = x
    room = max(max(lens), 1) + 3
    top = V if few is None else few
    hist = rng.integers(0, top, (S, room))
    hist[:, ::7] = V + 5                                       # tokens of no row of the table count nowhere
    hist[:, ::11] = -1
    hist[:, ::13] = -2 ** 31
    tok = rng.integers(0, top, (S, B))
    tok[:, ::5] = -3
    tok[:, 3::17] = -2 ** 31
    parents = [synth.random_tree(rng, B) for _ in range(S)] if parents is None else parents
    rep, freq, pres = rng.uniform(1, 2, S), rng.uniform(-.5, 1, S), rng.uniform(-.5, 1, S)
    b = {"none": None, "one": rng.standard_normal(V), "own": rng.standard_normal((S, V))}[bias]
    words = (V + 31) // 32 + 2
    m = None if mask == "none" else rng.integers(0, 2 ** 32, (S * B, words), dtype=np.uint32)
    if mask == "edges":
        m[0], m[-1] = 0, 0xFFFFFFFF                            # a row that its mask leaves nothing, and all
    logits0 = logits.clone()
    out = logits if in_place else torch.full_like(logits, 7.0)
    before = out.clone()
    got = goose.adjust_logits(
        logits, _i32(hist), _i32(lens), _i32(tok), _i32(parents), V=V, n_nodes=None if nodes is None else _i32(nodes),
        n_prompt=None if prompts is None else _i32(prompts), bias=None if b is None else _f32(b),
        mask=None if m is None else torch.tensor(m.view(np.int32), device="cuda"), out=out,
        **(dict(repetition=_f32(rep), frequency=_f32(freq), presence=_f32(pres)) if pen else {}))
    torch.cuda.synchronize()
    assert got is out and not goose.last_status(S).any()
    assert torch.equal(out[:, V:], before[:, V:])
    have, have0, was = out.float().cpu().numpy().astype(np.float64), logits0.float().cpu().numpy().astype(np.float64), before.float().cpu().numpy()
    rep, freq, pres = (np.float32(a).astype(np.float64) if pen else a * 0 + c for a, c in ((rep, 1), (freq, 0), (pres, 0)))
    for s in range(S):
        for i in range(B):
            r = s * B + i
            if nodes is not None and i >= nodes[s]:
                np.testing.assert_array_equal(have[r], was[r])
                continue
            allowed = np.ones(V, bool) if m is None else np.unpackbits(m[r].view(np.uint8), bitorder="little")[:V] == 1
            bb = np.zeros(V) if b is None else np.float32(b if b.ndim == 1 else b[s]).astype(np.float64)
            ref, size = _reference(have0[r, :V], hist[s, :lens[s]], 0 if prompts is None else prompts[s], tok[s, _path(parents[s], i)],
                                   rep[s], freq[s], pres[s], bb, allowed)
            y = have[r, :V]
            fine = np.isfinite(ref)
            np.testing.assert_array_equal(np.where(fine, 0, y), np.where(fine, 0, ref))
            assert (np.abs(y - np.where(fine, ref, 0))[fine] <= 2.0 ** -8 * np.abs(ref)[fine] + 2.0 ** -21 * size[fine]).all(), (s, i)


@pytest.mark.parametrize("V", [1, 7, 31, 2047, 2048, 2049, 4100, 32000])
@pytest.mark.parametrize("B", [1, 5])
def test_vocabularies(goose, V, B):
    _case(goose, 2, B, V, [100, 33], seed=V, mask="edges" if B > 1 else "random")


@pytest.mark.parametrize("mask,bias,pen", [("none", "none", True), ("random", "none", False), ("none", "own", False), ("edges", "own", True)])
def test_parts(goose, mask, bias, pen):
    _case(goose, 3, 9, 3001, [0, 1, 500], mask=mask, bias=bias, pen=pen, prompts=[0, 1, 200], extra=16)


def test_many_occurrences_of_few_tokens(goose):
    """Every token of the path and the history among 20: counts of hundreds, paths of 128 nodes that name a token several times."""
    B = 128
    _case(goose, 3, B, 2100, [4000, 10, 1000], few=20, parents=[synth.chain_tree(B), synth.star_tree(B), synth.kary_tree(B, 3)],
          prompts=[1000, 0, 5000])                             # (a prompt longer than the history: none of it counts as generated)


def test_node_counts(goose):
    _case(goose, 4, 33, 5000, [50, 60, 70, 80], nodes=[33, 0, 1, 20], prompts=[50, 0, 0, 40])


def test_in_place(goose):
    _case(goose, 2, 40, 2500, [300, 0], few=300, in_place=True)


def test_large_batch(goose):
    _case(goose, 33, 3, 2300, list(range(33)))


def test_special_values(goose):
    """Masked places may hold anything; elsewhere infinities stay and NaN stays."""
    V, inf = 64, float("inf")
    x = torch.zeros(1, V, dtype=torch.bfloat16, device="cuda")
    x[0, :8] = torch.tensor([float("nan"), inf, -inf, -3.3895e38, 3.3895e38, -0.0, 0.0, 1e-40])
    x[0, 32:40] = x[0, :8]
    mask = torch.tensor([[-1, 0]], dtype=torch.int32, device="cuda")
    hist = _i32([[1, 2, 3, 4, 5, 6, 7]])
    y = goose.adjust_logits(x, hist, _i32([7]), None, _i32([[-1]]), repetition=_f32([1.5]), mask=mask)[0].float().cpu()
    assert (y[32:] == -inf).all() and torch.isnan(y[0]) and y[1] == inf and y[2] == -inf and y[3] == -inf and 2e38 < y[4] < 2.3e38
    assert (y[5:7] == 0).all()
    am, ids, vals = goose.node_topk(y.bfloat16()[None].nan_to_num(0.0, inf, -inf).cuda(), 4)
    assert am.item() == 1
    empty = goose.adjust_logits(x, None, None, None, _i32([[-1]]), mask=torch.zeros_like(mask))
    am, ids, vals = goose.node_topk(empty, 3)
    assert (empty == -inf).all() and ids.tolist() == [[0, 1, 2]] and (vals == -inf).all()


def test_masked_rows_through_the_topk(goose):
    """A few tokens left of a large vocabulary: they come first, the rest of the k are the lowest masked tokens."""
    V, rows = 128256, 6
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(rows, V, generator=g, device="cuda").bfloat16()
    mask = np.zeros((rows, V // 32), np.uint32)
    left = [[5], [128255, 40000], [70000, 70001, 70002], [0], [131071 % V, 99], [64000]]
    for r, ids in enumerate(left):
        for v in ids:
            mask[r, v >> 5] |= np.uint32(1 << (v & 31))
    y = goose.adjust_logits(x, None, None, None, _i32([synth.chain_tree(rows)]), mask=torch.tensor(mask.view(np.int32), device="cuda"))
    am, ids, vals = goose.node_topk(y, 5)
    for r, want in enumerate(left):
        best = sorted(want, key=lambda v: (-x[r, v].item(), v))
        rest = [v for v in range(10) if v not in want]
        assert ids[r].tolist() == (best + rest)[:5] and am[r].item() == best[0]


def test_broken_sequences(goose):
    from paper_2604_02047_b200 import binding
    S, B, V = 4, 3, 100
    x = torch.ones(S * B, 104, dtype=torch.bfloat16, device="cuda")
    hist = torch.zeros(S, 10, dtype=torch.int32, device="cuda")
    y = goose.adjust_logits(x, hist, _i32([5, 11, -1, 5]), None, _i32([[-1, 0, 2], [-1, 0, 1], [-1, 0, 1], [-1, 0, 1]]), V=V,
                            repetition=_f32([2.0] * S), n_nodes=_i32([3, 3, 3, 4]), out=torch.full_like(x, 7.0))
    assert goose.last_status(S).tolist() == [binding.ST_BAD_PARENT, binding.ST_BAD_ROWS, binding.ST_BAD_ROWS, binding.ST_BAD_NODES]
    assert (y[:3, :V] == 0).all() and (y[3:9, :V] == 1).all() and (y[9:] == 7).all() and (y[:, V:] == 7).all()


def test_refusals(goose):
    from paper_2604_02047_b200.binding import GooseError
    z = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    i = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    par = _i32([[-1, 0], [-1, 0]])
    base = dict(logits=z(4, 64), hist=i(2, 8), hist_len=i(2), draft_tok=i(2, 2), parent=par)
    goose.adjust_logits(**base)
    for wrong in (dict(logits=z(4, 60)), dict(logits=z(3, 64)), dict(V=65), dict(V=0), dict(hist=i(3, 8)), dict(hist_len=i(3)), dict(draft_tok=i(2, 3)),
                  dict(bias=torch.zeros(63, device="cuda")), dict(bias=torch.zeros(3, 64, device="cuda")), dict(mask=i(4, 1)), dict(mask=i(2, 2)),
                  dict(repetition=torch.ones(3, device="cuda")), dict(out=z(4, 32)), dict(out=z(3, 64)), dict(n_nodes=i(3)), dict(logits=z(4, 64).float()),
                  dict(parent=i(41, 2), logits=z(82, 64)), dict(V=32, out=z(4, 32), logits=z(256).as_strided((4, 64), (64, 1)), mask=i(4, 0))):
        with pytest.raises(GooseError):
            goose.adjust_logits(**{**base, **wrong})
    shared = z(4, 64)
    with pytest.raises(GooseError):                            # in place with another stride
        goose.adjust_logits(**{**base, "logits": shared, "V": 32, "out": shared.view(-1)[:128].view(4, 32)})
    torch.cuda.synchronize()
    assert not goose.last_status(2).any()


# ------------------------------------------------------------------------------------------------ goose_append_tokens
def test_append_tokens(goose):
    S, B, room = 5, 9, 40
    rng = np.random.default_rng(0)
    tok = rng.integers(0, 1000, (S, B))
    hist = rng.integers(0, 1000, (S, room))
    path = np.full((S, B), -1)
    path[0, :1], path[1, :4], path[2, :9], path[3, :2], path[4, :3] = [0], [0, 2, 5, 8], range(9), [0, 3], [0, 1, 2]
    alen, lens, nodes = [0, 3, 8, 1, 2], [0, 36, 31, 7, 39], [9, 9, 9, 0, 9]
    h = _i32(hist)
    new = goose.append_tokens(_i32(tok), _i32(path), _i32(alen), h, _i32(lens), n_nodes=_i32(nodes))
    from paper_2604_02047_b200 import binding
    assert goose.last_status(S).tolist() == [0, 0, 0, 0, binding.ST_BAD_ROWS]    # sequence 4 has room for one token, not three
    want = hist.copy()
    for s in (0, 1, 2):
        want[s, lens[s]:lens[s] + alen[s] + 1] = tok[s, path[s, :alen[s] + 1]]
    np.testing.assert_array_equal(h.cpu().numpy(), want)
    assert new.tolist() == [1, 40, 40, 7, 39]


def test_append_tokens_refuses_what_is_no_path(goose):
    from paper_2604_02047_b200 import binding
    paths = [[0, 2, 1], [1, 2, -1], [0, 1, 3], [0, 1, 2], [0, 1, 2], [0, 1, 1]]
    alen = [2, 1, 2, 3, -1, 2]
    S = len(paths)
    hist = torch.full((S, 8), 7, dtype=torch.int32, device="cuda")
    new = goose.append_tokens(torch.zeros(S, 3, dtype=torch.int32, device="cuda"), _i32(paths), _i32(alen), hist, _i32([2] * S))
    assert goose.last_status(S).tolist() == [binding.ST_BAD_PATH] * S
    assert (hist == 7).all() and new.tolist() == [2] * S
    i = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    base = dict(draft_tok=i(2, 3), path=i(2, 3), accept_len=i(2), hist=i(2, 8), hist_len=i(2))
    for wrong in (dict(draft_tok=i(2, 4)), dict(hist=i(3, 8)), dict(accept_len=i(3)), dict(new_len=base["hist_len"]), dict(new_len=i(3)), dict(hist=i(2, 8).long())):
        with pytest.raises(binding.GooseError):
            goose.append_tokens(**{**base, **wrong})
