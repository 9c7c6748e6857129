"""goose_append_kv against the formula in 64 bits: norm, both kinds of rotation, trees and runs of tokens, parts of a wider tensor,
sequences that are short, gone or broken.

Tolerance.  An output is one fp32 result rounded to bf16: half a unit of its last place, at most 2^-8 of it
(eight bits of significand).  The fp32 part: a sum of 128 squares (eight in
a lane, then four levels: 12 roundings of positive terms), rsqrt (2 units), two products and a rotation of two terms: below 24 roundings of
2^-24 of the larger of the pair's elements, which for a small result of a large pair is more than its own half unit.  So: 2^-8 of the result
plus 2^-19 of the pair."""
import numpy as np
import pytest
import torch

from paper_2604_02047_b200 import synth

pytestmark = pytest.mark.gpu
D = 128


@pytest.fixture(scope="module")
def goose():
    from paper_2604_02047_b200 import binding, build
    build.build()
    g = binding.Goose(max_S=40, max_B=128, max_H=64)
    yield g
    g.close()


def _normal(g, *shape, scale=1.0):
    return (scale * torch.randn(shape, generator=g, device="cuda")).bfloat16()


def _i32(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


def _table(rot, rows):
    t = np.arange(rows)[:, None] * 10000.0 ** (-np.arange(0, rot, 2) / max(rot, 1))
    return torch.tensor(np.concatenate([np.cos(t), np.sin(t)], 1), dtype=torch.float32, device="cuda")


def _depths(parent):
    d = []
    for i, p in enumerate(parent):
        d.append(0 if i == 0 else d[p] + 1)
    return d


def _turned(x, w, table_rows, rot, interleaved, eps):
    """(result, the larger element of each element's pair), x [n][heads][D] in 64 bits."""
    x = x.double()
    if w is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * w.double()
    size = x.abs()
    if rot:
        j = torch.arange(rot // 2, device=x.device)
        a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + rot // 2)
        c, s = table_rows[:, None, :rot // 2].double(), table_rows[:, None, rot // 2:].double()
        y = x.clone()
        y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
        size[..., a] = size[..., b] = torch.maximum(size[..., a], size[..., b])
        x = y
    return x, size


def _close(got, ref, size):
    got = got.double()
    assert torch.isfinite(got).all()
    over = (got - ref).abs() - (2.0 ** -8 * ref.abs() + 2.0 ** -19 * size)
    assert over.max().item() <= 0, over.max().item()


def _run(goose, S, H, Hkv, B, ctxs, *, parents=None, nodes=None, norm=True, rot=D, interleaved=False, fused=True, pos_off=None, scale=1.0,
         seed=0, in_place=False):
    g = torch.Generator(device="cuda").manual_seed(seed)
    if fused:
        qkv = _normal(g, S, B, H + 2 * Hkv + 1, D, scale=scale)    # one head more: the token's stride is not its heads'
        q, k, v = qkv[:, :, :H], qkv[:, :, H:H + Hkv], qkv[:, :, H + Hkv:H + 2 * Hkv]
    else:
        q, k, v = (_normal(g, S, B, h, D, scale=scale) for h in (H, Hkv, Hkv))
    rows = [c + B + 3 for c in ctxs]
    off = np.concatenate([[5], 5 + np.cumsum(rows)[:-1]]).astype(np.int64)
    kc, vc = _normal(g, 5 + sum(rows), Hkv, D), _normal(g, 5 + sum(rows), Hkv, D)
    k_ref, v_ref = kc.clone(), vc.clone()
    pos = [0] * S if pos_off is None else pos_off
    table = _table(rot, max(p + c for p, c in zip(pos, ctxs)) + B)
    wq, wk = [(1 + 0.3 * torch.randn(D, generator=g, device="cuda")).bfloat16() if norm else None for _ in range(2)]
    out = torch.full((S, B, H, D), 7.0, dtype=torch.bfloat16, device="cuda")
    q0 = q.clone()
    if in_place:
        out = q
    goose.append_kv(q, k, v, kc, vc, torch.tensor(off, device="cuda"), _i32(ctxs), rope=table if rot else None,
                    parent=None if parents is None else _i32(parents), n_nodes=None if nodes is None else _i32(nodes),
                    pos_off=None if pos_off is None else _i32(pos_off), q_weight=wq, k_weight=wk, eps=1e-5, interleaved=interleaved, out=out)
    torch.cuda.synchronize()
    assert not goose.last_status(S).any()
    for s in range(S):
        n = B if nodes is None else nodes[s]
        depth = torch.arange(n) if parents is None else torch.tensor(_depths(parents[s])[:n], dtype=torch.long)
        at = table[(pos[s] + ctxs[s] + depth).cuda()]
        _close(out[s, :n], *_turned(q0[s, :n], wq, at, rot, interleaved, 1e-5)) if n else None
        assert torch.equal(out[s, n:], (q0 if in_place else torch.full_like(out, 7.0))[s, n:])
        new = slice(int(off[s]) + ctxs[s], int(off[s]) + ctxs[s] + n)
        if n:
            _close(kc[new], *_turned(k[s, :n], wk, at, rot, interleaved, 1e-5))
        k_ref[new] = kc[new]
        v_ref[new] = v[s, :n]
    assert torch.equal(kc, k_ref) and torch.equal(vc, v_ref)   # (values are bit patterns: no other row has moved)


@pytest.mark.parametrize("rot,interleaved", [(128, False), (128, True), (64, False), (16, True), (48, False), (16, False), (0, False)])
@pytest.mark.parametrize("norm", [True, False])
def test_forms(goose, rot, interleaved, norm):
    rng = np.random.default_rng(rot)
    parents = [synth.random_tree(rng, 21) for _ in range(3)]
    _run(goose, 3, 8, 2, 21, [0, 130, 17], parents=parents, rot=rot, interleaved=interleaved, norm=norm)


@pytest.mark.parametrize("H,Hkv", [(1, 1), (3, 1), (5, 5), (32, 8), (40, 40), (52, 52), (64, 4), (16, 1)])
@pytest.mark.parametrize("B", [1, 2, 128])
def test_heads(goose, H, Hkv, B):
    _run(goose, 2, H, Hkv, B, [3, 200], parents=[synth.chain_tree(B), synth.star_tree(B)], seed=H + B)


@pytest.mark.parametrize("B", [1, 127, 129, 1000, 5003])
def test_runs_of_tokens(goose, B):
    _run(goose, 2, 6, 2, B, [0, 9], nodes=[B, max(1, B - 1)], rot=64, seed=B)


def test_node_counts_and_offsets(goose):
    rng = np.random.default_rng(3)
    parents = [synth.kary_tree(60, 3), synth.random_tree(rng, 60), synth.chain_tree(60), synth.random_tree(rng, 60)]
    _run(goose, 4, 32, 8, 60, [10, 0, 3000, 7], parents=parents, nodes=[60, 0, 1, 33], pos_off=[0, 5, 20000, 512])


def test_separate_tensors_and_in_place(goose):
    _run(goose, 2, 8, 8, 33, [1, 2], parents=[synth.chain_tree(33)] * 2, fused=False)
    _run(goose, 2, 8, 8, 33, [1, 2], parents=[synth.chain_tree(33)] * 2, fused=False, in_place=True)


def test_magnitudes(goose):
    """Norms of rows far from 1: squares of 1e15 fit fp32, squares of 1e-15 vanish beside eps."""
    for scale in (1e15, 1e-15):
        _run(goose, 1, 4, 2, 9, [4], nodes=None, scale=scale)


def test_nan_stays_in_its_head(goose):
    g = torch.Generator(device="cuda").manual_seed(1)
    q, k, v = (_normal(g, 1, 4, h, D) for h in (4, 2, 2))
    q[0, 1, 2, 5] = float("nan")
    k[0, 3, 1, 7] = float("inf")
    kc, vc = torch.zeros(8, 2, D, dtype=torch.bfloat16, device="cuda"), torch.zeros(8, 2, D, dtype=torch.bfloat16, device="cuda")
    w = torch.ones(D, dtype=torch.bfloat16, device="cuda")
    out = goose.append_kv(q, k, v, kc, vc, torch.zeros(1, dtype=torch.int64, device="cuda"), _i32([2]), rope=_table(64, 16), q_weight=w, k_weight=w)
    bad = torch.isnan(out).any(-1).nonzero().tolist()
    assert bad == [[0, 1, 2]] and torch.isnan(kc).any(-1).nonzero().tolist() == [[5, 1]] and torch.equal(vc[2:6], v[0])


def test_broken_sequences(goose):
    """An invalid tree, rows outside the cache, a position outside the table, a count outside [0, B]: reported, zeros, no row written;
    the other sequences as ever."""
    from paper_2604_02047_b200 import binding
    g = torch.Generator(device="cuda").manual_seed(2)
    S, B, H, Hkv = 6, 5, 4, 2
    q, k, v = (_normal(g, S, B, h, D) for h in (H, Hkv, Hkv))
    kc = _normal(g, 100, Hkv, D)
    vc, k0 = kc.clone(), kc.clone()
    parents = [[-1, 0, 1, 2, 3], [-1, 0, 2, 1, 0], [-1, 0, 0, 0, 0], [-1, 0, 1, 2, 3], [-1] * 5, [-1, 0, 1, 2, 3]]
    off = torch.tensor([0, 10, 2 ** 62, 30, 40, 50], device="cuda")
    ctx = _i32([3, 3, 3, 17, 3, -1])
    out = goose.append_kv(q, k, v, kc, vc, off, ctx, rope=_table(128, 20), parent=_i32(parents), n_nodes=_i32([5, 5, 5, 5, 9, 5]),
                          out=torch.full_like(q, 7.0))
    assert goose.last_status(S).tolist() == [0, binding.ST_BAD_PARENT, binding.ST_BAD_ROWS, binding.ST_BAD_POS, binding.ST_BAD_NODES,
                                             binding.ST_BAD_ROWS | binding.ST_BAD_POS]
    assert not out[1].any() and not out[2].any() and not out[3, 3:].any() and (out[4] == 7).all() and not out[5].any()
    assert out[3, :3].any(-1).all() and out[0].any(-1).all()
    same = torch.ones(100, dtype=torch.bool, device="cuda")
    same[3:8] = False
    same[47:50] = False                                        # tokens 0..2 of sequence 3 have a place in the table
    assert torch.equal(kc[same], k0[same]) and torch.equal(vc[3:8], v[0]) and torch.equal(vc[47:50], v[3, :3])


def test_refusals(goose):
    from paper_2604_02047_b200.binding import GooseError
    z = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    base = dict(q=z(2, 4, 8, D), k=z(2, 4, 2, D), v=z(2, 4, 2, D), k_cache=z(64, 2, D), v_cache=z(64, 2, D),
                row_off=torch.zeros(2, dtype=torch.int64, device="cuda"), ctx_len=_i32([0, 0]), rope=_table(128, 64))
    goose.append_kv(**base)
    for wrong in (dict(k=z(2, 4, 3, D)), dict(q=z(2, 4, 8, D).float()), dict(q=z(2, 4, D, 8).transpose(2, 3)), dict(v=z(4, 2, 2, D).transpose(0, 1)),
                  dict(rope=_table(24, 64)), dict(rope=_table(144, 64)), dict(q=z(2, 4, 65, D)), dict(eps=-1.0), dict(eps=float("nan")),
                  dict(out=z(2, 4, 7, D)), dict(q_weight=z(64)), dict(ctx_len=_i32([0])), dict(parent=_i32([[-1, 0, 0, 0]])),
                  dict(n_nodes=_i32([1])), dict(k_cache=z(64, 2, 64), v_cache=z(64, 2, 64)), dict(q=z(41, 1, 8, D), k=z(41, 1, 2, D), v=z(41, 1, 2, D)),
                  dict(k=z(8 * 2 * D + 4)[4:].view(2, 4, 2, D))):
        with pytest.raises(GooseError):
            goose.append_kv(**{**base, **wrong})
    with pytest.raises(GooseError):                            # a tree of more nodes than a context's
        goose.append_kv(z(1, 129, 8, D), z(1, 129, 2, D), z(1, 129, 2, D), base["k_cache"], base["v_cache"], base["row_off"][:1], _i32([0]),
                        rope=_table(128, 200), parent=_i32([synth.chain_tree(129)]))
    torch.cuda.synchronize()
    assert not goose.last_status(2).any()
