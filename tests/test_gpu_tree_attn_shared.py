"""goose_tree_attn_shared against dense attention in 64 bits over the shared rows, the sequence's own and the node's ancestors.

Tolerance, element by element.  P is rounded to bf16: every term of sum p v is off by at most 2^-8 of itself, so the output by 2^-8 A with
A = sum p |v| / sum p; the output's own rounding is 2^-8 |out|.  The rest: scores from fp32 sums of 128 products (with standard normal
q and k at scale 128^-1/2 the sum of their sizes is about 7, times 128 * 2^-24: below 6e-5 in the exponent), exp2 (below 1e-4), partial results
in 11 bits, 2^-11 |x| < 0.13 * 2^-8 A: together below 0.2 * 2^-8 A.  So 2^-8 (1.2 A + |out|).  The log-sum-exp: the scores' 6e-5 and the
exponentials' 1e-4, 2e-4, and a few roundings of itself in 32 bits, 2^-20 of it."""
import math

import numpy as np
import pytest
import torch

from paper_2604_02047_b200 import synth

pytestmark = pytest.mark.gpu
D = 128
SCALE = D ** -0.5


@pytest.fixture(scope="module")
def goose():
    from paper_2604_02047_b200 import binding, build
    build.build()
    g = binding.Goose(max_S=64, max_B=128, max_H=64)
    yield g
    g.close()


def _i32(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


def _sees(parent, n):
    m = np.zeros((n, n), bool)
    for i in range(n):
        if i:
            m[i] = m[parent[i]]
        m[i, i] = True
    return torch.tensor(m, device="cuda")


def _reference(q, kc, vc, rows, visible, scale):
    """(out, A, lse) of one sequence: q [n][H][D], the cache rows `rows`, visible [n][keys]."""
    n, H, _ = q.shape
    Hkv = kc.shape[1]
    K, V = (c[rows].double().transpose(0, 1) for c in (kc, vc))                     # [Hkv][keys][D]
    qq = q.double().view(n, Hkv, H // Hkv, D).permute(1, 2, 0, 3)                    # [Hkv][g][n][D]
    x = scale * (qq @ K[:, None].transpose(2, 3))
    x = x.masked_fill(~visible, -math.inf)
    p = torch.softmax(x, -1)
    back = lambda t: t.permute(2, 0, 1, 3).reshape(n, H, D)  # noqa: E731
    return back(p @ V[:, None]), back(p @ V[:, None].abs()), torch.logsumexp(x, -1).permute(2, 0, 1).reshape(n, H)


class Case:
    def __init__(self, S, H, Hkv, B, shared, ctxs, *, parents=None, nodes=None, seed=0, spare=5, scale=SCALE, gap=1, rows=None):
        rng = np.random.default_rng([seed, S, H, B, shared])
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.S, self.B, self.H, self.shared, self.ctxs, self.nodes, self.scale = S, B, H, shared, list(ctxs), nodes, scale
        self.parents = [synth.random_tree(rng, B) for _ in range(S)] if parents is None else parents
        # the sequences stand in the cache in an order of their own, the shared rows among them
        order, at = rng.permutation(S + 1), gap
        self.off = [0] * S
        for x in order:
            if x == S:
                self.shared_row = at
                at += shared + spare
            else:
                self.off[x] = at
                at += self.ctxs[x] + B + spare
        total = at if rows is None else rows
        self.q = torch.randn(S, B, H, D, generator=g, device="cuda").bfloat16()
        self.k = torch.randn(total, Hkv, D, generator=g, device="cuda").bfloat16()
        self.v = torch.randn(total, Hkv, D, generator=g, device="cuda").bfloat16()

    def n(self, s):
        return self.B if self.nodes is None else self.nodes[s]

    def spoil(self):
        """NaN in every row that no sequence has, and in the queries of nodes that do not exist."""
        live = torch.zeros(self.k.shape[0], dtype=torch.bool, device="cuda")
        live[self.shared_row:self.shared_row + self.shared] = True
        for s in range(self.S):
            if self.n(s):
                live[self.off[s]:self.off[s] + self.ctxs[s] + self.n(s)] = True
            self.q[s, self.n(s):] = float("nan")
        self.k[~live] = float("nan")
        self.v[~live] = float("inf")
        return self

    def run(self, goose, **kw):
        out = torch.full_like(self.q, 7.0)
        lse = torch.full((self.S, self.B, self.H), 7.0, device="cuda")
        goose.tree_attn_shared(self.q, self.k, self.v, self.shared_row, self.shared, torch.tensor(self.off, dtype=torch.int64, device="cuda"),
                               _i32(self.ctxs), _i32(self.parents), self.scale, out=out, lse=lse,
                               n_nodes=None if self.nodes is None else _i32(self.nodes), **kw)
        return out, lse

    def check(self, goose, out=None, lse=None, skip=()):
        if out is None:
            out, lse = self.run(goose)
            torch.cuda.synchronize()
            assert not goose.last_status(self.S).any()
        for s in range(self.S):
            n = self.n(s)
            assert (out[s, n:] == 7).all() and (lse[s, n:] == 7).all()
            if n == 0 or s in skip:
                continue
            rows = torch.cat([self.shared_row + torch.arange(self.shared), self.off[s] + torch.arange(self.ctxs[s] + n)]).cuda()
            visible = torch.cat([torch.ones(n, self.shared + self.ctxs[s], dtype=torch.bool, device="cuda"), _sees(self.parents[s], n)], 1)
            ref, A, ref_lse = _reference(self.q[s, :n], self.k, self.v, rows, visible, self.scale)
            over = ((out[s, :n].double() - ref).abs() - 2.0 ** -8 * (1.2 * A + ref.abs())).max().item()
            assert over <= 0, (s, over)
            assert ((lse[s, :n].double() - ref_lse).abs() - 2.0 ** -20 * ref_lse.abs()).max().item() <= 2e-4, s


# group sizes 1..16, trees that fill 128-row tiles, leave them ragged or need several, odd numbers of tiles
SHAPES = [(8, 2, 32), (8, 2, 33), (8, 2, 128), (6, 2, 50), (16, 1, 20), (4, 4, 20), (2, 1, 64), (2, 1, 65), (32, 8, 1), (10, 2, 26), (12, 4, 1),
          (16, 1, 128), (64, 4, 128), (3, 3, 128), (5, 1, 7), (11, 1, 12), (40, 40, 1)]


@pytest.mark.parametrize("H,Hkv,B", SHAPES)
def test_shapes(goose, H, Hkv, B):
    Case(3, H, Hkv, B, 200, [300, 0, 129], seed=H + B).spoil().check(goose)


@pytest.mark.parametrize("shared", [0, 1, 127, 128, 129, 255, 1000])
@pytest.mark.parametrize("B", [1, 40])
def test_shared_lengths(goose, shared, B):
    Case(2, 4, 1, B, shared, [0, 77], seed=shared).spoil().check(goose)


@pytest.mark.parametrize("ctx", [0, 1, 64, 100, 127, 128, 255])
def test_own_lengths(goose, ctx):
    """The tree rows in one tile, over the edge of two, at the start of one."""
    Case(2, 8, 4, 60, 130, [ctx, 2 * ctx], parents=[synth.chain_tree(60), synth.kary_tree(60, 3)], seed=ctx).spoil().check(goose)


@pytest.mark.parametrize("S", [1, 2, 31, 33, 64])
def test_batches(goose, S):
    Case(S, 8, 2, 3, 700, [(37 * s) % 400 for s in range(S)], seed=S).spoil().check(goose)


def test_node_counts(goose):
    Case(5, 8, 2, 60, 500, [10, 20, 300, 0, 64], nodes=[60, 0, 1, 33, 59]).spoil().check(goose)
    Case(3, 8, 1, 100, 500, [10, 200, 300], nodes=[3, 17, 100]).spoil().check(goose)     # M tiles without a node
    Case(3, 8, 2, 9, 300, [5, 5, 5], nodes=[0, 0, 0]).check(goose)


def test_long_lists_split_over_all_ctas(goose):
    Case(2, 4, 1, 9, 30011, [9000, 40], seed=1).spoil().check(goose)
    Case(3, 16, 2, 128, 4000, [1500, 3, 700], seed=2).spoil().check(goose)
    Case(16, 8, 2, 64, 3000, [100 * s for s in range(16)], seed=3).spoil().check(goose)


@pytest.mark.parametrize("S,H,Hkv,B,shared,own", [
    (30, 16, 16, 8, 300, 140),      # a pair of M tiles over the shared rows, then single ones of a tile or two
    (40, 16, 16, 8, 130, 100),      # a pair and a single one over the shared rows, own rows of one tile
    (40, 64, 4, 24, 100, 250),      # a pair and a single M tile of every sequence and head in turn
    (60, 64, 4, 16, 1, 130),        # pairs of a tile or two
    (64, 32, 8, 2, 0, 300),         # no shared rows
])
def test_many_items_a_cta(goose, S, H, Hkv, B, shared, own):
    """Several changes of item a CTA, from either kind to either kind."""
    rng = np.random.default_rng(S)
    Case(S, H, Hkv, B, shared, rng.integers(0, own, S).tolist(), seed=S + B).spoil().check(goose)


def test_random_cases(goose):
    rng = np.random.default_rng(11)
    for i in range(40):
        g, Hkv = int(rng.integers(1, 17)), int(rng.integers(1, 5))
        S, B = int(2 ** rng.uniform(0, 5)), int(rng.choice([1, 2, 16, 60, int(rng.integers(1, 129))]))
        ctxs = rng.integers(0, int(2 ** rng.uniform(0, 11)) + 1, S).tolist()
        nodes = rng.integers(0, B + 1, S).tolist() if rng.random() < .5 else None
        Case(S, g * Hkv, Hkv, B, int(rng.choice([0, int(2 ** rng.uniform(0, 13))])), ctxs, nodes=nodes, seed=i).spoil().check(goose)


def test_rows_that_grow_from_tile_to_tile(goose):
    """Scores that rise along the keys: the running maximum changes in every tile, by more than the rescaling threshold and by less."""
    for step in (2.0, 40.0):
        c = Case(2, 4, 2, 16, 900, [300, 200])
        ramp = torch.arange(c.k.shape[0], device="cuda").float() * (step / 128)
        c.q[..., 0] = 1.0 / SCALE
        c.k[..., 0] = ramp[:, None].bfloat16()
        # (scores up to 2^8 * step are sums with one term that large: its fp32 rounding, 2^-24 of it, stays below the 6e-5 of the bound)
        c.check(goose)


def test_values_of_any_size(goose):
    """Partial results keep a row's power of two apart: values of 1e30 and of 1e-30."""
    for size in (1e30, 1e-30):
        c = Case(2, 4, 2, 16, 900, [300, 200])
        c.v = (c.v.float() * size).bfloat16()
        c.check(goose)


def test_a_sequence_is_its_own(goose):
    """Infinities and NaN in one sequence's own rows do not reach the others; in the shared rows they reach all."""
    c = Case(4, 8, 2, 5, 300, [200, 30, 64, 500])
    clean = c.run(goose)[0].clone()
    c.k[c.off[2] + 10] = float("nan")
    c.v[c.off[2] + 11] = float("inf")
    out, lse = c.run(goose)
    assert not torch.isfinite(out[2]).all()
    for s in (0, 1, 3):
        assert torch.equal(out[s], clean[s])
    c.v[c.shared_row + 7] = float("nan")
    assert torch.isnan(c.run(goose)[0]).all()


def test_the_same_bits_every_time(goose):
    c = Case(6, 32, 8, 33, 1000, [100, 2000, 3, 400, 0, 77])
    first = [t.clone() for t in c.run(goose)]
    other = Case(3, 8, 2, 128, 5000, [100, 200, 300], seed=5)
    for _ in range(3):
        other.run(goose)                                       # another call's results in the workspace
        assert all(torch.equal(a, b) for a, b in zip(first, c.run(goose)))


def test_other_stream_in_place_and_graph(goose):
    c = Case(4, 8, 2, 20, 600, [100, 0, 300, 50])
    want, want_lse = [t.clone() for t in c.run(goose)]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    args = (c.k, c.v, c.shared_row, c.shared, torch.tensor(c.off, device="cuda"), _i32(c.ctxs), _i32(c.parents), c.scale)
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        q = c.q.clone()
        out = goose.tree_attn_shared(q, *args, out=q)
    stream.synchronize()
    assert out is q and torch.equal(q, want)
    q, out = c.q.clone(), torch.zeros_like(want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        goose.tree_attn_shared(q, *args, out=out)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)


def test_a_graph_outlives_its_workspace():
    """A graph captured with a small workspace is replayed behind calls that needed a larger one."""
    from paper_2604_02047_b200 import binding
    g = binding.Goose(max_S=16, max_B=128, max_H=32)
    small, large = Case(2, 8, 2, 5, 600, [100, 30]), Case(16, 32, 8, 64, 700, [40] * 16)
    want = small.run(g)[0].clone()
    args = (small.k, small.v, small.shared_row, small.shared, torch.tensor(small.off, device="cuda"), _i32(small.ctxs), _i32(small.parents),
            small.scale)
    out, graph = torch.zeros_like(want), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        g.tree_attn_shared(small.q, *args, out=out)
    for _ in range(2):
        large.check(g)
        other = torch.full((large.S * 64 * 1024,), float("nan"), device="cuda")      # whatever was freed is somebody else's now
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.isnan(other).all()
    g.close()


def test_offsets_beyond_32_bits(goose):
    """Rows whose byte offset passes 2^32 (and whose element offset passes 2^31)."""
    rows = 2_200_000
    c = Case(2, 8, 8, 4, 300, [200, 100], gap=rows - 700, rows=1)
    c.k, c.v = (torch.empty(rows, 8, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for t in (c.k, c.v):
        t[rows - 1000:] = torch.randn(1000, 8, D, device="cuda").bfloat16()
    c.check(goose)


def test_broken_sequences(goose):
    from paper_2604_02047_b200 import binding
    parents = [[-1, 0, 1, 1], [-1, 0, 3, 1], [-1, 0, 0, 0], [-1, 0, 0, 0], [0, 0, 0, 0], [-1, 0, 1, 2], [-1, 0, 1, 2]]
    c = Case(7, 8, 2, 4, 200, [100, 100, 100, 100, 100, 100, 3], parents=parents)
    keep = c.off[2]
    c.off[2] = 2 ** 62                                          # rows outside the cache
    c.ctxs[3], c.nodes = -1, [4, 4, 4, 4, 4, 5, 4]
    out, lse = c.run(goose)
    B = binding
    assert goose.last_status(7).tolist() == [0, B.ST_BAD_PARENT, B.ST_BAD_ROWS, B.ST_BAD_ROWS, B.ST_BAD_PARENT, B.ST_BAD_NODES, 0]
    for s in (1, 2, 3, 4):
        assert not out[s].any() and not lse[s].any()
    assert (out[5] == 7).all()
    c.off[2], c.ctxs[3], c.nodes = keep, 100, [4, 4, 4, 4, 4, 0, 4]
    c.check(goose, out, lse, skip=(1, 2, 3, 4))


def test_refusals(goose):
    from paper_2604_02047_b200.binding import GooseError
    c = Case(2, 8, 2, 4, 100, [5, 6])
    base = dict(q=c.q, k_cache=c.k, v_cache=c.v, shared_row=0, shared_len=10, row_off=torch.tensor(c.off, device="cuda"), ctx_len=_i32(c.ctxs),
                parent=_i32(c.parents), scale=SCALE)
    goose.tree_attn_shared(**base)
    for wrong in (dict(shared_len=-1), dict(shared_row=-1), dict(shared_row=c.k.shape[0] - 9), dict(shared_len=2 ** 31 - 1), dict(scale=0.0),
                  dict(scale=float("nan")), dict(scale=1e31), dict(q=c.q[:, :, :7].contiguous()), dict(q=c.q.float()), dict(row_off=_i32(c.off)),
                  dict(parent=_i32(c.parents)[:1]), dict(ctx_len=_i32([1])), dict(out=torch.empty_like(c.q)[:, :2]), dict(v_cache=c.v[:, :1].contiguous()),
                  dict(n_nodes=_i32([1])), dict(q=torch.zeros(2, 4, 66, D, dtype=torch.bfloat16, device="cuda")),
                  dict(lse=torch.zeros(2, 4, 7, device="cuda")), dict(k_cache=c.k[..., :64].contiguous(), v_cache=c.v[..., :64].contiguous())):
        with pytest.raises(GooseError):
            goose.tree_attn_shared(**{**base, **wrong})
    torch.cuda.synchronize()
    assert not goose.last_status(2).any()
