"""goose_chunk_attn against dense attention in 64 bits over the sequence's rows, wherever its pages lie.

Tolerance, element by element.  P is rounded to bf16: every term of sum p v is off by at most 2^-8 of itself, so the output by 2^-8 A with
A = sum p |v| / sum p; the output's own rounding is 2^-8 |out|.  The rest: scores from fp32 sums of 128 products (with standard normal
q and k at scale 128^-1/2 the sum of their sizes is about 7, times 128 * 2^-24: below 6e-5 in the exponent), exp2 (below 1e-4), partial
results of 16 bits: together below 0.2 * 2^-8 A.  So 2^-8 (1.2 A + |out|).  The log-sum-exp: the scores' 6e-5 and the exponentials' 1e-4,
2e-4, and a few roundings of itself in 32 bits, 2^-20 of it."""
import numpy as np
import pytest
import torch

from _pages import D, Paged, attention, i32

pytestmark = pytest.mark.gpu
SCALE = D ** -0.5


@pytest.fixture(scope="module")
def goose():
    from paper_2604_02047_b200 import binding, build
    build.build()
    g = binding.Goose(max_S=70, max_B=16, max_H=64)
    yield g
    g.close()


class Case:
    def __init__(self, H, Hkv, B, ctxs, page, *, new=None, seed=0, scale=SCALE, **kw):
        self.S, self.H, self.B, self.ctxs, self.new, self.scale = len(ctxs), H, B, list(ctxs), new, scale
        self.n = [B] * self.S if new is None else list(new)
        self.c = Paged([x + n if n else 0 for x, n in zip(ctxs, self.n)], Hkv, page, seed=seed, **kw)
        g = torch.Generator(device="cuda").manual_seed(seed + 1)
        self.q = torch.randn(self.S, B, H, D, generator=g, device="cuda").bfloat16()
        for s, n in enumerate(self.n):
            self.q[s, n:] = float("nan")
        self.ctx, self.n_new = i32(ctxs), None if new is None else i32(new)

    def run(self, goose, **kw):
        out = torch.full_like(self.q, 7.0)
        lse = torch.full((self.S, self.B, self.H), 7.0, device="cuda")
        goose.chunk_attn(self.q, self.c.k, self.c.v, self.c.table, self.ctx, self.scale, **{**dict(out=out, lse=lse, n_new=self.n_new), **kw})
        return out, lse

    def check(self, goose, out=None, lse=None, skip=(), untouched=7.0):
        if out is None:
            out, lse = self.run(goose)
            torch.cuda.synchronize()
            assert not goose.last_status(self.S).any()
        for s, n in enumerate(self.n):
            if untouched is not None:
                assert (out[s, n:] == untouched).all() and (lse[s, n:] == untouched).all()
            if n == 0 or s in skip:
                continue
            K, V = (f(s, self.ctxs[s] + n) for f in (self.c.keys, self.c.values))
            step = max(1, 2 ** 24 // (self.ctxs[s] + n))       # heads at a time: memory
            Hkv, g = K.shape[1], self.H // K.shape[1]
            step = max(1, 2 ** 26 // ((self.ctxs[s] + n) * n * g))
            for h in range(0, Hkv, step):
                heads = slice(h * g, min(h + step, Hkv) * g)
                ref, A, l, _ = attention(self.q[s, :n, heads], K[:, h:h + step], V[:, h:h + step], self.ctxs[s], self.scale)
                got = out[s, :n, heads].double()
                assert torch.isfinite(got).all()
                over = (got - ref).abs() - 2.0 ** -8 * (1.2 * A + ref.abs())
                assert over.max().item() <= 0, (s, h, over.max().item())
                off = (lse[s, :n, heads].double() - l).abs() - 2e-4 - 2.0 ** -20 * l.abs()
                assert off.max().item() <= 0, (s, h, off.max().item())
        return out, lse


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256, 1024])
@pytest.mark.parametrize("B,ctxs", [(1, [0, 1, 127, 128, 1000]), (17, [0, 5, 111, 500, 16]), (130, [0, 126, 900])])
def test_pages(goose, page, B, ctxs):
    Case(8, 2, B, ctxs, page, seed=page + B).check(goose)


@pytest.mark.parametrize("H,Hkv", [(1, 1), (3, 1), (5, 5), (6, 2), (32, 8), (40, 40), (52, 52), (64, 4), (16, 1), (14, 2), (22, 2)])
@pytest.mark.parametrize("B", [1, 9, 150])
def test_heads(goose, H, Hkv, B):
    Case(H, Hkv, B, [3, 200], 32, seed=H + B).check(goose)


@pytest.mark.parametrize("B", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257])
def test_chunk_lengths(goose, B):
    """Around the tiles' edges, a group of four (tiles of 32 tokens) and heads of their own (128)."""
    Case(4, 1, B, [0, 100], 16, seed=B).check(goose)
    Case(2, 2, B, [0, 100], 16, seed=B).check(goose)


@pytest.mark.parametrize("ctx", [0, 1, 15, 16, 17, 127, 128, 129, 255, 256, 257, 1023])
def test_prefix_lengths(goose, ctx):
    Case(8, 2, 5, [ctx, 0, ctx], 16, seed=ctx).check(goose)


@pytest.mark.parametrize("H,Hkv,B,ctx", [(8, 2, 2000, 0), (4, 4, 1111, 777), (32, 8, 700, 5000), (16, 1, 333, 1)])
def test_long_chunks(goose, H, Hkv, B, ctx):
    Case(H, Hkv, B, [ctx], 64, seed=B).check(goose)


def test_ragged_batch(goose):
    Case(32, 8, 60, [10, 0, 5000, 7, 640, 128], 16, new=[60, 0, 1, 33, 0, 59], seed=1).check(goose)
    Case(5, 5, 700, [0, 0, 300, 9000], 128, new=[700, 3, 0, 1], seed=2).check(goose)


def test_many_sequences(goose):
    rng = np.random.default_rng(5)
    Case(8, 2, 1, rng.integers(0, 3000, 70).tolist(), 16, seed=3).check(goose)
    Case(8, 8, 3, rng.integers(0, 300, 70).tolist(), 32, new=rng.integers(0, 4, 70).tolist(), seed=4).check(goose)


def test_one_long_sequence(goose):
    """A token over many rows: the rows are split over the device."""
    Case(16, 2, 1, [70000], 16, seed=5).check(goose)
    Case(4, 4, 2, [70001], 256, seed=6).check(goose)


def test_no_sequence_and_nothing_new(goose):
    c = Case(8, 2, 4, [3, 5], 16, new=[0, 0])
    out, lse = c.check(goose)
    z = torch.zeros(0, 4, 8, D, dtype=torch.bfloat16, device="cuda")
    assert goose.chunk_attn(z, c.c.k, c.c.v, torch.zeros(0, 1, dtype=torch.int32, device="cuda"), i32([]), SCALE).shape == z.shape


def test_shared_pages(goose):
    """Two sequences that have pages of a common prefix."""
    c = Case(8, 2, 6, [100, 90], 16, seed=8, spare=8)
    c.c.table_host[1, :4] = c.c.table_host[0, :4]
    c.c.table = i32(c.c.table_host)
    c.check(goose)


def test_out_is_q(goose):
    for c in (Case(8, 2, 300, [50, 3000], 32, seed=9, new=[300, 11]), Case(32, 8, 1, [500] * 5, 16, seed=10)):
        want = c.run(goose)
        keep = c.q.clone()
        out, lse = c.run(goose, out=c.q)
        for s, n in enumerate(c.n):
            assert torch.equal(c.q[s, :n], want[0][s, :n]) and torch.equal(lse[s, :n], want[1][s, :n])
        c.q = keep


def test_extreme_scores(goose):
    """Rows of one dominant key, scores far from 0, all scores alike; infinities and NaN in queries stay in their rows."""
    c = Case(4, 2, 40, [300], 16, seed=11)
    c.c.k.flatten(0, 1)[c.c.rows(0, 17, 18)] *= 20
    out, lse = c.run(goose)
    K, V = c.c.keys(0, 340), c.c.values(0, 340)
    ref, A, l, _ = attention(c.q[0], K, V, 300, SCALE)
    # the scores of row 17 are twenty times as large: so is their error
    assert ((out[0].double() - ref).abs() - (2.0 ** -8 * (1.2 * A + ref.abs()) + 2.4e-3 * A)).max() <= 0
    assert ((lse[0].double() - l).abs() - 1.4e-3 - 2.0 ** -20 * l.abs()).max() <= 0
    same = Case(4, 2, 40, [300], 16, seed=12)
    same.c.k.flatten(0, 1)[same.c.rows(0, 0, 340)] = 0
    same.check(goose)
    same.q[0, 3, 1, 5] = float("nan")
    out, lse = same.run(goose)
    bad = torch.isnan(out).any(-1)
    assert bad[0, 3, 1] and bad.sum() == 1 and torch.isnan(lse).sum() == 1


def test_keys_behind_a_token_reach_nothing(goose):
    """NaN among the keys of a chunk's last token: the tokens in front of it are as they were."""
    c = Case(4, 2, 40, [300], 16, seed=13)
    want, want_lse = c.run(goose)
    c.c.k.flatten(0, 1)[c.c.rows(0, 339, 340)] = float("nan")
    out, lse = c.run(goose)
    assert torch.equal(out[:, :39], want[:, :39]) and torch.equal(lse[:, :39], want_lse[:, :39]) and torch.isnan(out[:, 39]).all()


def test_the_same_bits_again(goose):
    for c in (Case(32, 8, 1, [9000, 100, 3], 16, seed=14), Case(8, 2, 500, [1000], 32, seed=15)):
        first = c.run(goose)
        for _ in range(5):
            again = c.run(goose)
            assert all(torch.equal(a, b) for a, b in zip(first, again))


def test_broken_sequences(goose):
    """Lengths outside the table, a page outside the pool, counts outside [0, B]: reported, zeros; the others as ever."""
    from paper_2604_02047_b200 import binding
    c = Case(8, 2, 5, [40, 60, 33, 20, 90, 10, 12], 16, new=[5, 5, 5, 5, 5, 5, 5], seed=16)
    ctx, new = [40, -1, 2 ** 31 - 3, 20, 108, 10, 12], [5, 5, 5, 9, 5, -2, 5]
    c.c.table_host[6, 0] = -5
    c.c.table = i32(c.c.table_host)
    c.ctx, c.n_new = i32(ctx), i32(new)
    out, lse = c.run(goose)
    assert c.c.table.shape[1] == 7                             # 112 rows: 108 + 5 do not fit
    assert goose.last_status(7).tolist() == [0, binding.ST_BAD_ROWS, binding.ST_BAD_ROWS, binding.ST_BAD_NODES, binding.ST_BAD_ROWS,
                                             binding.ST_BAD_NODES, binding.ST_BAD_ROWS]
    for s in (1, 2, 4, 6):
        assert not out[s].any() and not lse[s].any()
    for s in (3, 5):
        assert (out[s] == 7).all() and (lse[s] == 7).all()
    c.check(goose, out, lse, skip=range(1, 7), untouched=None)


@pytest.mark.parametrize("B,ctx,broken", [(1, 9000, 500), (300, 200, 30), (300, 4000, 100)])
def test_a_page_outside_the_pool(goose, B, ctx, broken):
    """Tokens that see it are zeros, wherever the work on their rows was split; other sequences are as ever."""
    from paper_2604_02047_b200 import binding
    c = Case(8, 2, B, [ctx, 100], 16, seed=17)
    c.c.table_host[0, broken] = c.c.n_pages
    c.c.table = i32(c.c.table_host)
    out, lse = c.run(goose)
    assert goose.last_status(2).tolist() == [binding.ST_BAD_ROWS, 0]
    first = max(0, broken * 16 - ctx)
    assert not out[0, first:].any() and not lse[0, first:].any()
    c.check(goose, out, lse, skip=[0])


def test_captured_and_replayed(goose):
    """A graph, replayed with other lengths and queries in the same arrays, beside eager calls of a larger size in between."""
    c = Case(32, 8, 3, [2000, 40], 16, seed=18)
    out, lse = c.run(goose)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            goose.chunk_attn(c.q, c.c.k, c.c.v, c.c.table, c.ctx, SCALE, out=out, lse=lse)
    torch.cuda.current_stream().wait_stream(stream)
    for ctxs in ([2000, 40], [17, 30], [1999, 0]):
        Case(32, 8, 600, [3000, 500], 64, seed=19).run(goose)
        c.ctxs = ctxs
        c.ctx.copy_(i32(ctxs))
        c.q.normal_()
        graph.replay()
        torch.cuda.synchronize()
        c.check(goose, out, lse)
    assert not goose.last_status(2).any()


def test_refusals(goose):
    from paper_2604_02047_b200.binding import GooseError
    z = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    base = dict(q=z(2, 4, 8, D), k_cache=z(9, 16, 2, D), v_cache=z(9, 16, 2, D), page_table=i32(np.zeros((2, 4))), ctx_len=i32([0, 0]), scale=1.0)
    goose.chunk_attn(**base)
    for wrong in (dict(q=z(2, 4, 8, 64)), dict(q=z(2, 4, 8, D).float()), dict(q=z(2, 4, 7, D)), dict(q=z(2, 4, 65, D)), dict(q=z(2, 8, 4, D).transpose(1, 2)),
                  dict(k_cache=z(9, 8, 2, D), v_cache=z(9, 8, 2, D)), dict(k_cache=z(9, 48, 2, D), v_cache=z(9, 48, 2, D)),
                  dict(v_cache=z(9, 16, 4, D)), dict(page_table=i32(np.zeros((1, 4)))), dict(page_table=torch.zeros(2, 4, device="cuda")),
                  dict(page_table=i32(np.zeros((2, 0)))), dict(page_table=i32(np.zeros((2, 65537)))), dict(ctx_len=i32([0])), dict(scale=0.0),
                  dict(scale=float("nan")), dict(scale=1e30), dict(n_new=i32([1])), dict(out=z(2, 4, 8, 64)), dict(lse=torch.zeros(2, 4, 7, device="cuda")),
                  dict(q=z(71, 1, 8, D), page_table=i32(np.zeros((71, 1))), ctx_len=i32(np.zeros(71))),
                  dict(k_cache=z(0, 16, 2, D), v_cache=z(0, 16, 2, D)), dict(q=z(2 * 4 * 8 * D + 4)[4:].view(2, 4, 8, D)),
                  dict(q=z(2, 0, 8, D)), dict(k_cache=z(9, 16, 1, D), v_cache=z(9, 16, 1, D), q=z(2, 4, 17, D))):
        with pytest.raises(GooseError):
            goose.chunk_attn(**{**base, **wrong})
    torch.cuda.synchronize()
    assert not goose.last_status(2).any()
