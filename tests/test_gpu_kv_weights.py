"""goose_kv_weights against sums of the attention's probabilities in 64 bits.

Tolerance, of a row's new weight.  A term exp(x - lse) of it: x from an fp32 sum of 128 products (with standard normal q and k at scale
128^-1/2 the sum of their sizes is about 7, times 128 * 2^-24: below 6e-5), the exponential and the roundings of x and lse in units of log 2 (below 40
in size, a few times 2^-24 of that: 1e-5): 1e-4 of the term.  The sum of N positive terms in fp32, in any order: N * 2^-24 of it.  What was there
before and the last addition: 2^-23 of the result."""
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
    def __init__(self, H, Hkv, B, ctxs, page, *, new=None, seed=0, room=None, **kw):
        self.S, self.H, self.Hkv, self.B, self.ctxs, self.new = len(ctxs), H, Hkv, B, list(ctxs), new
        self.n = [B] * self.S if new is None else list(new)
        rows = [x + n if n else 0 for x, n in zip(ctxs, self.n)]
        self.c = Paged(rows, Hkv, page, seed=seed, **kw)
        self.c.v = None
        g = torch.Generator(device="cuda").manual_seed(seed + 1)
        self.q = torch.randn(self.S, B, H, D, generator=g, device="cuda").bfloat16()
        self.ctx, self.n_new = i32(ctxs), None if new is None else i32(new)
        self.before = torch.rand(self.S, Hkv, max(rows) + 3 if room is None else room, generator=g, device="cuda")
        self.lse = torch.full((self.S, B, H), float("nan"), device="cuda")
        self.p = [None] * self.S
        for s, n in enumerate(self.n):
            self.q[s, n:] = float("nan")
            if n:
                K = self.c.keys(s, rows[s])
                _, _, l, p = attention(self.q[s, :n], K, K, ctxs[s], SCALE)
                # (the probabilities that belong to the rounded lse)
                self.lse[s, :n] = l.float()
                off = (l - self.lse[s, :n].double()).view(n, Hkv, H // Hkv).permute(1, 2, 0)
                self.p[s] = p * torch.exp(off)[..., None]

    def run(self, goose, **kw):
        weight = self.before.clone()
        goose.kv_weights(self.q, self.lse, self.c.k, self.c.table, self.ctx, SCALE, weight, **{**dict(n_new=self.n_new), **kw})
        return weight

    def check(self, goose, weight=None, n=None):
        if weight is None:
            weight = self.run(goose)
            torch.cuda.synchronize()
            assert not goose.last_status(self.S).any()
        for s, k in enumerate(self.n if n is None else n):
            rows = self.ctxs[s] + k if k else 0
            assert torch.equal(weight[s, :, rows:], self.before[s, :, rows:])
            if k:
                ref = self.p[s][:, :, :k, :rows].sum((1, 2))
                total = ref + self.before[s, :, :rows].double()
                terms = k * self.H // self.Hkv
                over = (weight[s, :, :rows].double() - total).abs() - (1e-4 + terms * 2.0 ** -24) * ref - 2.0 ** -23 * total
                assert over.max().item() <= 0, (s, over.max().item())
        return weight


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256, 1024])
@pytest.mark.parametrize("B,ctxs", [(1, [0, 1, 127, 128, 1000]), (17, [0, 5, 111, 500, 16]), (130, [0, 126, 900])])
def test_pages(goose, page, B, ctxs):
    Case(8, 2, B, ctxs, page, seed=page + B).check(goose)


@pytest.mark.parametrize("H,Hkv", [(1, 1), (3, 1), (5, 5), (6, 2), (32, 8), (40, 40), (52, 52), (64, 4), (16, 1), (14, 2), (22, 2)])
@pytest.mark.parametrize("B", [1, 9, 150])
def test_heads(goose, H, Hkv, B):
    Case(H, Hkv, B, [3, 200], 32, seed=H + B).check(goose)


@pytest.mark.parametrize("B", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257])
def test_chunk_lengths(goose, B):
    Case(4, 1, B, [0, 100], 16, seed=B).check(goose)
    Case(2, 2, B, [0, 100], 16, seed=B).check(goose)


@pytest.mark.parametrize("H,Hkv,B,ctx", [(8, 2, 1500, 0), (4, 4, 1111, 777), (32, 8, 300, 5000), (16, 1, 333, 1)])
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
    Case(16, 2, 1, [70000], 16, seed=5).check(goose)


def test_of_the_attention(goose):
    """With the attention's own log-sum-exp: a token's probabilities add up to one."""
    c = Case(32, 8, 20, [1000, 3], 16, seed=6)
    V = torch.zeros_like(c.c.k)
    _, lse = goose.chunk_attn(c.q, c.c.k, V, c.c.table, c.ctx, SCALE, want_lse=True)
    weight = torch.zeros_like(c.before)
    goose.kv_weights(c.q, lse, c.c.k, c.c.table, c.ctx, SCALE, weight)
    sums = weight.double().sum(-1)
    assert (sums / (20 * 4) - 1).abs().max() < 5e-4             # (2e-4 of lse, 1e-4 of a term, the sums)


def test_fewer_tokens_than_the_attention_had(goose):
    """The accepted part of a draft."""
    c = Case(8, 2, 17, [500, 60, 0], 16, seed=7)
    c.check(goose, c.run(goose, n_new=i32([5, 0, 17])), n=[5, 0, 17])


def test_rows_of_nothing(goose):
    """A head of a token whose lse is -infinity adds nothing (its scores may be anything)."""
    c = Case(8, 2, 5, [40], 16, seed=8)
    c.q[0, 2, 3] = float("nan")
    c.lse[0, 2, 3] = -torch.inf
    c.p[0][0, 3, 2] = 0
    c.check(goose)


def test_nan_stays_in_its_row(goose):
    c = Case(8, 2, 5, [40], 16, seed=9)
    c.c.k.flatten(0, 1)[c.c.rows(0, 7, 8), 1] = float("nan")
    weight = c.run(goose)
    assert torch.isnan(weight).nonzero().tolist() == [[0, 1, 7]]


def test_the_same_bits_again(goose):
    for c in (Case(32, 8, 1, [9000, 100, 3], 16, seed=14), Case(8, 2, 500, [1000], 32, seed=15)):
        first = c.run(goose)
        for _ in range(5):
            assert torch.equal(first, c.run(goose))


def test_broken_sequences(goose):
    from paper_2604_02047_b200 import binding
    c = Case(8, 2, 5, [40, 60, 33, 20, 90, 10, 12], 16, new=[5, 5, 5, 5, 5, 5, 5], seed=16, room=200)
    ctx, new = [40, -1, 2 ** 31 - 3, 20, 108, 10, 12], [5, 5, 5, 9, 5, -2, 5]
    c.c.table_host[6, 0] = -5
    c.c.table = i32(c.c.table_host)
    c.ctx, c.n_new = i32(ctx), i32(new)
    weight = c.run(goose)
    assert goose.last_status(7).tolist() == [0, binding.ST_BAD_ROWS, binding.ST_BAD_ROWS, binding.ST_BAD_NODES, binding.ST_BAD_ROWS,
                                             binding.ST_BAD_NODES, binding.ST_BAD_ROWS]
    assert torch.equal(weight[1:6], c.before[1:6]) and torch.equal(weight[6, :, :16], c.before[6, :, :16])
    c.n = [5] + [0] * 5
    c.check(goose, weight, n=[5, 0, 0, 0, 0, 0])
    # the array beside the pages is too short
    c = Case(8, 2, 5, [40, 60], 16, seed=17, room=64)
    weight = c.run(goose)
    assert goose.last_status(2).tolist() == [0, binding.ST_BAD_ROWS] and torch.equal(weight[1], c.before[1])


def test_captured_and_replayed(goose):
    c = Case(32, 8, 3, [2000, 40], 16, seed=18)
    weight = c.run(goose)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            goose.kv_weights(c.q, c.lse, c.c.k, c.c.table, c.ctx, SCALE, weight)
    torch.cuda.current_stream().wait_stream(stream)
    want = c.run(goose)
    for _ in range(3):
        weight.copy_(c.before)
        Case(8, 2, 300, [100, 50, 7], 32, seed=19).run(goose)
        graph.replay()
        assert torch.equal(weight, want)


def test_refusals(goose):
    from paper_2604_02047_b200.binding import GooseError
    z = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    f = lambda *s: torch.zeros(s, device="cuda")  # noqa: E731
    base = dict(q=z(2, 4, 8, D), lse=f(2, 4, 8), k_cache=z(9, 16, 2, D), page_table=i32(np.zeros((2, 4))), ctx_len=i32([0, 0]), scale=1.0,
                row_weight=f(2, 2, 64))
    goose.kv_weights(**base)
    for wrong in (dict(q=z(2, 4, 8, 64)), dict(lse=f(2, 4, 7)), dict(lse=z(2, 4, 8)), dict(k_cache=z(9, 24, 2, D)), dict(row_weight=f(2, 1, 64)),
                  dict(row_weight=f(2, 2, 0)), dict(row_weight=f(2, 2, 128)[..., ::2]), dict(page_table=i32(np.zeros((2, 65537)))), dict(scale=-1.0),
                  dict(n_new=i32([1, 1, 1])), dict(ctx_len=i32([0, 0]).long()), dict(q=z(2, 4, 66, D), lse=f(2, 4, 66))):
        with pytest.raises(GooseError):
            goose.kv_weights(**{**base, **wrong})
    torch.cuda.synchronize()
    assert not goose.last_status(2).any()
