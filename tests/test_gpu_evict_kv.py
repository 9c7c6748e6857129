"""goose_evict_kv against its definition, bit by bit: which rows stay, where they lie, their weights and positions; what is not moved keeps its bits."""
import numpy as np
import pytest
import torch

from _pages import D, Paged, i32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def goose():
    from paper_2604_02047_b200 import binding, build
    build.build()
    g = binding.Goose(max_S=70, max_B=16, max_H=64)
    yield g
    g.close()


def _choice(weight, pos, budget, sink, recent_from):
    """The rows that stay, as the definition has them: the protected ones, then by weight (NaN last), the lower row of equal ones."""
    safe = (pos < sink) | (pos >= recent_from)
    w = weight.astype(np.float64)
    order = sorted(range(len(w)), key=lambda j: (not safe[j], 0 if safe[j] else np.isnan(w[j]), 0 if safe[j] or np.isnan(w[j]) else -w[j], j))
    keep = np.zeros(len(w), bool)
    keep[order[:budget]] = True
    return keep


class Case:
    def __init__(self, Hkv, ctxs, page, budget, sink, recent, *, off=None, seed=0, weights=None, room=None, new_room=None, **kw):
        self.S, self.Hkv, self.ctxs, self.budget, self.sink, self.recent = len(ctxs), Hkv, list(ctxs), budget, sink, recent
        self.c = Paged(ctxs, Hkv, page, seed=seed, **kw)
        # (bits that no arithmetic would leave alone: every row is its own)
        for t in (self.c.k, self.c.v):
            t.copy_(torch.randint(-2 ** 15, 2 ** 15, t.shape, dtype=torch.int16, device="cuda").view(torch.bfloat16))
        rng = np.random.default_rng(seed)
        room = max(max(ctxs), 1) + 5 if room is None else room
        self.off = [0] * self.S if off is None else list(off)
        self.weight = (rng.standard_normal((self.S, Hkv, room)) if weights is None else weights(rng, (self.S, Hkv, room))).astype(np.float32)
        # positions: what is left of off + ctx of them, in no order (rows have changed places before)
        self.pos = np.full((self.S, Hkv, room), -77, np.int64)
        for s, x in enumerate(ctxs):
            for h in range(Hkv):
                late = np.arange(self.off[s] + x - min(recent, x), self.off[s] + x)
                early = rng.permutation(self.off[s] + x - len(late))[:x - len(late)]
                p = np.concatenate([early, late])
                self.pos[s, h, :x] = rng.permutation(p) if self.off[s] else p
        self.new_room = room if new_room is None else new_room
        self.ctx, self.pos_off = i32(ctxs), None if off is None else i32(off)

    def run(self, goose, **kw):
        w, p = torch.tensor(self.weight, device="cuda"), i32(self.pos)
        k, v = self.c.k.clone(), self.c.v.clone()
        nw = torch.full((self.S, self.Hkv, self.new_room), 7.0, device="cuda")
        np_ = torch.full((self.S, self.Hkv, self.new_room), 7, dtype=torch.int32, device="cuda")
        r = goose.evict_kv(k, v, self.c.table, self.ctx, w, p, self.budget, self.sink, self.recent, self.pos_off, new_weight=nw, new_pos=np_, **kw)
        assert r[2] is nw and r[3] is np_
        return k, v, nw, np_, r[0], r[1]

    def check(self, goose, got=None, skip=()):
        if got is None:
            got = self.run(goose)
            torch.cuda.synchronize()
            assert not goose.last_status(self.S).any()
        k, v, nw, np_, new_ctx, new_off = [t.view(torch.int16).cpu().numpy().reshape(-1, self.Hkv, D) if t.dtype == torch.bfloat16 else t.cpu().numpy() for t in got]
        k0, v0 = [t.view(torch.int16).cpu().numpy().reshape(-1, self.Hkv, D).copy() for t in (self.c.k, self.c.v)]
        for s, x in enumerate(self.ctxs):
            if s in skip:
                continue
            left = min(x, self.budget)
            assert new_ctx[s] == left and new_off[s] == self.off[s] + x - left
            rows = self.c.rows(s, 0, x).cpu().numpy()
            for h in range(self.Hkv):
                w, p = self.weight[s, h, :x].copy(), self.pos[s, h, :x].copy()
                if x > self.budget:
                    keep = _choice(w, p, self.budget, self.sink, self.off[s] + x - self.recent)
                    to, of = np.nonzero(~keep[:self.budget])[0], self.budget + np.nonzero(keep[self.budget:])[0]
                    w[to], p[to] = w[of], p[of]
                    for c0 in (k0, v0):
                        c0[rows[to], h] = c0[rows[of], h]
                assert np.array_equal(nw[s, h, :left].view(np.int32), w[:left].view(np.int32)) and np.array_equal(np_[s, h, :left], p[:left])
                assert (nw[s, h, left:] == 7).all() and (np_[s, h, left:] == 7).all()
        assert np.array_equal(k, k0) and np.array_equal(v, v0)
        return got


@pytest.mark.parametrize("page", [16, 64, 256])
@pytest.mark.parametrize("budget,sink,recent", [(1, 0, 0), (1, 1, 0), (1, 0, 1), (31, 4, 10), (32, 0, 32), (33, 4, 20), (100, 100, 0), (100, 0, 50), (500, 4, 64), (1000, 16, 300)])
def test_budgets(goose, page, budget, sink, recent):
    Case(2, [1, 32, 33, 100, 101, 500, 1001, 1500], page, budget, sink, recent, seed=budget).check(goose)


@pytest.mark.parametrize("Hkv", [1, 3, 8, 40, 64])
def test_heads_and_positions(goose, Hkv):
    """Positions that are left of a longer past, in no order."""
    Case(Hkv, [300, 777], 32, 200, 4, 60, off=[0, 5000], seed=Hkv).check(goose)


@pytest.mark.parametrize("name", ["equal", "zeros", "few", "signed zeros", "infinities", "nan", "subnormal", "one digit"])
def test_weights(goose, name):
    """Ties by the hundred, signs, values that differ in their last bits alone."""
    def make(rng, shape):
        n = rng.standard_normal(shape)
        return {"equal": lambda: np.full(shape, 0.25), "zeros": lambda: np.zeros(shape), "few": lambda: rng.integers(-1, 3, shape),
                "signed zeros": lambda: np.where(n > 0, 0.0, -0.0), "infinities": lambda: np.where(n > 0.6, np.inf, np.where(n < -1, -np.inf, n)),
                "nan": lambda: np.where(n > 0.2, np.nan, n) * np.where(rng.random(shape) < 0.5, -1, 1), "subnormal": lambda: 1e-41 * n,
                "one digit": lambda: (np.float32(1).view(np.int32) + rng.integers(0, 200, shape)).astype(np.int32).view(np.float32)}[name]()
    Case(4, [700, 650, 1999], 16, 600, 4, 50, weights=make, seed=3).check(goose)
    Case(2, [700], 16, 600, 0, 0, weights=make, seed=4).check(goose)


@pytest.mark.parametrize("ctx,budget", [(40000, 20000), (33000, 1000), (20001, 20000), (70000, 64)])
def test_long(goose, ctx, budget):
    Case(1, [ctx], 128, budget, 4, budget // 3, seed=budget, weights=lambda r, s: np.exp(2 * r.standard_normal(s))).check(goose)


def test_many_sequences(goose):
    rng = np.random.default_rng(1)
    Case(2, rng.integers(0, 900, 70).tolist(), 16, 300, 4, 40, seed=6).check(goose)


def test_nothing_to_do(goose):
    Case(2, [0, 5, 300], 16, 300, 4, 40, seed=7).check(goose)
    Case(2, [0, 5, 300], 16, 5000, 4, 40, seed=7).check(goose)    # more than the table has


def test_shorter_new_arrays(goose):
    Case(2, [400, 100], 16, 120, 4, 40, seed=8, new_room=120).check(goose)


def test_twice(goose):
    """A cache that has been cut before: the second cut works on rows that have changed places."""
    c = Case(2, [400], 16, 300, 4, 50, seed=9)
    k, v, w, p, ctx, off = c.check(goose)
    d = Case(2, [300], 16, 100, 4, 50, off=[100], seed=9)
    d.c = c.c
    d.c.k, d.c.v = k, v
    d.weight, d.pos, d.new_room = w.cpu().numpy(), p.cpu().numpy().astype(np.int64), w.shape[-1]
    d.ctx, d.pos_off = ctx, off
    _, _, _, p, ctx, off = d.check(goose)
    assert ctx.item() == 100 and off.item() == 300
    for h in range(2):
        left = set(p[0, h, :100].tolist())
        assert {0, 1, 2, 3} | set(range(350, 400)) <= left and len(left) == 100


def test_broken_sequences(goose):
    from paper_2604_02047_b200 import binding
    c = Case(2, [400, 300, 200, 350, 390], 16, 120, 4, 40, seed=10)
    c.c.table_host[1, 18] = c.c.n_pages                         # the last of its nineteen pages
    c.c.table_host[4, 24] = -1
    c.c.table = i32(c.c.table_host)
    c.ctx = i32([400, 300, -3, 10 ** 9, 390])
    got = c.run(goose)
    assert goose.last_status(5).tolist() == [0] + [binding.ST_BAD_ROWS] * 4
    assert got[4].tolist() == [120, 300, -3, 10 ** 9, 390] and got[5].tolist() == [280, 0, 0, 0, 0]
    assert (got[2][1:] == 7).all() and (got[3][1:] == 7).all()
    c.check(goose, got, skip=[1, 2, 3, 4])
    c = Case(2, [400, 100], 16, 120, 4, 40, seed=11, new_room=110)   # more rows stay than the new arrays have
    got = c.run(goose)
    assert goose.last_status(2).tolist() == [binding.ST_BAD_ROWS, 0] and got[4].tolist() == [400, 100]
    c.check(goose, got, skip=[0])


def test_captured_and_replayed(goose):
    c = Case(4, [700, 90], 16, 256, 4, 40, seed=12)
    want = c.run(goose)
    k, v, w, p = c.c.k.clone(), c.c.v.clone(), torch.tensor(c.weight, device="cuda"), i32(c.pos)
    nw, np_, ctx, off = [torch.full_like(t, 7) for t in want[2:]]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            goose.evict_kv(k, v, c.c.table, c.ctx, w, p, 256, 4, 40, new_weight=nw, new_pos=np_, new_ctx_len=ctx, new_pos_off=off)
    torch.cuda.current_stream().wait_stream(stream)
    for _ in range(3):
        k.copy_(c.c.k), v.copy_(c.c.v), nw.fill_(7), np_.fill_(7)
        Case(4, [3000, 90, 1000], 16, 1500, 4, 40, seed=13).run(goose)
        graph.replay()
        torch.cuda.synchronize()
        c.check(goose, (k, v, nw, np_, ctx, off))


def test_refusals(goose):
    from paper_2604_02047_b200.binding import GooseError
    z = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    f = lambda *s: torch.zeros(s, device="cuda")  # noqa: E731
    base = dict(k_cache=z(9, 16, 2, D), v_cache=z(9, 16, 2, D), page_table=i32([[0, 1, 2], [3, 4, 5]]), ctx_len=i32([40, 10]), row_weight=f(2, 2, 48),
                row_pos=i32(np.tile(np.arange(48), (2, 2, 1))), budget=20, sink=4, recent=8)
    goose.evict_kv(**base)
    for wrong in (dict(budget=0), dict(sink=-1), dict(recent=-1), dict(sink=13), dict(recent=17), dict(v_cache=z(9, 16, 1, D)), dict(k_cache=z(9, 16, 2, 64), v_cache=z(9, 16, 2, 64)),
                  dict(row_weight=f(2, 2, 40)), dict(row_pos=f(2, 2, 48)), dict(new_weight=base["row_weight"]), dict(new_pos=base["row_pos"]),
                  dict(new_ctx_len=base["ctx_len"]), dict(new_pos_off=base["ctx_len"]), dict(pos_off=(p := i32([0, 0])), new_pos_off=p),
                  dict(new_ctx_len=(c := i32([0, 0])), new_pos_off=c), dict(new_weight=f(2, 1, 48)), dict(new_weight=f(2, 2, 20), new_pos=i32(np.zeros((2, 2, 21)))),
                  dict(pos_off=i32([0])), dict(page_table=i32(np.zeros((2, 65537))))):
        with pytest.raises(GooseError):
            goose.evict_kv(**{**base, **wrong})
    with pytest.raises(OverflowError):
        goose.evict_kv(**{**base, "budget": 2 ** 31})
    torch.cuda.synchronize()
    assert not goose.last_status(2).any()


@pytest.mark.parametrize("Hkv,S,page", [(8, 20, 16), (5, 64, 32), (64, 3, 16), (64, 6, 64), (20, 15, 16)])
def test_more_heads_than_the_device_has_sms(goose, Hkv, S, page):
    """All sizes of blocks, ragged sequences, some that lose nothing; ties."""
    rng = np.random.default_rng([Hkv, S])
    ctxs = rng.integers(0, 700, S).tolist()
    ctxs[0], ctxs[-1] = 300, 301
    Case(Hkv, ctxs, page, 300, 3, 20, off=rng.integers(0, 50, S).tolist(), seed=S).check(goose)
    Case(Hkv, ctxs, page, 129, 0, 0, seed=S + 1, weights=lambda r, shape: r.integers(0, 3, shape)).check(goose)


def test_more_heads_with_long_tables(goose):
    """Room for more keys than two or four blocks an SM have, sequences short and long."""
    Case(64, [500, 30, 700, 129, 128, 0], 16, 128, 4, 10, seed=20, width=900).check(goose)
    Case(40, [500, 30, 700, 129, 128, 0], 16, 128, 4, 10, seed=21, width=32768, room=40000).check(goose)
    Case(2, [17000] + [90] * 69, 16, 100, 4, 10, seed=22, room=25000, width=1700).check(goose)
    Case(2, [26000] + [90] * 69, 16, 25000, 4, 10, seed=23, room=26100, width=1700).check(goose)
