"""The calls on a cache in pages at the ends of what they allow: pools behind 2^32 elements, work lists that need 64 bits, another stream than the
default one, two graphs that share a workspace, results on 16 bytes only.  Tolerances are those of each call's own tests; elsewhere the bits agree."""
import numpy as np
import pytest
import torch

from _pages import D, Paged, i32
from test_gpu_chunk_attn import Case as Chunk
from test_gpu_evict_kv import Case as Evict
from test_gpu_kv_weights import Case as Weights

pytestmark = pytest.mark.gpu
SCALE = D ** -0.5


@pytest.fixture(scope="module")
def goose():
    from paper_2604_02047_b200 import binding, build
    build.build()
    g = binding.Goose(max_S=70, max_B=16, max_H=64)
    yield g
    g.close()


def _near(c, n_pages, seed):
    """The pages of the sequences of ``c`` in a pool of n_pages, some of them at its end and around the 2^31-th and 2^32-th element: (k, v, table)."""
    p = c.c
    per = p.page * p.k.shape[2] * D
    spots = [n_pages - 1 - i for i in range(8)] + [x // per + i for x in (2 ** 31, 2 ** 32) for i in (-1, 0, 1)] + [0, 1]
    rng = np.random.default_rng(seed)
    used = [int(x) for x in np.unique(p.table_host[(p.table_host >= 0) & (p.table_host < p.n_pages)])]
    assert max(spots) < n_pages and len(set(spots)) == len(spots) and len(used) >= len(spots)
    rest = [x for x in rng.choice(n_pages, len(used) + len(spots), replace=False).tolist() if x not in spots]
    to = rng.permutation(spots + rest[:len(used) - len(spots)])
    at = dict(zip(used, to.tolist()))
    old, new = torch.tensor(used, device="cuda"), torch.tensor([at[x] for x in used], device="cuda")
    out = []
    for t in (p.k, p.v):
        big = torch.zeros(n_pages, *t.shape[1:], dtype=t.dtype, device="cuda") if t is not None else None
        if t is not None:
            big[new] = t[old]
        out.append(big)
    table = p.table_host.copy()
    for a, b in at.items():
        table[p.table_host == a] = b
    return *out, i32(table)


N_FAR = 2 ** 32 // (16 * 8 * D) + 37            # pages of 16 rows, 8 heads


def test_far_attention(goose):
    for c in (Chunk(32, 8, 3, [700, 90], 16, seed=1), Chunk(8, 8, 200, [150], 16, seed=2)):
        k, v, table = _near(c, N_FAR, 1)
        want = c.run(goose)
        out, lse = torch.full_like(c.q, 7.0), torch.full((c.S, c.B, c.H), 7.0, device="cuda")
        goose.chunk_attn(c.q, k, v, table, c.ctx, SCALE, out=out, lse=lse)
        assert not goose.last_status(c.S).any()
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
        c.check(goose, out, lse)
        del k, v


def test_far_weights(goose):
    for c in (Weights(32, 8, 3, [700, 90], 16, seed=3), Weights(8, 8, 200, [150], 16, seed=4)):
        k, _, table = _near(c, N_FAR, 2)
        weight = c.before.clone()
        goose.kv_weights(c.q, c.lse, k, table, c.ctx, SCALE, weight)
        assert not goose.last_status(c.S).any()
        assert torch.equal(weight, c.run(goose))
        c.check(goose, weight)
        del k


def test_far_eviction(goose):
    c = Evict(8, [400, 60], 16, 50, 4, 10, seed=5)
    want = c.run(goose)
    k, v, table = _near(c, N_FAR, 3)
    moved = [t[table[s, :-(-x // 16)].long()].flatten(0, 1)[:x].clone() for t in (k, v) for s, x in enumerate(c.ctxs)]
    r = goose.evict_kv(k, v, table, c.ctx, torch.tensor(c.weight, device="cuda"), i32(c.pos), c.budget, c.sink, c.recent)
    assert not goose.last_status(c.S).any()
    i = 0
    for t, w in ((k, want[0]), (v, want[1])):
        for s, x in enumerate(c.ctxs):
            got = t[table[s, :-(-x // 16)].long()].flatten(0, 1)[:x].view(torch.int16)
            ref = w.flatten(0, 1)[c.c.rows(s, 0, x)].view(torch.int16)
            assert torch.equal(got, ref) and not torch.equal(got, moved[i].view(torch.int16))
            i += 1
    assert torch.equal(r[0], want[4]) and torch.equal(r[1], want[5])


def test_far_rows_appended(goose):
    c = Chunk(8, 8, 150, [100, 0], 16, seed=6)
    k, v, table = _near(c, N_FAR, 4)
    kk, vv = c.c.k.clone(), c.c.v.clone()
    x = [torch.randn(2, 150, 8, D, device="cuda").bfloat16() for _ in range(3)]
    a = goose.append_kv_paged(*x, k, v, table, c.ctx)
    b = goose.append_kv_paged(*x, kk, vv, c.c.table, c.ctx)
    assert not goose.last_status(2).any() and torch.equal(a, b)
    for t, w in ((k, kk), (v, vv)):
        for s, n in enumerate((250, 150)):
            got = t[table[s, :-(-n // 16)].long()].flatten(0, 1)[:n]
            assert torch.equal(got, w.flatten(0, 1)[c.c.rows(s, 0, n)])


WIDE = 524288 // 16                             # entries of the longest table


def test_long_work_lists(goose):
    """The tables leave room for more places than 32 bits hold: the same split as with short tables, the same bits."""
    ctxs, new = [0, 3000, 7, 128] * 17, [600, 1, 33, 0] * 17
    args = (8, 2, 600, ctxs, 16)
    for a, b in ((Chunk(*args, new=new, seed=7), Chunk(*args, new=new, seed=7, width=WIDE)),):
        want, got = a.run(goose), b.run(goose)
        assert not goose.last_status(b.S).any()
        for s, n in enumerate(new):
            assert torch.equal(got[0][s, :n], want[0][s, :n]) and torch.equal(got[1][s, :n], want[1][s, :n])
    del a, b, want, got
    a, b = Weights(*args, new=new, seed=8, room=3700), Weights(*args, new=new, seed=8, width=WIDE, room=524288)
    b.before[:, :, :3700] = a.before
    want, got = a.run(goose), b.run(goose)
    assert not goose.last_status(b.S).any()
    assert torch.equal(got[:, :, :3700], want) and torch.equal(got[:, :, 3700:], b.before[:, :, 3700:])
    a.check(goose, want)


def test_longest_tables(goose):
    """Rows at the end of the longest sequence that the calls allow."""
    n = 524288
    c = Chunk(2, 1, 3, [n - 3], 16, seed=9, width=WIDE)
    c.check(goose)
    w = Weights(2, 1, 3, [n - 3], 16, seed=9, width=WIDE, room=n)
    w.check(goose)
    e = Evict(1, [n], 16, 1000, 4, 100, seed=10, width=WIDE, room=n, new_room=1000)
    e.check(goose)


def test_other_streams(goose):
    """Calls on a stream whose earlier work is still to come when they are made; the default stream has work of its own."""
    c, w, e = Chunk(32, 8, 20, [500, 60], 16, seed=11), Weights(32, 8, 20, [500, 60], 16, seed=12), Evict(8, [400, 300], 16, 100, 4, 10, seed=13)
    want = c.run(goose), w.run(goose), e.run(goose)
    q, lse, pos = c.q.clone(), w.lse.clone(), i32(e.pos)
    weight0 = torch.tensor(e.weight, device="cuda")
    busy = torch.randn(4096, 4096, device="cuda")
    c.q.zero_(), w.lse.zero_()
    k, v = e.c.k.clone(), e.c.v.clone()
    ew = torch.zeros_like(weight0)
    out, l = torch.full_like(q, 7.0), torch.full_like(want[0][1], 7.0)
    weight = torch.zeros_like(w.before)
    nw, npos = torch.full_like(want[2][2], 7.0), torch.full_like(want[2][3], 7)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        for _ in range(20):
            torch.mm(busy, busy)
        c.q.copy_(q), w.lse.copy_(lse), ew.copy_(weight0), weight.copy_(w.before)
        goose.chunk_attn(c.q, c.c.k, c.c.v, c.c.table, c.ctx, SCALE, out=out, lse=l)
        goose.kv_weights(w.q, w.lse, w.c.k, w.c.table, w.ctx, SCALE, weight)
        r = goose.evict_kv(k, v, e.c.table, e.ctx, ew, pos, e.budget, e.sink, e.recent, new_weight=nw, new_pos=npos)
    torch.mm(busy, busy)
    stream.synchronize()
    assert torch.equal(out, want[0][0]) and torch.equal(l, want[0][1]) and torch.equal(weight, want[1])
    e.check(goose, (k, v, nw, npos, r[0], r[1]))


def test_two_graphs(goose):
    """Two graphs of the same context and its workspace, replayed in turn."""
    cases = [(Chunk(32, 8, n, x, 16, seed=n), Weights(32, 8, n, x, 16, seed=n), Evict(8, x, 16, 100, 4, 10, seed=n)) for n, x in ((1, [5000, 100]), (300, [40, 3000, 0]))]
    graphs, held, wants = [], [], []
    for c, w, e in cases:
        wants.append((c.run(goose), w.run(goose), e.run(goose)))
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        for (c, w, e), want in zip(cases, wants):
            t = dict(out=torch.empty_like(c.q), lse=torch.empty_like(want[0][1]), weight=w.before.clone(), k=e.c.k.clone(), v=e.c.v.clone(),
                     ew=torch.tensor(e.weight, device="cuda"), pos=i32(e.pos), nw=torch.full_like(want[2][2], 7.0), np=torch.full_like(want[2][3], 7))
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                goose.chunk_attn(c.q, c.c.k, c.c.v, c.c.table, c.ctx, SCALE, out=t["out"], lse=t["lse"])
                goose.kv_weights(w.q, w.lse, w.c.k, w.c.table, w.ctx, SCALE, t["weight"])
                t["r"] = goose.evict_kv(t["k"], t["v"], e.c.table, e.ctx, t["ew"], t["pos"], e.budget, e.sink, e.recent, new_weight=t["nw"], new_pos=t["np"])
            graphs.append(graph), held.append(t)
        for _ in range(3):
            for (c, w, e), t in zip(cases, held):
                t["out"].fill_(7.0), t["weight"].copy_(w.before), t["k"].copy_(e.c.k), t["v"].copy_(e.c.v)
            for g in graphs:
                g.replay()
            stream.synchronize()
            for (c, w, e), t, want in zip(cases, held, wants):
                assert torch.equal(t["out"], want[0][0]) and torch.equal(t["lse"], want[0][1]) and torch.equal(t["weight"], want[1])
                e.check(goose, (t["k"], t["v"], t["nw"], t["np"], t["r"][0], t["r"][1]))


def test_sixteen_bytes(goose):
    """q and out that begin on 16 bytes and on no more."""
    for c in (Chunk(8, 2, 300, [70], 16, seed=14), Chunk(40, 40, 8, [200, 30], 16, seed=15)):
        want = c.run(goose)
        q, out = [torch.full((c.q.numel() + 8,), 7.0, dtype=torch.bfloat16, device="cuda")[8:].view(c.q.shape) for _ in range(2)]
        q.copy_(c.q)
        assert q.data_ptr() % 32 == 16 and out.data_ptr() % 32 == 16
        goose.chunk_attn(q, c.c.k, c.c.v, c.c.table, c.ctx, SCALE, out=out)
        assert torch.equal(out, want[0])
        w = Weights(8, 2, 20, [70], 16, seed=16)
        a = w.run(goose)
        wq = torch.empty(w.q.numel() + 8, dtype=torch.bfloat16, device="cuda")[8:].view(w.q.shape)
        w.q = wq.copy_(w.q)
        assert torch.equal(w.run(goose), a)


def test_weights_of_any_lse(goose):
    """+infinity: nothing (2^-126 at most); NaN: NaN for the rows that the token sees, no other."""
    w = Weights(8, 2, 150, [200], 16, seed=17)
    a = w.run(goose)
    w.lse[0, 40, 5] = torch.inf
    p = w.p[0][1, 1, 40].clone()
    w.p[0][1, 1, 40] = 0
    w.check(goose)
    w.p[0][1, 1, 40] = p
    w.lse[0, 40, 5] = torch.nan
    b = w.run(goose)
    assert torch.isnan(b[0, 1, :241]).all() and torch.equal(b[0, 0], a[0, 0]) and torch.equal(b[0, 1, 241:], a[0, 1, 241:])
