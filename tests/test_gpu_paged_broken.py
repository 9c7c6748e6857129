"""Tables with a page outside the pool and sequences that do not fit: what the calls that belong together make of one another's results.  Tolerances are those
of each call's own tests."""
import pytest
import torch

from _pages import D, attention, i32
from test_gpu_chunk_attn import Case as Chunk
from test_gpu_evict_kv import Case as Evict

pytestmark = pytest.mark.gpu
SCALE = D ** -0.5


@pytest.fixture(scope="module")
def goose():
    from paper_2604_02047_b200 import binding, build
    build.build()
    g = binding.Goose(max_S=70, max_B=16, max_H=64)
    yield g
    g.close()


def _added(c, s, lse):
    """What the tokens of sequence s that have been computed add to its rows, in 64 bits, [Hkv][rows]."""
    n, ctx = c.n[s], c.ctxs[s]
    K = c.c.keys(s, ctx + n)
    _, _, l, p = attention(c.q[s, :n], K, K, ctx, SCALE)
    Hkv = K.shape[1]
    off = (l - lse[s, :n].double()).view(n, Hkv, -1).permute(1, 2, 0)
    there = (lse[s, :n] != 0).view(n, Hkv, -1).permute(1, 2, 0)
    return (p * torch.where(there, torch.exp(off), 0.0)[..., None]).sum((1, 2))


@pytest.mark.parametrize("repaired", [False, True])
@pytest.mark.parametrize("B,ctx,broken", [(1, 9000, 500), (300, 200, 30), (300, 4000, 100), (17, 500, 31)])
def test_tokens_that_could_not_be_computed_add_nothing(goose, B, ctx, broken, repaired):
    """chunk_attn over a page outside the pool, kv_weights with its lse, before and after the table has been put right."""
    from paper_2604_02047_b200 import binding
    c = Chunk(8, 2, B, [ctx, 100], 16, seed=17)
    right = c.c.table
    wrong = right.clone()
    wrong[0, broken] = c.c.n_pages
    c.c.table = wrong
    out, lse = c.run(goose)
    assert goose.last_status(2).tolist() == [binding.ST_BAD_ROWS, 0]
    first = max(0, broken * 16 - ctx)
    assert not lse[0, first:].any()
    before = torch.rand(2, 2, ctx + B, device="cuda")
    weight = before.clone()
    goose.kv_weights(c.q, lse, c.c.k, right if repaired else wrong, c.ctx, SCALE, weight)
    assert goose.last_status(2).tolist() == [0 if repaired else binding.ST_BAD_ROWS, 0]
    for s in range(2):
        rows = c.ctxs[s] + B
        ref = _added(c, s, lse)
        if s == 0:
            page = slice(broken * 16, broken * 16 + 16)
            if not repaired:
                assert torch.equal(weight[0, :, page], before[0, :, page])
                ref[:, page] = 0
            if first == 0:
                assert torch.equal(weight[0], before[0])
        total = ref + before[s, :, :rows].double()
        over = (weight[s, :, :rows].double() - total).abs() - (1e-4 + B * 4 * 2.0 ** -24) * ref - 2.0 ** -23 * total
        assert over.max().item() <= 0, (s, over.max().item())
        assert torch.equal(weight[s, :, rows:], before[s, :, rows:])


def test_a_chunk_that_did_not_fit_and_a_part_of_it_that_does(goose):
    """The draft runs over the sequence's room, its first token alone would not: what the attention could not compute adds nothing."""
    from paper_2604_02047_b200 import binding
    c = Chunk(8, 2, 5, [59, 40], 16, seed=3, width=4)
    c.ctxs[0], c.ctx = 62, i32([62, 40])
    out, lse = c.run(goose)
    assert goose.last_status(2).tolist() == [binding.ST_BAD_ROWS, 0] and not out[0].any() and not lse[0].any()
    before = torch.rand(2, 2, 64, device="cuda")
    weight = before.clone()
    goose.kv_weights(c.q, lse, c.c.k, c.c.table, c.ctx, SCALE, weight, n_new=i32([1, 5]))
    assert not goose.last_status(2).any()
    assert torch.equal(weight[0], before[0]) and not torch.equal(weight[1], before[1])


@pytest.mark.parametrize("B,ctx,broken", [(300, 200, 30), (300, 4000, 260), (1000, 3000, 230), (60, 5000, 314)])
def test_tokens_in_front_of_a_broken_page(goose, B, ctx, broken):
    """Right or zeros, every token and head for itself, wherever the work on their rows was split; zeros from the first that sees the page on."""
    from paper_2604_02047_b200 import binding
    c = Chunk(8, 2, B, [ctx, 100], 16, seed=B)
    c.c.table_host[0, broken] = -1
    K, V = c.c.keys(0, ctx + B), c.c.values(0, ctx + B)        # (the page's rows are of some other one here, which no token in front of it sees)
    c.c.table = i32(c.c.table_host)
    out, lse = c.run(goose)
    assert goose.last_status(2).tolist() == [binding.ST_BAD_ROWS, 0]
    first = broken * 16 - ctx
    assert 0 < first < B and not out[0, first:].any() and not lse[0, first:].any()
    K[broken * 16:], V[broken * 16:] = 0, 0
    ref, A, l, _ = attention(c.q[0], K, V, ctx, SCALE)
    zero = (out[0, :first] == 0).all(-1)
    assert torch.equal(zero, lse[0, :first] == 0)
    near = ((out[0, :first].double() - ref[:first]).abs() <= 2.0 ** -8 * (1.2 * A + ref.abs())[:first]).all(-1)
    assert (zero | near).all()
    near = (lse[0, :first].double() - l[:first]).abs() <= 2e-4 + 2.0 ** -20 * l[:first].abs()
    assert (zero | near).all()
    c.check(goose, out, lse, skip=[0])


@pytest.mark.parametrize("given", [(), ("new_weight",), ("new_pos",)])
def test_a_sequence_that_cannot_be_cut_keeps_weights_and_positions(goose, given):
    """In arrays that the call makes; the next call ranks its rows by them."""
    from paper_2604_02047_b200 import binding
    c = Evict(2, [400, 300, 90], 16, 120, 4, 40, seed=10)
    c.c.table_host[1, 18] = c.c.n_pages
    c.c.table = i32(c.c.table_host)
    w, p = torch.tensor(c.weight, device="cuda"), i32(c.pos)
    spoilt = [torch.full_like(t, 7) for t in (w, p)]           # (what the allocator hands out next)
    del spoilt
    new = {n: {"new_weight": torch.full((2 * 3 * 310,), 9.0, device="cuda").view(3, 2, 310), "new_pos": torch.full_like(p, 9)}[n] for n in given}
    r = goose.evict_kv(c.c.k, c.c.v, c.c.table, c.ctx, w, p, 120, 4, 40, **new)
    assert goose.last_status(3).tolist() == [0, binding.ST_BAD_ROWS, 0] and r[0].tolist() == [120, 300, 90] and r[1].tolist() == [280, 0, 0]
    for got, old, name in ((r[2], w, "new_weight"), (r[3], p, "new_pos")):
        if name in given:
            assert (got[1] == 9).all()
        else:
            assert torch.equal(got[1, :, :300], old[1, :, :300])
        assert torch.equal(got[2, :, :90], old[2, :, :90])


def test_new_arrays_of_an_eviction_lie_in_nothing_that_it_reads(goose):
    """Refused ahead of any launch: the table and the caches too."""
    from paper_2604_02047_b200.binding import GooseError
    c = Evict(1, [300, 90], 16, 120, 4, 40, seed=11)
    w, p, k, v = torch.tensor(c.weight, device="cuda"), i32(c.pos), c.c.k, c.c.v
    ld = c.c.table.shape[1]
    inside = [dict(new_pos=c.c.table.view(2, 1, ld), new_weight=torch.zeros(2, 1, ld, device="cuda")),
              dict(new_weight=c.c.table.view(torch.float32).view(2, 1, ld), new_pos=torch.zeros(2, 1, ld, dtype=torch.int32, device="cuda")),
              dict(new_ctx_len=c.c.table.flatten()[3:5]), dict(new_pos_off=c.c.table.flatten()[-2:])]
    for cache in (k, v):
        words = cache.flatten().view(torch.int32)
        inside += [dict(new_ctx_len=words[:2]), dict(new_pos_off=words[-2:]), dict(new_pos=words[100:100 + p.numel()].view(p.shape)),
                   dict(new_weight=words[100:100 + p.numel()].view(torch.float32).view(p.shape))]
    before = [t.clone() for t in (c.c.table, k, v)]
    for new in inside:
        with pytest.raises(GooseError):
            goose.evict_kv(k, v, c.c.table, c.ctx, w, p, 120, 4, 40, **new)
    torch.cuda.synchronize()
    assert all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip((c.c.table, k, v), before)) and not goose.last_status(2).any()
    # arrays next to one another are allowed
    both = torch.zeros(2, *p.shape, dtype=torch.int32, device="cuda")
    lens = torch.zeros(4, dtype=torch.int32, device="cuda")
    r = goose.evict_kv(k, v, c.c.table, c.ctx, w, p, 120, 4, 40, new_weight=both[0].view(torch.float32), new_pos=both[1], new_ctx_len=lens[:2], new_pos_off=lens[2:])
    assert r[0].tolist() == [120, 90] and lens.tolist() == [120, 90, 180, 0] and not goose.last_status(2).any()
