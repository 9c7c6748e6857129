"""goose_append_kv_paged: what goose_append_kv does with a run of tokens, into pages; the new rows' weights and positions.  Formula and tolerance are
test_gpu_append_kv's."""
import numpy as np
import pytest
import torch

from _pages import D, Paged, i32
from test_gpu_append_kv import _close, _normal, _table, _turned

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def goose():
    from paper_2604_02047_b200 import binding, build
    build.build()
    g = binding.Goose(max_S=40, max_B=16, max_H=64)
    yield g
    g.close()


def _run(goose, H, Hkv, B, ctxs, page, *, new=None, norm=True, rot=D, interleaved=False, pos_off=None, seed=0, in_place=False, arrays="wp"):
    S = len(ctxs)
    g = torch.Generator(device="cuda").manual_seed(seed)
    if in_place:
        q, k, v = (_normal(g, S, B, h, D) for h in (H, Hkv, Hkv))
    else:
        q, k, v = _normal(g, S, B, H + 2 * Hkv + 1, D)[:, :, :H + 2 * Hkv].split([H, Hkv, Hkv], 2)
    n = [B] * S if new is None else new
    c = Paged([x + m if m else 0 for x, m in zip(ctxs, n)], Hkv, page, seed=seed)
    k0, v0 = c.k.clone(), c.v.clone()
    pos = [0] * S if pos_off is None else pos_off
    table = _table(rot, max(p + x for p, x in zip(pos, ctxs)) + B)
    wq, wk = [(1 + 0.3 * torch.randn(D, generator=g, device="cuda")).bfloat16() if norm else None for _ in range(2)]
    out = q if in_place else torch.full((S, B, H, D), 7.0, dtype=torch.bfloat16, device="cuda")
    q0 = q.clone()
    room = max(x + B for x in ctxs) + 2
    weight = torch.full((S, Hkv, room), 7.0, device="cuda") if "w" in arrays else None
    row_pos = torch.full((S, Hkv, room), 7, dtype=torch.int32, device="cuda") if "p" in arrays else None
    goose.append_kv_paged(q, k, v, c.k, c.v, c.table, i32(ctxs), rope=table if rot else None, n_new=None if new is None else i32(new),
                          pos_off=None if pos_off is None else i32(pos_off), q_weight=wq, k_weight=wk, eps=1e-5, interleaved=interleaved,
                          row_weight=weight, row_pos=row_pos, out=out)
    torch.cuda.synchronize()
    assert not goose.last_status(S).any()
    for s in range(S):
        at = table[pos[s] + ctxs[s]:][:n[s]]
        assert torch.equal(out[s, n[s]:], (q0 if in_place else torch.full_like(out, 7.0))[s, n[s]:])
        rows = c.rows(s, ctxs[s], ctxs[s] + n[s])
        if n[s]:
            _close(out[s, :n[s]], *_turned(q0[s, :n[s]], wq, at, rot, interleaved, 1e-5))
            _close(c.k.flatten(0, 1)[rows], *_turned(k[s, :n[s]], wk, at, rot, interleaved, 1e-5))
        k0.flatten(0, 1)[rows] = c.k.flatten(0, 1)[rows]
        v0.flatten(0, 1)[rows] = v[s, :n[s]]
        for t, want in ((weight, torch.zeros(n[s], device="cuda")), (row_pos, pos[s] + ctxs[s] + torch.arange(n[s], device="cuda"))):
            if t is not None:
                assert (t[s, :, ctxs[s]:ctxs[s] + n[s]] == want).all() and (t[s, :, :ctxs[s]] == 7).all() and (t[s, :, ctxs[s] + n[s]:] == 7).all()
    for got, want in ((c.k, k0), (c.v, v0)):
        assert torch.equal(got.view(torch.int16), want.view(torch.int16))


@pytest.mark.parametrize("rot,interleaved", [(128, False), (128, True), (64, False), (16, True), (0, False)])
@pytest.mark.parametrize("norm", [True, False])
def test_forms(goose, rot, interleaved, norm):
    _run(goose, 8, 2, 21, [0, 130, 17], 16, rot=rot, interleaved=interleaved, norm=norm)


@pytest.mark.parametrize("H,Hkv", [(1, 1), (3, 1), (32, 8), (40, 40), (52, 52), (64, 4), (16, 1)])
@pytest.mark.parametrize("B,page", [(1, 16), (2, 32), (300, 64)])
def test_heads(goose, H, Hkv, B, page):
    _run(goose, H, Hkv, B, [3, 200], page, seed=H + B)


@pytest.mark.parametrize("page", [16, 128, 1024])
def test_ragged(goose, page):
    _run(goose, 8, 2, 1000, [0, 15, 16, 3000], page, new=[1000, 0, 1, 999], pos_off=[0, 5, 20000, 512], rot=64)
    _run(goose, 8, 2, 7, [0, 15, 16, 3000], page, arrays="w")
    _run(goose, 8, 2, 7, [0, 15, 16, 3000], page, arrays="p", in_place=True)
    _run(goose, 8, 2, 7, [0, 15, 16, 3000], page, arrays="", rot=0, norm=False)


def test_the_same_as_without_pages(goose):
    """Bit by bit what goose_append_kv puts into consecutive rows."""
    g = torch.Generator(device="cuda").manual_seed(5)
    B, H, Hkv = 200, 8, 2
    q, k, v = (_normal(g, 2, B, h, D) for h in (H, Hkv, Hkv))
    w, table = _normal(g, D), _table(D, 400)
    c = Paged([30 + B, 50 + B], Hkv, 16, seed=5)
    out = goose.append_kv_paged(q, k, v, c.k, c.v, c.table, i32([30, 50]), rope=table, q_weight=w, k_weight=w)
    kc, vc = (torch.zeros(600, Hkv, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    want = goose.append_kv(q, k, v, kc, vc, torch.tensor([0, 300], device="cuda"), i32([30, 50]), rope=table, q_weight=w, k_weight=w)
    assert torch.equal(out, want)
    for s, (off, ctx) in enumerate(((0, 30), (300, 50))):
        rows = c.rows(s, ctx, ctx + B)
        assert torch.equal(c.k.flatten(0, 1)[rows], kc[off + ctx:][:B]) and torch.equal(c.v.flatten(0, 1)[rows], vc[off + ctx:][:B])


def test_broken_sequences(goose):
    """Rows that do not fit, a page outside the pool (its tokens alone), positions outside the table or an int32, counts outside [0, B]."""
    from paper_2604_02047_b200 import binding
    g = torch.Generator(device="cuda").manual_seed(2)
    S, B, H, Hkv = 6, 20, 4, 2
    q, k, v = (_normal(g, S, B, h, D) for h in (H, Hkv, Hkv))
    c = Paged([40] * S, Hkv, 16, seed=2, width=3)
    c.table_host[2, 1] = c.n_pages
    c.table = i32(c.table_host)
    k0, v0 = c.k.clone(), c.v.clone()
    weight = torch.full((S, Hkv, 48), 7.0, device="cuda")
    out = goose.append_kv_paged(q, k, v, c.k, c.v, c.table, i32([3, 29, 10, 17, 3, -1]), rope=_table(128, 40), pos_off=i32([0, 0, 0, 10, 0, 0]),
                                n_new=i32([20, 20, 20, 20, 21, 20]), row_weight=weight, out=torch.full_like(q, 7.0))
    assert goose.last_status(S).tolist() == [0, binding.ST_BAD_ROWS | binding.ST_BAD_POS, binding.ST_BAD_ROWS, binding.ST_BAD_POS, binding.ST_BAD_NODES,
                                             binding.ST_BAD_ROWS | binding.ST_BAD_POS]
    assert out[0].any(-1).all() and not out[1].any() and not out[2, 6:].any() and out[2, :6].any(-1).all() and not out[3, 13:].any()
    assert (out[4] == 7).all() and not out[5].any()
    live = {0: range(3, 23), 2: range(10, 16), 3: range(17, 30)}
    for s in range(S):
        for j in live.get(s, ()):
            row = c.rows(s, j, j + 1)
            k0.flatten(0, 1)[row], v0.flatten(0, 1)[row] = c.k.flatten(0, 1)[row], v[s, j - live[s].start]
        mine = torch.zeros(48, dtype=torch.bool, device="cuda")
        mine[list(live.get(s, ()))] = True
        assert (weight[s, :, mine] == 0).all() and (weight[s, :, ~mine] == 7).all()
    for got, want in ((c.k, k0), (c.v, v0)):
        assert torch.equal(got.view(torch.int16), want.view(torch.int16))
    # positions that are no int32; an array that is too short
    pos = torch.full((1, Hkv, 48), 7, dtype=torch.int32, device="cuda")
    c = Paged([40], Hkv, 16, seed=3)
    goose.append_kv_paged(q[:1], k[:1], v[:1], c.k, c.v, c.table, i32([10]), pos_off=i32([2 ** 31 - 20]), row_pos=pos)
    assert goose.last_status(1).tolist() == [binding.ST_BAD_POS] and (pos[..., 10:20] > 0).all() and (pos[..., 20:] == 7).all()
    goose.append_kv_paged(q[:1], k[:1], v[:1], c.k, c.v, c.table, i32([10]), row_pos=pos[..., :29].contiguous())
    assert goose.last_status(1).tolist() == [binding.ST_BAD_ROWS]


def test_refusals(goose):
    from paper_2604_02047_b200.binding import GooseError
    z = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    base = dict(q=z(2, 4, 8, D), k=z(2, 4, 2, D), v=z(2, 4, 2, D), k_cache=z(9, 16, 2, D), v_cache=z(9, 16, 2, D), page_table=i32([[0, 1], [2, 3]]),
                ctx_len=i32([0, 0]), rope=_table(128, 64), row_weight=torch.zeros(2, 2, 32, device="cuda"), row_pos=i32(np.zeros((2, 2, 32))))
    goose.append_kv_paged(**base)
    for wrong in (dict(k=z(2, 4, 3, D)), dict(q=z(2, 4, 8, D).float()), dict(v=z(4, 2, 2, D).transpose(0, 1)), dict(rope=_table(24, 64)), dict(q=z(2, 4, 65, D)),
                  dict(eps=-1.0), dict(out=z(2, 4, 7, D)), dict(q_weight=z(64)), dict(ctx_len=i32([0])), dict(n_new=i32([1])), dict(k_cache=z(9, 8, 2, D), v_cache=z(9, 8, 2, D)),
                  dict(k_cache=z(3, 48, 2, D), v_cache=z(3, 48, 2, D)), dict(page_table=i32([[0, 1]])), dict(row_weight=torch.zeros(2, 2, 31, device="cuda")),
                  dict(row_pos=torch.zeros(2, 2, 32, device="cuda")), dict(row_weight=torch.zeros(2, 1, 32, device="cuda")), dict(page_table=i32(np.zeros((2, 0))))):
        with pytest.raises(GooseError):
            goose.append_kv_paged(**{**base, **wrong})
    torch.cuda.synchronize()
    assert not goose.last_status(2).any()
