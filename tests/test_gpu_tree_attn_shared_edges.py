"""goose_tree_attn_shared where its parts meet what they must not see or must not lose; reference and tolerance as in
test_gpu_tree_attn_shared.py."""
import pytest
import torch

from test_gpu_tree_attn_shared import Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def goose():
    from paper_2604_02047_b200 import binding, build
    build.build()
    g = binding.Goose(max_S=64, max_B=128, max_H=64)
    yield g
    g.close()


def test_rows_behind_the_last_key_in_tiles_of_one_warp(goose):
    """Four query rows a tile: three of the four warps that write the zeros behind the last key have no row themselves.  Every ragged length, the rows
    behind it infinite, time after time."""
    ctxs = [1 + (37 * s) % 127 for s in range(64)]
    c = Case(64, 32, 8, 1, 129, ctxs, seed=3).spoil()
    c.check(goose)
    first = [t.clone() for t in c.run(goose)]
    for _ in range(200):
        out, lse = c.run(goose)
        assert torch.equal(out, first[0]) and torch.equal(lse, first[1])


def _columns(c, powers):
    """The values' column d times 2^powers[d]."""
    c.v = (c.v.float() * torch.exp2(torch.tensor(powers, dtype=torch.float32, device="cuda"))).bfloat16()
    return c


# one column above all others, columns beside one another that differ, every column of a size of its own
COLUMNS = {"one, 2^16": [16.0 * (d == 37) for d in range(128)], "one, 2^24": [24.0 * (d == 64) for d in range(128)],
           "every other, 2^20": [20.0 * (d % 2) for d in range(128)], "2^-80 to 2^80": [float((53 * d) % 161 - 80) for d in range(128)]}


@pytest.mark.parametrize("powers", COLUMNS.values(), ids=COLUMNS.keys())
@pytest.mark.parametrize("S,H,Hkv,B,shared,ctxs", [(2, 4, 2, 16, 900, [300, 200]), (5, 8, 2, 1, 700, [30, 0, 500, 64, 129]), (1, 2, 1, 128, 20000, [7])])
def test_values_whose_columns_differ_in_size(goose, S, H, Hkv, B, shared, ctxs, powers):
    """Every column has its own bits in a partial result: the tolerance is element by element, A of an element being a sum over its column."""
    _columns(Case(S, H, Hkv, B, shared, ctxs, seed=B), powers).check(goose)


def test_an_infinite_value_stays_in_its_column(goose):
    """(The sizes of the other columns include some that half precision has no numbers for.)"""
    for size in (1.0, 1e6, 1e-10):
        c = Case(3, 8, 2, 9, 500, [100, 0, 300], seed=4)
        c.v = (c.v.float() * size).bfloat16()
        clean, lse = c.run(goose)
        c.check(goose, clean, lse)
        clean = clean.clone()
        c.v[c.shared_row + 7, :, 50] = float("inf")
        out, _ = c.run(goose)
        assert not torch.isfinite(out[..., 50]).any()
        assert torch.equal(out[..., :50], clean[..., :50]) and torch.equal(out[..., 51:], clean[..., 51:])


@pytest.mark.parametrize("S,H,Hkv,B,shared", [(64, 40, 40, 1, 1000), (64, 32, 8, 1, 1000), (1, 32, 8, 1, 500), (4, 16, 2, 128, 300), (16, 6, 2, 50, 0)])
def test_the_workspace_is_the_headers(S, H, Hkv, B, shared):
    """Device memory that a context's first call takes: goose.h's formula, and no more than a page or two."""
    from paper_2604_02047_b200 import binding
    sms, t = torch.cuda.get_device_properties(0).multi_processor_count, 128 // (H // Hkv)
    pairs, k = (lambda n: -(-(-(-n // t)) // 2)), (lambda n: max(2 ** e for e in range(6) if 2 ** e * min(n, t) * (H // Hkv) <= 128))
    up = lambda n, d: -(-n // d)  # noqa: E731
    formula = 51200 * ((up(2 * Hkv * pairs(S * B), k(S * B)) if shared else 0) + up(2 * S * Hkv * pairs(B), k(B)) + up(4 * sms, k(S * B) if shared else k(B)))
    goose = binding.Goose(max_S=S, max_B=128, max_H=64)
    c = Case(S, H, Hkv, B, shared, [20] * S)
    c.run(_another_context())                                      # (whatever a first call loads is there: another context's)
    torch.cuda.synchronize()
    before = torch.cuda.mem_get_info()[0]
    reserved = torch.cuda.memory_reserved()
    out, lse = c.run(goose)
    torch.cuda.synchronize()
    taken = before - torch.cuda.mem_get_info()[0] - (torch.cuda.memory_reserved() - reserved)
    assert 0 < taken <= formula + (4 << 20), (taken, formula)
    c.check(goose, out, lse)
    goose.close()


_warm = []


def _another_context():
    from paper_2604_02047_b200 import binding
    if not _warm:
        _warm.append(binding.Goose(max_S=64, max_B=128, max_H=64))
    return _warm[0]
