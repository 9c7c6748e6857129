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
