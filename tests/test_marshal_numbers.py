"""Numbers on their way to the C entry points: one that its C type does not hold is refused, not cut to what is left of it (a shared prefix of
2^32 + 5 rows is none of 5 rows).  No GPU: the numbers are looked at before the call."""
import pytest

from paper_2604_02047_b200 import binding, build


@pytest.fixture(scope="module")
def marshal():
    build.build()
    return binding.load_marshal()


INT_MAX = 2 ** 31 - 1
# arguments of goose_tree_attn_shared: context, q, caches, kv_rows, shared_row (64 bits), shared_len (32), row_off, ctx_len, parent, n_nodes, S, B, ...
SHARED = [None, None, None, None, 100, 0, 5, None, None, None, None, 1, 1, 1, 1, 128, 1.0, None, None]
# of goose_node_topk: context, logits, rows, V, ldl (64 bits), k, n_nodes, B, argmax, ids, values
TOPK = [None, None, 1, 100, 104, 4, None, 0, None, None, None]


@pytest.mark.parametrize("entry,args,at", [("tree_attn_shared", SHARED, i) for i in (6, 11, 12, 13, 14, 15)] + [("node_topk", TOPK, i) for i in (2, 3, 5, 7)])
@pytest.mark.parametrize("value", [2 ** 31, 2 ** 32, 2 ** 32 + 5, -2 ** 31 - 1, 2 ** 63 - 1, 2 ** 64])
def test_numbers_beyond_32_bits(marshal, entry, args, at, value):
    with pytest.raises(OverflowError):
        getattr(marshal, entry)(*[value if i == at else a for i, a in enumerate(args)])


@pytest.mark.parametrize("entry,args,at", [("tree_attn_shared", SHARED, 4), ("tree_attn_shared", SHARED, 5), ("node_topk", TOPK, 4)])
def test_numbers_beyond_64_bits(marshal, entry, args, at):
    with pytest.raises(OverflowError):
        getattr(marshal, entry)(*[2 ** 63 if i == at else a for i, a in enumerate(args)])


def test_no_number(marshal):
    with pytest.raises(TypeError):
        marshal.tree_attn_shared(*[("five" if i == 6 else a) for i, a in enumerate(SHARED)])
