"""More sequences than a grid has rows (65535), in a context that allows them: the operators around the step refuse them as an argument, with nothing
enqueued.  The largest number that they take is computed."""
import pytest
import torch

pytestmark = pytest.mark.gpu
D, MOST = 128, 65535


@pytest.fixture(scope="module")
def goose():
    from paper_2604_02047_b200 import binding, build
    build.build()
    g = binding.Goose(max_S=MOST + 1, max_B=1, max_H=1)
    yield g
    g.close()


def _bf16(*shape):
    return torch.randn(shape, device="cuda").bfloat16()


def _calls(goose, S):
    i32 = lambda v: torch.full((S,), v, dtype=torch.int32, device="cuda")  # noqa: E731
    row_off, parent = torch.arange(S, device="cuda"), i32(-1).view(S, 1)
    q, k, v = _bf16(S, 1, 1, D), _bf16(S, 1, 1, D), _bf16(S, 1, 1, D)
    kc, vc = k.view(S, 1, D).clone(), v.view(S, 1, D).clone()
    logits = _bf16(S, 8)
    return {"append_kv": lambda: torch.equal(goose.append_kv(q, k, v, kc, vc, row_off, i32(0)), q),
            # a node that sees itself alone: its value
            "tree_attn_shared": lambda: torch.equal(goose.tree_attn_shared(q, kc, vc, 0, 0, row_off, i32(0), parent, 0.1), v),
            "adjust_logits": lambda: torch.equal(goose.adjust_logits(logits, None, None, None, parent), logits)}


@pytest.mark.parametrize("call", ["append_kv", "tree_attn_shared", "adjust_logits"])
def test_as_many_as_a_grid_has_and_one_more(goose, call):
    from paper_2604_02047_b200.binding import GooseError
    assert _calls(goose, MOST)[call]()
    torch.cuda.synchronize()
    launched = goose.launch_count()
    with pytest.raises(GooseError, match="invalid argument"):
        _calls(goose, MOST + 1)[call]()
    assert goose.launch_count() == launched
    torch.cuda.synchronize()
    assert not goose.last_status(MOST).any()
