"""The exponentials of goose_kv_weights, each by itself, against 64 bits: all keys are zero, and every (sequence, head) has one token whose log-sum-exp is
finite, in any column of a tile of 128 query rows, so that a row's weight is exp(-lse) of it.  (+infinity elsewhere: 0 or, of the
polynomial, 2^-126, from 32 columns in all: 2^-121 of the sum.)

Tolerance, relative.  Every fourth pair of columns comes of a polynomial, 1.7e-7; the others of the special function unit, two units in the last place, 2.4e-7.
Its argument in units of log 2: -lse in three parts, added in the tensor cores to 2^-22 of it; log2(e) and the product with it 2^-24 each.  In exp that is 1.5 * 2^-22 * |lse|."""
import pytest
import torch

from _pages import D, Paged, i32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def goose():
    from paper_2604_02047_b200 import binding, build
    build.build()
    g = binding.Goose(max_S=16, max_B=16, max_H=64)
    yield g
    g.close()


@pytest.mark.parametrize("low,high", [(-0.7, 0.7), (-2.0, 10.0), (-30.0, 80.0)])
def test_every_exponential(goose, low, high):
    S, H, B, ctx = 16, 64, 128, 256
    c = Paged([ctx + B] * S, H, 64)
    c.k.zero_()
    q = torch.zeros(S, B, H, D, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(int(high))
    heads = torch.arange(H, device="cuda")
    for turn in range(8):
        x = low + (high - low) * torch.rand(S, H, generator=g, device="cuda")
        lse = torch.full((S, B, H), torch.inf, device="cuda")
        column = (torch.arange(S * H, device="cuda").view(S, H) + 16 * turn) % B
        lse[torch.arange(S, device="cuda")[:, None], column, heads] = x
        weight = torch.zeros(S, H, ctx + B, device="cuda")
        goose.kv_weights(q, lse, c.k, c.table, i32([ctx] * S), 1.0, weight)
        assert not goose.last_status(S).any()
        ref = torch.exp(-x.double())[..., None]
        off = (weight[..., :ctx].double() / ref - 1).abs() - 2.4e-7 - (1.5 * 2.0 ** -22 * x.double().abs())[..., None] - 2.0 ** -121 / ref
        assert off.max().item() <= 0, off.max().item()


@pytest.mark.parametrize("size", [3.3895e38, 3.3953e38, 3.3961e38, 3.4e38, 3.4028e38, float("inf")])
def test_the_largest_log_sum_exps(goose, size):
    """-lse / scale of a size that bf16 has just, or rounds to infinity: nothing is added where exp(-lse) is 0, and rows that do not see the token are as they were."""
    scale = 2.0 ** -97
    c = Paged([300], 2, 16)
    c.k.zero_()
    q = torch.zeros(1, 140, 2, D, dtype=torch.bfloat16, device="cuda")
    lse = torch.zeros(1, 140, 2, device="cuda")
    plain = torch.zeros(1, 2, 300, device="cuda")
    goose.kv_weights(q, lse, c.k, c.table, i32([160]), scale, plain)
    lse[0, 6, 0] = lse[0, 135, 0] = torch.tensor(size).float() * scale
    weight = torch.zeros(1, 2, 300, device="cuda")
    goose.kv_weights(q, lse, c.k, c.table, i32([160]), scale, weight)
    assert not goose.last_status(1).any()
    sees = (torch.arange(300, device="cuda") <= 160 + 6).float() + (torch.arange(300, device="cuda") <= 160 + 135).float()
    assert torch.equal(weight[0, 1], plain[0, 1])
    # (140 terms of exp(0): each to 2.4e-7, sums of them to 2^-24 an addition)
    assert (weight[0, 0] - (plain[0, 0] - sees)).abs().max() <= 140 * (2.4e-7 + 2.0 ** -24 * 140)
