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
