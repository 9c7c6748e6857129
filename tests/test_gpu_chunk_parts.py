"""goose_chunk_attn where an item's keys are split over the device and the parts nearly cancel: what the parts have must be joined as it was summed.

All keys are zero, so that every score is 0, every term p = exp2(0) = 1 and its rounding to bf16 exact; values are multiples of 2^-8, three quarters of them of size
128 to 255, and for each of those there is its negative.  A part's sums are below 2^16 for the parts of up to 256 rows here, 24 bits with their last one: fp32
holds them exactly, in any order.  With signs that change every 256 rows (``block``) that goes for the sum of the parts so far as well, so an output is off
by its own rounding to bf16, 2^-8 of it, and by those of 1 / l and of the product with it, 2^-23 together.  With all negatives in the second half of the rows the sum so far grows
beyond that: every part that is added, one a CTA at most, then costs 2^-24 of what it is at its largest."""
import pytest
import torch

from _pages import D, Paged, i32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def goose():
    from paper_2604_02047_b200 import binding, build
    build.build()
    g = binding.Goose(max_S=4, max_B=16, max_H=64)
    yield g
    g.close()


@pytest.mark.parametrize("block", [256, None])
@pytest.mark.parametrize("H,Hkv,B,rows", [(2, 1, 1, 20001), (16, 1, 1, 20001), (1, 1, 256, 20256), (4, 1, 60, 20060), (4, 2, 3, 9003)])
def test_parts_keep_their_bits(goose, H, Hkv, B, rows, block):
    c = Paged([rows], Hkv, 16, seed=H + B)
    g = torch.Generator(device="cuda").manual_seed(B)
    half, ctx = (rows - B) // 2, rows - B
    V = (128 + torch.randint(0, 128, (rows, Hkv, D), generator=g, device="cuda")).double()
    small = torch.rand(rows, 1, 1, generator=g, device="cuda") < 0.25
    if block:
        at = torch.arange(rows, device="cuda")
        of = at % (2 * block)
        mirror = at - of + torch.where(of >= block, 2 * block - 1 - of, of)
        V = torch.where((of >= block)[:, None, None], -V[mirror], V)
        small = small[mirror]
        small[ctx // (2 * block) * 2 * block:] = True
    else:
        V[ctx - half:ctx] = -V[:half].flip(0)
        small[ctx - half:ctx] = small[:half].flip(0)
        small[half:ctx - half] = True
        small[ctx:] = True
    fraction = (torch.randint(-255, 256, V.shape, generator=g, device="cuda").double() / 256)
    V = torch.where(small, fraction, V)
    assert torch.equal(V.bfloat16().double(), V) and not block or V.cumsum(0).abs().max() < 2 ** 16
    at = c.rows(0, 0, rows)
    c.k.flatten(0, 1)[at], c.v.flatten(0, 1)[at] = 0, V.bfloat16()
    q = torch.randn(1, B, H, D, generator=g, device="cuda").bfloat16()
    out, lse = goose.chunk_attn(q, c.k, c.v, c.table, i32([ctx]), 1.0, want_lse=True)
    assert not goose.last_status(1).any()
    seen = torch.arange(ctx + 1, rows + 1, device="cuda").double()
    ref = (V.cumsum(0)[ctx:] / seen[:, None, None]).repeat_interleave(H // Hkv, 1)
    parts = torch.cuda.get_device_properties(0).multi_processor_count
    joined = 0 if block else parts * 2.0 ** -24 * V.cumsum(0).abs().max().item() / ctx
    over = (out[0].double() - ref).abs() - (2.0 ** -8 + 2.0 ** -23) * ref.abs() - joined
    assert over.max().item() <= 0, over.max().item()
    assert (lse[0].double() - seen.log()[:, None]).abs().max().item() < 1e-5
