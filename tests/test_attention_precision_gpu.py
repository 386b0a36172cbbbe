"""Tree attention where its arithmetic is narrowest: long sums, and softmax weights far apart.

A context repeats one page many times, so that a long one costs little memory and its reference in 64 bits is a sum over
one page's slots with the number of times that each occurs.
"""
import math

import pytest
import torch

from cache_reference import UNIT

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16
PAGE = 128


def tolerance(dtype, D, slots, reach, weight, out):
    """Elementwise bound on |out - reference| of the tensor-core kernel for a unit that one CTA walks through.

    Scores: sums of D products in 32 bits. Weights: twice a score's error, the exponential's few units, one rounding to
    the type. Sums: each of two groups adds half of the slots, 16 an instruction, which may cut off (a unit in the last
    place is 2u) where a sum rounds (u). f16 weights below 2^-14 are off by half their spacing, 2^-25, where the largest
    is 2^7. The result is rounded once.
    """
    u = 2.0 ** -24
    rel = 2 * (D + 2) * u * reach + 2.0 ** -21 + 2 * u * (slots / 32)
    tol = rel * weight + UNIT[dtype] * (weight + out.abs())
    return tol + (slots * 2.0 ** -32 if dtype == F16 else 0.0)


@pytest.mark.parametrize("at", [0, 977, 1952], ids=["first", "middle", "last"])
@pytest.mark.parametrize("ahead", [10.0, 20.6, 23.0, 25.1])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_one_strong_key_and_many_weak_ones(asd, dtype, D, ahead, at):
    """The weak keys' weights, 2^-ahead of the strong one's each, add up to a share of the result that counts."""
    B, H, G, pages = 19, 8, 2, 1954  # a unit a CTA, or nearly: no piece without the strong key
    slots = pages * PAGE
    g = torch.Generator().manual_seed(int(ahead * 10) + D)
    k = torch.randn(2, PAGE, H, D, generator=g) * 0.05
    v = 0.5 + torch.rand(2, PAGE, H, D, generator=g)
    k[1], v[1] = k[0], v[0]
    k[:, :, :, 0] = 0
    k[1, 5, :, 0] = ahead * math.log(2)
    v[1, 5] = 0
    k, v = k.to(dtype), v.to(dtype)
    q = torch.randn(B, 1, H * G, D, generator=g)
    q[..., 0] = 1
    q = q.to(dtype)
    table = torch.zeros(B, pages, dtype=torch.int32)
    table[:, at] = 1
    cache = asd.KVCache(k.cuda(), v.cuda(), table.cuda())
    kv_len = torch.full((B,), slots - 1, dtype=torch.int32, device="cuda")
    got = asd.tree_attention(q.cuda(), cache, kv_len, scale=1.0)

    x = q.double().view(B, H, G, D)
    z = torch.einsum("bhgd,pshd->bhgps", x, k.double())
    times = torch.tensor([pages - 1.0, 1.0], dtype=torch.float64)[:, None]
    top = z.amax((-1, -2), keepdim=True)
    w = (z - top).exp() * times
    total = w.sum((-1, -2))
    want = torch.einsum("bhgps,pshd->bhgd", w, v.double()) / total[..., None]
    reach = torch.einsum("bhgd,pshd->bhgps", x.abs(), k.double().abs()).amax((-1, -2))[..., None]
    far = (got["out"].cpu().double().view_as(want) - want).abs() - tolerance(dtype, D, slots, reach, want, want)
    assert float(far.max()) <= 0, f"{float(far.max()):.3g} further off than it may be"
    lse = (top[..., 0, 0] + total.log())
    gap = (got["lse"].cpu().double().view_as(lse) - lse).abs()
    # a thread adds 128 weights a tile, half of the tiles in turn, and the tiles' sums one after the other
    may = (D + 2) * 2.0 ** -24 * reach[..., 0] + 2.0 ** -20 + (slots / 256 + 40) * 2.0 ** -24 + lse.abs() * 2.0 ** -22
    assert float((gap - may).max()) <= 0
