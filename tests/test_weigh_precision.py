"""How precise the exponents of asd_kv_weigh are, where products are exact.

A weight is exp(scale z - lse), worked out as exp2(scale log2(e) z - lse log2(e)). Where scores and lse are large, a
rounding of either product is an error of the exponent that all weights of a row share, so both come in two parts (the
scale's, and of the lse what its rounded product lost). Keys and queries here are small whole numbers whose products are
exact in any order and precision, so that no rounding of the scores hides this.

The bound. In log2 units t is the exponent that is left, at most S + |z' - x| where rows of one offset differ by S. Its
two additions are rounded, 2^-24 |t| each, a relative error of ln 2 times that in the weight; the exponential has 2^-22;
the factor for what the lse's rounding lost and that for the row's distance from its offset are exponentials by exp2f,
two units (2 * 2^-23) each; three products are rounded, 2^-24 each, and a sum of n terms, n 2^-24.
"""
import math

import numpy as np
import pytest
import torch

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
U = 2.0 ** -24


def bound(exponent, spread, n):
    t = spread + 1 + exponent  # an offset is a whole number above the largest
    return 2 * U * t * math.log(2) + 2.0 ** -22 + 2 * 2.0 ** -22 + (3 + n) * U


class Problem:
    """Scores of about 9 sqrt(D) that differ by a few, an lse near them."""

    def __init__(self, dtype, B, T, Hq, Hkv, D, ctx, spread, seed=0):
        g = torch.Generator().manual_seed(seed)
        self.B, self.T, self.Hq, self.Hkv, self.D, self.ctx, self.spread = B, T, Hq, Hkv, D, ctx, spread
        self.q = torch.full((B, T, Hq, D), 8.0)
        self.q[..., : D // 4] -= torch.randint(2, (B, T, Hq, D // 4), generator=g)
        pages = B * -(-(ctx + T) // 16)
        self.table = torch.randperm(pages, generator=g).to(torch.int32).view(B, -1)
        self.k = torch.full((pages, 16, Hkv, D), 9.0)
        at = torch.randint(D, (pages, 16, Hkv, 2), generator=g)
        self.k.scatter_add_(3, at, -torch.ones(at.shape))
        self.q, self.k = self.q.to(dtype), self.k.to(dtype)
        self.scale = 1 / math.sqrt(D)
        slots = torch.arange(ctx + T)
        self.keys = self.k.double()[self.table.long()[:, slots // 16], slots % 16]  # [B, slots, Hkv, D]
        G = Hq // Hkv
        self.z = torch.einsum("bthd,bshd->bths", self.q.double(), self.keys.repeat_interleave(G, 2))
        near = self.z.mean(-1) * self.scale
        self.lse = (near + spread * (torch.rand(near.shape, generator=g) - 0.5) * math.log(2)).float()

    def exact(self):
        """Weights [B, Hkv, slots] and their bound."""
        see = torch.arange(self.ctx + self.T)[None, :] <= self.ctx + torch.arange(self.T)[:, None]  # [T, slots]
        away = self.z * self.scale - self.lse.double()[..., None]
        p = torch.exp(away) * see[:, None, :]

        def heads(x):
            return x.sum(1).view(self.B, self.Hkv, self.Hq // self.Hkv, -1).sum(2)
        rows = self.lse.double().view(self.B, self.T, self.Hkv, -1)
        apart = ((rows.amax((1, 3)) - rows.amin((1, 3))) / math.log(2)).repeat_interleave(self.Hq // self.Hkv, 1)
        n = self.T * self.Hq // self.Hkv
        return heads(p), heads(p * bound(away.abs() / math.log(2), apart[:, None, :, None], n))


def f32(x):
    return np.float64(np.float32(x))


def model(z, lse, scale, lost=True, rest=True, rest_first=False):
    """One row's weights with the roundings that the kernels have, products in 64 bits in between."""
    log2e = 1.4426950408889634
    by = f32(scale * log2e)
    short = f32(scale * log2e - by) if rest else 0.0
    x = f32(f32(lse) * f32(log2e))
    y = np.exp2(-(lse * log2e - x)) if lost else 1.0
    t = f32(z * by + f32(z * short - x)) if rest_first else f32(z * short + f32(z * by - x))
    return np.exp2(t) * y


@pytest.mark.parametrize("D", (72, 20, 136))
def test_the_bound_tells_one_part_from_two(D):
    """Mistakes in the model: without what the lse's product lost, without the scale's second part, and with that part
    added to the whole of the lse first, where it is rounded away."""
    p = Problem(F32, 6, 1, 1, 1, D, 300, 0.0, seed=D)
    exact, tol = p.exact()

    def off(**kw):
        worst = 0.0
        for b in range(p.B):
            got = np.array([model(float(z), float(p.lse[b, 0, 0]), p.scale, **kw) for z in p.z[b, 0, 0]])
            worst = max(worst, float((np.abs(got - exact[b, 0].numpy()) / tol[b, 0].numpy()).max()))
        return worst
    assert off() < 0.7
    for mistake in (dict(lost=False), dict(rest=False), dict(rest_first=True)):
        assert off(**mistake) > 2, mistake


@pytest.mark.gpu
@pytest.mark.parametrize("D", (72, 20, 136))
@pytest.mark.parametrize("dtype", (F32, F16, BF16), ids=("f32", "f16", "bf16"))
@pytest.mark.parametrize("T,Hq,Hkv,spread", [(1, 1, 1, 0.0), (5, 8, 2, 3.0), (40, 8, 2, 3.0)])
def test_exact_products(asd, dtype, D, T, Hq, Hkv, spread):
    p = Problem(dtype, 6, T, Hq, Hkv, D, 300, spread, seed=D)
    exact, tol = p.exact()
    cache = asd.KVCache(p.k.cuda(), p.k.cuda(), p.table.cuda())
    out = torch.full((6, Hkv, 300 + T), -1.0, device="cuda")
    asd.kv_weigh(p.q.cuda(), p.lse.cuda(), cache, torch.full((6,), 300, dtype=torch.int32, device="cuda"), None, decay=0.0,
                 out=out, scale=p.scale)
    off = (out.cpu().double() - exact).abs() / tol
    assert float(off.max()) <= 1
