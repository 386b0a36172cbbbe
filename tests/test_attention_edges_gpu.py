"""asd_tree_attention at further edges, against the plain 64-bit implementation or from the definition."""
import math

import pytest
import torch

from test_attention_gpu import BF16, F16, F32, Problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,D", [(F32, 64), (F32, 200), (F16, 64), (BF16, 128), (F16, 256), (BF16, 36)])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("new", [False, True], ids=["context", "new-token"])
def test_what_a_row_does_see_reaches_it_however_small_its_weight(asd, dtype, D, bad, new):
    """A value that is not finite, of a key whose weight is less than the smallest fp32 number: no softmax weight is
    zero, so the rows that see it are not finite in that element, and all the others are as without it."""
    T, B = 4, 2
    ctx = [100, 20]  # beyond a tile of 64 and within one
    parents = torch.tensor([[-1, 0, 0, 1]] * B)
    p = Problem(dtype, T, 4, 2, D, 16, ctx=ctx, seed=31)
    p.mask = asd.tree_mask(parents)
    p.scale = 1.0
    p.q[..., 0] = 16.0
    slots = [c + 1 if new else c - 7 for c in ctx]
    for b in range(B):
        for s in range(ctx[b] + T):
            page, place = p.place(b, s)
            p.k[page, place, :, 0] = 0.0
        page, place = p.place(b, slots[b])
        p.k[page, place, :, 0] = -32.0  # a score 512 below the others': exp(-512) < 2^-700
    good, good_lse, _ = p.run(asd)
    p.check(good, good_lse)
    for b in range(B):
        page, place = p.place(b, slots[b])
        p.v[page, place, 1, 9] = bad
    out, lse, status = p.run(asd)
    assert not status.any() and torch.equal(lse, good_lse)
    hit = torch.zeros(B, T, 4, D, dtype=torch.bool)
    hit[:, [1, 3] if new else slice(None), 2:, 9] = True
    assert not bool(out[hit].isfinite().any())
    assert torch.equal(out[~hit], good[~hit])
