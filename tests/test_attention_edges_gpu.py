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


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("tree", [False, True], ids=["chain", "tree"])
def test_the_last_slots_that_31_bits_count(asd, dtype, tree):
    """A context of 2^31 - 3 slots, nearly all of them on one page, and two new tokens: what is masked in the last tile
    still is. The new tokens' keys outweigh the context by e^-40 a slot."""
    page, width, D = 65536, 32768, 8
    k = torch.zeros(2, page, 1, D, dtype=dtype)
    v = torch.ones_like(k)
    k[1, -1] = v[1, -1] = math.nan  # slot 2^31 - 1, which no length reaches
    k[1, -3, 0, 0], k[1, -2, 0, 0] = 40.0, 48.0
    v[1, -3], v[1, -2] = 3.0, 5.0
    if tree:
        v[1, -2, 0, 4] = math.nan
    table = torch.zeros(1, width, dtype=torch.int32)
    table[0, -1] = 1
    q = torch.zeros(1, 2, 1, D, dtype=dtype)
    q[..., 0] = 1
    cache = asd.KVCache(k.cuda(), v.cuda(), table.cuda())
    mask = asd.tree_mask(torch.tensor([[-1, 0]])).cuda() if tree else None
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    o = asd.tree_attention(q.cuda(), cache, torch.tensor([2 ** 31 - 3], dtype=torch.int32, device="cuda"), scale=1.0,
                           tree_mask=mask, status=status)
    out, lse = o["out"].cpu().double()[0, :, 0], o["lse"].cpu().double()[0, :, 0]
    assert not status.any()
    w = math.exp(-8)  # of token 0 for token 1; the context's weights are under 2^31 e^-40 = 1e-8 together
    want = torch.tensor([3.0, (5.0 + 3.0 * w) / (1 + w)], dtype=torch.float64)[:, None].expand(2, D).clone()
    if tree:
        want[1, 4] = math.nan
    assert torch.equal(out.isnan(), want.isnan())
    assert float((out - want).nan_to_num(0).abs().max()) <= 5.0 * (2.0 ** -8 if dtype == BF16 else 1e-6)
    assert float((lse - torch.tensor([40.0, 48 + math.log1p(w)], dtype=torch.float64)).abs().max()) <= 1e-4
