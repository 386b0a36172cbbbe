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


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_a_replayed_graph_follows_the_lengths(asd, dtype):
    """Every replay against the 64-bit form of its own lengths, log-sum-exp included; a context that is shorter than at
    capture lies in slots that are filled."""
    p = Problem(dtype, 9, 10, 2, 128, 16, ctx=[3000, 0, 40], tree=True, seed=17)
    cache = p.device(asd)
    q, kv_len, mask = p.q.cuda(), p.kv_len.cuda(), p.mask.cuda()
    new_len = torch.full((3,), 9, dtype=torch.int32, device="cuda")
    ws = asd.attention_workspace(cache, p.T, p.Hq)
    out = {"out": torch.zeros(3, 9, 10, 128, dtype=dtype, device="cuda"),
           "lse": torch.zeros(3, 9, 10, dtype=torch.float32, device="cuda")}
    asd.tree_attention(q, cache, kv_len, tree_mask=mask, new_len=new_len, scale=p.scale, workspace=ws, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        asd.tree_attention(q, cache, kv_len, tree_mask=mask, new_len=new_len, scale=p.scale, workspace=ws, out=out)
    for ctx, new in (([3000, 0, 40], [9, 9, 9]), ([10, 0, 40], [9, 1, 0]), ([2000, 0, 0], [3, 9, 9]),
                     ([1, 0, 31], [0, 0, 9]), ([2990, 0, 17], [9, 5, 9])):
        p.kv_len, p.new_len = (torch.tensor(x, dtype=torch.int32) for x in (ctx, new))
        kv_len.copy_(p.kv_len)
        new_len.copy_(p.new_len)
        out["out"].fill_(7)
        out["lse"].fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        p.check(out["out"].cpu(), out["lse"].cpu())
    assert ws.error() == 0


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("T,Hq,Hkv,D", [(1, 130, 1, 64), (3, 150, 1, 128), (2, 600, 2, 64), (1, 128, 1, 64), (3, 127, 1, 64)])
def test_wide_groups(asd, dtype, T, Hq, Hkv, D):
    """Up to and more than 128 query heads on a key/value head: row tiles begin inside a token."""
    for tree in (False, True):
        p = Problem(dtype, T, Hq, Hkv, D, 16, ctx=[150, 0, 700], tree=tree, seed=Hq)
        out, lse, status = p.run(asd)
        p.check(out, lse)
        assert not status.any()


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("T,Hq,Hkv,D", [(1000, 5, 1, 64), (517, 4, 2, 128), (300, 8, 1, 96)])
def test_prompts(asd, dtype, T, Hq, Hkv, D):
    """Hundreds of new tokens, with and without a context, fewer in one request than in the others."""
    p = Problem(dtype, T, Hq, Hkv, D, 48, ctx=[0, 300, 77], new=[T, T - 131, 1], seed=T)
    out, lse, status = p.run(asd)
    p.check(out, lse)
    assert not status.any()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_prompts_under_a_mask_of_many_words(asd, dtype):
    """The same as a chain where the mask is a chain's; and a tree of 300 nodes."""
    T = 300
    p = Problem(dtype, T, 6, 2, 64, 16, ctx=[40, 0], seed=3)
    chain, chain_lse, _ = p.run(asd)
    p.check(chain, chain_lse)
    p.mask = asd.tree_mask(torch.arange(T)[None].expand(2, T) - 1)
    out, lse, _ = p.run(asd)
    p.check(out, lse)
    p = Problem(dtype, T, 6, 2, 64, 16, ctx=[40, 0], tree=True, seed=4)
    out, lse, _ = p.run(asd)
    p.check(out, lse)
