"""asd_kv_evict against a plain implementation: equal bit for bit."""
import math

import pytest
import torch

import rules_reference as ref

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


class Problem:
    def __init__(self, dtype, layers, heads, D, page, ctx, keep, first=0, last=0, seed=0, kind="normal", width=None):
        g = torch.Generator().manual_seed(seed)
        B = len(ctx)
        self.kv_len, self.first, self.last = torch.tensor(ctx, dtype=torch.int32), first, last
        self.keep = torch.tensor(keep, dtype=torch.int32)
        need = [-(-c // page) for c in ctx]
        pages = sum(need) + 2
        order = torch.randperm(pages, generator=g).to(torch.int32)
        self.table = torch.full((B, max(max(need), 1)), 2 ** 31 - 1, dtype=torch.int32)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = order[at:at + n]
            at += n
        self.k = torch.randn(layers, pages, page, heads, D, generator=g).to(dtype)
        self.v = torch.randn(layers, pages, page, heads, D, generator=g).to(dtype)
        shape = (layers, B, heads, width or max(ctx) + 3)
        if kind == "normal":
            self.weight = torch.exp(2 * torch.randn(shape, generator=g))
        elif kind == "ties":
            self.weight = torch.randint(3, shape, generator=g).float()
        elif kind == "equal":
            self.weight = torch.full(shape, 0.25)
        else:  # everything a float can be
            pick = torch.tensor([math.nan, math.inf, -math.inf, 0.0, -0.0, 1e-45, -1.0, 3e38, 1.0, 1.0000001])
            self.weight = pick[torch.randint(len(pick), shape, generator=g)]

    def check(self, asd, layout="tokens", out=False, **kw):
        k, v = self.k.cuda(), self.v.cuda()
        if layout == "heads":
            k, v = (x.transpose(2, 3).contiguous().transpose(2, 3) for x in (k, v))
        elif layout == "loose":
            def loose(x):
                store = torch.full((x[..., 0].numel() * (x.shape[-1] + 3) + 1,), 9.0, dtype=x.dtype, device="cuda")
                return store[1:].view(*x.shape[:-1], x.shape[-1] + 3)[..., :-3].copy_(x)
            k, v = loose(k), loose(v)
        w = self.weight.cuda()
        to = torch.full_like(w, 5.0) if out else w
        cache = asd.KVCache(k, v, self.table.cuda())
        got = asd.kv_evict(cache, self.kv_len.cuda(), w, self.keep.cuda(), self.first, self.last,
                           out=to if out else None, **kw)
        ek, ev, ew, en = ref.evicted(self.k, self.v, self.table, self.kv_len, self.weight, self.keep, self.first,
                                     self.last)
        assert torch.equal(got.cpu(), en)
        assert torch.equal(k.cpu(), ek) and torch.equal(v.cpu(), ev)
        if out:
            for b, n in enumerate(en.tolist()):
                assert bool((to[:, b, :, n:] == 5).all())
                ew[:, b, :, n:] = 5.0
            assert torch.equal(w.cpu().view(torch.int32), self.weight.view(torch.int32))
        assert torch.equal(to.cpu().view(torch.int32), ew.view(torch.int32))


CASES = [(BF16, 2, 2, 128, 64, [300, 129, 64], [200, 129, 1], 4, 16), (F32, 1, 3, 96, 24, [100], [99], 0, 0),
         (F16, 3, 1, 64, 5, [1, 2, 33], [1, 1, 32], 0, 1), (BF16, 1, 4, 80, 48, [500, 400], [250, 300], 4, 64),
         (BF16, 2, 1, 20, 16, [77], [40], 1, 3), (F32, 1, 2, 7, 3, [40, 9], [13, 8], 2, 2),
         (F32, 1, 1, 256, 16, [70], [35], 0, 8), (BF16, 1, 2, 1, 16, [90], [30], 0, 0),
         (BF16, 1, 1, 64, 32, [2000], [1000], 10, 100), (F16, 1, 1, 64, 32, [5000, 4100], [64, 4099], 4, 32)]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(x).replace("torch.", "") for x in c).replace(" ", ""))
@pytest.mark.parametrize("kind", ("normal", "ties", "equal", "any"))
def test_evict(asd, case, kind):
    Problem(*case, kind=kind, seed=1).check(asd)
    Problem(*case, kind=kind, seed=2).check(asd, out=True)


@pytest.mark.parametrize("layout", ("tokens", "heads", "loose"))
@pytest.mark.parametrize("dtype", (BF16, F32), ids=("bf16", "f32"))
def test_layouts(asd, dtype, layout):
    Problem(dtype, 2, 2, 64, 16, [200, 90], [100, 45], 2, 8, seed=3).check(asd, layout)


@pytest.mark.parametrize("first,last,keep", [(0, 0, 0), (0, 0, 50), (50, 0, 50), (0, 50, 50), (1000, 1000, 50),
                                             (20, 1000, 50), (20, 30, 50), (0, 100, 99), (2 ** 31 - 1, 2 ** 31 - 1, 7),
                                             (4, 4, 2 ** 31 - 1)])
def test_what_always_stays(asd, first, last, keep):
    p = Problem(F16, 1, 2, 64, 16, [100, 51, 50, 0], [keep] * 4, first, last, seed=4)
    p.check(asd)
    p.check(asd, out=True)


def test_one_layer_without_its_dimension(asd):
    p = Problem(BF16, 1, 2, 64, 16, [60], [30], seed=5)
    k, w = p.k.cuda(), p.weight.cuda()
    asd.kv_evict(asd.KVCache(k, p.v.cuda(), p.table.cuda()), p.kv_len.cuda(), w[0], p.keep.cuda())
    ek, _, ew, _ = ref.evicted(p.k, p.v, p.table, p.kv_len, p.weight, p.keep, 0, 0)
    assert torch.equal(k.cpu(), ek) and torch.equal(w.cpu(), ew)


def test_flags(asd):
    p = Problem(F32, 2, 2, 64, 16, [60, 60, 60, 60, 64], [30, -1, 30, 30, 64], seed=6)
    p.kv_len[2], p.kv_len[3] = -5, 65  # before the first slot, past the table (64 slots; the weights have 67)
    status = torch.zeros(5, dtype=torch.int32, device="cuda")
    k, v, w = p.k.cuda(), p.v.cuda(), p.weight.cuda()
    got = asd.kv_evict(asd.KVCache(k, v, p.table.cuda()), p.kv_len.cuda(), w, p.keep.cuda(), status=status)
    L = asd.STATUS_LENGTH
    assert status.tolist() == [0, L, L, L, 0] and got.tolist() == [30, 60, -5, 65, 64]
    p.kv_len[1:] = torch.tensor([0, 0, 0, 64])
    p.keep[1] = 0
    ek, ev, ew, _ = ref.evicted(p.k, p.v, p.table, p.kv_len, p.weight, p.keep, 0, 0)
    assert torch.equal(k.cpu(), ek) and torch.equal(v.cpu(), ev) and torch.equal(w.cpu(), ew)
    status.zero_()
    short = p.weight[..., :59].contiguous().cuda()  # room for 59 of 60 slots
    asd.kv_evict(asd.KVCache(k, v, p.table.cuda()), p.kv_len.cuda(), short, p.keep.cuda(), status=status)
    assert status.tolist() == [L, 0, 0, 0, L]


def test_pages_out_of_range_are_left_out(asd):
    p = Problem(F32, 1, 1, 64, 16, [64], [32], seed=7, kind="equal")
    p.weight[..., 32:] = 1.0  # the upper half stays and goes down
    p.table[0, 3] = 10 ** 6   # from there nothing can be read
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    k = p.k.cuda()
    got = asd.kv_evict(asd.KVCache(k, p.v.cuda(), p.table.cuda()), p.kv_len.cuda(), p.weight.cuda(), p.keep.cuda(),
                       status=status)
    assert status.tolist() == [asd.STATUS_PAGE] and got.tolist() == [32]
    at = p.table[0].tolist()
    want = p.k.clone()
    want[0, at[0]] = p.k[0, at[2]]
    assert torch.equal(k.cpu(), want)


@pytest.mark.parametrize("ctx,keep", [(9000, 4000), (40000, 39000), (70001, 20000), (300000, 299000)])
@pytest.mark.parametrize("kind", ("normal", "ties"))
def test_long_contexts(asd, ctx, keep, kind):
    """One head, one element: clusters of several CTAs, and what a sort says."""
    g = torch.Generator(device="cuda").manual_seed(ctx)
    page = 64
    n = -(-ctx // page)
    table = torch.randperm(n, generator=g, device="cuda").to(torch.int32).view(1, n).contiguous()
    k = torch.randn(1, n, page, 1, 8, generator=g, device="cuda")
    v = torch.randn(1, n, page, 1, 8, generator=g, device="cuda")
    w = torch.randn(1, 1, 1, ctx, generator=g, device="cuda")
    if kind == "ties":
        w = (w * 2).round()
    first, last = 4, 100
    score = w.flatten().clone()
    score[:first], score[-last:] = math.inf, math.inf
    stay = torch.zeros(ctx, dtype=torch.bool, device="cuda")
    stay[score.sort(descending=True, stable=True).indices[:keep]] = True
    src, dst = keep + stay[keep:].nonzero().flatten(), (~stay[:keep]).nonzero().flatten()
    at = torch.arange(ctx, device="cuda")
    at[dst] = src
    at = at[:keep]

    def rows(x):
        return x[0, table[0].long()].view(-1, 8)
    wk, wv, ww = rows(k)[at], rows(v)[at], w.flatten()[at]
    got = asd.kv_evict(asd.KVCache(k, v, table), torch.tensor([ctx], dtype=torch.int32, device="cuda"), w,
                       torch.tensor([keep], dtype=torch.int32, device="cuda"), first, last)
    assert got.tolist() == [keep]
    assert torch.equal(rows(k)[:keep], wk) and torch.equal(rows(v)[:keep], wv) and torch.equal(w.flatten()[:keep], ww)


def test_twice_and_captured(asd):
    """An eviction of what is within its budget moves nothing; a graph follows the lengths it finds."""
    p = Problem(BF16, 2, 2, 64, 16, [200, 90], [100, 45], 2, 8, seed=8)
    k, v, w = p.k.cuda(), p.v.cuda(), p.weight.cuda()
    cache, kv, keep = asd.KVCache(k, v, p.table.cuda()), p.kv_len.cuda(), p.keep.cuda()
    new = torch.zeros_like(kv)
    asd.kv_evict(cache, kv, w, keep, 2, 8, new_len=new)
    after = k.clone(), v.clone(), w.clone()
    again = asd.kv_evict(cache, new, w, keep, 2, 8)
    assert torch.equal(again, new)
    for a, b in zip(after, (k, v, w)):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        asd.kv_evict(cache, kv, w, keep, 2, 8, new_len=new)
    for ctx in ([200, 90], [150, 45], [100, 46]):
        k.copy_(p.k), v.copy_(p.v), w.copy_(p.weight), kv.copy_(torch.tensor(ctx, dtype=torch.int32))
        graph.replay()
        ek, ev, ew, en = ref.evicted(p.k, p.v, p.table, torch.tensor(ctx), p.weight, p.keep, 2, 8)
        assert torch.equal(k.cpu(), ek) and torch.equal(v.cpu(), ev) and torch.equal(w.cpu(), ew)
        assert torch.equal(new.cpu(), en)


def test_attention_after_an_eviction(asd):
    """Order does not matter to attention: what stayed, in any order, gives the same result."""
    B, heads, D, page, ctx, keep = 2, 2, 64, 16, 200, 120
    p = Problem(F32, 1, heads, D, page, [ctx, 150], [keep, keep], 4, 16, seed=9)
    cache = asd.KVCache(p.k.cuda(), p.v.cuda(), p.table.cuda())
    new = asd.kv_evict(cache, p.kv_len.cuda(), p.weight.cuda(), p.keep.cuda(), 4, 16)
    q = torch.randn(B, 1, heads, D, generator=torch.Generator().manual_seed(1)).cuda()
    got = asd.tree_attention(q, cache, new - 1, scale=0.2)["out"].cpu()
    for b in range(B):
        n = int(p.kv_len[b])
        slots = torch.arange(n)
        at = p.table[b].long()[slots // page], slots % page
        for h in range(heads):
            w = p.weight[0, b, h, :n].clone()
            w[:4], w[n - 16:] = math.inf, math.inf
            stay = w.sort(descending=True, stable=True).indices[:keep]
            kk, vv = p.k[0][at][stay, h].double(), p.v[0][at][stay, h].double()
            want = torch.softmax(kk @ q[b, 0, h].cpu().double() * 0.2, 0) @ vv
            assert float((got[b, 0, h].double() - want).abs().max()) < 1e-5
