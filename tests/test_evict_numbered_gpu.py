"""Evictions that know each slot's token: the newest tokens stay however few come between two of them."""
import importlib.util
import math
import os

import pytest
import torch

import numbered_reference as nref
import rules_reference as ref

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


class Chat:
    """Requests whose caches grow by tokens with rows of their own, on the CPU and on the GPU alike."""

    def __init__(self, dtype, layers, heads, D, page, B, slots, seed=0, loose=False):
        self.g = torch.Generator().manual_seed(seed)
        self.layers, self.heads, self.D, self.page, self.B = layers, heads, D, page, B
        width = -(-slots // page)
        self.table = torch.randperm(B * width, generator=self.g).to(torch.int32).view(B, width)
        self.k = torch.zeros(layers, B * width, page, heads, D, dtype=dtype)
        self.v = torch.zeros_like(self.k)
        self.weight = torch.zeros(layers, B, heads, slots)
        self.numbers = torch.full(self.weight.shape, -1, dtype=torch.int32)
        self.kv_len, self.tokens = torch.zeros(B, dtype=torch.int32), torch.zeros(B, dtype=torch.int32)
        self.rows = [[] for _ in range(B)]  # every token's keys [layers, heads, D]

        def put(x):
            if not loose:
                return x.cuda()
            store = torch.full((x[..., 0].numel() * (D + 3) + 1,), 9.0, dtype=x.dtype, device="cuda")
            return store[1:].view(*x.shape[:-1], D + 3)[..., :-3].copy_(x)
        self.gk, self.gv, self.gtable = put(self.k), put(self.v), self.table.cuda()
        self.gw, self.gn = self.weight.cuda(), self.numbers.cuda()

    def append(self, counts, weigh):
        for b, n in enumerate(counts):
            for _ in range(n):
                s = int(self.kv_len[b])
                at = int(self.table[b, s // self.page]), s % self.page
                k, v = (torch.randn(self.layers, self.heads, self.D, generator=self.g).to(self.k.dtype) for _ in "kv")
                self.k[(slice(None), *at)], self.v[(slice(None), *at)] = k, v
                self.gk[(slice(None), *at)], self.gv[(slice(None), *at)] = k.cuda(), v.cuda()
                self.rows[b].append(k)
                self.weight[:, b, :, s] = 0.0  # nothing has seen it yet
                self.kv_len[b] += 1
                self.tokens[b] += 1
            m = int(self.kv_len[b])
            self.weight[:, b, :, :m] += weigh(self.layers, self.heads, m)
        self.gw.copy_(self.weight)

    def evict(self, asd, keep, first, last, out=False, **kw):
        cache = asd.KVCache(self.gk, self.gv, self.gtable)
        to = torch.full_like(self.gw, 5.0) if out else self.gw
        got = asd.kv_evict(cache, self.kv_len.cuda(), self.gw, torch.tensor(keep, dtype=torch.int32).cuda(), first, last,
                           out=to if out else None, numbers=self.gn, tokens=self.tokens.cuda(), **kw)
        was = self.weight
        self.k, self.v, self.weight, self.numbers, new = nref.evicted(
            self.k, self.v, self.table, self.kv_len, self.weight, self.numbers, self.tokens, keep, first, last)
        self.kv_len = torch.tensor(new, dtype=torch.int32)
        assert got.tolist() == new
        assert torch.equal(self.gk.cpu(), self.k) and torch.equal(self.gv.cpu(), self.v)
        assert torch.equal(self.gn.cpu(), self.numbers)
        if out:
            assert torch.equal(self.gw.cpu().view(torch.int32), was.view(torch.int32))
            for b, n in enumerate(new):
                assert bool((to[:, b, :, n:] == 5).all())
                assert torch.equal(to[:, b, :, :n].cpu().view(torch.int32),
                                   self.weight[:, b, :, :n].contiguous().view(torch.int32))
            self.gw = to
            self.gw.copy_(self.weight)
        assert torch.equal(self.gw.cpu().view(torch.int32), self.weight.view(torch.int32))

    def newest_are_there(self, last, keep):
        """By the rows themselves: the newest `last` tokens' keys are in the cache of every layer and head."""
        for b in range(self.B):
            n = int(self.kv_len[b])
            slots = torch.arange(n)
            have = self.gk.cpu()[:, self.table[b].long()[slots // self.page], slots % self.page]  # [layers, n, heads, D]
            assert n == min(keep[b], len(self.rows[b]))
            for row in self.rows[b][len(self.rows[b]) - min(last, n):]:
                assert bool((have == row[:, None]).all(-1).any(1).all())


@pytest.mark.parametrize("dtype,layers,heads,D,page,loose", [(BF16, 2, 2, 64, 16, False), (F32, 1, 3, 20, 5, False),
                                                             (F16, 1, 2, 8, 3, False), (BF16, 1, 1, 24, 16, True)])
@pytest.mark.parametrize("most", (1, 5, 9))
def test_rounds_of_a_few_tokens(asd, dtype, layers, heads, D, page, loose, most):
    """Evicted after every round of one to `most` tokens, new tokens being the lightest: the window never loses one."""
    first, last, keep = 2, 12, [30, 17]
    c = Chat(dtype, layers, heads, D, page, 2, 64, seed=most, loose=loose)

    def weigh(L, H, m):
        return torch.rand(L, H, m, generator=c.g) * torch.linspace(3, 0.1, m)
    c.append([34, 9], weigh)
    for i in range(18):
        c.evict(asd, keep, first, last, out=i % 3 == 2)
        c.newest_are_there(last, keep)
        c.append(torch.randint(1, most + 1, (2,), generator=c.g).tolist(), weigh)


@pytest.mark.parametrize("kind", ("ties", "any"))
def test_weights_of_all_kinds(asd, kind):
    pick = torch.tensor([0.0, 1.0, 2.0] if kind == "ties" else
                        [math.nan, math.inf, -math.inf, 0.0, -0.0, 1e-45, -1.0, 3e38, 1.0, 1.0000001])
    c = Chat(F32, 2, 2, 8, 16, 3, 96, seed=4)
    c.append([70, 40, 25], lambda L, H, m: torch.zeros(L, H, m))
    for _ in range(6):
        for b in range(3):
            n = int(c.kv_len[b])
            c.weight[:, b, :, :n] = pick[torch.randint(len(pick), (2, 2, n), generator=c.g)]
        c.gw.copy_(c.weight)
        c.evict(asd, [40, 40, 20], 3, 10)
        c.newest_are_there(10, [40, 40, 20])
        c.append([2, 7, 1], lambda L, H, m: torch.zeros(L, H, m))


def test_limits_that_change(asd):
    """keep, first and last from call to call: what an earlier call let go is not there, the rest fills up."""
    c = Chat(BF16, 1, 2, 16, 16, 2, 128, seed=5)

    def weigh(L, H, m):
        return torch.rand(L, H, m, generator=c.g)
    c.append([80, 50], weigh)
    for keep, first, last in (([60, 60], 4, 10), ([30, 3], 4, 40), ([40, 40], 0, 40), ([20, 40], 50, 7), ([0, 12], 2, 3),
                              ([9, 12], 2 ** 31 - 1, 2 ** 31 - 1), ([9, 9], 0, 0), ([2 ** 31 - 1] * 2, 1, 1)):
        c.evict(asd, keep, first, last)
        c.append([3, 5], weigh)


def test_without_moves_before_it_equals_the_last_slots(asd):
    c = Chat(BF16, 2, 2, 64, 16, 2, 160, seed=6)
    c.append([150, 90], lambda L, H, m: torch.rand(L, H, m, generator=c.g))
    k, v, w, n = ref.evicted(c.k, c.v, c.table, c.kv_len, c.weight, torch.tensor([100, 45]), 4, 16)
    c.evict(asd, [100, 45], 4, 16)
    assert torch.equal(c.k, k) and torch.equal(c.v, v) and torch.equal(c.weight, w) and torch.equal(c.kv_len, n)


def test_flags(asd):
    c = Chat(F32, 1, 2, 8, 16, 4, 64, seed=7)
    c.append([40, 40, 40, 40], lambda L, H, m: torch.rand(L, H, m, generator=c.g))
    c.gn[0, 1, 1, :40] = 39  # every slot the newest token
    c.gn[0, 2, 0, 5] = 2 ** 31 - 1  # one number too large: a token that counts as new
    tokens = c.tokens.cuda()
    tokens[3] = 39
    status = torch.zeros(4, dtype=torch.int32, device="cuda")
    cache = asd.KVCache(c.gk, c.gv, c.gtable)
    got = asd.kv_evict(cache, c.kv_len.cuda(), c.gw, torch.full((4,), 24, dtype=torch.int32).cuda(), 2, 6, status=status,
                       numbers=c.gn, tokens=tokens)
    assert status.tolist() == [0, asd.STATUS_POSITION, 0, asd.STATUS_LENGTH] and got.tolist() == [24, 24, 24, 40]
    slots = torch.arange(40)

    def rows(x, b):
        return x.cpu()[0, c.table[b].long()[slots // 16], slots % 16]
    assert torch.equal(rows(c.gk, 1)[:, 1], rows(c.k, 1)[:, 1])  # that head moved nothing
    assert torch.equal(rows(c.gk, 3), rows(c.k, 3)) and bool((c.gn[0, 3] == -1).all())
    assert bool((c.gn[0, 1, 1, 24:] == -1).all()) and bool((c.gn[0, 1, 1, :24] == 39).all())
    good = nref.evicted(c.k, c.v, c.table, c.kv_len, c.weight, torch.full_like(c.numbers, -1), c.tokens, [24] * 4, 2, 6)
    assert torch.equal(rows(c.gk, 0), rows(good[0], 0)) and torch.equal(rows(c.gk, 1)[:, 0], rows(good[0], 1)[:, 0])
    assert torch.equal(c.gn[0, 0].cpu(), good[3][0, 0])


@pytest.mark.parametrize("ctx,keep,add", [(3000, 2990, 7), (9000, 4000, 3), (70001, 69000, 64), (300000, 299000, 100)])
def test_long_contexts(asd, ctx, keep, add):
    """One head and clusters of several CTAs; a second eviction after few tokens, against a sort."""
    g = torch.Generator(device="cuda").manual_seed(ctx)
    first, last, page = 4, 500, 64
    n = -(-(ctx + add) // page)
    table = torch.randperm(n, generator=g, device="cuda").to(torch.int32).view(1, n).contiguous()
    k = torch.randn(1, n, page, 1, 8, generator=g, device="cuda")
    v = torch.randn(1, n, page, 1, 8, generator=g, device="cuda")
    cache = asd.KVCache(k, v, table)
    w = torch.rand(1, 1, 1, ctx + add, generator=g, device="cuda")
    numbers = torch.full(w.shape, -1, dtype=torch.int32, device="cuda")

    def word(x):
        return torch.tensor([x], dtype=torch.int32, device="cuda")

    def rows(x):
        return x[0, table[0].long()].view(-1, 8)
    length, total = ctx, ctx
    token = torch.arange(ctx, device="cuda")
    for _ in range(2):
        score = w.flatten()[:length].clone()
        score[:first] = math.inf
        score[token >= total - last] = math.inf
        stay = torch.zeros(length, dtype=torch.bool, device="cuda")
        stay[score.sort(descending=True, stable=True).indices[:keep]] = True
        src, dst = keep + stay[keep:].nonzero().flatten(), (~stay[:keep]).nonzero().flatten()
        at = torch.arange(length, device="cuda")
        at[dst] = src
        at = at[:keep]
        wk, wv, ww, wt = rows(k)[at], rows(v)[at], w.flatten()[at], token[at]
        got = asd.kv_evict(cache, word(length), w, word(keep), first, last, numbers=numbers, tokens=word(total))
        assert got.tolist() == [keep] and torch.equal(numbers.flatten()[:keep], wt.int())
        assert bool((numbers.flatten()[keep:] == -1).all())
        assert torch.equal(rows(k)[:keep], wk) and torch.equal(rows(v)[:keep], wv) and torch.equal(w.flatten()[:keep], ww)
        assert bool(torch.isin(torch.arange(total - last, total, device="cuda"), wt).all())
        token = torch.cat([wt, torch.arange(total, total + add, device="cuda")])
        w.flatten()[keep:keep + add] = 0.0
        length, total = keep + add, total + add


def test_captured_and_on_a_stream(asd):
    c = Chat(BF16, 2, 2, 64, 16, 2, 160, seed=8)
    c.append([120, 100], lambda L, H, m: torch.rand(L, H, m, generator=c.g))
    cache, keep = asd.KVCache(c.gk, c.gv, c.gtable), torch.tensor([100, 45], dtype=torch.int32).cuda()
    kv, tokens, new = c.kv_len.cuda(), c.tokens.cuda(), torch.zeros(2, dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    first = [x.clone() for x in (c.gk, c.gv, c.gw, c.gn)]
    side.wait_stream(torch.cuda.current_stream())
    asd.kv_evict(cache, kv, c.gw, keep, 2, 8, new_len=new, numbers=c.gn, tokens=tokens, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    want = nref.evicted(c.k, c.v, c.table, c.kv_len, c.weight, c.numbers, c.tokens, [100, 45], 2, 8)
    for got, x in zip((c.gk, c.gv, c.gw, c.gn), want):
        assert torch.equal(got.cpu(), x)
    for got, x in zip((c.gk, c.gv, c.gw, c.gn), first):
        got.copy_(x)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        asd.kv_evict(cache, kv, c.gw, keep, 2, 8, new_len=new, numbers=c.gn, tokens=tokens)
    for _ in range(2):
        for got, x in zip((c.gk, c.gv, c.gw, c.gn), first):
            got.copy_(x)
        graph.replay()
        for got, x in zip((c.gk, c.gv, c.gw, c.gn), want):
            assert torch.equal(got.cpu(), x)
        assert new.tolist() == [100, 45]


@pytest.mark.parametrize("dtype", (F32, BF16), ids=("f32", "bf16"))
def test_decoding_keeps_its_newest_tokens(asd, dtype, monkeypatch):
    """examples/tree_decode.py evicts after rounds of one to K + 1 tokens; every layer and head keeps the last K + 1."""
    spec = importlib.util.spec_from_file_location("tree_decode", os.path.join(ROOT, "examples", "tree_decode.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    depth, evict = example.Tree().depth, asd.kv_evict
    seen, held, checked = {}, {}, []  # of a request: all its tokens' keys, the slots that it had after the last call

    def watched(cache, kv_len, *args, **kw):
        def rows(b, n):
            slots = torch.arange(n, device="cuda")
            return cache.k[:, cache.page_table[b].long()[slots // cache.page_size], slots % cache.page_size].cpu()
        for b, n in enumerate(kv_len.tolist()):
            seen[b] = torch.cat([seen[b], rows(b, n)[:, held[b]:]], 1) if b in seen else rows(b, n)
        new = evict(cache, kv_len, *args, **kw)
        for b, n in enumerate(new.tolist()):
            held[b] = n
            have, newest = rows(b, n), seen[b][:, -min(depth + 1, n):]
            found = (newest[:, :, None] == have[:, None]).all(-1).any(2)  # [layers, newest, heads]
            checked.append(n < kv_len.tolist()[b])
            assert bool(found.all()), f"request {b}, {seen[b].shape[1]} tokens"
        return new
    monkeypatch.setattr(example.asd, "kv_evict", watched)
    example.decode(example.Decoder(dtype), [[1, 2, 3, 4, 5], [7], [11, 13, 17, 19, 23, 29, 31, 37, 41]], 30, keep=14)
    assert sum(checked) > 40
