"""asd_kv_weigh against a plain 64-bit implementation."""
import math

import pytest
import torch

import cache_reference as cref
import rules_reference as ref

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


class Problem:
    """Inputs on the CPU: a paged cache whose unused places hold NaN."""

    def __init__(self, dtype, rows, Hq, Hkv, D, page, ctx, new=None, T=None, decay=1.0, seed=0, spare=3):
        g = torch.Generator().manual_seed(seed)
        self.B, self.rows, self.Hq, self.Hkv, self.D, self.page, self.dtype = len(ctx), rows, Hq, Hkv, D, page, dtype
        self.T = T or rows
        self.kv_len = torch.tensor(ctx, dtype=torch.int32)
        self.new_len = None if new is None else torch.tensor(new, dtype=torch.int32)
        need = [-(-(c + rows) // page) for c in ctx]
        pages = sum(need) + spare
        order = torch.randperm(pages, generator=g).to(torch.int32)
        self.table = torch.full((self.B, max(need)), 2 ** 31 - 1, dtype=torch.int32)  # ids of no page where unused
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = order[at:at + n]
            at += n
        self.k = torch.full((pages, page, Hkv, D), math.nan).to(dtype)
        for b in range(self.B):
            n = rows if new is None else new[b]
            slots = torch.arange(ctx[b] + n)
            self.k[self.table[b].long()[slots // page], slots % page] = \
                torch.randn(len(slots), Hkv, D, generator=g).to(dtype)
        self.q = (1.5 * torch.randn(self.B, self.T, Hq, D, generator=g)).to(dtype)
        self.scale, self.decay = 1.0 / math.sqrt(D), decay
        spread = (self.q.double() ** 2).sum(-1) / (2 * D)
        self.lse = (spread + torch.log(self.kv_len.double() + 1)[:, None, None]).float()
        self.path = None
        if T:
            self.path = torch.stack([torch.randperm(T, generator=g)[:rows].sort().values for _ in ctx]).to(torch.int32)
        self.width = max(c + rows for c in ctx) + 5
        self.before = torch.rand(self.B, Hkv, self.width, generator=g)

    def cache(self, asd, layout="tokens"):
        k = self.k.cuda()
        if layout == "heads":  # [pages, heads, page, D]
            k = k.transpose(1, 2).contiguous().transpose(1, 2)
        elif layout == "loose":  # rows that start on no boundary
            P, n, H, D = k.shape
            store = torch.full((P * n * H * (D + 3) + 1,), math.nan, dtype=k.dtype, device="cuda")
            k = store[1:].view(P, n, H, D + 3)[..., :D].copy_(k)
        return asd.KVCache(k, k, self.table.cuda())

    def run(self, asd, layout="tokens", q=None, out=None, **kw):
        dev = [None if x is None else x.cuda() for x in (self.new_len, self.path)]
        return asd.kv_weigh(self.q.cuda() if q is None else q, self.lse.cuda(), self.cache(asd, layout),
                            self.kv_len.cuda(), self.before.cuda(), decay=self.decay, new_len=dev[0], path=dev[1],
                            scale=self.scale, out=out, **kw)

    def check(self, got):
        want, tol = ref.weighed(self.q, self.lse, self.k, self.table, self.kv_len, self.new_len, self.path, self.scale,
                                self.decay, self.before)
        got = got.cpu()
        written = ~want.isnan()
        assert torch.equal(got[~written], self.before[~written])  # the rest is left
        off = (got.double() - want).abs()[written] / tol[written]
        assert off.numel() == 0 or float(off.max()) <= 1.0, float(off.max())


CASES = [(BF16, 1, 8, 2, 128, 64, [700], None), (BF16, 1, 5, 5, 64, 16, [0], None), (F16, 1, 4, 4, 64, 5, [1, 0, 127], None),
         (BF16, 9, 10, 2, 128, 64, [300, 129, 64], None), (F16, 5, 8, 1, 96, 48, [130, 31, 0, 515], [5, 3, 0, 1]),
         (BF16, 3, 32, 1, 128, 24, [200, 90], None), (F16, 33, 8, 1, 64, 32, [70, 260], [33, 20]),
         (BF16, 70, 4, 1, 80, 256, [100], None), (BF16, 200, 4, 2, 128, 16, [40, 0], None),
         (F16, 17, 16, 1, 128, 12, [400], None), (BF16, 2, 6, 3, 8, 64, [50, 128], None),
         (F32, 1, 4, 2, 96, 24, [90, 0, 200], None), (F32, 17, 16, 4, 96, 24, [130, 64], [17, 9]),
         (F32, 40, 4, 1, 128, 7, [65], None), (F32, 3, 2, 1, 256, 16, [30], None), (F32, 2, 2, 2, 1, 1, [9], None),
         (BF16, 4, 4, 2, 20, 16, [77], None), (F16, 6, 4, 2, 256, 16, [33], None), (F32, 5, 6, 2, 7, 3, [12, 70], None)]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(x).replace("torch.", "") for x in c).replace(" ", ""))
@pytest.mark.parametrize("decay", (0.0, 0.9))
def test_weigh(asd, case, decay):
    p = Problem(*case, decay=decay, seed=3)
    p.check(p.run(asd))


@pytest.mark.parametrize("dtype", (BF16, F16, F32), ids=("bf16", "f16", "f32"))
@pytest.mark.parametrize("case", [(150, 10, 2, 64, 16, [140, 300]), (150, 10, 2, 64, 5, [140]), (70, 5, 1, 128, 64, [400, 1]),
                                  (90, 4, 1, 128, 7, [130])], ids=str)
def test_more_rows_than_stay(asd, dtype, case):
    """Queries that are read again and again while the keys of several tiles wait."""
    p = Problem(dtype, *case, seed=13)
    p.check(p.run(asd))


@pytest.mark.parametrize("dtype", (BF16, F32), ids=("bf16", "f32"))
@pytest.mark.parametrize("spread", (30.0, 60.0, 200.0))
def test_rows_whose_sums_are_far_apart(asd, dtype, spread):
    """Weights of 2^-80 beside weights of 2^80: neither loses its bits to the other's scale."""
    p = Problem(dtype, 20, 4, 1, 64, 16, [200], seed=14, decay=0.0)
    sign = torch.where(torch.arange(20 * 4) % 3 == 0, 1.0, -0.25).view(20, 4)
    p.lse += spread * sign
    p.check(p.run(asd))
    p.lse = torch.where(sign > 0, p.lse, torch.tensor(math.inf))  # only the small ones
    p.check(p.run(asd))


@pytest.mark.parametrize("dtype", (BF16, F32), ids=("bf16", "f32"))
@pytest.mark.parametrize("scale", (0.0, -0.07, 0.5, 1e-20))
def test_any_scale(asd, dtype, scale):
    p = Problem(dtype, 5, 4, 2, 64, 16, [150, 20], seed=15)
    p.scale = scale
    p.lse = p.lse + 40 * abs(scale)
    p.check(p.run(asd))


@pytest.mark.parametrize("dtype", (BF16, F32), ids=("bf16", "f32"))
@pytest.mark.parametrize("layout", ("tokens", "heads", "loose"))
def test_layouts_and_strided_queries(asd, dtype, layout):
    p = Problem(dtype, 4, 8, 2, 64, 16, [150, 37], seed=4)
    rows = torch.full((p.B, p.T, 3 * p.Hq, p.D), math.nan, dtype=dtype, device="cuda")
    q = rows[:, :, p.Hq:2 * p.Hq].copy_(p.q)
    p.check(p.run(asd, layout, q=q))


@pytest.mark.parametrize("dtype", (F16, F32), ids=("f16", "f32"))
def test_paths(asd, dtype):
    p = Problem(dtype, 6, 8, 2, 64, 16, [150, 260, 3], new=[6, 2, 4], T=21, seed=5)
    p.check(p.run(asd))
    p.path[1, 1], p.path[2, 0] = 21, -1  # rows that lead nowhere add nothing
    status = torch.zeros(3, dtype=torch.int32, device="cuda")
    p.check(p.run(asd, status=status))
    assert status.tolist() == [0, asd.STATUS_PATH, asd.STATUS_PATH]


@pytest.mark.parametrize("dtype", (BF16, F32), ids=("bf16", "f32"))
def test_rows_with_infinite_lse_add_nothing(asd, dtype):
    p = Problem(dtype, 3, 4, 2, 64, 16, [100], seed=6)
    p.lse[0, 1], p.lse[0, 2, 0] = -math.inf, math.inf
    p.q[0, 1, 0] = math.nan
    p.check(p.run(asd))
    p.lse[:] = math.inf
    got = p.run(asd)
    assert torch.equal(got[:, :, :100].cpu(), p.before[:, :, :100]) and not bool(got[:, :, 100:103].any())


@pytest.mark.parametrize("dtype", (BF16, F32), ids=("bf16", "f32"))
def test_what_a_row_does_not_see(asd, dtype):
    """New slots behind a row's own may hold anything: row 0 leaves them alone, and row 2's own NaN reaches its slot only."""
    p = Problem(dtype, 3, 4, 2, 64, 16, [60], seed=7)
    bad = cref.slot_place(p.table[0], 62, 16)
    p.k[bad[0], bad[1]] = math.nan
    got = p.run(asd)
    assert bool(got[0, :, 62].isnan().all()) and not bool(got[0, :, :62].isnan().any())
    p.lse[0, 2] = math.inf  # the only row that sees it
    got = p.run(asd)
    assert not bool(got.isnan().any()) and not bool(got[0, :, 62].any())


@pytest.mark.parametrize("dtype", (BF16, F32), ids=("bf16", "f32"))
def test_in_place_and_nothing_before(asd, dtype):
    p = Problem(dtype, 2, 4, 2, 64, 16, [90, 300], seed=8)
    w = p.before.cuda()
    dev = (p.q.cuda(), p.lse.cuda(), p.cache(asd), p.kv_len.cuda())
    assert asd.kv_weigh(*dev, w, scale=p.scale) is w
    p.check(w)
    out = torch.full_like(w, 7.0)
    asd.kv_weigh(*dev, None, decay=0.0, scale=p.scale, out=out)
    p.decay, p.before = 0.0, torch.full_like(p.before, 7.0)
    p.check(out)
    nan = torch.full_like(w, math.nan)  # with decay 0 what was there does not matter
    asd.kv_weigh(*dev, nan, decay=0.0, scale=p.scale, out=out)
    p.check(out)


@pytest.mark.parametrize("dtype", (BF16, F32), ids=("bf16", "f32"))
def test_lengths_and_pages_out_of_range(asd, dtype):
    p = Problem(dtype, 2, 4, 2, 64, 16, [90, 40, 50, 60], seed=9)
    good = p.run(asd).cpu()
    status = torch.zeros(4, dtype=torch.int32, device="cuda")
    kv = torch.tensor([90, -1, p.table.shape[1] * 16 - 1, 60], dtype=torch.int32)
    p.table[3, 1] = 10 ** 6
    dev = (p.q.cuda(), p.lse.cuda(), p.cache(asd), kv.cuda())
    got = asd.kv_weigh(*dev, p.before.cuda(), scale=p.scale, status=status).cpu()
    assert status.tolist() == [0, asd.STATUS_LENGTH, asd.STATUS_LENGTH, asd.STATUS_PAGE]
    assert torch.equal(got[0], good[0]) and torch.equal(got[1:3], p.before[1:3])
    w = torch.exp(-p.lse[3]).double().view(2, 2, 2).sum((0, 2))  # keys of zeros: exp(-lse) of every row
    assert float((got[3, :, 16:32].double() - p.before[3, :, 16:32].double() - w[:, None]).abs().max()) <= 4e-7
    assert torch.equal(got[3, :, :16], good[3, :, :16])
    narrow = torch.zeros(4, 2, 61, device="cuda")  # the weights have room for 61 slots: 60 + 2 are too many
    status.zero_()
    asd.kv_weigh(p.q.cuda(), p.lse.cuda(), p.cache(asd), p.kv_len.cuda(), None, decay=0.0, out=narrow, status=status)
    assert (status & asd.STATUS_LENGTH).tolist() == [asd.STATUS_LENGTH, 0, 0, asd.STATUS_LENGTH]


@pytest.mark.parametrize("dtype", (BF16, F16, F32), ids=("bf16", "f16", "f32"))
def test_with_the_attention_that_leaves_its_lse(asd, dtype):
    """The weights of a pass add up to one a row."""
    p = Problem(dtype, 7, 8, 2, 64, 16, [500, 129, 1], seed=10)
    cache = p.cache(asd)
    q, kv = p.q.cuda(), p.kv_len.cuda()
    got = asd.tree_attention(q, cache, kv, scale=p.scale)
    w = asd.kv_weigh(q, got["lse"], cache, kv, torch.zeros_like(p.before).cuda(), scale=p.scale)
    assert float((w.double().sum(-1) - 7 * 4).abs().max()) < 28 * 2e-5
    p.lse, p.before = got["lse"].cpu(), torch.zeros_like(p.before)
    p.check(w)


@pytest.mark.parametrize("dtype", (BF16, F32), ids=("bf16", "f32"))
def test_long_contexts_whose_every_slot_is_checked(asd, dtype):
    """Keys that differ slot by slot in a way that the score shows, over many tiles and several requests a CTA."""
    B, Hkv, D, page, ctx = 6, 2, 64, 32, 30000
    g = torch.Generator(device="cuda").manual_seed(1)
    k = torch.randn(B * (ctx // page + 1), page, Hkv, D, generator=g, device="cuda").to(dtype)
    table = torch.randperm(k.shape[0], generator=g, device="cuda").to(torch.int32).view(B, -1).contiguous()
    kv = torch.tensor([ctx, 17, ctx - 1000, 128, ctx - 129, 9000], dtype=torch.int32, device="cuda")
    q = torch.randn(B, 2, 4, D, generator=g, device="cuda").to(dtype)
    lse = torch.full((B, 2, 4), 9.0, device="cuda")
    w = asd.kv_weigh(q, lse, asd.KVCache(k, k, table), kv, None, decay=0.0,
                     out=torch.full((B, Hkv, ctx + 2), -1.0, device="cuda"))
    for b in range(B):
        n = int(kv[b])
        keys = k[table[b].long()].view(-1, Hkv, D)[:n].double()
        z = torch.einsum("thgd,shd->hstg", q[b].view(2, Hkv, 2, D).double(), keys) / math.sqrt(D)
        want = torch.exp(z - 9.0).sum((2, 3))
        assert float(((w[b, :, :n].double() - want) / want).abs().max()) < 2e-5
        assert bool((w[b, :, n + 2:] == -1).all()) and bool((w[b, :, n:n + 2] >= 0).all())


@pytest.mark.parametrize("dtype", (BF16, F16), ids=("bf16", "f16"))
@pytest.mark.parametrize("case", [(1, 4, 1, 256, 64, [700, 1]), (9, 16, 2, 256, 16, [300, 0, 129]), (40, 8, 2, 192, 32, [400, 60]),
                                  (5, 6, 3, 136, 12, [150, 33]), (100, 4, 1, 256, 48, [0, 300]), (3, 8, 4, 200, 5, [90]),
                                  (64, 16, 4, 248, 24, [640, 513])], ids=str)
def test_wide_heads(asd, dtype, case):
    p = Problem(dtype, *case, seed=21)
    p.check(p.run(asd))
    p.check(p.run(asd, layout="heads"))


@pytest.mark.parametrize("dtype,D,page", ((BF16, 128, 16), (F16, 64, 48), (BF16, 64, 5), (BF16, 256, 16), (F32, 32, 24)), ids=str)
def test_prompts_that_see_themselves(asd, dtype, D, page):
    """Many tiles a CTA, of which the later ones are seen by ever fewer rows; every weight, with the bound of
    rules_reference.weighed."""
    B, T, Hkv, G, u = 16, 1300, 8, 3, 2.0 ** -24
    g = torch.Generator(device="cuda").manual_seed(D)
    kv = torch.tensor([0, 0, 1, 127, 200, 0, 511, 512, 0, 64, 3, 0, 900, 0, 0, 31], dtype=torch.int32, device="cuda")
    new = torch.tensor([T, T - 1, T, 700, T, 1, T, 129, 1024, T, 1153, 43, T, T, 1280, T], dtype=torch.int32, device="cuda")
    width = -(-(900 + T) // page)
    k = torch.randn(B * width, page, Hkv, D, generator=g, device="cuda").to(dtype)
    table = torch.randperm(k.shape[0], generator=g, device="cuda").to(torch.int32).view(B, -1).contiguous()
    q = torch.randn(B, T, Hkv * G, D, generator=g, device="cuda").to(dtype)
    lse = torch.empty(B, T, Hkv * G, device="cuda")
    want, tol = [], []
    for b in range(B):
        ctx, n = int(kv[b]), int(new[b])
        keys = k[table[b].long()].view(-1, Hkv, D)[:ctx + n].double()
        rows = q[b, :n].view(n, Hkv, G, D).double()
        z = torch.einsum("thgd,shd->hstg", rows, keys) * D ** -0.5
        sees = torch.arange(ctx + n, device="cuda")[:, None] <= ctx + torch.arange(n, device="cuda")
        z.masked_fill_(~sees[None, :, :, None], -math.inf)
        lse[b, :n] = torch.logsumexp(z, 1).permute(1, 0, 2).reshape(n, Hkv * G).float()
        ref_lse = lse[b, :n].view(n, Hkv, G).permute(1, 0, 2)[:, None].double()
        weight = torch.exp(z - ref_lse)
        reach = torch.einsum("thgd,shd->hstg", rows.abs(), keys.abs()) * D ** -0.5
        off = weight * ((D + 2) * u * reach + 4 * u * (z.masked_fill(z.isinf(), 0.0).abs() + ref_lse.abs()) + 2.0 ** -22)
        want.append(weight.sum((2, 3)))
        tol.append(1.01 * off.sum((2, 3)) + (n * G + 2) * u * want[b] + 1e-37)
    out = asd.kv_weigh(q, lse, asd.KVCache(k, k, table), kv, None, decay=0.0, new_len=new,
                       out=torch.full((B, Hkv, 900 + T + 3), -1.0, device="cuda"))
    for b in range(B):
        n = want[b].shape[1]
        assert float(((out[b, :, :n].double() - want[b]).abs() / tol[b]).max()) <= 1.0, b
        assert bool((out[b, :, n:] == -1).all())


def test_results_do_not_depend_on_the_batch(asd):
    """Other requests cut the work differently; a request's weights stay the same bit for bit."""
    p = Problem(BF16, 5, 8, 2, 128, 64, [3000, 700, 1500, 2500, 1], seed=11)
    all_of = p.run(asd)
    cache = p.cache(asd)
    for b in range(5):
        one = asd.KVCache(cache.k, cache.v, cache.page_table[b:b + 1].contiguous())
        got = asd.kv_weigh(p.q[b:b + 1].cuda(), p.lse[b:b + 1].cuda(), one, p.kv_len[b:b + 1].cuda(),
                           p.before[b:b + 1].cuda(), scale=p.scale)
        assert torch.equal(got[0], all_of[b])


@pytest.mark.parametrize("dtype", (BF16, F32), ids=("bf16", "f32"))
def test_captured_replayed_and_on_another_stream(asd, dtype):
    p = Problem(dtype, 3, 8, 2, 64, 16, [400, 90], seed=12)
    q, lse, cache, kv = p.q.cuda(), p.lse.cuda(), p.cache(asd), p.kv_len.cuda()
    before, out = p.before.cuda(), p.before.cuda()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    asd.kv_weigh(q, lse, cache, kv, before, scale=p.scale, out=out, stream=side)
    side.synchronize()
    p.check(out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for _ in range(2):
            asd.kv_weigh(q, lse, cache, kv, before, scale=p.scale, out=out)
    for ctx in ([400, 90], [17, 395], [0, 1]):
        kv.copy_(torch.tensor(ctx, dtype=torch.int32))
        out.copy_(p.before)
        graph.replay()
        p.kv_len = torch.tensor(ctx, dtype=torch.int32)
        if max(ctx[0] - 400, ctx[1] - 90) <= 0:
            p.check(out)
        else:  # slots that the problem has no keys for hold NaN
            assert bool(out.isnan().any())
