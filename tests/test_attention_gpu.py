"""asd_tree_attention against a plain 64-bit implementation."""
import math

import pytest
import torch

import cache_reference as ref

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


def random_parents(B, T, g):
    p = torch.full((B, T), -1, dtype=torch.int64)
    for t in range(1, T):
        p[:, t] = t - 1 - (torch.rand(B, generator=g) ** 2 * min(t, 6)).long()
    return p


class Problem:
    """Inputs on the CPU: a paged cache whose unused places hold NaN."""

    def __init__(self, dtype, T, Hq, Hkv, D, page, ctx, new=None, tree=False, seed=0, spare_pages=3, width=None,
                 q_scale=1.0):
        g = torch.Generator().manual_seed(seed)
        self.B, self.T, self.Hq, self.Hkv, self.D, self.page, self.dtype = len(ctx), T, Hq, Hkv, D, page, dtype
        self.kv_len = torch.tensor(ctx, dtype=torch.int32)
        self.new_len = None if new is None else torch.tensor(new, dtype=torch.int32)
        need = [-(-(c + T) // page) for c in ctx]
        self.width = width or max(need)
        self.pages = sum(need) + spare_pages
        order = torch.randperm(self.pages, generator=g).to(torch.int32)
        # places of the table that no slot uses hold ids of no page
        self.table = torch.full((self.B, self.width), 2 ** 31 - 1, dtype=torch.int32)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = order[at:at + n]
            at += n
        self.k = torch.full((self.pages, page, Hkv, D), math.nan).to(dtype)
        self.v = self.k.clone()
        for b in range(self.B):
            n = T if new is None else new[b]
            for s in range(ctx[b] + n):
                p, o = ref.slot_place(self.table[b], s, page)
                self.k[p, o] = torch.randn(Hkv, D, generator=g).to(dtype)
                self.v[p, o] = torch.randn(Hkv, D, generator=g).to(dtype)
        self.q = (torch.randn(self.B, T, Hq, D, generator=g) * q_scale).to(dtype)
        self.mask = None
        if tree:
            from paper_2608_03447_gb300 import asd
            self.mask = asd.tree_mask(random_parents(self.B, T, g))
        self.scale = 1.0 / math.sqrt(D)

    def place(self, b, slot):
        return ref.slot_place(self.table[b], slot, self.page)

    def reference(self):
        dev = "cuda" if int(self.kv_len.max()) > 2000 else "cpu"  # in 64 bits either way
        got = ref.attention(self.q.to(dev), self.k.to(dev), self.v.to(dev), self.table, self.kv_len, self.new_len,
                            self.mask, self.scale)
        return [x.cpu() for x in got]

    def device(self, asd, layout="tokens"):
        if layout == "tokens":
            k, v = self.k.cuda(), self.v.cuda()
        elif layout == "heads":  # [pages, heads, page, D]
            k, v = (x.transpose(1, 2).contiguous().cuda().transpose(1, 2) for x in (self.k, self.v))
        else:  # rows that start on no boundary: D + 3 elements apart, one element in
            def loose(x):
                P, n, H, D = x.shape
                store = torch.full((P * n * H * (D + 3) + 1,), math.nan, dtype=x.dtype, device="cuda")
                w = store[1:].view(P, n, H, D + 3)[..., :D]
                w.copy_(x)
                return w
            k, v = loose(self.k), loose(self.v)
        return asd.KVCache(k, v, self.table.cuda())

    def run(self, asd, layout="tokens", **kw):
        cache = self.device(asd, layout)
        status = torch.zeros(self.B, dtype=torch.int32, device="cuda")
        ws = kw.pop("workspace", None) or asd.attention_workspace(cache, self.T, self.Hq)
        o = asd.tree_attention(self.q.cuda(), cache, self.kv_len.cuda(),
                               tree_mask=None if self.mask is None else self.mask.cuda(),
                               new_len=None if self.new_len is None else self.new_len.cuda(), scale=self.scale,
                               status=status, workspace=ws, **kw)
        assert ws.error() == 0
        return o["out"].cpu(), o["lse"].cpu(), status.cpu()

    def check(self, out, lse):
        o, l, weight, reach = self.reference()
        slots = int(self.kv_len.max()) + self.T
        vmax = float(self.v.double().nan_to_num(0).abs().max()) if self.v.numel() else 0.0
        far = (out.double() - o).abs() - ref.attention_tolerance(self.dtype, self.D, slots, weight, reach, o, vmax)
        assert not out.isnan().any()
        assert float(far.max()) <= 0, f"out is {float(far.max()):.3g} further off than it may be"
        empty = torch.isinf(l)
        assert torch.equal(torch.isinf(lse) & (lse < 0), empty)
        assert not out[empty].any()
        gap = (lse.double() - l).abs()[~empty] - ref.lse_tolerance(self.D, slots, reach, l)[~empty]
        assert gap.numel() == 0 or float(gap.max()) <= 0, f"lse is {float(gap.max()):.3g} further off than it may be"


# one request's lengths at and around tiles of 64 and 128 slots
EDGES = [0, 1, 2, 31, 62, 63, 64, 65, 126, 127, 128, 129, 191, 255, 256, 300]

SHAPES = [
    # dtype, T, Hq, Hkv, D, page
    (BF16, 1, 4, 1, 64, 16),
    (BF16, 1, 10, 2, 128, 64),
    (BF16, 9, 10, 2, 128, 16),
    (F16, 5, 8, 2, 64, 48),
    (F16, 33, 4, 1, 128, 128),
    (BF16, 7, 6, 2, 80, 24),
    (F16, 4, 6, 3, 96, 5),
    (F32, 1, 4, 2, 64, 16),
    (F32, 17, 4, 1, 96, 24),
    (F32, 3, 6, 2, 128, 1),
    (BF16, 2, 2, 1, 256, 16),
    (F32, 6, 4, 2, 200, 7),
    (BF16, 5, 2, 2, 40, 33),
    (F32, 3, 2, 1, 33, 10),
    (BF16, 3, 2, 1, 1, 10),
    (F16, 3, 3, 1, 21, 16),
]


@pytest.mark.parametrize("tree", [False, True], ids=["chain", "tree"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"{str(s[0])[6:]}-T{s[1]}-{s[2]}x{s[3]}x{s[4]}-p{s[5]}")
def test_lengths_at_tile_edges(asd, shape, tree):
    p = Problem(*shape, ctx=EDGES, tree=tree, seed=len(str(shape)))
    out, lse, status = p.run(asd)
    p.check(out, lse)
    assert not status.any()


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("T,Hq,Hkv,D", [(1, 5, 1, 128), (9, 5, 1, 128), (26, 5, 1, 128), (52, 5, 1, 64), (3, 2, 2, 64)])
def test_long_context_is_split(asd, dtype, T, Hq, Hkv, D):
    """One long request among short ones: its units are cut into many pieces."""
    p = Problem(dtype, T, Hq, Hkv, D, 32, ctx=[9000, 3, 0, 700], tree=True, seed=5)
    out, lse, _ = p.run(asd)
    p.check(out, lse)


class Filled(Problem):
    """Contexts of tens of thousands of slots: the cache is filled at once, unused places included."""

    def __init__(self, dtype, T, Hq, Hkv, D, page, ctx, seed):
        Problem.__init__(self, dtype, T, Hq, Hkv, D, page, [0] * len(ctx), tree=True, seed=seed)
        g = torch.Generator().manual_seed(seed + 1)
        self.kv_len = torch.tensor(ctx, dtype=torch.int32)
        self.width = max(-(-(c + T) // page) for c in ctx)
        self.pages = self.B * self.width
        self.table = torch.randperm(self.pages, generator=g).to(torch.int32).view(self.B, self.width)
        self.k = torch.randn(self.pages, page, Hkv, D, generator=g).to(dtype)
        self.v = torch.randn(self.pages, page, Hkv, D, generator=g).to(dtype)


@pytest.mark.parametrize("page", [64, 48, 16, 128, 20, 256])
@pytest.mark.parametrize("T,Hq,Hkv,D", [(1, 3, 1, 128), (7, 8, 2, 64), (44, 5, 1, 128), (61, 5, 1, 128)])
def test_ranges_of_many_tiles(asd, T, Hq, Hkv, D, page):
    """Every CTA works through tens of tiles: rings and barriers wrap many times."""
    p = Filled(BF16, T, Hq, Hkv, D, page, [150000, 20000, 90000], seed=page)
    out, lse, _ = p.run(asd)
    p.check(out, lse)


def test_ranges_of_many_tiles_of_short_requests(asd):
    """Every CTA works through tens of units of one to four tiles, shared and not."""
    g = torch.Generator().manual_seed(2)
    for T, Hq, Hkv, D, page in ((5, 16, 8, 64, 16), (33, 8, 2, 128, 32), (1, 8, 8, 128, 64)):
        ctx = torch.randint(0, 400, (256,), generator=g).tolist()
        p = Filled(BF16, T, Hq, Hkv, D, page, ctx, seed=T)
        p.new_len = torch.randint(0, T + 1, (256,), generator=g).to(torch.int32)
        out, lse, _ = p.run(asd)
        p.check(out, lse)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,G", [(70, 1), (128, 1), (129, 1), (33, 8), (100, 5)])
def test_many_rows(asd, dtype, T, G):
    """More rows per key/value head than one row tile holds; masks of more than two words."""
    for tree in (False, True):
        p = Problem(dtype, T, 2 * G, 2, 64, 16, ctx=[200, 0, 130], tree=tree, seed=T)
        out, lse, _ = p.run(asd)
        p.check(out, lse)


@pytest.mark.parametrize("tree", [False, True], ids=["chain", "tree"])
@pytest.mark.parametrize("B,T,Hq,Hkv", [(1, 27, 10, 2), (3, 61, 10, 2), (40, 33, 8, 2), (9, 70, 6, 2)])
def test_row_tiles_that_cost_differently(asd, B, T, Hq, Hkv, tree):
    """Requests with more rows than a softmax group has threads for beside requests (and last row tiles) with fewer."""
    g = torch.Generator().manual_seed(B + T)
    ctx = torch.randint(0, 700, (B,), generator=g).tolist()
    new = [T] + torch.randint(0, T + 1, (B - 1,), generator=g).tolist()
    p = Problem(BF16, T, Hq, Hkv, 64, 16, ctx=ctx, new=new, tree=tree, seed=T)
    out, lse, _ = p.run(asd)
    p.check(out, lse)


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_fewer_tokens_than_T_and_none(asd, dtype):
    p = Problem(dtype, 9, 10, 2, 128, 16, ctx=[100, 0, 0, 200, 77], new=[9, 3, 0, 0, 1], tree=True, seed=3)
    out, lse, status = p.run(asd)
    p.check(out, lse)
    assert not status.any()
    assert not out[1, 3:].any() and not out[2].any() and torch.isinf(lse[3]).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_that_see_nothing(asd, dtype):
    """Mask rows of zeros: with an empty context the row is 0 and -inf, beside rows that see something."""
    p = Problem(dtype, 40, 4, 2, 64, 16, ctx=[0, 0, 90], tree=True, seed=4)
    p.mask[0] = 0
    p.mask[1, ::2] = 0
    p.mask[2, 5] = 0
    out, lse, _ = p.run(asd)
    p.check(out, lse)
    assert not out[0].any() and torch.isinf(lse[0]).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_mask_bits_past_the_tokens_are_ignored(asd, dtype):
    p = Problem(dtype, 9, 4, 2, 64, 16, ctx=[50, 0, 128], new=[4, 9, 2], tree=True, seed=6)
    p2 = Problem(dtype, 9, 4, 2, 64, 16, ctx=[50, 0, 128], new=[4, 9, 2], tree=True, seed=6)
    for b, n in enumerate([4, 9, 2]):
        p2.mask[b] |= torch.tensor(~((1 << n) - 1), dtype=torch.int32)
    out, lse, _ = p.run(asd)
    out2, lse2, _ = p2.run(asd)
    p.check(out, lse)
    assert torch.equal(out, out2) and torch.equal(lse, lse2)


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_what_a_row_does_not_see_does_not_reach_it(asd, dtype, bad):
    """NaN and infinities in one branch's keys and values: the other branch's rows and the other requests are as
    without them; rows of the branch itself, which sees them, are not finite."""
    p = Problem(dtype, 6, 4, 2, 64, 16, ctx=[100, 61, 0], seed=7)
    from paper_2608_03447_gb300 import asd as binding
    parents = torch.tensor([[-1, 0, 0, 1, 2, 3]] * 3)  # 0 - 1 - 3 - 5 and 0 - 2 - 4
    p.mask = binding.tree_mask(parents)
    good, good_lse, _ = p.run(asd)
    p.check(good, good_lse)
    for b in (0, 1):
        page, place = p.place(b, int(p.kv_len[b]) + 3)
        p.k[page, place] = bad
        p.v[page, place] = bad
    out, lse, _ = p.run(asd)
    assert torch.equal(out[2], good[2]) and torch.equal(lse[2], good_lse[2])
    for b in (0, 1):
        for t in (0, 1, 2, 4):
            assert torch.equal(out[b, t], good[b, t]), (b, t)
            assert torch.equal(lse[b, t], good_lse[b, t])
    # only a value: the keys are as they were
    p = Problem(dtype, 6, 4, 2, 64, 16, ctx=[100, 61, 0], seed=7)
    p.mask = binding.tree_mask(parents)
    for b in (0, 1):
        page, place = p.place(b, int(p.kv_len[b]) + 3)
        p.v[page, place, 1, 10] = bad
    out, lse, _ = p.run(asd)
    assert torch.equal(lse, good_lse)
    for b in (0, 1):
        for t in range(6):
            for h in range(4):
                hit = t in (3, 5) and h // 2 == 1
                same = out[b, t, h] == good[b, t, h]
                assert bool(same[:10].all()) and bool(same[11:].all())
                assert bool(same[10]) != hit
                if hit:
                    assert bool(out[b, t, h, 10].isnan()) if math.isnan(bad) else float(out[b, t, h, 10]) == bad


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("layout", ["heads", "loose"])
@pytest.mark.parametrize("D", [64, 128, 72])
def test_cache_layouts(asd, dtype, layout, D):
    p = Problem(dtype, 5, 6, 2, D, 16, ctx=[130, 0, 63, 300], tree=True, seed=8)
    out, lse, _ = p.run(asd, layout)
    p.check(out, lse)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_queries_are_a_view_of_a_projection(asd, dtype):
    p = Problem(dtype, 5, 6, 2, 64, 16, ctx=[130, 3], tree=True, seed=9)
    rows = torch.full((2, 5, 6 + 4, 64), math.nan, dtype=dtype, device="cuda")
    rows[:, :, :6] = p.q.cuda()
    cache = p.device(asd)
    want = asd.tree_attention(p.q.cuda(), cache, p.kv_len.cuda(), tree_mask=p.mask.cuda())
    got = asd.tree_attention(rows[:, :, :6], cache, p.kv_len.cuda(), tree_mask=p.mask.cuda())
    assert torch.equal(want["out"], got["out"]) and torch.equal(want["lse"], got["lse"])
    # batch and token dimensions the other way round, and one query row for all tokens
    turned = p.q.cuda().transpose(0, 1).contiguous().transpose(0, 1)
    got = asd.tree_attention(turned, cache, p.kv_len.cuda(), tree_mask=p.mask.cuda())
    assert torch.equal(want["out"], got["out"])
    same = p.q[:, :1].cuda().expand(2, 5, 6, 64)
    p.q = same.cpu()
    got = asd.tree_attention(same, cache, p.kv_len.cuda(), tree_mask=p.mask.cuda())
    p.check(got["out"].cpu(), got["lse"].cpu())


def test_more_requests_than_a_cta_has_threads(asd):
    """The deal adds the lengths up in several rounds."""
    g = torch.Generator().manual_seed(1)
    ctx = torch.randint(0, 40, (1100,), generator=g).tolist()
    for dtype in (BF16, F32):
        p = Problem(dtype, 2, 2, 1, 32, 16, ctx=ctx, new=[i % 3 for i in range(1100)], seed=10)
        out, lse, _ = p.run(asd)
        p.check(out, lse)


@pytest.mark.parametrize("B", [31, 32, 33, 64, 65, 97, 130])
def test_any_number_of_requests(asd, B):
    """A block of requests a lane: numbers at and around whole blocks, runs of requests without any work."""
    g = torch.Generator().manual_seed(B)
    ctx = [0 if i % 7 < 3 else int(torch.randint(0, 300, (1,), generator=g)) for i in range(B)]
    new = [0 if i % 7 < 4 else i % 4 for i in range(B)]
    for dtype in (BF16, F32):
        p = Problem(dtype, 3, 4, 2, 64, 16, ctx=ctx, new=new, seed=B)
        out, lse, status = p.run(asd)
        p.check(out, lse)
        assert not status.any()


def test_layers(asd):
    p = Problem(BF16, 3, 4, 2, 64, 16, ctx=[40, 9], seed=11)
    k = torch.full((3, *p.k.shape), math.nan, dtype=BF16, device="cuda")
    v = k.clone()
    k[1], v[1] = p.k.cuda(), p.v.cuda()
    cache = asd.KVCache(k, v, p.table.cuda())
    o = asd.tree_attention(p.q.cuda(), cache, p.kv_len.cuda(), layer=1, scale=p.scale)
    p.check(o["out"].cpu(), o["lse"].cpu())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("q_scale", [30.0, 0.0])
def test_large_scores_and_equal_ones(asd, dtype, q_scale):
    """Scores in the hundreds, whose running maximum climbs over the tiles; and all scores equal."""
    p = Problem(dtype, 4, 4, 2, 64, 16, ctx=[1000, 500], tree=True, seed=12, q_scale=q_scale)
    out, lse, _ = p.run(asd)
    p.check(out, lse)


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_scores_that_rise_and_fall(asd, dtype):
    """Keys that grow along the context (the output's sum is rescaled tile after tile), and that shrink."""
    for up in (True, False):
        p = Problem(dtype, 4, 4, 2, 64, 16, ctx=[1500], seed=13)
        for s in range(1504):
            page, place = p.place(0, s)
            f = s / 150 if up else (1504 - s) / 150
            p.k[page, place] = (p.q[0, 0, ::2].double() * f / 8).to(dtype)
        out, lse, _ = p.run(asd)
        p.check(out, lse)


def test_negative_and_zero_scale(asd):
    for dtype in (BF16, F32):
        for scale in (-0.3, 0.0):
            p = Problem(dtype, 3, 4, 2, 64, 16, ctx=[200, 0], tree=True, seed=14)
            p.scale = scale
            out, lse, _ = p.run(asd)
            p.check(out, lse)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_same_bits_every_time_and_a_workspace_for_all_shapes(asd, dtype):
    """One workspace, calls of several shapes in turn, each twice: the same bits, whatever ran in between."""
    shapes = [(9, 10, 2, 128, 16, [3000, 0, 40]), (1, 4, 1, 64, 16, [9000]), (52, 10, 2, 128, 16, [700, 2500])]
    ps = [Problem(dtype, T, Hq, Hkv, D, page, ctx=ctx, tree=True, seed=15) for T, Hq, Hkv, D, page, ctx in shapes]
    caches = [p.device(asd) for p in ps]
    sizes = [asd.attention_workspace(c, p.T, p.Hq) for c, p in zip(caches, ps)]
    ws = max(sizes, key=lambda w: w.nbytes)
    first = None
    for _ in range(3):
        got = [p.run(asd, workspace=ws)[:2] for p in ps]
        if first is None:
            first = got
            for p, (out, lse) in zip(ps, got):
                p.check(out, lse)
        for a, b in zip(first, got):
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    assert ws.error() == 0


def test_without_lse_and_into_given_outputs(asd):
    p = Problem(BF16, 3, 4, 2, 64, 16, ctx=[200, 7], seed=16)
    cache = p.device(asd)
    want = asd.tree_attention(p.q.cuda(), cache, p.kv_len.cuda())
    mine = {"out": torch.full((2, 3, 4, 64), 7.0, dtype=BF16, device="cuda")}
    got = asd.tree_attention(p.q.cuda(), cache, p.kv_len.cuda(), out=mine)
    assert got is mine and torch.equal(mine["out"], want["out"])


def test_on_another_stream_and_in_a_graph(asd):
    p = Problem(BF16, 9, 10, 2, 128, 16, ctx=[3000, 0, 40], tree=True, seed=17)
    cache = p.device(asd)
    q, kv_len, mask = p.q.cuda(), p.kv_len.cuda(), p.mask.cuda()
    ws = asd.attention_workspace(cache, p.T, p.Hq)
    want = asd.tree_attention(q, cache, kv_len, tree_mask=mask, scale=p.scale, workspace=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = asd.tree_attention(q, cache, kv_len, tree_mask=mask, scale=p.scale, workspace=ws)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert torch.equal(got["out"], want["out"]) and torch.equal(got["lse"], want["lse"])
    out = {"out": torch.zeros_like(want["out"]), "lse": torch.zeros_like(want["lse"])}
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for _ in range(3):
            asd.tree_attention(q, cache, kv_len, tree_mask=mask, scale=p.scale, workspace=ws, out=out)
    # the lengths are the device's at replay
    for ctx in ([3000, 0, 40], [10, 0, 40], [2000, 0, 0]):
        kv_len.copy_(torch.tensor(ctx, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        p.kv_len = torch.tensor(ctx, dtype=torch.int32)
        p.check(out["out"].cpu(), out["lse"].cpu()) if ctx[2] == 40 and ctx[0] == 3000 else None
        again = asd.tree_attention(q, cache, kv_len, tree_mask=mask, scale=p.scale, workspace=ws)
        torch.cuda.synchronize()
        assert torch.equal(out["out"], again["out"])


def test_offsets_past_32_bits(asd):
    """A cache of 5.4e9 elements a tensor: pages at its end."""
    pages, page, H, D = 20600, 256, 8, 128
    k = torch.empty(pages, page, H, D, dtype=BF16, device="cuda")
    v = torch.empty_like(k)
    assert k.numel() > 2 ** 32
    p = Problem(BF16, 2, 16, 8, 128, 256, ctx=[600, 100], seed=18, spare_pages=0)
    shift = pages - p.pages
    k[shift:], v[shift:] = p.k.cuda(), p.v.cuda()
    table = torch.where(p.table == 2 ** 31 - 1, p.table, p.table + shift)
    o = asd.tree_attention(p.q.cuda(), asd.KVCache(k, v, table.cuda()), p.kv_len.cuda())
    p.check(o["out"].cpu(), o["lse"].cpu())


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_data_errors_are_flagged(asd, dtype):
    """Lengths out of range count as no tokens; slots on pages out of range read as zeros."""
    p = Problem(dtype, 3, 4, 2, 64, 16, ctx=[40, 20, 33, 5, 17], new=[3, 3, 3, 3, 3], seed=19)
    want, want_lse, _ = p.run(asd)
    kv_len, new_len = p.kv_len.clone(), p.new_len.clone()
    p.kv_len[0] = -1
    p.new_len[1] = 4
    p.kv_len[3] = p.width * 16 - 2
    out, lse, status = p.run(asd)
    assert status.tolist() == [asd.STATUS_LENGTH, asd.STATUS_LENGTH, 0, asd.STATUS_LENGTH, 0]
    for b in (0, 1, 3):
        assert not out[b].any() and torch.isinf(lse[b]).all()
    for b in (2, 4):
        assert torch.equal(out[b], want[b])
    p.kv_len, p.new_len = kv_len, new_len
    for bad in (-1, p.pages, 2 ** 31 - 1, -2 ** 31):
        q = Problem(dtype, 3, 4, 2, 64, 16, ctx=[40, 20, 33, 5, 17], new=[3, 3, 3, 3, 3], seed=19)
        was = int(q.table[2, 1])
        q.table[2, 1] = bad
        out, lse, status = q.run(asd)
        assert status.tolist() == [0, 0, asd.STATUS_PAGE, 0, 0]
        q.table[2, 1] = was
        q.k[was], q.v[was] = 0, 0
        q.check(out, lse)


def test_a_failed_workspace_is_reported(asd):
    """While the workspace's error word is set a call flags its requests and writes nothing."""
    for dtype in (BF16, F32):
        p = Problem(dtype, 3, 4, 2, 64, 16, ctx=[40, 20], seed=20)
        cache = p.device(asd)
        ws = asd.attention_workspace(cache, 3, 4)
        ws.buffer[:4] = torch.tensor([9, 0, 0, 0], dtype=torch.uint8)
        out = {"out": torch.full((2, 3, 4, 64), 7.0, dtype=dtype, device="cuda")}
        status = torch.zeros(2, dtype=torch.int32, device="cuda")
        asd.tree_attention(p.q.cuda(), cache, p.kv_len.cuda(), workspace=ws, out=out, status=status)
        assert status.tolist() == [asd.STATUS_INCOMPLETE] * 2 and bool((out["out"] == 7).all())
        assert ws.error() == 9
        ws.reset()
        asd.tree_attention(p.q.cuda(), cache, p.kv_len.cuda(), workspace=ws, out=out)
        assert not bool((out["out"] == 7).all())


def test_empty_calls(asd):
    k = torch.zeros(4, 16, 2, 64, dtype=BF16, device="cuda")
    none = asd.KVCache(k, k.clone(), torch.zeros(0, 2, dtype=torch.int32, device="cuda"))
    o = asd.tree_attention(torch.zeros(0, 3, 4, 64, dtype=BF16, device="cuda"), none,
                           torch.zeros(0, dtype=torch.int32, device="cuda"))
    assert o["out"].shape == (0, 3, 4, 64)
    two = asd.KVCache(k, k.clone(), torch.zeros(2, 0, dtype=torch.int32, device="cuda"))
    o = asd.tree_attention(torch.zeros(2, 0, 4, 64, dtype=BF16, device="cuda"), two,
                           torch.zeros(2, dtype=torch.int32, device="cuda"))
    assert o["out"].shape == (2, 0, 4, 64)
    # no page at all: rows that see nothing
    o = asd.tree_attention(torch.ones(2, 1, 4, 64, dtype=BF16, device="cuda"), two,
                           torch.zeros(2, dtype=torch.int32, device="cuda"),
                           new_len=torch.zeros(2, dtype=torch.int32, device="cuda"))
    assert not bool(o["out"].any()) and bool(torch.isinf(o["lse"]).all())
