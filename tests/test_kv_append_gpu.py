"""asd_kv_append and asd_kv_compact against plain 64-bit implementations."""
import math

import pytest
import torch

import cache_reference as ref

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


class Append:
    def __init__(self, dtype, T, Hq, Hkv, D, rot, page, ctx, new=None, norm=True, interleaved=False, seed=0,
                 positions=True):
        g = torch.Generator().manual_seed(seed)
        self.B, self.T, self.Hq, self.Hkv, self.D, self.rot, self.page = len(ctx), T, Hq, Hkv, D, rot, page
        self.dtype, self.interleaved, self.eps = dtype, interleaved, 1e-6
        self.kv_len = torch.tensor(ctx, dtype=torch.int32)
        self.new_len = None if new is None else torch.tensor(new, dtype=torch.int32)
        self.width = max(-(-(c + T) // page) for c in ctx)
        self.pages = self.B * self.width + 2
        self.table = torch.randperm(self.pages, generator=g)[:self.B * self.width].to(torch.int32).view(self.B, -1)
        self.rows = torch.randn(self.B, T, Hq + 2 * Hkv, D, generator=g).to(dtype)
        far = max(ctx) + T
        self.positions = torch.randint(0, far, (self.B, T), generator=g).to(torch.int32) if positions else None
        angle = torch.randn(far, max(rot // 2, 1), generator=g) * 3
        self.cos, self.sin = (angle.cos(), angle.sin()) if rot else (None, None)
        self.q_norm = (1 + 0.3 * torch.randn(D, generator=g)).to(dtype) if norm else None
        self.k_norm = (1 + 0.3 * torch.randn(D, generator=g)).to(dtype) if norm else None

    def reference(self):
        """{(b, t): (q, k, v rows)} of the tokens that exist."""
        got = {}
        for b in range(self.B):
            for t in range(self.T if self.new_len is None else int(self.new_len[b])):
                pos = int(self.kv_len[b]) + t if self.positions is None else int(self.positions[b, t])
                row = self.rows[b, t]

                def turn(h, w):
                    return ref.turned(row[h], w, self.eps, self.cos, self.sin, pos, self.rot, self.interleaved)
                got[b, t] = ([turn(h, self.q_norm) for h in range(self.Hq)],
                             [turn(self.Hq + h, self.k_norm) for h in range(self.Hkv)],
                             row[self.Hq + self.Hkv:])
        return got

    def run(self, asd, rows=None, cache=None, **kw):
        rows = self.rows.cuda() if rows is None else rows
        Hq, Hkv = self.Hq, self.Hkv
        if cache is None:
            k = torch.full((self.pages, self.page, Hkv, self.D), 7.0, dtype=self.dtype, device="cuda")
            cache = asd.KVCache(k, k.clone(), self.table.cuda())
        status = torch.zeros(self.B, dtype=torch.int32, device="cuda")

        def dev(x):
            return None if x is None else x.cuda()
        q_out = torch.full((self.B, self.T, Hq, self.D), 7.0, dtype=self.dtype, device="cuda") if Hq else None
        q_out = kw.pop("q_out", q_out)
        asd.kv_append(rows[:, :, Hq:Hq + Hkv], rows[:, :, Hq + Hkv:], cache, dev(self.kv_len),
                      q=rows[:, :, :Hq] if Hq else None, q_out=q_out, positions=dev(self.positions),
                      new_len=dev(self.new_len), cos=dev(self.cos), sin=dev(self.sin), interleaved=self.interleaved,
                      q_norm=dev(self.q_norm) if Hq else None, k_norm=dev(self.k_norm), eps=self.eps, status=status,
                      **kw)
        torch.cuda.synchronize()
        return None if q_out is None else q_out.cpu(), cache.k[0].cpu(), cache.v[0].cpu(), status.cpu()

    def check(self, q_out, k, v):
        want = self.reference()
        written = torch.zeros(self.pages, self.page, dtype=torch.bool)
        exists = torch.zeros(self.B, self.T, dtype=torch.bool)
        for (b, t), (qs, ks, vs) in want.items():
            page, place = ref.slot_place(self.table[b], int(self.kv_len[b]) + t, self.page)
            written[page, place] = exists[b, t] = True
            for got, rows in ((q_out[b, t] if self.Hq else [], qs), (k[page, place], ks)):
                for x, y in zip(got, rows):
                    far = (x.double() - y).abs() - ref.append_tolerance(self.dtype, self.D, None, None, y)
                    assert float(far.max()) <= 0, (b, t, float(far.max()))
            assert torch.equal(v[page, place], vs), (b, t)
        assert bool((k[~written] == 7).all()) and bool((v[~written] == 7).all()), "a place of no token was written"
        if self.Hq:
            assert bool((q_out[~exists] == 7).all())


SHAPES = [
    # dtype, T, Hq, Hkv, D, rot, page
    (BF16, 1, 5, 1, 128, 128, 64),
    (BF16, 9, 10, 2, 128, 128, 16),
    (F16, 5, 4, 4, 64, 64, 5),
    (F32, 7, 4, 1, 96, 32, 24),
    (BF16, 3, 3, 1, 80, 40, 16),
    (F16, 3, 3, 1, 96, 24, 16),
    (BF16, 3, 2, 1, 256, 256, 16),
    (F32, 3, 2, 1, 256, 64, 1),
    (BF16, 2, 3, 2, 33, 10, 7),
    (F32, 2, 3, 2, 50, 6, 7),
    (BF16, 2, 1, 1, 2, 2, 7),
    (F32, 2, 1, 1, 1, 0, 7),
    (F16, 70, 2, 3, 64, 0, 32),
    (BF16, 4, 0, 2, 128, 64, 32),
    (F32, 2, 2, 1, 200, 200, 9),
    (F16, 2, 2, 1, 250, 120, 9),
]


@pytest.mark.parametrize("interleaved", [False, True], ids=["halves", "neighbours"])
@pytest.mark.parametrize("norm", [False, True], ids=["plain", "norm"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"{str(s[0])[6:]}-T{s[1]}-{s[2]}q{s[3]}x{s[4]}-r{s[5]}-p{s[6]}")
def test_append(asd, shape, norm, interleaved):
    a = Append(*shape, ctx=[0, 1, 31, 100], norm=norm, interleaved=interleaved, seed=shape[4])
    q, k, v, status = a.run(asd)
    a.check(q, k, v)
    assert not status.any()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_fewer_tokens_and_positions_by_slot(asd, dtype):
    a = Append(dtype, 9, 4, 2, 64, 64, 16, ctx=[0, 20, 5, 6], new=[9, 0, 4, 1], seed=2, positions=False)
    q, k, v, status = a.run(asd)
    a.check(q, k, v)
    assert not status.any()


def test_layouts_and_in_place_queries(asd):
    """A cache by heads, rows that start on no boundary, and queries turned where they are."""
    for dtype in (BF16, F32):
        a = Append(dtype, 5, 4, 2, 64, 32, 16, ctx=[3, 40], seed=3)
        base = torch.full((a.pages, 2, 16, 64), 7.0, dtype=dtype, device="cuda")
        cache = asd.KVCache(base.transpose(1, 2), base.clone().transpose(1, 2), a.table.cuda())
        q, k, v, _ = a.run(asd, cache=cache)
        a.check(q, k, v)
        store = torch.zeros(2 * 5 * 8 * 67 + 1, dtype=dtype, device="cuda")
        loose = store[1:].view(2, 5, 8, 67)[..., :64]
        loose.copy_(a.rows)
        q2, k2, v2, _ = a.run(asd, rows=loose)
        a.check(q2, k2, v2)
        only_q = a.rows[:, :, :4].cuda().contiguous()
        rows = a.rows.cuda()
        k = torch.full((a.pages, 16, 2, 64), 7.0, dtype=dtype, device="cuda")
        cache = asd.KVCache(k, k.clone(), a.table.cuda())
        asd.kv_append(rows[:, :, 4:6], rows[:, :, 6:], cache, a.kv_len.cuda(), q=only_q, q_out=only_q,
                      positions=a.positions.cuda(), cos=a.cos.cuda(), sin=a.sin.cuda(), q_norm=a.q_norm.cuda(),
                      k_norm=a.k_norm.cuda())
        a.check(only_q.cpu(), cache.k[0].cpu(), cache.v[0].cpu())


def test_layer_and_pages_past_32_bits(asd):
    """The last pages of the second layer of a cache of 4.3e9 elements a tensor."""
    a = Append(BF16, 3, 4, 2, 128, 128, 256, ctx=[300, 7], seed=4)
    pages = 32800
    k = torch.empty(2, pages, 256, 2, 128, dtype=BF16, device="cuda")
    v = torch.empty_like(k)
    assert k.numel() > 2 ** 32
    k[1, -a.pages:] = 7
    v[1, -a.pages:] = 7
    cache = asd.KVCache(k, v, a.table.cuda() + (pages - a.pages))
    q, _, _, _ = a.run(asd, cache=cache, layer=1)
    a.check(q, k[1, -a.pages:].cpu(), v[1, -a.pages:].cpu())


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_infinities_and_nan_stay_with_the_elements_they_turn_with(asd, dtype, interleaved):
    """Without a norm an element reaches itself and its partner, and one past the rotation itself alone."""
    for D, rot in ((64, 32), (33, 10), (96, 48)):
        a = Append(dtype, 2, 1, 1, D, rot, 8, ctx=[3], norm=False, interleaved=interleaved, seed=7)
        clean, _, _, _ = a.run(asd)
        bad_at = [1, rot // 2, rot, D - 1]
        for bad in (math.nan, math.inf):
            for at in bad_at:
                rows = a.rows.clone()
                rows[0, 0, 0, at] = bad
                q, _, _, _ = a.run(asd, rows=rows.cuda())
                if at >= rot:
                    hit = {at}
                elif interleaved:
                    hit = {at, at ^ 1}
                else:
                    hit = {at, at + rot // 2 if at < rot // 2 else at - rot // 2}
                for i in range(D):
                    if i in hit:
                        assert not math.isfinite(float(q[0, 0, 0, i]))
                    else:
                        assert torch.equal(q[0, 0, 0, i], clean[0, 0, 0, i]), (D, at, i)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype,D,rot", [(BF16, 128, 128), (F16, 64, 32), (F32, 96, 96), (BF16, 80, 40), (BF16, 66, 6)])
def test_prompts(asd, dtype, D, rot, interleaved):
    """Thousands of tokens: several items a group of lanes, the last round ragged."""
    check_prompts(asd, dtype, D, rot, interleaved, 1501, 9, 3)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype,D,rot,Hq,Hkv", [(BF16, 128, 128, 5, 1), (F16, 64, 64, 1, 1), (BF16, 80, 40, 5, 1),
                                                (BF16, 128, 64, 2, 2), (F16, 96, 48, 0, 1), (F32, 64, 64, 5, 1)])
def test_prompts_of_few_heads(asd, dtype, D, rot, Hq, Hkv, interleaved):
    """As many tokens, with fewer heads than a group of lanes takes at a time."""
    check_prompts(asd, dtype, D, rot, interleaved, 4099, Hq, Hkv)


def check_prompts(asd, dtype, D, rot, interleaved, T, Hq, Hkv):
    a = Append(dtype, T, Hq, Hkv, D, rot, 16, ctx=[5, 0, 70], new=[T, 700, T - 1], interleaved=interleaved, seed=8)
    q, k, v, status = a.run(asd)
    assert not status.any()
    x = a.rows.double()
    w = torch.cat([a.q_norm.double().expand(Hq, D), a.k_norm.double().expand(Hkv, D)])
    q = q if Hq else torch.full((3, T, 0, D), 7.0, dtype=dtype)
    x = x[:, :, :Hq + Hkv] / (x[:, :, :Hq + Hkv].square().mean(-1, keepdim=True) + a.eps).sqrt() * w
    cos, sin = a.cos.double()[a.positions.long()][:, :, None], a.sin.double()[a.positions.long()][:, :, None]
    y = x.clone()
    lo, hi = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    y[..., lo], y[..., hi] = x[..., lo] * cos - x[..., hi] * sin, x[..., hi] * cos + x[..., lo] * sin
    big = y.abs().amax(-1, keepdim=True) * math.sqrt(2.0)
    tol = ref.UNIT[dtype] * y.abs() + (D + 16) * 2.0 ** -24 * big + (2.0 ** -24 if dtype == F16 else 1e-30)
    t = torch.arange(T)
    for b in range(3):
        n = int(a.new_len[b])
        assert bool(((q[b, :n].double() - y[b, :n, :Hq]).abs() <= tol[b, :n, :Hq]).all())
        assert bool((q[b, n:] == 7).all())
        slots = int(a.kv_len[b]) + t[:n]
        pages, places = a.table[b].long()[slots // 16], slots % 16
        assert bool(((k[pages, places].double() - y[b, :n, Hq:]).abs() <= tol[b, :n, Hq:]).all())
        assert torch.equal(v[pages, places], a.rows[b, :n, Hq + Hkv:])
    assert int((k != 7).any(-1).any(-1).sum()) == int(a.new_len.sum())


def test_append_data_errors(asd):
    a = Append(F32, 3, 2, 1, 32, 32, 8, ctx=[4, 5, 6, 7, 8, 9], new=[3, 3, 3, 3, 3, 3], seed=5)
    a.kv_len[0] = -2
    a.new_len[1] = 4
    a.kv_len[2] = a.width * 8 - 2
    a.table[3, 1] = a.pages           # kv_len 7: token 0 is on the page before it
    a.positions[4, 1] = a.cos.shape[0]
    a.positions[5, 2] = -1
    q, k, v, status = a.run(asd)
    assert status.tolist() == [asd.STATUS_LENGTH] * 3 + [asd.STATUS_PAGE] + [asd.STATUS_POSITION] * 2
    # what is left: tokens (3, 0), (4, 0), (4, 2), (5, 0), (5, 1), and the queries of all of request 3
    b = Append(F32, 3, 2, 1, 32, 32, 8, ctx=[4, 5, 6, 7, 8, 9], new=[0, 0, 0, 3, 3, 3], seed=5)
    q2, k2, v2, status2 = b.run(asd)
    assert not status2.any()
    assert bool((q[:3] == 7).all()) and torch.equal(q[3], q2[3])
    for req, t in ((4, 0), (4, 2), (5, 0), (5, 1)):
        assert torch.equal(q[req, t], q2[req, t])
    assert bool((q[4, 1] == 7).all()) and bool((q[5, 2] == 7).all())
    for req, t in ((3, 1), (3, 2), (4, 1), (5, 2)):
        page, place = ref.slot_place(b.table[req], int(b.kv_len[req]) + t, 8)
        k2[page, place] = v2[page, place] = 7
    assert torch.equal(k, k2) and torch.equal(v, v2)


def test_append_then_attend_is_ordered_without_synchronising(asd):
    """Launched back to back, attention reads what the append wrote."""
    a = Append(BF16, 9, 10, 2, 128, 128, 16, ctx=[100, 0, 40], seed=6)
    g = torch.Generator(device="cuda").manual_seed(1)
    k = torch.randn(a.pages, 16, 2, 128, generator=g, device="cuda").to(BF16)
    v = torch.randn(a.pages, 16, 2, 128, generator=g, device="cuda").to(BF16)
    rows, kv_len = a.rows.cuda(), a.kv_len.cuda()
    args = dict(positions=a.positions.cuda(), cos=a.cos.cuda(), sin=a.sin.cuda(), q_norm=a.q_norm.cuda(),
                k_norm=a.k_norm.cuda())
    want = None
    for sync in (True, False, False, False):
        cache = asd.KVCache(k.clone(), v.clone(), a.table.cuda())
        ws = asd.attention_workspace(cache, 9, 10)
        torch.cuda.synchronize()
        q = asd.kv_append(rows[:, :, 10:12], rows[:, :, 12:], cache, kv_len, q=rows[:, :, :10], **args)
        if sync:
            torch.cuda.synchronize()
        o = asd.tree_attention(q, cache, kv_len, workspace=ws)
        torch.cuda.synchronize()
        if want is None:
            want = o
        assert torch.equal(o["out"], want["out"]) and torch.equal(o["lse"], want["lse"])


# ---------------------------------------------------------------- compaction

def compact_reference(k, v, table, kv_len, path, path_len, page):
    k2, v2 = k.clone(), v.clone()
    for b in range(table.shape[0]):
        for i in range(int(path_len[b])):
            sp, so = ref.slot_place(table[b], int(kv_len[b]) + int(path[b, i]), page)
            dp, do = ref.slot_place(table[b], int(kv_len[b]) + i, page)
            k2[:, dp, do], v2[:, dp, do] = k[:, sp, so], v[:, sp, so]
    return k2, v2


@pytest.mark.parametrize("dtype,H,D", [(BF16, 8, 128), (F16, 3, 40), (F32, 2, 64), (BF16, 1, 33), (F32, 3, 7)])
@pytest.mark.parametrize("layers", [1, 5])
@pytest.mark.parametrize("by_heads", [False, True])
def test_compact(asd, dtype, H, D, layers, by_heads):
    g = torch.Generator().manual_seed(D)
    B, T, P, page, width = 6, 70, 20, 7, 25
    pages = B * width
    shape = (layers, pages, H, page, D) if by_heads else (layers, pages, page, H, D)
    k = torch.randn(shape, generator=g).to(dtype)
    v = torch.randn(shape, generator=g).to(dtype)
    table = torch.randperm(pages, generator=g).to(torch.int32).view(B, width)
    kv_len = torch.tensor([0, 3, 50, 90, 7, 100], dtype=torch.int32)
    path_len = torch.tensor([20, 1, 0, 20, 9, 20], dtype=torch.int32)
    path = torch.stack([torch.randperm(T, generator=g)[:P].sort().values for _ in range(B)]).to(torch.int32)
    path[3] = torch.arange(P)          # all in place
    path[0] = torch.arange(P) + 1      # every node one further on: each source is the next one's destination
    path[1, 1:] = 0                    # past path_len: not looked at
    kd, vd = k.cuda(), v.cuda()
    if by_heads:
        kd, vd, k, v = kd.transpose(2, 3), vd.transpose(2, 3), k.transpose(2, 3), v.transpose(2, 3)
    status = torch.zeros(B, dtype=torch.int32, device="cuda")
    asd.kv_compact(asd.KVCache(kd, vd, table.cuda()), kv_len.cuda(), path.cuda(), path_len.cuda(), status=status)
    torch.cuda.synchronize()
    k2, v2 = compact_reference(k, v, table, kv_len, path, path_len, page)
    assert torch.equal(kd.cpu(), k2) and torch.equal(vd.cpu(), v2) and not bool(status.any())


def test_compact_data_errors(asd):
    B, page, width = 7, 4, 6
    k = torch.randn(2, B * width, page, 2, 16).cuda()
    v = torch.randn(2, B * width, page, 2, 16).cuda()
    table = torch.arange(B * width, dtype=torch.int32).view(B, width)
    table[5, 2] = -1
    kv_len = torch.tensor([-1, 0, 0, 0, 22, 5, 5], dtype=torch.int32)
    path = torch.tensor([[0, 1, 2], [0, 2, 2], [0, 0, 5], [1, 2, 3], [0, 1, 2], [1, 4, 6], [0, 2, 4]],
                        dtype=torch.int32)
    path_len = torch.tensor([3, 3, 3, 4, 3, 3, 3], dtype=torch.int32)
    k0, v0 = k.cpu(), v.cpu()
    status = torch.zeros(B, dtype=torch.int32, device="cuda")
    asd.kv_compact(asd.KVCache(k, v, table.cuda()), kv_len.cuda(), path.cuda(), path_len.cuda(), status=status)
    torch.cuda.synchronize()
    assert status.tolist() == [asd.STATUS_LENGTH, asd.STATUS_PATH, asd.STATUS_PATH, asd.STATUS_LENGTH,
                               asd.STATUS_LENGTH, asd.STATUS_PAGE, 0]
    good = torch.tensor([0, 0, 0, 0, 0, 0, 3], dtype=torch.int32)
    k2, v2 = compact_reference(k0, v0, table, kv_len, path, good, page)
    assert torch.equal(k.cpu(), k2) and torch.equal(v.cpu(), v2)
