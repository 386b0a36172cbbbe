"""Logits under rules against a plain implementation that rounds every operation once: equal bit for bit."""
import math

import numpy as np
import pytest
import torch

import rules_reference as ref
from oracle import oracle

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


class Problem:
    def __init__(self, dtype, B, K, V, said=40, biased=5, grammar="third", seed=0, penalties=True, odd=True):
        g = torch.Generator().manual_seed(seed)
        self.dtype, self.B, self.K, self.V = dtype, B, K, V
        self.z = (3 * torch.randn(B, K + 1, V, generator=g)).to(dtype)
        self.z[torch.rand(B, K + 1, V, generator=g) < 0.02] = 0.0
        text = torch.randint(V, (B, said), generator=g)
        self.seen = torch.zeros(B, V, dtype=torch.int32)
        for b in range(B):
            for i, x in enumerate(text[b].tolist()):
                self.seen[b, x] = self.seen[b, x] | ref.PROMPT if i < said // 3 else self.seen[b, x] + 1
        self.bias = torch.zeros(B, V)
        self.marked = self.seen != 0
        for b in range(B):
            for x in torch.randint(V, (biased,), generator=g).tolist():
                self.bias[b, x] = 4 * torch.randn(1, generator=g)
                self.marked[b, x] = True
        # drafts: the text's tokens, leaders of their rows, twice the same
        self.draft = torch.randint(V, (B, K), generator=g).to(torch.int32)
        for b in range(B):
            for j in range(K):
                c = (b + j) % 4
                if c == 0 and said:
                    self.draft[b, j] = int(text[b, j % said])
                elif c == 1:
                    self.draft[b, j] = int(self.z[b, j].float().argmax())
                elif c == 2 and j:
                    self.draft[b, j] = self.draft[b, j - 1]
        self.repetition = 0.8 + 0.7 * torch.rand(B, generator=g) if penalties else None
        self.frequency = 0.6 * torch.rand(B, generator=g) - 0.1 if penalties else None
        self.presence = 0.7 * torch.rand(B, generator=g) if penalties else None
        self.allow = None
        if grammar:
            share = {"third": 0.33, "few": 0.02, "most": 0.97}[grammar]
            self.allow = torch.rand(B, K + 1, V, generator=g) < share

    def rules(self, asd):
        records = torch.stack([self.seen, self.bias.view(torch.int32)], -1)
        # what has no mark is not read
        junk = torch.tensor([77, int(torch.tensor(1000.0).view(torch.int32))], dtype=torch.int32)
        records = torch.where(self.marked[:, :, None], records, junk)
        marks = ref.words_of(self.marked)
        if self.V % 32:  # bits past the vocabulary may be anything
            marks[:, -1] |= -1 << (self.V % 32)
        dev = [None if x is None else x.cuda() for x in (self.repetition, self.frequency, self.presence)]
        return asd.TokenRules(marks.cuda(), records.contiguous().cuda(), *dev)

    def mask(self):
        return None if self.allow is None else ref.words_of(self.allow).cuda()

    def logits(self, off=0):
        """On the GPU, `off` elements past a 16-byte boundary."""
        store = torch.empty(self.z.numel() + 16, dtype=self.dtype, device="cuda")
        at = store[off:off + self.z.numel()].view(self.z.shape)
        return at.copy_(self.z)

    def changed(self):
        out = []
        for b in range(self.B):
            pen = [None if x is None else float(x[b]) for x in (self.repetition, self.frequency, self.presence)]
            out.append(ref.changed(self.z[b], self.draft[b].tolist(), self.marked[b], self.seen[b], self.bias[b], *pen,
                                   None if self.allow is None else self.allow[b]))
        return torch.stack(out)


def same(got, want):
    """Bit for bit, but for the sign of a zero and a NaN's payload."""
    return torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(0.0), want.nan_to_num(0.0))


def check_verify(asd, p, off=0, strict=False, gate=1.0, cap=2, budget=8.0, nan_rows=False):
    """nan_rows: a request flagged for a NaN has an unspecified argmax, and what follows from it, in the NaN's row."""
    led = asd.make_ledger(p.B, budget, 0.5)
    want = oracle.verify(p.changed().float().numpy(), p.draft.numpy(), led.cpu().numpy(), gate, cap, strict)
    ws = asd.Workspace(p.B, p.K, p.V, asd.BF16 if p.dtype == BF16 else asd.F32)
    for _ in range(2):  # the workspace is left as it was
        led = asd.make_ledger(p.B, budget, 0.5)
        got = asd.rules_verify(p.logits(off), p.draft.cuda(), None if strict else led, gate, cap, p.rules(asd),
                               allow=p.mask(), workspace=ws)
        ok = (want["status"] & oracle.STATUS_NAN_LOGIT) == 0 if nan_rows else np.ones(p.B, bool)
        for name in ("accepted_len", "status"):
            assert np.array_equal(got[name].cpu().numpy(), want[name]), name
        for name in ("committed", "recovery", "row_argmax"):
            assert np.array_equal(got[name].cpu().numpy()[ok], want[name][ok]), name
        assert np.array_equal(got["row_regret"].cpu().numpy()[ok], want["row_regret"][ok], equal_nan=True)
        if not strict:
            assert np.array_equal(led.cpu().numpy(), want["ledger"])
    assert int(ws.buffer.count_nonzero()) == 0


def check_logits(asd, p, off=0, to=0, in_place=False):
    want = p.changed().float().to(p.dtype)
    z = p.logits(off)
    out = z
    if not in_place:
        store = torch.full((p.z.numel() + 16,), 9.0, dtype=p.dtype, device="cuda")
        out = store[to:to + p.z.numel()].view(p.z.shape)
    got = asd.rules_logits(z, p.draft.cuda() if p.K else None, p.rules(asd), allow=p.mask(), out=out)
    assert got is out and same(got.cpu(), want)
    if not in_place:
        assert bool((store[:to] == 9).all() and (store[to + p.z.numel():] == 9).all()) and same(z.cpu(), p.z)


SHAPES = [(1, 0, 1), (2, 3, 7), (1, 8, 33), (3, 1, 1000), (2, 31, 513), (2, 8, 2049), (1, 5, 4096), (5, 10, 6001),
          (1, 0, 32001), (1, 4, 151936), (40, 4, 4099)]


@pytest.mark.parametrize("B,K,V", SHAPES)
@pytest.mark.parametrize("dtype", (BF16, F32), ids=("bf16", "f32"))
@pytest.mark.parametrize("grammar", (None, "third"))
def test_verify(asd, dtype, B, K, V, grammar):
    p = Problem(dtype, B, K, V, said=min(V, 60), biased=min(V, 9), grammar=grammar, seed=V + K)
    check_verify(asd, p)


@pytest.mark.parametrize("B,K,V", SHAPES)
@pytest.mark.parametrize("dtype", (BF16, F32), ids=("bf16", "f32"))
@pytest.mark.parametrize("grammar", (None, "third"))
def test_logits(asd, dtype, B, K, V, grammar):
    p = Problem(dtype, B, K, V, said=min(V, 60), biased=min(V, 9), grammar=grammar, seed=V + K + 1)
    check_logits(asd, p)


@pytest.mark.parametrize("dtype", (BF16, F32), ids=("bf16", "f32"))
@pytest.mark.parametrize("off", (1, 3, 7))
@pytest.mark.parametrize("V", (2048, 3001))
def test_logits_that_start_anywhere(asd, dtype, off, V):
    p = Problem(dtype, 3, 4, V, grammar="most", seed=off)
    check_verify(asd, p, off=off)
    check_logits(asd, p, off=off, to=(off * 3) % 8)
    check_logits(asd, p, off=off, to=off)
    check_logits(asd, p, off=off, in_place=True)


@pytest.mark.parametrize("case", ("no rules", "all tokens", "few allowed", "bias only", "penalties only"))
@pytest.mark.parametrize("dtype", (BF16, F32), ids=("bf16", "f32"))
def test_kinds_of_rules(asd, dtype, case):
    kw = {"no rules": dict(said=0, biased=0, grammar=None, penalties=False),
          "all tokens": dict(said=9000, biased=400),
          "few allowed": dict(grammar="few"), "bias only": dict(said=0, biased=50, grammar=None, penalties=False),
          "penalties only": dict(biased=0, grammar=None)}[case]
    p = Problem(dtype, 2, 6, 2500, seed=5, **kw)
    check_verify(asd, p)
    check_verify(asd, p, strict=True)
    check_verify(asd, p, gate=math.inf, cap=2 ** 31 - 1, budget=math.inf)
    check_logits(asd, p)
    check_logits(asd, p, in_place=True)


@pytest.mark.parametrize("dtype", (BF16, F32), ids=("bf16", "f32"))
@pytest.mark.parametrize("V,off", ((5000, 0), (3001, 3), (700, 0)))
@pytest.mark.parametrize("grammar", (None, "third"))
def test_most_of_the_vocabulary_is_lowered(asd, dtype, V, off, grammar):
    """Bans and large penalties on nearly every token: the best one that is left may be far down."""
    p = Problem(dtype, 4, 5, V, said=3 * V, biased=0, grammar=grammar, seed=V)
    p.repetition, p.frequency, p.presence = p.repetition.clamp(min=1.0), p.frequency.abs() + 3, p.presence + 9
    p.marked = torch.rand(4, V, generator=torch.Generator().manual_seed(3)) < torch.tensor([0.97, 0.5, 1.0, 1.0])[:, None]
    p.seen[2:] = torch.where(p.seen[2:] == 0, torch.tensor(1, dtype=torch.int32), p.seen[2:])
    p.bias[0] = -80.0
    p.bias[3] = -math.inf
    p.z[1, 2, 20:40] = math.inf  # infinite logits, some lowered, some not
    if p.allow is not None:
        p.allow[1, 2, 20:40] = True
    check_verify(asd, p, off=off)
    check_verify(asd, p, off=off, strict=True)


def test_strict_equals_zero_budget(asd):
    p = Problem(BF16, 4, 8, 5000, seed=8)
    strict = asd.rules_verify(p.logits(), p.draft.cuda(), None, 1.0, 2, p.rules(asd), allow=p.mask())
    zero = asd.rules_verify(p.logits(), p.draft.cuda(), asd.make_ledger(4, 0.0), 1.0, 2, p.rules(asd), allow=p.mask())
    for name in ("accepted_len", "committed", "recovery", "row_argmax"):
        assert torch.equal(strict[name], zero[name])


def test_no_rules_equal_verify(asd):
    p = Problem(BF16, 6, 8, 9001, said=0, biased=0, grammar=None, seed=9)
    led = [asd.make_ledger(6, 8.0) for _ in range(2)]
    rules = asd.TokenRules.empty(6, 9001)
    a = asd.rules_verify(p.logits(), p.draft.cuda(), led[0], 1.0, 2, rules)
    b = asd.verify(p.logits(), p.draft.cuda(), led[1], 1.0, 2)
    for name in a:
        assert torch.equal(a[name], b[name]), name
    assert torch.equal(*led)


@pytest.mark.parametrize("dtype", (BF16, F32), ids=("bf16", "f32"))
@pytest.mark.parametrize("V,off", ((3001, 3), (4096, 0)))
def test_many_rows(asd, dtype, V, off):
    """Enough rows for the largest units: ordinary requests, nearly banned vocabularies, infinities and NaN side by side."""
    p = Problem(dtype, 170, 15, V, said=60, biased=9, grammar="third", seed=V + 1)
    g = torch.Generator().manual_seed(2)
    for b in range(0, 40):  # most tokens said and lowered, or banned
        p.marked[b] = torch.rand(V, generator=g) < (0.97, 0.5, 1.0, 1.0)[b % 4]
        p.seen[b] = torch.where(p.seen[b] == 0, torch.tensor(1, dtype=torch.int32), p.seen[b])
        p.bias[b] = (0.0, -80.0, 0.0, -math.inf)[b % 4]
        p.repetition[b], p.frequency[b], p.presence[b] = 1.3, 3.0, 9.0
    p.z[40:50, 2, 20:40] = math.inf
    p.allow[41:50, 2, 20:40] = True
    p.z[50:60, 3, 50], p.allow[50:60, 3, 50] = math.nan, False
    p.z[55, 4, 51], p.allow[55, 4, 51], p.marked[55, 51] = math.nan, True, False
    p.z[60:70, :, 60:90] = -math.inf
    p.bias[60:70, 60:64], p.marked[60:70, 60:64] = 2.0, True
    p.allow[70:80, 5] = False
    check_verify(asd, p, off=off, nan_rows=True)
    check_verify(asd, p, off=off, strict=True, nan_rows=True)
    check_logits(asd, p, off=off, to=(off * 3) % 8)
    check_logits(asd, p, off=off, to=off)
    p.allow = None
    p.z[50:60, 3, 50] = 0.0
    check_verify(asd, p, off=off, nan_rows=True)
    check_logits(asd, p, off=off, in_place=True)


@pytest.mark.parametrize("dtype", (BF16, F32), ids=("bf16", "f32"))
def test_infinities_and_nan(asd, dtype):
    p = Problem(dtype, 5, 3, 700, grammar="most", seed=11)
    p.allow[0] = False                                                 # a request without a token that may come
    p.allow[1, 2] = False                                              # a row without one
    p.z[2, :, 10:20], p.allow[2, :, 10:20] = math.nan, False           # NaN where the grammar allows nothing
    p.z[2, :, 30:40], p.allow[2, :, 30:40] = math.inf, False
    p.z[3, 1, 50], p.allow[3, 1, 50], p.marked[3, 50] = math.nan, True, False  # a NaN that counts
    p.draft[3, 0] = 51
    p.z[4, :, 60:90] = -math.inf
    p.bias[4, 60:64], p.marked[4, 60:64] = 2.0, True                   # -infinity stays
    p.bias[4, 100], p.bias[4, 101] = -math.inf, math.inf               # banned; forced
    p.marked[4, 100:102], p.allow[4, :, 100:102] = True, True
    check_verify(asd, p)
    check_logits(asd, p)
    got = asd.rules_verify(p.logits(), p.draft.cuda(), asd.make_ledger(5, 8.0), 1.0, 2, p.rules(asd), allow=p.mask())
    assert got["status"].tolist() == [0, 0, 0, asd.STATUS_NAN_LOGIT, 0]
    assert got["row_argmax"][0].tolist() == [0] * 4 and got["row_argmax"][4].tolist() == [101] * 4


def test_a_marked_nan_is_flagged(asd):
    p = Problem(F32, 2, 2, 300, grammar=None, seed=12)
    p.bias[1, 7], p.marked[1, 7] = math.nan, True
    check = asd.rules_verify(p.logits(), p.draft.cuda(), asd.make_ledger(2, 8.0), 1.0, 2, p.rules(asd))
    assert check["status"].tolist() == [0, asd.STATUS_NAN_LOGIT] and check["accepted_len"].tolist()[1] == 0
    assert same(asd.rules_logits(p.logits(), p.draft.cuda(), p.rules(asd)).cpu(), p.changed().float())


def test_drafts_out_of_range_count_for_nothing(asd):
    p = Problem(BF16, 3, 4, 1200, seed=13)
    p.draft[0, 1], p.draft[1, 0], p.draft[2, 3] = -1, 1200, 2 ** 31 - 1
    check_verify(asd, p)
    check_logits(asd, p)


def test_masks_with_strides(asd):
    p = Problem(BF16, 3, 4, 1000, grammar="third", seed=14)
    p.allow[:] = p.allow[:1, :1]
    one = ref.words_of(p.allow[:1, :1]).cuda().expand(3, 5, 32)
    want = p.changed().float().to(BF16)
    assert same(asd.rules_logits(p.logits(), p.draft.cuda(), p.rules(asd), allow=one).cpu(), want)
    wide = torch.zeros(5, 3, 40, dtype=torch.int32, device="cuda")
    view = wide.transpose(0, 1)[:, :, 3:35]
    view.copy_(one)
    assert same(asd.rules_logits(p.logits(), p.draft.cuda(), p.rules(asd), allow=view).cpu(), want)


def test_without_drafts_rows_see_the_text_only(asd):
    p = Problem(F32, 2, 3, 900, seed=15)
    got = asd.rules_logits(p.logits(), None, p.rules(asd), allow=p.mask())
    p.draft = torch.full((2, 3), -1, dtype=torch.int32)
    assert same(got.cpu(), p.changed().float())


# ---------------------------------------------------------------- token records

@pytest.mark.parametrize("n,V", ((300, 1001), (2048, 1001), (4097, 40000), (9000, 64)))
def test_tokens_record(asd, n, V):
    B = 5
    g = torch.Generator().manual_seed(n)
    rules = asd.TokenRules.empty(B, V)
    seen = torch.zeros(B, V, dtype=torch.int32)
    for call in range(3):
        tokens = torch.randint(-2, V if call else 4, (B, n), generator=g).to(torch.int32)
        length = torch.tensor([n, 0, 1, 77, n - 1], dtype=torch.int32) if call else None
        asd.tokens_record(tokens.cuda(), rules, prompt=call == 1, token_len=None if length is None else length.cuda())
        for b in range(B):
            for x in tokens[b, :n if length is None else int(length[b])].tolist():
                if x >= 0:
                    seen[b, x] = seen[b, x] | ref.PROMPT if call == 1 else seen[b, x] + 1
    assert torch.equal(rules.records[:, :, 0].cpu(), seen)
    assert int(rules.records[:, :, 1].count_nonzero()) == 0
    assert torch.equal(rules.marks.cpu(), ref.words_of(seen != 0))
    rules.clear(3)
    assert int(rules.records[3].count_nonzero()) == 0 and int(rules.marks[3].count_nonzero()) == 0
    assert torch.equal(rules.records[4, :, 0].cpu(), seen[4])


@pytest.mark.parametrize("n", (7, 5000))
def test_tokens_record_skips_what_is_out_of_range(asd, n):
    rules = asd.TokenRules.empty(3, 100)
    tokens = torch.arange(3 * n).view(3, n).to(torch.int32) % 130 - 10
    status = torch.zeros(3, dtype=torch.int32, device="cuda")
    length = torch.tensor([n, n + 1, n - 3], dtype=torch.int32)
    asd.tokens_record(tokens.cuda(), rules, token_len=length.cuda(), status=status)
    seen = torch.zeros(3, 100, dtype=torch.int32)
    want = [0, asd.STATUS_LENGTH, 0]
    for b in (0, 2):
        mine = tokens[b, :int(length[b])]
        want[b] = asd.STATUS_TOKEN if bool((mine >= 100).any()) else 0
        seen[b] = torch.bincount(mine[(mine >= 0) & (mine < 100)], minlength=100).int()
    assert status.tolist() == want and torch.equal(rules.records[:, :, 0].cpu(), seen)
    assert torch.equal(rules.marks.cpu(), ref.words_of(seen != 0))


def test_tokens_record_flags(asd):
    rules = asd.TokenRules.empty(4, 50)
    status = torch.zeros(4, dtype=torch.int32, device="cuda")
    tokens = torch.tensor([[1, 50], [2, 3], [4, 2 ** 31 - 1], [5, -7]], dtype=torch.int32).cuda()
    asd.tokens_record(tokens, rules, token_len=torch.tensor([2, 3, -1, 2], dtype=torch.int32).cuda(), status=status)
    assert status.tolist() == [asd.STATUS_TOKEN, asd.STATUS_LENGTH, asd.STATUS_LENGTH, 0]
    seen = rules.records[:, :, 0].cpu()
    assert [r.nonzero().flatten().tolist() for r in seen] == [[1], [], [], [5]]


@pytest.mark.parametrize("n", (1, 33, 1024))
def test_tokens_bias(asd, n):
    B, V = 3, 400
    g = torch.Generator().manual_seed(n)
    rules = asd.TokenRules.empty(B, V)
    ids = torch.randint(-1, V, (B, n), generator=g).to(torch.int32)
    value = torch.randn(B, n, generator=g)
    length = torch.tensor([n, n // 2, 0], dtype=torch.int32)
    for _ in range(2):
        asd.tokens_bias(ids.cuda(), value.cuda(), rules, length=length.cuda())
    want, marked = torch.zeros(B, V), torch.zeros(B, V, dtype=torch.bool)
    for b in range(B):
        for i in range(int(length[b])):
            if ids[b, i] >= 0:
                want[b, ids[b, i]], marked[b, ids[b, i]] = value[b, i], True
    assert torch.equal(rules.records[:, :, 1].cpu(), want.view(torch.int32))
    assert torch.equal(rules.marks.cpu(), ref.words_of(marked))
    status = torch.zeros(B, dtype=torch.int32, device="cuda")
    ids[1, 0] = V
    asd.tokens_bias(ids.cuda(), value.cuda(), rules, length=torch.tensor([n + 1, 1, 0]).int().cuda(), status=status)
    assert status.tolist() == [asd.STATUS_LENGTH, asd.STATUS_TOKEN, 0]


# ---------------------------------------------------------------- as they are used

def test_a_round_and_the_next(asd):
    """verify, commit, record: the second round's penalties know what the first one emitted."""
    B, K, V = 4, 6, 3000
    p = Problem(BF16, B, K, V, grammar=None, seed=20)
    rules = p.rules(asd)
    p.marked = p.marked.clone()
    for call in range(2):
        check = p.changed().float()
        led = asd.make_ledger(B, 6.0)
        want = oracle.verify(check.numpy(), p.draft.numpy(), led.cpu().numpy(), 1.0, 2)
        got = asd.rules_verify(p.logits(), p.draft.cuda(), led, 1.0, 2, rules)
        assert np.array_equal(got["committed"].cpu().numpy(), want["committed"])
        asd.tokens_record(got["committed"], rules)
        # the plain state: the same tokens said once more
        p.bias = torch.where(p.marked, p.bias, torch.zeros(()))
        p.seen = torch.where(p.marked, p.seen, torch.full((), 77, dtype=torch.int32))
        for b in range(B):
            for x in want["committed"][b]:
                if x >= 0:
                    if not p.marked[b, x]:  # rules() fills what has no mark with junk, which then counts
                        p.bias[b, x] = 1000.0
                    p.seen[b, x] += 1
                    p.marked[b, x] = True


def test_captured_and_replayed(asd):
    p = Problem(BF16, 3, 5, 7000, seed=21)
    rules, mask, draft, z = p.rules(asd), p.mask(), p.draft.cuda(), p.logits()
    led = asd.make_ledger(3, 8.0)
    ws = asd.Workspace(3, 5, 7000, asd.BF16)
    out, to = asd.alloc_outputs(3, 5), torch.empty_like(z)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        asd.rules_verify(z, draft, led, 1.0, 2, rules, allow=mask, workspace=ws, out=out)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        asd.rules_verify(z, draft, led, 1.0, 2, rules, allow=mask, workspace=ws, out=out)
        asd.rules_logits(z, draft, rules, allow=mask, out=to)
        asd.tokens_record(out["committed"], rules)
    other = Problem(BF16, 3, 5, 7000, seed=22)
    for q in (p, other, p):
        fresh = q.rules(asd)
        rules.marks.copy_(fresh.marks), rules.records.copy_(fresh.records)
        for name in ("repetition", "frequency", "presence"):
            getattr(rules, name).copy_(getattr(fresh, name))
        z.copy_(q.z), draft.copy_(q.draft), mask.copy_(q.mask())
        led.copy_(asd.make_ledger(3, 8.0))
        graph.replay()
        torch.cuda.synchronize()
        want = oracle.verify(q.changed().float().numpy(), q.draft.numpy(), asd.make_ledger(3, 8.0).cpu().numpy(), 1.0, 2)
        for name in ("accepted_len", "committed", "recovery", "row_argmax"):
            assert np.array_equal(out[name].cpu().numpy(), want[name]), name
        assert same(to.cpu(), q.changed().float().to(BF16))


def test_on_streams_at_once(asd):
    """Two calls, each with rules and a workspace of its own, on two streams, outputs allocated by the call."""
    ps = [Problem(BF16, 8, 8, 20000, seed=s) for s in (30, 31)]
    args = [(p.logits(), p.draft.cuda(), asd.make_ledger(8, 8.0), 1.0, 2, p.rules(asd), p.mask()) for p in ps]
    streams = [torch.cuda.Stream() for _ in ps]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for i, (a, s) in enumerate(zip(args, streams)):
            a[2][:, 1] = 0.0
            s.wait_stream(torch.cuda.current_stream())
            got[i].append(asd.rules_verify(*a[:6], allow=a[6], stream=s))
            torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    for p, outs in zip(ps, got):
        want = oracle.verify(p.changed().float().numpy(), p.draft.numpy(), asd.make_ledger(8, 8.0).cpu().numpy(), 1.0, 2)
        for o in outs:
            assert np.array_equal(o["committed"].cpu().numpy(), want["committed"])


def test_records_past_2_31_bytes(asd):
    """Rows and records whose offsets do not fit 32 bits: the last request's are right."""
    B, V = 2200, 151936  # 2.7 GB of records, 0.67 GB of logits
    rules = asd.TokenRules.empty(B, V, presence=torch.full((B,), 2.0, device="cuda"))
    z = torch.zeros(B, 1, V, dtype=BF16, device="cuda")
    z[:, 0, V - 1], z[:, 0, V - 2] = 3.0, 2.0
    asd.tokens_record(torch.full((B, 1), V - 1, dtype=torch.int32, device="cuda"), rules)
    draft = torch.empty(B, 0, dtype=torch.int32, device="cuda")
    got = asd.rules_verify(z, draft, None, 1.0, 2, rules)
    assert bool((got["recovery"] == V - 2).all())
    out = asd.rules_logits(z, None, rules)
    assert out[-1, 0, V - 2:].tolist() == [2.0, 1.0] and out[0, 0, V - 2:].tolist() == [2.0, 1.0]
