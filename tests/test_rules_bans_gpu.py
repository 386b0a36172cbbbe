"""What may not come is not committed: drafts that the grammar or a bias of -infinity bans, whatever gate and budget are,
and rows in which no token may come."""
import math

import pytest
import torch

import rules_reference as ref

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
ANY_GATE = dict(gate=math.inf, cap=2 ** 31 - 1)


class Problem:
    """Drafts of which about every third is banned; each row's best token is one that may come."""

    def __init__(self, dtype, B, K, V, how, seed=0):
        g = torch.Generator().manual_seed(seed)
        self.B, self.K, self.V, self.dtype = B, K, V, dtype
        self.z = torch.randn(B, K + 1, V, generator=g).to(dtype)
        self.draft = torch.randint(V, (B, K), generator=g).to(torch.int32)
        self.may = torch.ones(B, K + 1, V, dtype=torch.bool)
        ban = torch.rand(B, K, generator=g) < 0.35
        for b in range(B):
            for j in range(K):
                if ban[b, j]:  # a bias bans a token in every row
                    self.may[b, slice(None) if how == "bias" else j, self.draft[b, j]] = False
        self.rule = how

    def verify(self, asd, ledger, gate, cap, **kw):
        rules = asd.TokenRules.empty(self.B, self.V)
        allow = None
        if self.rule == "bias":
            banned = ~self.may[:, 0]
            rules.marks.copy_(ref.words_of(banned))
            bias = torch.zeros(self.B, self.V).masked_fill(banned, -math.inf)
            rules.records[:, :, 1] = bias.view(torch.int32).cuda()
        else:
            allow = ref.words_of(self.may).cuda()
        return asd.rules_verify(self.z.cuda(), self.draft.cuda(), ledger, gate, cap, rules, allow=allow, **kw)

    def nothing_banned(self, committed):
        for b in range(self.B):
            for j, x in enumerate(committed[b].tolist()):
                assert x == -1 or bool(self.may[b, j, x]), (b, j, x)


@pytest.mark.parametrize("how", ("grammar", "bias"))
@pytest.mark.parametrize("dtype", (BF16, F32), ids=("bf16", "f32"))
@pytest.mark.parametrize("B,K,V", ((20, 1, 40), (40, 8, 300), (3, 31, 2500), (2, 6, 20000)))
def test_banned_drafts_under_an_infinite_gate_and_budget(asd, dtype, how, B, K, V):
    """Everything that may come is accepted, up to the first draft that may not."""
    p = Problem(dtype, B, K, V, how, seed=V)
    led = asd.make_ledger(B, math.inf)
    got = p.verify(asd, led, **ANY_GATE)
    barred = ~p.may[:, :K].gather(2, p.draft[:, :, None].long())[:, :, 0]
    want = [row.index(True) if True in row else K for row in barred.tolist()]
    assert any(a < K for a in want) and any(a > 0 for a in want)
    assert got["accepted_len"].tolist() == want and not got["status"].any()
    p.nothing_banned(got["committed"])
    assert bool(led[:, 1].isfinite().all())
    changed = p.z.float().masked_fill(~p.may, -math.inf)
    top = changed.amax(-1)
    for b, a in enumerate(want):
        assert got["recovery"].tolist()[b] == int(changed[b, a].argmax())
        spent = torch.zeros(())
        for j in range(a):  # Eq. 8 and 13 in fp32; matches add nothing
            spent = spent + (top[b, j] - changed[b, j, p.draft[b, j]])
        assert float(led[b, 1]) == float(spent)
    r = got["row_regret"].cpu()
    assert torch.equal(r.isinf(), barred)


@pytest.mark.parametrize("budget", (None, 0.0, 5.0, math.inf), ids=("strict", "0", "5", "inf"))
@pytest.mark.parametrize("how", ("grammar", "bias"))
def test_no_ledger_relaxes_a_ban(asd, how, budget):
    p = Problem(F32, 60, 5, 200, how, seed=3)
    for b in range(0, 60, 2):  # drafts near the top, so that some are accepted
        for j in range(5):
            p.z[b, j, p.draft[b, j]] = 9.0
    led = None if budget is None else asd.make_ledger(60, budget)
    got = p.verify(asd, led, **ANY_GATE)
    p.nothing_banned(got["committed"])
    assert int(got["accepted_len"].max()) > 0 and not got["status"].any()


@pytest.mark.parametrize("how", ("grammar", "bias"))
@pytest.mark.parametrize("mode", ("strict", "budget", "anything"))
def test_a_row_without_tokens(asd, how, mode):
    """y* is 0 there, which a draft of 0 does not match; the status tells where that row's token was to be emitted."""
    B, K, V = 5, 4, 100
    p = Problem(F32, B, K, V, how, seed=4)
    p.may[:] = True
    p.draft[:] = p.z[:, :K].argmax(-1)
    empty = [0, 2, K, 3, None]  # the row without tokens, of each request
    for b, row in enumerate(empty):
        if row is None:
            continue
        if how == "bias":  # a bias bans in all rows
            p.may[b] = False
        else:
            p.may[b, row] = False
        if row < K:
            p.draft[b, row] = 0
    p.draft[3, 1] = (p.draft[3, 1] + 1) % V  # ends before its empty row, but where anything goes
    args = {"strict": (None, 1.0, 2), "budget": (asd.make_ledger(B, 1e-6), 1.0, 2),
            "anything": (asd.make_ledger(B, math.inf), math.inf, 9)}[mode]
    reach = [0, 2, K, 3 if mode == "anything" else 1, K] if how == "grammar" else [0, 0, 0, 0, K]
    got = p.verify(asd, *args, flag_empty=True)
    assert got["accepted_len"].tolist() == reach
    meets = [how == "bias" and row is not None or row == a for row, a in zip(empty, reach)]
    assert got["status"].tolist() == [asd.STATUS_EMPTY_ROW if x else 0 for x in meets]
    assert [got["recovery"].tolist()[b] for b in range(B) if meets[b]] == [0] * sum(meets)
    for b, a in enumerate(reach):
        assert got["committed"][b, :a].tolist() == p.draft[b, :a].tolist()
    if args[0] is not None:
        assert bool(args[0][:, 1].isfinite().all())
    plain = p.verify(asd, None if args[0] is None else asd.make_ledger(B, float(args[0][0, 0])), *args[1:])
    assert not plain["status"].any()
    for name in ("accepted_len", "committed", "recovery", "row_argmax"):
        assert torch.equal(plain[name], got[name])


def test_the_flag_changes_nothing_else(asd):
    p = Problem(BF16, 30, 6, 700, "grammar", seed=5)
    a, b = (p.verify(asd, asd.make_ledger(30, 8.0), 1.0, 2, flag_empty=f) for f in (False, True))
    for name in a:
        assert torch.equal(a[name].view(torch.int32), b[name].view(torch.int32)), name
