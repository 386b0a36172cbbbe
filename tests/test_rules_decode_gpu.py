"""The decoding example under rules and with a limit on its cache: every operator of a round, as they are used together."""
import importlib.util
import os

import pytest
import torch

import rules_reference as ref

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROMPTS = [[1, 2, 3, 4, 5], [7], [11, 13, 17, 19, 23, 29, 31, 37, 41]]


@pytest.fixture(scope="module")
def example(asd):
    spec = importlib.util.spec_from_file_location("tree_decode", os.path.join(ROOT, "examples", "tree_decode.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16), ids=("f32", "bf16"))
def test_a_large_presence_penalty_repeats_nothing(example, dtype):
    """Every row counts what was emitted and the drafts before it, so no token comes twice, accepted drafts included."""
    m = example.Decoder(dtype)
    out, rate = example.decode(m, PROMPTS, 14, presence=1e4)
    assert all(len(set(t)) == len(t) >= 14 for t in out)
    plain, _ = example.decode(m, PROMPTS, 14)
    assert any(len(set(t)) < len(t) for t in plain), "the model has to repeat itself for this to say anything"


def test_without_a_penalty_rules_change_nothing(example):
    m = example.Decoder(torch.float32)
    assert example.decode(m, PROMPTS, 10, presence=0.0) == example.decode(m, PROMPTS, 10)


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16), ids=("f32", "bf16"))
def test_a_cache_within_its_limit_is_not_touched(example, dtype):
    m = example.Decoder(dtype)
    assert example.decode(m, PROMPTS, 10, keep=1000) == example.decode(m, PROMPTS, 10)


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16), ids=("f32", "bf16"))
def test_a_limited_cache(example, dtype):
    """The cache stays at its limit; what is emitted before the limit is reached stays the same."""
    m, seen = example.Decoder(dtype), []
    out, _ = example.decode(m, PROMPTS, 20, keep=16, lengths_seen=seen)
    free, _ = example.decode(m, PROMPTS, 20)
    assert max(map(max, seen)) == 16 and all(len(t) >= 20 for t in out)
    for b, prompt in enumerate(PROMPTS):
        until = next(i for i, n in enumerate(seen) if n[b] == 16)  # a token a round at least
        assert out[b][:until] == free[b][:until]


def test_a_round_by_hand(asd):
    """append, attend, verify under rules, compact, weigh, commit, record, evict of one layer, each checked by its plain
    form on what the ones before it left."""
    dtype, B, K, heads, G, D, page, V = torch.float32, 2, 3, 2, 2, 16, 8, 60
    g = torch.Generator().manual_seed(5)
    table = torch.randperm(12, generator=g).to(torch.int32).view(B, 6)
    k0, v0 = torch.randn(2, 1, 12, page, heads, D, generator=g)
    kv = torch.tensor([30, 21], dtype=torch.int32)
    k, v = k0.cuda(), v0.cuda()
    cache = asd.KVCache(k, v, table.cuda())
    new_k, new_v, q = (torch.randn(B, K + 1, n, D, generator=g) for n in (heads, heads, heads * G))
    asd.kv_append(new_k.cuda(), new_v.cuda(), cache, kv.cuda())
    got = asd.tree_attention(q.cuda(), cache, kv.cuda())
    rules = asd.TokenRules.empty(B, V, presence=torch.tensor([0.5, 9.0]).cuda())
    said = torch.randint(V, (B, 9), generator=g).to(torch.int32)
    asd.tokens_record(said.cuda(), rules)
    z = 2 * torch.randn(B, K + 1, V, generator=g)
    draft = z[:, :K].argmax(-1).to(torch.int32)
    seen = torch.zeros(B, V, dtype=torch.int32)
    for b in range(B):
        seen[b] += torch.bincount(said[b], minlength=V).int()
    block = asd.rules_verify(z.cuda(), draft.cuda(), asd.make_ledger(B, 3.0), 1.0, 2, rules)
    from oracle import oracle
    changed = torch.stack([ref.changed(z[b], draft[b].tolist(), seen[b] != 0, seen[b], torch.zeros(V), None, None,
                                       [0.5, 9.0][b], None) for b in range(B)])
    want = oracle.verify(changed.float().numpy(), draft.numpy(), [[3.0, 0.0]] * B, 1.0, 2)
    accepted = block["accepted_len"].cpu()
    assert accepted.tolist() == want["accepted_len"].tolist()
    path = torch.arange(K + 1, dtype=torch.int32).expand(B, -1).contiguous()
    asd.kv_compact(cache, kv.cuda(), path.cuda(), (accepted + 1).cuda())
    weight = torch.rand(1, B, heads, 48, generator=g)
    w = weight.cuda()
    asd.kv_weigh(q.cuda(), got["lse"], cache, kv.cuda(), w[0], path=path.cuda(), new_len=(accepted + 1).cuda())
    exact, tol = ref.weighed(q, got["lse"].cpu(), k.cpu()[0], table, kv, accepted + 1, path, D ** -0.5, 1.0, weight[0])
    written = ~exact.isnan()
    assert bool(((w[0].cpu().double() - exact).abs() <= tol)[written].all())
    length = kv.cuda()
    asd.commit(block["accepted_len"], block["committed"], kv_len=length)
    asd.tokens_record(block["committed"], rules)
    for b in range(B):
        tokens = [t for t in want["committed"][b] if t >= 0]
        seen[b] += torch.bincount(torch.tensor(tokens), minlength=V).int()
    assert torch.equal(rules.records[:, :, 0].cpu(), seen) and torch.equal(rules.marks.cpu(), ref.words_of(seen != 0))
    before = k.cpu(), v.cpu(), w.cpu()
    keep = torch.full((B,), 15, dtype=torch.int32)
    new = asd.kv_evict(cache, length, w, keep.cuda(), first=2, last=4)
    ek, ev, ew, en = ref.evicted(*before[:2], table, length.cpu(), before[2], keep, 2, 4)
    assert torch.equal(new.cpu(), en) and torch.equal(k.cpu(), ek) and torch.equal(v.cpu(), ev) and torch.equal(w.cpu(), ew)
