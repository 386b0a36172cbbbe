"""The decoding example: cache operators, verification and commit together, against plain decoding in 64 bits."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example(asd):
    spec = importlib.util.spec_from_file_location("tree_decode", os.path.join(ROOT, "examples", "tree_decode.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def plain_logits(m, tokens):
    """The model over one whole sequence, no cache, in 64 bits: [T, V]."""
    def w(t):
        return t.double().cpu()

    def norm(t):
        return t * torch.rsqrt(t.square().mean(-1, keepdim=True) + 1e-6)

    def turn(t, weight):  # [T, heads, D]
        t = norm(t) * w(weight)
        c, s = w(m.cos)[:len(tokens), None], w(m.sin)[:len(tokens), None]
        a, b = t.chunk(2, -1)
        return torch.cat((a * c - b * s, b * c + a * s), -1)

    T, G = len(tokens), m.q_heads // m.heads
    x = w(m.embed)[tokens]
    for i in range(m.layers):
        q, k, v = (norm(x) @ w(m.qkv[i]).T).view(T, -1, m.D).split((m.q_heads, m.heads, m.heads), 1)
        q, k = turn(q, m.q_norm[i]), turn(k, m.k_norm[i])
        k, v = k.repeat_interleave(G, 1), v.repeat_interleave(G, 1)
        s = torch.einsum("qhd,khd->hqk", q, k) * m.D ** -0.5
        s = s.masked_fill(torch.ones(T, T).triu(1).bool(), -float("inf"))
        x = x + torch.einsum("hqk,khd->qhd", s.softmax(-1), v).reshape(T, -1) @ w(m.out[i]).T
        x = x + torch.relu(norm(x) @ w(m.up[i]).T) @ w(m.down[i]).T
    return norm(x) @ w(m.head).T


PROMPTS = [[1, 2, 3, 4, 5], [7], [11, 13, 17, 19, 23, 29, 31, 37, 41]]


@pytest.mark.parametrize("seed", [0, 1])
def test_without_a_budget_it_is_greedy_decoding(example, seed):
    """A budget of zero emits the target's own greedy tokens, whatever the drafts: each emitted token is the argmax
    after those before it, up to what 32 bits may be off (1e-3 on logits of a few units)."""
    m = example.Decoder(torch.float32, seed=seed)
    out, rate = example.decode(m, PROMPTS, 10)
    assert rate > 0.2, "the drafts have to be accepted now and then, or no path is ever moved"
    for prompt, tokens in zip(PROMPTS, out):
        z = plain_logits(m, prompt + tokens)[len(prompt) - 1:-1]
        assert len(tokens) >= 10 and len(z) == len(tokens)
        chosen = z.gather(1, torch.tensor(tokens)[:, None])[:, 0]
        assert bool((chosen >= z.max(1).values - 1e-3).all())


def test_a_budget_accepts_more_and_spends_no_more(example):
    m = example.Decoder(torch.bfloat16)
    strict, strict_rate = example.decode(m, PROMPTS, 12)
    loose, loose_rate = example.decode(m, PROMPTS, 12, budget=1000.0, gate=1000.0, cap=4)
    assert loose_rate == 4.0  # every draft fits the budget
    assert strict_rate < loose_rate and all(len(t) == 12 * 5 for t in loose)
