"""What a list of biases leaves of the lists before it."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


def test_unlisted_biases_stay(asd):
    """asd_tokens_bias writes the ids that it is given; a caller resets the others with 0, or the request as a whole."""
    V = 100
    rules = asd.TokenRules.empty(2, V)

    def bias(ids, values):
        asd.tokens_bias(torch.tensor([ids, ids], dtype=torch.int32).cuda(), torch.tensor([values, values]).cuda(), rules)

    def logits():
        return asd.rules_logits(torch.ones(2, 1, V, device="cuda"), None, rules)[:, 0].cpu()
    want = torch.ones(2, V)
    bias([3, 64, 99], [2.0, -math.inf, 0.5])
    want[:, [3, 64, 99]] = torch.tensor([3.0, -math.inf, 1.5])
    assert torch.equal(logits(), want)
    bias([7, 3], [1.0, -1.0])  # another list: 64 stays banned
    want[:, [7, 3]] = torch.tensor([2.0, 0.0])
    assert torch.equal(logits(), want)
    bias([64, 99], [0.0, 0.0])
    want[:, [64, 99]] = 1.0
    assert torch.equal(logits(), want)
    rules.clear(0)
    want[0] = 1.0
    assert torch.equal(logits(), want)
