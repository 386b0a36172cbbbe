"""Rows whose lse is finite but whose lse in log2 units is not: their weights are 0, or infinite, as the formula says."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,D", [(torch.float32, 64), (torch.bfloat16, 64), (torch.float16, 20)],
                         ids=("f32", "tensor cores", "16-bit on the CUDA cores"))
@pytest.mark.parametrize("T", (3, 60))
def test_lse_near_the_largest(asd, dtype, D, T):
    g = torch.Generator().manual_seed(T)
    k = torch.randn(1, 10, 16, 2, D, generator=g).to(dtype).cuda()
    cache = asd.KVCache(k, k, torch.arange(10, dtype=torch.int32, device="cuda")[None])
    q = torch.randn(1, T, 4, D, generator=g).to(dtype).cuda()
    kv_len = torch.full((1,), 90, dtype=torch.int32, device="cuda")

    def weigh(lse):
        out = torch.full((1, 2, 160), 7.0, device="cuda")
        return asd.kv_weigh(q, lse.cuda(), cache, kv_len, None, decay=0.0, out=out).cpu()
    lse = torch.full((1, T, 4), 4.0)
    without = lse.clone()
    without[0, 1, :] = math.inf  # adds nothing
    want = weigh(without)
    for value in (2.4e38, 3.4e38):
        lse[0, 1, :] = value
        assert torch.equal(weigh(lse), want)
    lse[0, 1, 2:] = -3e38  # the second key/value head's
    got = weigh(lse)
    assert torch.equal(got[:, 0], want[:, 0])
    assert bool((got[0, 1, :92] == math.inf).all()) and torch.equal(got[0, 1, 92:], want[0, 1, 92:])
