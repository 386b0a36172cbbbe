"""``stream=`` with torch's current stream elsewhere: results are as on one stream, whatever the current one does."""
import pytest
import torch

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
SLEEP = 20_000_000  # cycles, some ten milliseconds: long after every call of a test has been queued


def inputs(asd, dtype, B=3, T=5, Hq=8, Hkv=2, D=64, page=16, ctx=200):
    g = torch.Generator(device="cuda").manual_seed(1)
    width = -(-(ctx + T) // page)
    shape = (B * width, page, Hkv, D)
    k, v = (torch.randn(shape, generator=g, device="cuda").to(dtype) for _ in range(2))
    table = torch.randperm(B * width, generator=g, device="cuda").to(torch.int32).view(B, width)
    cache = asd.KVCache(k, v, table)
    q, kn, vn = (torch.randn(B, T, n, D, generator=g, device="cuda").to(dtype) for n in (Hq, Hkv, Hkv))
    kv_len = torch.tensor([ctx, 0, 77], dtype=torch.int32, device="cuda")
    w = torch.ones(D, dtype=dtype, device="cuda")
    return cache, q, kn, vn, kv_len, w


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("handle", [False, True], ids=["Stream", "int"])
def test_queries_appended_on_another_stream_stay(asd, dtype, handle):
    """The current stream is busy when the call is made: nothing of the call may wait there and run afterwards."""
    cache, q, kn, vn, kv_len, w = inputs(asd, dtype)
    want = asd.kv_append(kn, vn, cache, kv_len, q=q, q_norm=w, k_norm=w)
    want_k, want_v = cache.k.clone(), cache.v.clone()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(SLEEP)
    got = asd.kv_append(kn, vn, cache, kv_len, q=q, q_norm=w, k_norm=w, stream=side.cuda_stream if handle else side)
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.equal(cache.k, want_k) and torch.equal(cache.v, want_v)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("handle", [False, True], ids=["Stream", "int"])
def test_a_dropped_workspace_is_not_handed_out_before_the_call_has_run(asd, dtype, handle):
    cache, q, _, _, kv_len, _ = inputs(asd, dtype)
    want = asd.tree_attention(q, cache, kv_len)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(SLEEP)
    got = asd.tree_attention(q, cache, kv_len, stream=side.cuda_stream if handle else side)
    # on the current stream, before the call runs: whatever the allocator has, filled
    size = asd.attention_workspace(cache, q.shape[1], q.shape[2]).nbytes
    taken = [torch.full((size,), 255, dtype=torch.uint8, device="cuda") for _ in range(4)]
    torch.cuda.synchronize()
    assert torch.equal(got["out"], want["out"]) and torch.equal(got["lse"], want["lse"])
    assert all(bool((t == 255).all()) for t in taken)


def test_two_streams_with_a_workspace_each(asd):
    """Calls of both dtypes on two streams at once, over the same cache: each as on its own."""
    for dtype in (BF16, F32):
        cache, q, _, _, kv_len, _ = inputs(asd, dtype, T=9, ctx=1500)
        other = (q.flip(1).contiguous(), kv_len.flip(0).contiguous())
        want = [asd.tree_attention(q, cache, kv_len), asd.tree_attention(other[0], cache, other[1])]
        streams = [torch.cuda.Stream() for _ in range(2)]
        ws = [asd.attention_workspace(cache, 9, 8) for _ in range(2)]
        torch.cuda.synchronize()
        got = [[], []]
        for _ in range(20):
            for i, (x, n) in enumerate(((q, kv_len), other)):
                got[i].append(asd.tree_attention(x, cache, n, workspace=ws[i], stream=streams[i]))
        torch.cuda.synchronize()
        for i in range(2):
            assert ws[i].error() == 0
            for o in got[i]:
                assert torch.equal(o["out"], want[i]["out"]) and torch.equal(o["lse"], want[i]["lse"])


def test_verification_on_another_stream(asd):
    """Outputs, workspace, counts and host copies of calls on a side stream that is behind the current one."""
    B, K, V = 4, 5, 5003
    g = torch.Generator(device="cuda").manual_seed(2)
    z = torch.randn(B, K + 1, V, generator=g, device="cuda")
    x = z[:, :K].argmax(-1).to(torch.int32)
    x[:, 2] = 7
    ledger = asd.make_ledger(B, 100.0)
    want = asd.verify(z, x, ledger.clone(), 100.0, 2)
    counts = asd.opportunity(want["row_argmax"], x, want["row_regret"], [0.5, 100.0], [1, 2])
    side = torch.cuda.Stream()
    zh, xh = z.cpu().pin_memory(), x.cpu().pin_memory()
    ws, out = asd.Workspace(B, K, V, asd.F32), asd.alloc_outputs(B, K)
    host = {n: torch.zeros_like(out[n], device="cpu").pin_memory() for n in ("accepted_len", "committed", "recovery")}
    ledgers = [ledger.clone(), ledger.clone()]
    torch.cuda.synchronize()
    torch.cuda._sleep(SLEEP)
    seen = asd.opportunity(want["row_argmax"], x, want["row_regret"], [0.5, 100.0], [1, 2], stream=side)
    with torch.cuda.stream(side):
        torch.cuda._sleep(SLEEP)
    got = asd.verify(z, x, ledgers[0], 100.0, 2, stream=side)
    taken = [torch.full((ws.nbytes,), 255, dtype=torch.uint8, device="cuda") for _ in range(4)]
    asd.verify_from_host(zh, xh, ledgers[1], 100.0, 2, ws, out, host, stream=side)
    side.synchronize()
    for n in host:
        assert torch.equal(host[n], want[n].cpu()), n
    torch.cuda.synchronize()
    for n in want:
        assert torch.equal(got[n], want[n]), n
    assert torch.equal(seen, counts) and int(counts[-1]) > 0
    assert all(bool((t == 255).all()) for t in taken)
