"""asd_kv_evict_numbered on the host: refusals before any CUDA call (no GPU needed)."""
import ctypes
import types

import pytest
import torch

from paper_2608_03447_gb300 import asd

NULL, SHAPE, ALIGN = 1, 2, 6


def evict(number=0x6000, tokens=0x7000, cache=None, **kw):
    c = dict(k=0x10000, v=0x20000, dtype=asd.BF16, layers=2, pages=4, page_size=16, heads=2, head_dim=64,
             layer_stride=4 * 2048, page_stride=2048, token_stride=128, head_stride=64, page_table=0x30000, B=3,
             table_width=2)
    c.update(cache or {})
    c = asd._Cache(*[c[n] for n, _ in asd._Cache._fields_])
    a = dict(w=0x1000, out=0x1000, kv_len=0x2000, new=0x3000, keep=0x4000, status=0, first=0, last=0, width=32,
             reserved=0)
    a.update(kw)
    return asd.load().asd_kv_evict_numbered(ctypes.addressof(c), asd._EVICT.pack(*a.values()), number, tokens, None)


@pytest.mark.parametrize("kw,code", [(dict(number=None), NULL), (dict(tokens=None), NULL), (dict(new=0x7000), SHAPE),
                                     (dict(number=0x6002), ALIGN), (dict(tokens=0x7001), ALIGN), (dict(w=0), NULL),
                                     (dict(first=-1), SHAPE), (dict(reserved=1), SHAPE), (dict(new=0x2000), SHAPE)],
                         ids=str)
def test_bad_arguments(kw, code):
    assert evict(**kw) == code


def test_nothing():
    assert evict(number=None, tokens=None, cache=dict(B=0)) == 0
    assert asd.load().asd_kv_evict_numbered(None, None, None, None, None) == NULL


def test_the_binding_checks_its_tensors(monkeypatch):
    calls = []
    lib = types.SimpleNamespace(asd_kv_evict=lambda *a: calls.append("plain") or 0,
                                asd_kv_evict_numbered=lambda *a: calls.append("numbered") or 0)
    monkeypatch.setattr(asd, "load", lambda: lib)
    c = asd.KVCache.__new__(asd.KVCache)
    c.k = c.v = torch.ones(1, 4, 16, 2, 8)
    c.dtype, c.device, c.index, c.layers, c.B, c.heads, c.head_dim, c._ref = torch.float32, c.k.device, -1, 1, 2, 2, 8, 0
    stream = types.SimpleNamespace(cuda_stream=0x5eed)

    def i32(*shape):
        return torch.ones(*shape, dtype=torch.int32)

    def call(**kw):
        asd.kv_evict(c, i32(2), torch.ones(2, 2, 30), i32(2), new_len=i32(2), stream=stream, **kw)
    call()
    call(numbers=i32(2, 2, 30), tokens=i32(2))
    assert calls == ["plain", "numbered"]
    for kw in (dict(numbers=i32(2, 2, 30)), dict(tokens=i32(2)), dict(numbers=i32(2, 2, 29), tokens=i32(2)),
               dict(numbers=i32(2, 2, 30).long(), tokens=i32(2)), dict(numbers=i32(2, 2, 30), tokens=i32(3)),
               dict(numbers=torch.ones(2, 2, 30), tokens=i32(2)), dict(numbers=i32(2, 2, 60)[..., ::2], tokens=i32(2))):
        with pytest.raises(ValueError):
            call(**kw)
    assert calls == ["plain", "numbered"]
