"""The entry points for rules, weights and evictions on the host: refusals before any CUDA call, and the binding's own
checks (no GPU needed)."""
import contextlib
import ctypes
import math
import types

import pytest
import torch

from paper_2608_03447_gb300 import asd

STREAM = types.SimpleNamespace(cuda_stream=0x5eed)
NULL, SHAPE, DTYPE, CONTROL, WORKSPACE, ALIGN = 1, 2, 3, 4, 5, 6


@pytest.fixture(scope="module")
def lib():
    return asd.load()


def cache(**kw):
    a = dict(k=0x10000, v=0x20000, dtype=asd.BF16, layers=2, pages=4, page_size=16, heads=2, head_dim=64,
             layer_stride=4 * 2048, page_stride=2048, token_stride=128, head_stride=64, page_table=0x30000, B=3,
             table_width=2)
    a.update(kw)
    return asd._Cache(*[a[n] for n, _ in asd._Cache._fields_])


def rules(**kw):
    a = dict(marks=0x1000, records=0x2000, repetition=0, frequency=0, presence=0, allow=0, batch=0, row=0, B=2, V=100)
    a.update(kw)
    return asd._RULES.pack(*a.values())


def verify(lib, r, **kw):
    a = dict(logits=0x4000, draft=0x5000, ledger=0x6000, a=0x7000, c=0x7100, rec=0x7200, arg=0, reg=0, status=0,
             ws=0x10000, wsb=1 << 30, dtype=asd.BF16, K=3, gate=1.0, cap=2)
    a.update({n: 0 if x is None else x for n, x in kw.items()})
    return lib.asd_rules_verify(r, asd._RULES_BLOCK.pack(*a.values()), None)


BAD_RULES = [(dict(marks=0), NULL), (dict(records=0), NULL), (dict(B=-1), SHAPE), (dict(V=0), SHAPE),
             (dict(batch=-1), SHAPE), (dict(row=-4), SHAPE), (dict(marks=0x1002), ALIGN), (dict(records=0x2004), ALIGN),
             (dict(allow=0x11), ALIGN), (dict(repetition=0x12), ALIGN), (dict(frequency=0x13), ALIGN),
             (dict(presence=0x11), ALIGN)]


@pytest.mark.parametrize("kw,code", BAD_RULES, ids=[str(k) for k, _ in BAD_RULES])
def test_bad_rules(lib, kw, code):
    r = rules(**kw)
    assert verify(lib, r) == code
    assert lib.asd_rules_logits(r, 0x4000, asd.F32, 4, None, 0x8000, None) == code
    assert lib.asd_tokens_record(r, 0x4000, 5, None, 0, None, None) == code
    assert lib.asd_tokens_bias(r, 0x4000, 0x5000, 5, None, None, None) == code


def test_no_rules(lib):
    assert verify(lib, None) == NULL and lib.asd_rules_verify(rules(), None, None) == NULL
    assert lib.asd_rules_logits(None, 0x4000, asd.F32, 4, None, 0x8000, None) == NULL
    assert lib.asd_tokens_record(None, 0x4000, 5, None, 0, None, None) == NULL
    assert lib.asd_tokens_bias(None, 0x4000, 0x5000, 5, None, None, None) == NULL


BAD_VERIFY = [(dict(dtype=asd.F16), DTYPE), (dict(dtype=asd.BF16 | asd.RESIDENT_INPUTS), DTYPE), (dict(K=-1), SHAPE),
              (dict(K=32), SHAPE), (dict(logits=None), NULL), (dict(draft=None), NULL), (dict(a=None), NULL),
              (dict(c=None), NULL), (dict(rec=None), NULL), (dict(ws=None), NULL), (dict(gate=-1.0), CONTROL),
              (dict(gate=math.nan), CONTROL), (dict(cap=-1), CONTROL), (dict(wsb=100), WORKSPACE),
              (dict(ws=0x10008), ALIGN), (dict(logits=0x4001), ALIGN), (dict(dtype=asd.F32, logits=0x4002), ALIGN)]


@pytest.mark.parametrize("kw,code", BAD_VERIFY, ids=[str(k) for k, _ in BAD_VERIFY])
def test_bad_verify_arguments(lib, kw, code):
    assert verify(lib, rules(), **kw) == code
    if code == CONTROL:  # strict verification has no controls
        assert verify(lib, rules(B=0), ledger=None, **kw) == 0


def test_bad_logits_arguments(lib):
    r = rules()

    def call(z=0x4000, dtype=asd.F32, rows=4, out=0x8000, r=r):
        return lib.asd_rules_logits(r, z, dtype, rows, None, out, None)
    assert call(dtype=asd.F16) == DTYPE and call(rows=0) == SHAPE and call(rows=33) == SHAPE
    assert call(z=None) == NULL and call(out=None) == NULL
    assert call(z=0x4002) == ALIGN and call(out=0x8002) == ALIGN and call(out=0x8001, dtype=asd.BF16) == ALIGN
    assert call(r=rules(B=2 ** 24, V=2 ** 31 - 1)) == SHAPE  # more ranges than a grid has CTAs


def test_bad_token_arguments(lib):
    r = rules()
    assert lib.asd_tokens_record(r, None, 5, None, 0, None, None) == NULL
    assert lib.asd_tokens_record(r, 0x4000, -1, None, 0, None, None) == SHAPE
    assert lib.asd_tokens_record(r, None, 0, None, 0, None, None) == 0
    assert lib.asd_tokens_record(rules(B=2 ** 30), 0x4000, 2 ** 30, None, 0, None, None) == SHAPE
    assert lib.asd_tokens_record(r, 0x4002, 5, None, 0, None, None) == ALIGN
    assert lib.asd_tokens_bias(r, None, 0x5000, 5, None, None, None) == NULL
    assert lib.asd_tokens_bias(r, 0x4000, None, 5, None, None, None) == NULL
    assert lib.asd_tokens_bias(r, 0x4000, 0x5000, 1025, None, None, None) == SHAPE
    assert lib.asd_tokens_bias(r, 0x4000, 0x5000, -1, None, None, None) == SHAPE
    assert lib.asd_tokens_bias(r, None, None, 0, None, None, None) == 0
    assert lib.asd_tokens_bias(r, 0x4000, 0x5001, 5, None, None, None) == ALIGN


def weigh(lib, c, **kw):
    a = dict(q=0x1000, lse=0x2000, s0=768, s1=256, s2=64, w=0x3000, out=0x3000, kv_len=0x4000, new_len=0, path=0,
             status=0, scale=0.1, decay=1.0, layer=0, T=3, rows=3, q_heads=4, width=32)
    a.update(kw)
    return lib.asd_kv_weigh(None if c is None else ctypes.addressof(c), asd._WEIGH.pack(*a.values()), None)


BAD_WEIGH = [(dict(layer=-1), SHAPE), (dict(layer=2), SHAPE), (dict(T=-1, rows=-1), SHAPE), (dict(rows=4), SHAPE),
             (dict(rows=-1, path=0x5000), SHAPE), (dict(q_heads=0), SHAPE), (dict(q_heads=3), SHAPE),
             (dict(width=-1), SHAPE), (dict(T=2 ** 28, rows=2 ** 28), SHAPE),
             (dict(scale=math.inf), CONTROL), (dict(scale=math.nan), CONTROL), (dict(scale=3e38), CONTROL), (dict(decay=-0.5), CONTROL),
             (dict(decay=math.inf), CONTROL), (dict(decay=math.nan), CONTROL), (dict(q=0), NULL), (dict(lse=0), NULL),
             (dict(w=0), NULL), (dict(out=0), NULL), (dict(kv_len=0), NULL), (dict(q=0x1001), ALIGN),
             (dict(lse=0x2002), ALIGN), (dict(w=0x3001), ALIGN), (dict(out=0x3002), ALIGN), (dict(kv_len=0x4001), ALIGN),
             (dict(new_len=0x4001), ALIGN), (dict(path=0x5002), ALIGN), (dict(status=0x5001), ALIGN)]


@pytest.mark.parametrize("kw,code", BAD_WEIGH, ids=[str(k) for k, _ in BAD_WEIGH])
def test_bad_weigh_arguments(lib, kw, code):
    assert weigh(lib, cache(), **kw) == code


def test_weigh_of_nothing(lib):
    assert weigh(lib, cache(), T=0, rows=0) == 0 and weigh(lib, cache(B=0)) == 0
    assert weigh(lib, None) == NULL and lib.asd_kv_weigh(ctypes.addressof(cache()), None, None) == NULL
    assert weigh(lib, cache(dtype=7)) == DTYPE


def evict(lib, c, **kw):
    a = dict(w=0x1000, out=0x1000, kv_len=0x2000, new=0x3000, keep=0x4000, status=0, first=0, last=0, width=32,
             reserved=0)
    a.update(kw)
    return lib.asd_kv_evict(None if c is None else ctypes.addressof(c), asd._EVICT.pack(*a.values()), None)


BAD_EVICT = [(dict(first=-1), SHAPE), (dict(last=-1), SHAPE), (dict(width=-1), SHAPE),
             (dict(width=asd.MAX_EVICT_SLOTS + 1), SHAPE), (dict(reserved=1), SHAPE), (dict(new=0x2000), SHAPE), (dict(new=0x4000), SHAPE),
             (dict(w=0), NULL), (dict(out=0), NULL), (dict(kv_len=0), NULL), (dict(new=0), NULL), (dict(keep=0), NULL),
             (dict(w=0x1001), ALIGN), (dict(out=0x1002), ALIGN), (dict(kv_len=0x2001), ALIGN), (dict(new=0x3002), ALIGN),
             (dict(keep=0x4001), ALIGN), (dict(status=0x5002), ALIGN)]


@pytest.mark.parametrize("kw,code", BAD_EVICT, ids=[str(k) for k, _ in BAD_EVICT])
def test_bad_evict_arguments(lib, kw, code):
    assert evict(lib, cache(), **kw) == code


def test_evict_of_nothing(lib):
    assert evict(lib, cache(B=0)) == 0
    assert evict(lib, None) == NULL and lib.asd_kv_evict(ctypes.addressof(cache()), None, None) == NULL
    assert evict(lib, cache(heads=0)) == SHAPE


# ---------------------------------------------------------------- the binding

class Library:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def entry(*args):
            self.calls.append((name, args))
            if name.endswith("_size"):
                args[-1]._obj.value = 1024
            return 0
        return entry


@pytest.fixture
def fake(monkeypatch):
    """A library that takes every call, and the stream that torch allocates on."""
    lib = Library()
    lib.stream, lib.allocated = None, []
    monkeypatch.setattr(asd, "load", lambda: lib)

    @contextlib.contextmanager
    def on(stream):
        was, lib.stream = lib.stream, stream
        yield
        lib.stream = was
    monkeypatch.setattr(torch.cuda, "stream", on)
    for how in ("zeros", "empty"):
        make = getattr(torch, how)

        def recorded(*a, _make=make, **kw):
            lib.allocated.append(lib.stream)
            kw.pop("device", None)
            return _make(*a, **kw)
        monkeypatch.setattr(torch, how, recorded)
    monkeypatch.setattr(asd, "_shape", lambda z, x: (z.shape[0], z.shape[1] - 1, z.shape[2]))
    return lib


def host_rules(B=2, V=100):
    r = asd.TokenRules.__new__(asd.TokenRules)
    r.marks, r.records = torch.ones(B, -(-V // 32), dtype=torch.int32), torch.ones(B, V, 2, dtype=torch.int32)
    r.B, r.V, r.words, r.device, r.index = B, V, -(-V // 32), r.marks.device, r.marks.get_device()
    r._head, r._plain = (1, 2, 0, 0, 0), asd._RULES.pack(1, 2, 0, 0, 0, 0, 0, 0, B, V)
    return r


def host_cache(B=2, heads=2, D=8):
    c = asd.KVCache.__new__(asd.KVCache)
    c.k = c.v = torch.ones(1, 4, 16, heads, D)
    c.dtype, c.device, c.index, c.layers = torch.float32, c.k.device, c.k.get_device(), 1
    c.B, c.heads, c.head_dim, c._ref = B, heads, D, 0
    return c


def i32(*shape):
    return torch.ones(*shape, dtype=torch.int32)


def test_calls_allocate_on_their_stream(fake):
    z = torch.ones(2, 4, 100)
    asd.rules_verify(z, i32(2, 3), torch.ones(2, 2), 1.0, 2, host_rules(), stream=STREAM)
    asd.rules_logits(z, i32(2, 3), host_rules(), stream=STREAM)
    asd.kv_evict(host_cache(), i32(2), torch.ones(1, 2, 2, 30), i32(2), stream=STREAM)
    assert len(fake.allocated) >= 8 and all(s is STREAM for s in fake.allocated)
    assert all(a[-1] == STREAM.cuda_stream for n, a in fake.calls if not n.endswith("_size"))
    fake.allocated.clear()
    q = torch.ones(2, 3, 4, 8)
    asd.kv_weigh(q, torch.ones(2, 3, 4), host_cache(), i32(2), torch.ones(2, 2, 30), stream=STREAM)
    asd.tokens_record(i32(2, 5), host_rules(), stream=STREAM)
    asd.tokens_bias(i32(2, 5), torch.ones(2, 5), host_rules(), stream=STREAM)
    asd.kv_evict(host_cache(), i32(2), torch.ones(2, 2, 30), i32(2), new_len=i32(2), stream=STREAM)
    assert fake.allocated == [] and fake.calls[-1][1][-1] == STREAM.cuda_stream


def test_wrong_tensors_are_refused(fake):
    r, c, z = host_rules(), host_cache(), torch.ones(2, 4, 100)
    led, w, q, lse = torch.ones(2, 2), torch.ones(2, 2, 30), torch.ones(2, 3, 4, 8), torch.ones(2, 3, 4)
    bad = [
        lambda: asd.rules_verify(torch.ones(3, 4, 100), i32(3, 3), led, 1.0, 2, r),
        lambda: asd.rules_verify(torch.ones(2, 4, 99), i32(2, 3), led, 1.0, 2, r),
        lambda: asd.rules_verify(z, i32(2, 3).long(), led, 1.0, 2, r),
        lambda: asd.rules_verify(z, i32(2, 3), led.double(), 1.0, 2, r),
        lambda: asd.rules_verify(z, i32(2, 3), led, 1.0, 2, r, allow=i32(2, 4, 3)),
        lambda: asd.rules_verify(z, i32(2, 3), led, 1.0, 2, r, allow=i32(2, 4, 8)[:, :, ::2]),
        lambda: asd.rules_verify(z, i32(2, 3), led, 1.0, 2, r, allow=torch.ones(2, 4, 4)),
        lambda: asd.rules_logits(z, i32(2, 2), r), lambda: asd.rules_logits(z[:, :, :50], None, r),
        lambda: asd.rules_logits(z, None, r, out=z.bfloat16()), lambda: asd.rules_logits(z[:1], None, r),
        lambda: asd.tokens_record(i32(10), r), lambda: asd.tokens_record(i32(3, 5), r),
        lambda: asd.tokens_record(i32(2, 5), r, token_len=i32(3)), lambda: asd.tokens_record(i32(2, 5).long(), r),
        lambda: asd.tokens_record(i32(2, 10)[:, ::2], r), lambda: asd.tokens_bias(i32(2, 5), torch.ones(2, 4), r),
        lambda: asd.tokens_bias(i32(2, 5), torch.ones(2, 5).double(), r),
        lambda: asd.kv_weigh(q, lse[:, :2], c, i32(2), w), lambda: asd.kv_weigh(q, lse, c, i32(2), None),
        lambda: asd.kv_weigh(q, lse, c, i32(2), w[:, :1]), lambda: asd.kv_weigh(q, lse, c, i32(2), w, out=w[:, :, :9]),
        lambda: asd.kv_weigh(q.half(), lse, c, i32(2), w), lambda: asd.kv_weigh(q, lse, c, i32(2), w, path=i32(3, 3)),
        lambda: asd.kv_weigh(q, lse, c, i32(2), w, new_len=i32(1)),
        lambda: asd.kv_evict(c, i32(2), w[0], i32(2)), lambda: asd.kv_evict(c, i32(2), w, i32(3)),
        lambda: asd.kv_evict(c, i32(2), w, i32(2), out=w[:, :, :9]),
        lambda: asd.kv_evict(c, i32(2), w, i32(2), new_len=i32(2).long()),
    ]
    for i, call in enumerate(bad):
        with pytest.raises((ValueError, TypeError)):
            call()
            pytest.fail(f"call {i} was taken")
    assert [n for n, _ in fake.calls if not n.endswith(("_size", "_init"))] == []


def test_rules_need_tensors_alike():
    m, rec = i32(2, 4), i32(2, 100, 2)
    for args in ((m, rec[:, :, :1]), (m[:, :3], rec), (m.float(), rec), (m, rec.float()), (m, rec)):  # the last: on the CPU
        with pytest.raises(ValueError):
            asd.TokenRules(*args)


def test_tensors_of_another_device_are_refused(fake, monkeypatch):
    """Without a stream of their own, calls run on the current device."""
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    r, c, z, q = host_rules(), host_cache(), torch.ones(2, 4, 100), torch.ones(2, 3, 4, 8)
    ws = types.SimpleNamespace(buffer=torch.ones(8), nbytes=1 << 20)
    out = {n: i32(2, 4) for n in ("accepted_len", "committed", "recovery")}
    calls = [lambda: asd.rules_verify(z, i32(2, 3), None, 1.0, 2, r, workspace=ws, out=out),
             lambda: asd.rules_logits(z, None, r, out=z), lambda: asd.tokens_record(i32(2, 5), r),
             lambda: asd.tokens_bias(i32(2, 5), torch.ones(2, 5), r),
             lambda: asd.kv_weigh(q, torch.ones(2, 3, 4), c, i32(2), torch.ones(2, 2, 30)),
             lambda: asd.kv_evict(c, i32(2), torch.ones(2, 2, 30), i32(2), new_len=i32(2))]
    for call in calls:
        with pytest.raises(ValueError, match="current device"):
            call()
    assert fake.calls == []


def test_streams_of_another_device_are_refused(fake):
    r, c, z, q = host_rules(), host_cache(), torch.ones(2, 4, 100), torch.ones(2, 3, 4, 8)
    other = types.SimpleNamespace(cuda_stream=0x5eed, device=torch.device("cuda", 3))
    ws = types.SimpleNamespace(buffer=torch.ones(8), nbytes=1 << 20)
    out = {n: i32(2, 4) for n in ("accepted_len", "committed", "recovery")}
    calls = [lambda s: asd.rules_verify(z, i32(2, 3), None, 1.0, 2, r, workspace=ws, out=out, stream=s),
             lambda s: asd.rules_logits(z, None, r, out=z, stream=s), lambda s: asd.tokens_record(i32(2, 5), r, stream=s),
             lambda s: asd.tokens_bias(i32(2, 5), torch.ones(2, 5), r, stream=s),
             lambda s: asd.kv_weigh(q, torch.ones(2, 3, 4), c, i32(2), torch.ones(2, 2, 30), stream=s),
             lambda s: asd.kv_evict(c, i32(2), torch.ones(2, 2, 30), i32(2), new_len=i32(2), stream=s)]
    for call in calls:
        with pytest.raises(ValueError, match="its stream is on cuda:3"):
            call(other)
    assert fake.calls == []
    for call in calls:
        call(STREAM)
    assert len(fake.calls) == len(calls)
