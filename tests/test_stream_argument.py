"""``stream=``: what a call allocates for itself belongs to the stream that its kernels run on, its fills included.

On the CPU: the library is a stand-in, and torch's stream context and allocations are recorded. A tensor that belonged
to the current stream would be filled in no order with the kernels, and could be another's before they have run.
"""
import contextlib
import types

import pytest
import torch

from paper_2608_03447_gb300 import asd

STREAM = types.SimpleNamespace(cuda_stream=0x5eed)


class Library:
    """Every entry point succeeds; what it was called with is kept."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def entry(*args):
            self.calls.append((name, args))
            if name.endswith("_size"):
                args[-1]._obj.value = 1024
            return 0
        return entry


class Recorder:
    def __init__(self):
        self.stream = None
        self.allocated = []  # (how, the stream it was allocated on)


@pytest.fixture
def record(monkeypatch):
    r, lib = Recorder(), Library()
    monkeypatch.setattr(asd, "load", lambda: lib)
    r.lib = lib

    @contextlib.contextmanager
    def on(stream):
        was, r.stream = r.stream, stream
        yield
        r.stream = was

    monkeypatch.setattr(torch.cuda, "stream", on)
    for how in ("zeros", "empty"):
        make = getattr(torch, how)

        def recorded(*a, _make=make, _how=how, **kw):
            r.allocated.append((_how, r.stream))
            kw.pop("device", None)
            return _make(*a, **kw)
        monkeypatch.setattr(torch, how, recorded)
    return r


def cpu_cache(B=2, heads=2, D=8):
    """A KVCache over host tensors, which its constructor refuses: only the arguments matter here."""
    c = asd.KVCache.__new__(asd.KVCache)
    c.k = c.v = torch.ones(4, 16, heads, D)[None]
    c.page_table = torch.ones(B, 2, dtype=torch.int32)
    c.dtype, c.device, c.index = torch.float32, c.k.device, c.k.get_device()
    c.B, c.heads, c.head_dim, c._ref = B, heads, D, 0
    return c


def test_append_allocates_its_queries_on_the_stream(record):
    k, q = torch.ones(2, 3, 2, 8), torch.ones(2, 3, 4, 8)
    out = asd.kv_append(k, k, cpu_cache(), torch.ones(2, dtype=torch.int32), q=q, stream=STREAM)
    assert out.shape == q.shape
    assert record.allocated == [("zeros", STREAM)]
    name, args = record.lib.calls[-1]
    assert name == "asd_kv_append" and args[-1] == STREAM.cuda_stream


def test_attention_allocates_outputs_and_workspace_on_the_stream(record):
    q = torch.ones(2, 3, 4, 8)
    asd.tree_attention(q, cpu_cache(), torch.ones(2, dtype=torch.int32), stream=STREAM)
    assert record.allocated == [("empty", STREAM)] * 3
    assert [name for name, _ in record.lib.calls] == ["asd_attention_workspace_size", "asd_workspace_init",
                                                      "asd_tree_attention"]
    assert all(args[-1] == STREAM.cuda_stream for _, args in record.lib.calls[1:])


def test_nothing_is_allocated_beside_given_tensors(record):
    k, q = torch.ones(2, 3, 2, 8), torch.ones(2, 3, 4, 8)
    n = torch.ones(2, dtype=torch.int32)
    asd.kv_append(k, k, cpu_cache(), n, q=q, q_out=q, stream=STREAM)
    asd.kv_append(k, k, cpu_cache(), n, stream=STREAM)
    assert record.allocated == []


@pytest.fixture
def shapes(monkeypatch):
    """The older calls check that logits are on a GPU; here they are not."""
    monkeypatch.setattr(asd, "_shape", lambda logits, draft: (logits.shape[0], logits.shape[1] - 1, logits.shape[2]))
    monkeypatch.setattr(asd, "_lm_shapes", lambda h, w: (h.shape[0], w.shape[0], h.shape[1]))


def test_verification_allocates_on_the_stream(record, shapes):
    B, K, V = 2, 3, 10
    z, x, led = torch.ones(B, K + 1, V), torch.ones(B, K, dtype=torch.int32), torch.ones(B, 2)
    h, w = torch.ones(B * (K + 1), 8), torch.ones(V, 8)
    s = dict(stream=STREAM)
    asd.verify(z, x, led, 1.0, 2, **s)
    asd.verify_noalloc(z, x, led, 1.0, 2, **s)
    asd.verify_strict(z, x, **s)
    asd.lmhead_verify(h, w, x, led, 1.0, 2, **s)
    asd.lmhead_partials(h, w, x, 0, V, **s)
    asd.lmhead_logits(h, w, **s)
    asd.shard_partials(z, x, 0, V, **s)
    asd.shard_combine(torch.ones(1, B * (K + 1), asd.PARTIAL_WORDS, dtype=torch.int32), x, led, 1.0, 2, V, **s)
    asd.blocks_workspace(2, B, K, V, asd.F32, device="cpu", **s)
    assert len(record.allocated) > 30
    assert [a for a in record.allocated if a[1] is not STREAM] == []
    assert all(args[-1] == STREAM.cuda_stream for name, args in record.lib.calls if not name.endswith("_size"))


def test_opportunity_counts_are_zeroed_on_the_stream(record):
    rows, x, regret = torch.ones(4, 3, dtype=torch.int32), torch.ones(4, 2, dtype=torch.int32), torch.ones(4, 2)
    asd.opportunity(rows, x, regret, [0.5], [1], stream=STREAM)
    assert record.allocated == [("zeros", STREAM)]


def test_results_are_copied_to_the_host_on_the_stream(record, monkeypatch):
    copied = []

    class Result:
        def data_ptr(self):
            return 64

    class HostResult:
        def copy_(self, src, non_blocking):
            copied.append((non_blocking, record.stream))

    class Pinned:
        dtype, shape = torch.float32, (2, 4, 10)

        def dim(self):
            return 3

        def is_pinned(self):
            return True

    monkeypatch.setattr(asd, "_alias", lambda t: 64)
    monkeypatch.setattr(asd, "_ptr", lambda t: 64)
    names = ("accepted_len", "committed", "recovery")
    ws = types.SimpleNamespace(ptr=64, nbytes=1024)
    asd.verify_from_host(Pinned(), Pinned(), Result(), 1.0, 2, ws, {n: Result() for n in names},
                         {n: HostResult() for n in names}, stream=STREAM)
    assert copied == [(True, STREAM)] * 3
