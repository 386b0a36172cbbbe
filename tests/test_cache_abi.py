"""The cache entry points on the host: sizes, and the refusal of bad arguments before any CUDA call (no GPU needed)."""
import ctypes
import math

import pytest
import torch

from paper_2608_03447_gb300 import asd


@pytest.fixture(scope="module")
def lib():
    return asd.load()


def cache(**kw):
    a = dict(k=0x10000, v=0x20000, dtype=asd.BF16, layers=2, pages=4, page_size=16, heads=2, head_dim=64,
             layer_stride=4 * 2048, page_stride=2048, token_stride=128, head_stride=64, page_table=0x30000, B=3,
             table_width=2)
    a.update(kw)
    return asd._Cache(*[a[n] for n, _ in asd._Cache._fields_])


def append(lib, c=None, **kw):
    a = dict(layer=0, T=3, k=0x1000, ks=(384, 128, 64), v=0x2000, vs=(384, 128, 64), q=0, qs=(0, 0, 0), q_heads=0,
             q_out=0, kv_len=0x3000, new_len=0, positions=0, cos=0, sin=0, rot=0, table=0, inter=0, qw=0, kw=0,
             eps=1e-6, status=0)
    a.update({n: 0 if x is None else x for n, x in kw.items()})
    block = asd._APPEND.pack(a["k"], a["v"], a["q"], a["q_out"], *a["ks"], *a["vs"], *a["qs"], a["kv_len"],
                             a["new_len"], a["positions"], a["cos"], a["sin"], a["qw"], a["kw"], a["status"],
                             a["layer"], a["T"], a["q_heads"], a["rot"], a["table"], a["inter"], a["eps"], 0)
    return lib.asd_kv_append(ctypes.addressof(c) if c is not None else None, block, None)


def attend(lib, c=None, **kw):
    a = dict(layer=0, T=3, q=0x1000, qs=(768, 256, 64), q_heads=4, kv_len=0x3000, new_len=0, mask=0, scale=0.1,
             out=0x4000, lse=0, status=0, ws=0x50000, wsb=1 << 40)
    a.update({n: 0 if x is None else x for n, x in kw.items()})
    block = asd._ATTENTION.pack(a["q"], a["out"], a["lse"], *a["qs"], a["kv_len"], a["new_len"], a["mask"],
                                a["status"], a["ws"], a["wsb"], a["layer"], a["T"], a["q_heads"], a["scale"])
    return lib.asd_tree_attention(ctypes.addressof(c) if c is not None else None, block, None)


def compact(lib, c=None, **kw):
    a = dict(P=4, kv_len=0x1000, path=0x2000, path_len=0x3000, status=None)
    a.update(kw)
    ref = ctypes.addressof(c) if c is not None else None
    return lib.asd_kv_compact(ref, a["P"], a["kv_len"], a["path"], a["path_len"], a["status"], None)


BAD_CACHES = [(dict(dtype=3), 3), (dict(dtype=asd.BF16 | asd.RESIDENT_INPUTS), 3), (dict(layers=0), 2),
              (dict(pages=-1), 2), (dict(page_size=0), 2), (dict(heads=0), 2), (dict(head_dim=0), 2),
              (dict(head_dim=257), 2), (dict(B=-1), 2), (dict(table_width=-1), 2), (dict(page_stride=-1), 2),
              (dict(token_stride=-1), 2), (dict(head_stride=-8), 2), (dict(layer_stride=-8), 2), (dict(k=None), 1),
              (dict(v=None), 1), (dict(page_table=None), 1), (dict(k=0x10001), 6), (dict(v=0x20001), 6),
              (dict(page_table=0x30002), 6)]


@pytest.mark.parametrize("kw,code", BAD_CACHES, ids=[str(k) for k, _ in BAD_CACHES])
def test_bad_caches(lib, kw, code):
    c = cache(**kw)
    n = ctypes.c_size_t(0)
    assert append(lib, c) == code
    assert attend(lib, c) == code
    assert compact(lib, c) == code
    assert lib.asd_attention_workspace_size(ctypes.addressof(c), 3, 4, ctypes.byref(n)) == code


def test_no_cache_and_no_arguments(lib):
    n = ctypes.c_size_t(0)
    c = cache()
    assert lib.asd_kv_append(ctypes.addressof(c), None, None) == 1
    assert lib.asd_tree_attention(ctypes.addressof(c), None, None) == 1
    assert append(lib) == attend(lib) == compact(lib) == 1
    assert lib.asd_attention_workspace_size(None, 3, 4, ctypes.byref(n)) == 1


@pytest.mark.parametrize("kw,code", [
    (dict(layer=2), 2), (dict(layer=-1), 2), (dict(T=-1), 2), (dict(q_heads=-1), 2), (dict(k=None), 1),
    (dict(v=None), 1), (dict(kv_len=None), 1), (dict(q_heads=4), 1), (dict(q_heads=4, q=0x5000), 1),
    (dict(cos=0x6000), 1), (dict(sin=0x6000), 1), (dict(cos=0x6000, sin=0x7000, rot=0, table=4), 2),
    (dict(cos=0x6000, sin=0x7000, rot=7, table=4), 2), (dict(cos=0x6000, sin=0x7000, rot=66, table=4), 2),
    (dict(cos=0x6000, sin=0x7000, rot=64, table=-1), 2), (dict(rot=64), 2), (dict(inter=2), 2), (dict(eps=-1.0), 4),
    (dict(eps=math.nan), 4), (dict(k=0x1001), 6), (dict(kv_len=0x3002), 6), (dict(status=0x3001), 6),
    (dict(qw=0x3001), 6), (dict(T=0), 0)], ids=str)
def test_append_refusals(lib, kw, code):
    assert append(lib, cache(), **kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(layer=2), 2), (dict(T=-1), 2), (dict(q_heads=3), 2), (dict(q_heads=0), 2), (dict(T=1 << 28), 2),
    (dict(q=None), 1), (dict(kv_len=None), 1), (dict(out=None), 1), (dict(ws=None), 1), (dict(scale=math.nan), 4),
    (dict(scale=math.inf), 4), (dict(q=0x1001), 6), (dict(out=0x4001), 6), (dict(lse=0x4002), 6),
    (dict(mask=0x4002), 6), (dict(wsb=1000), 5), (dict(ws=0x50008), 6), (dict(T=0), 0)], ids=str)
def test_attention_refusals(lib, kw, code):
    assert attend(lib, cache(), **kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(P=-1), 2), (dict(P=257), 2), (dict(kv_len=None), 1), (dict(path=None), 1), (dict(path_len=None), 1),
    (dict(path=0x2002), 6), (dict(P=0), 0)], ids=str)
def test_compact_refusals(lib, kw, code):
    assert compact(lib, cache(), **kw) == code


def test_argument_blocks_lie_as_in_the_header(tmp_path):
    """The packed blocks' sizes and the last fields' places, as the C compiler has them."""
    import subprocess
    from paper_2608_03447_gb300 import build
    (tmp_path / "shim.cpp").write_text("""
#include "asd.h"
#include <stddef.h>
extern "C" int at(int i) {
  const size_t x[] = {sizeof(asd_append), offsetof(asd_append, kv_len), offsetof(asd_append, status),
                      offsetof(asd_append, eps), sizeof(asd_attention), offsetof(asd_attention, kv_len),
                      offsetof(asd_attention, workspace_bytes), offsetof(asd_attention, scale), sizeof(asd_kv_cache)};
  return static_cast<int>(x[i]);
}
""")
    out = str(tmp_path / "shim.so")
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC", f"-I{build.INCLUDE}",
                    str(tmp_path / "shim.cpp"), "-o", out], check=True)
    at = ctypes.CDLL(out).at
    assert at(0) == asd._APPEND.size and at(4) == asd._ATTENTION.size and at(8) == ctypes.sizeof(asd._Cache)
    assert (at(1), at(2), at(3)) == (104, 160, 192)
    assert (at(5), at(6), at(7)) == (48, 88, 108)


def test_empty_batches(lib):
    c = cache(B=0, page_table=None)
    assert append(lib, c) == attend(lib, c) == compact(lib, c) == 0


def test_workspace_size(lib):
    n = ctypes.c_size_t(0)
    for dtype in (asd.F32, asd.BF16, asd.F16):
        for T, heads in ((1, 2), (9, 4), (200, 10)):
            c = cache(dtype=dtype)
            assert lib.asd_attention_workspace_size(ctypes.addressof(c), T, heads, ctypes.byref(n)) == 0
            assert n.value % 256 == 0 and 0 < n.value < 1 << 29
    assert lib.asd_attention_workspace_size(ctypes.addressof(cache()), 3, 4, None) == 1


def test_tree_mask():
    m = asd.tree_mask(torch.tensor([[-1, 0, 0, 2, -1, 4]]))
    assert m.tolist() == [[[0b1], [0b11], [0b101], [0b1101], [0b10000], [0b110000]]]
    chain = asd.tree_mask(torch.arange(40)[None] - 1)
    assert chain.shape == (1, 40, 2) and chain[0, 39].tolist() == [-1, 255] and chain[0, 31].tolist() == [-1, 0]
    with pytest.raises(ValueError):
        asd.tree_mask(torch.tensor([[0]]))
    with pytest.raises(ValueError):
        asd.tree_mask(torch.tensor([[-1, -2]]))


def test_the_binding_refuses_tensors_that_do_not_fit():
    k = torch.zeros(4, 16, 2, 64)
    table = torch.zeros(3, 2, dtype=torch.int32)
    with pytest.raises(ValueError):
        asd.KVCache(k, k, table)                       # not on a GPU
    with pytest.raises(TypeError):
        asd.KVCache(k.double(), k.double(), table)
    with pytest.raises(ValueError):
        asd.KVCache(k, k[:, :8], table)
    with pytest.raises(ValueError):
        asd.KVCache(k, k, table.long())
    with pytest.raises(ValueError):
        asd.KVCache(k[..., ::2], k[..., ::2], table)   # last dimension not contiguous
