"""ctypes binding of libasd (include/asd.h): argument marshalling only.

Every step of the verifier runs in the library's CUDA kernels; this module
turns torch tensors into device pointers, passes torch's current CUDA stream,
and raises on a non-zero return code. There is no fallback: if libasd.so is
missing the first call raises.

Entry points mirror the C names: ``verify`` (asd_verify), ``verify_strict``
(asd_verify_strict), ``workspace_size``, ``workspace_init``, ``status_string``.
Ledgers are float32 tensors of shape [B, 2] holding (budget, spent), the
memory layout of ``asd_ledger``. The cache side of a block: ``KVCache``
(asd_kv_cache), ``kv_append``, ``tree_mask``, ``tree_attention``, ``kv_compact``,
``kv_weigh``, ``weigh_error``, ``kv_evict`` (asd_kv_evict, asd_kv_evict_numbered). Logits under penalties, biases and grammars:
``TokenRules`` (asd_token_rules), ``rules_verify``, ``rules_logits``,
``tokens_record``, ``tokens_bias``.
"""
from __future__ import annotations

import contextlib
import ctypes
import os
import re
import struct
import threading

import torch

PKG = os.path.dirname(os.path.abspath(__file__))
LIBRARY = os.path.join(PKG, "libasd.so")
HEADER = os.path.join(os.path.dirname(PKG), "include", "asd.h")

F32 = 0
BF16 = 1
F16 = 2

OK = 0
STATUS_DRAFT_RANGE = 1
STATUS_NAN_LOGIT = 2
STATUS_BAD_LEDGER = 4
STATUS_OVERFLOW = 8
STATUS_INCOMPLETE = 16
STATUS_LENGTH = 32
STATUS_PAGE = 64
STATUS_POSITION = 128
STATUS_PATH = 256
STATUS_TOKEN = 512
STATUS_EMPTY_ROW = 1024
MAX_K = 31
MAX_HEAD_DIM = 256
MAX_PATH = 256
MAX_BIAS = 1024
MAX_EVICT_SLOTS = 360448
TOKEN_PROMPT = -2**31  # ASD_TOKEN_PROMPT as an int32, of a record's first word
RESIDENT_INPUTS = 0x100  # ASD_RESIDENT_INPUTS, ORed into the dtype code
FLAG_EMPTY_ROWS = 0x200  # ASD_FLAG_EMPTY_ROWS, ORed into rules_verify's dtype code
INT32_MAX = 2**31 - 1

_lock = threading.Lock()
_lib = None


class AsdError(RuntimeError):
    def __init__(self, fn: str, code: int):
        self.code = code
        super().__init__(f"{fn} returned {code}: {status_string(code) if _lib else code}")


def _declare(lib: ctypes.CDLL) -> ctypes.CDLL:
    vp, i32, f32, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_size_t
    lib.asd_workspace_size.argtypes = [i32, i32, i32, i32, ctypes.POINTER(sz)]
    lib.asd_workspace_size.restype = i32
    lib.asd_workspace_init.argtypes = [vp, sz, vp]
    lib.asd_workspace_init.restype = i32
    lib.asd_workspace_error.argtypes = [vp, ctypes.POINTER(i32), vp]
    lib.asd_workspace_error.restype = i32
    lib.asd_selftest_wait_timeout.argtypes = [vp, sz, vp]
    lib.asd_selftest_wait_timeout.restype = i32
    lib.asd_verify.argtypes = [vp, i32, i32, i32, i32, vp, vp, f32, i32, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.asd_verify.restype = i32
    lib.asd_verify_strict.argtypes = [vp, i32, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.asd_verify_strict.restype = i32
    lib.asd_status_string.argtypes = [i32]
    lib.asd_status_string.restype = ctypes.c_char_p
    lib.asd_host_alias.argtypes = [vp, ctypes.POINTER(vp)]
    lib.asd_host_alias.restype = i32
    lib.asd_verify_launches.argtypes = [i32, i32, i32, i32, ctypes.POINTER(i32)]
    lib.asd_verify_launches.restype = i32
    lib.asd_blocks_workspace_size.argtypes = [i32, i32, i32, i32, i32, ctypes.POINTER(sz)]
    lib.asd_blocks_workspace_size.restype = i32
    lib.asd_verify_blocks.argtypes = [vp, i32, i32, i32, i32, i32, vp, vp, f32, i32, vp, vp, vp, vp, vp, vp, vp, sz,
                                      vp]
    lib.asd_verify_blocks.restype = i32
    lib.asd_shard_partials.argtypes = [vp, i32, i32, i32, i32, i32, i32, vp, vp, vp, sz, vp]
    lib.asd_shard_partials.restype = i32
    lib.asd_shard_combine.argtypes = [vp, i32, i32, i32, i32, vp, vp, f32, i32, vp, vp, vp, vp, vp, vp, vp]
    lib.asd_shard_combine.restype = i32
    lib.asd_commit.argtypes = [i32, i32, vp, vp, i32, vp, vp, vp, i32, vp, vp]
    lib.asd_commit.restype = i32
    lib.asd_opportunity.argtypes = [vp, vp, vp, vp, i32, i32, vp, i32, vp, i32, vp, vp]
    lib.asd_opportunity.restype = i32
    if hasattr(lib, "asd_verify_noalloc"):
        lib.asd_verify_noalloc.argtypes = [vp, i32, i32, i32, i32, vp, vp, f32, i32, vp, vp, vp, vp, vp, vp, vp]
        lib.asd_verify_noalloc.restype = i32
    lib.asd_lmhead_workspace_size.argtypes = [i32, i32, i32, i32, ctypes.POINTER(sz)]
    lib.asd_lmhead_workspace_size.restype = i32
    lib.asd_lmhead_verify.argtypes = [vp, vp, i32, i32, i32, i32, vp, vp, f32, i32,
                                      vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.asd_lmhead_verify.restype = i32
    lib.asd_lmhead_logits.argtypes = [vp, vp, i32, i32, i32, vp, vp]
    lib.asd_lmhead_logits.restype = i32
    lib.asd_lmhead_partials.argtypes = [vp, vp, i32, i32, i32, i32, i32, i32, vp, vp, vp, sz, vp]
    lib.asd_lmhead_partials.restype = i32
    lib.asd_kv_append.argtypes = [vp, vp, vp]
    lib.asd_kv_append.restype = i32
    lib.asd_attention_workspace_size.argtypes = [vp, i32, i32, ctypes.POINTER(sz)]
    lib.asd_attention_workspace_size.restype = i32
    lib.asd_tree_attention.argtypes = [vp, vp, vp]
    lib.asd_tree_attention.restype = i32
    lib.asd_kv_compact.argtypes = [vp, i32, vp, vp, vp, vp, vp]
    lib.asd_kv_compact.restype = i32
    lib.asd_kv_weigh.argtypes = [vp, vp, vp]
    lib.asd_kv_weigh.restype = i32
    lib.asd_weigh_error.argtypes = [ctypes.POINTER(i32), vp]
    lib.asd_weigh_error.restype = i32
    lib.asd_kv_evict.argtypes = [vp, vp, vp]
    lib.asd_kv_evict.restype = i32
    lib.asd_kv_evict_numbered.argtypes = [vp, vp, vp, vp, vp]
    lib.asd_kv_evict_numbered.restype = i32
    lib.asd_rules_verify.argtypes = [vp, vp, vp]
    lib.asd_rules_verify.restype = i32
    lib.asd_rules_logits.argtypes = [vp, vp, i32, i32, vp, vp, vp]
    lib.asd_rules_logits.restype = i32
    lib.asd_tokens_record.argtypes = [vp, vp, i32, vp, i32, vp, vp]
    lib.asd_tokens_record.restype = i32
    lib.asd_tokens_bias.argtypes = [vp, vp, vp, i32, vp, vp, vp]
    lib.asd_tokens_bias.restype = i32
    lib.asd_set_launch_options.argtypes = [vp]
    lib.asd_set_launch_options.restype = i32
    lib.asd_get_launch_options.argtypes = [vp]
    lib.asd_get_launch_options.restype = i32
    return lib


class _LaunchOptions(ctypes.Structure):
    _fields_ = [("path", ctypes.c_int), ("fused_select", ctypes.c_int), ("no_pdl", ctypes.c_int)]


PATHS = {"auto": 0, "small": 1, "stream": 2, "tma": 3}


def set_launch_options(path: str = "auto", fused_select: bool = False, pdl: bool = True) -> None:
    """asd_set_launch_options: which row-stage kernel the verify calls use (process-wide)."""
    opt = _LaunchOptions(PATHS[path], int(fused_select), int(not pdl))
    _check("asd_set_launch_options", load().asd_set_launch_options(ctypes.byref(opt)))


def get_launch_options() -> dict:
    opt = _LaunchOptions()
    _check("asd_get_launch_options", load().asd_get_launch_options(ctypes.byref(opt)))
    names = {v: k for k, v in PATHS.items()}
    return {"path": names[opt.path], "fused_select": bool(opt.fused_select), "pdl": not opt.no_pdl}


def reset_launch_options() -> None:
    _check("asd_set_launch_options", load().asd_set_launch_options(None))


def load(path: str = LIBRARY) -> ctypes.CDLL:
    """Open libasd.so (once). Raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    with _lock:
        if _lib is None:
            if not os.path.exists(path):
                raise RuntimeError(f"{path} is missing: build it with __graft_entry__.build() "
                                   "(python -m paper_2608_03447_gb300.build)")
            _lib = _declare(ctypes.CDLL(path))
    return _lib


def declared_functions(header: str = HEADER) -> list[str]:
    """Names of the functions that include/asd.h declares."""
    with open(header) as f:
        text = f.read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    return sorted(set(re.findall(r"\b(asd_[a-z0-9_]+)\s*\(", text)))


def status_string(code: int) -> str:
    return load().asd_status_string(int(code)).decode()


def _check(fn: str, rc: int) -> None:
    if rc != OK:
        raise AsdError(fn, rc)


def _ptr(t: torch.Tensor | None) -> int | None:
    if t is None:
        return None
    return t.data_ptr()


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream) -> int:
    if stream is None:
        # the handle of torch.cuda.current_stream() without building a Stream object around it: 2.9 us of an eager
        # call's 12.4 us (8.7 us with load() answering before its lock, too)
        if _raw_stream is not None:
            return _raw_stream(torch.cuda.current_device())
        stream = torch.cuda.current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _stream_at(stream, index: int) -> int:
    """The handle of a call's stream. Kernels run on the current device, in a stream of its own: tensors of another one
    are refused (a raw handle does not show its device; the current one is compared all the same)."""
    if stream is not None:
        device = getattr(stream, "device", None)
        if device is not None and device.index != index:
            raise ValueError(f"the call's tensors are on cuda:{index}, its stream is on {device}")
        if index < 0:  # not of any GPU
            return _stream(stream)
    current = torch.cuda.current_device()
    if current != index:
        raise ValueError(f"the call's tensors are on cuda:{index}, the current device is cuda:{current}")
    if stream is None and _raw_stream is not None:
        return _raw_stream(current)
    return _stream(stream)


def _torch_on(stream):
    """A context in which torch allocates and launches on a call's stream, as the call's own kernels do.

    Memory that a call allocates belongs to that stream: its first fill is ordered before the kernels, and memory that
    is dropped on return is handed out again only behind them.
    """
    if stream is None:
        return contextlib.nullcontext()
    return torch.cuda.stream(stream if hasattr(stream, "cuda_stream") else torch.cuda.ExternalStream(int(stream)))


def _flag(resident: bool) -> int:
    return RESIDENT_INPUTS if resident else 0


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.bfloat16:
        return BF16
    raise TypeError(f"logits must be float32 or bfloat16, got {t.dtype}")


def host_alias(t: torch.Tensor) -> int:
    """asd_host_alias: device address of a pinned host tensor's data (for reading it from kernels)."""
    if t.is_cuda or not t.is_pinned():
        raise ValueError("host_alias needs a pinned host tensor")
    out = ctypes.c_void_p(0)
    _check("asd_host_alias", load().asd_host_alias(t.data_ptr(), ctypes.byref(out)))
    return out.value


def verify_launches(B: int, K: int, V: int, dtype: int) -> int:
    """asd_verify_launches: kernels one asd_verify call launches for this shape."""
    n = ctypes.c_int(0)
    _check("asd_verify_launches", load().asd_verify_launches(B, K, V, dtype, ctypes.byref(n)))
    return n.value


def workspace_size(B: int, K: int, V: int, dtype: int) -> int:
    n = ctypes.c_size_t(0)
    _check("asd_workspace_size", load().asd_workspace_size(B, K, V, dtype, ctypes.byref(n)))
    return n.value


class Workspace:
    """Device scratch for one stream of verify calls; zeroed once at creation."""

    def __init__(self, B: int, K: int, V: int, dtype: int, device=None, stream=None):
        self.nbytes = workspace_size(B, K, V, dtype)
        with _torch_on(stream):
            self.buffer = torch.empty(self.nbytes, dtype=torch.uint8, device=device or "cuda")
        _check("asd_workspace_init", load().asd_workspace_init(self.buffer.data_ptr(), self.nbytes, _stream(stream)))

    @property
    def ptr(self) -> int:
        return self.buffer.data_ptr()

    def error(self, stream=None) -> int:
        """The sticky error word (asd_workspace_error); synchronises the stream."""
        word = ctypes.c_int(0)
        _check("asd_workspace_error", load().asd_workspace_error(self.ptr, ctypes.byref(word), _stream(stream)))
        return word.value

    def reset(self, stream=None) -> None:
        """Zero the workspace again (asd_workspace_init), e.g. after a non-zero error word."""
        _check("asd_workspace_init", load().asd_workspace_init(self.ptr, self.nbytes, _stream(stream)))


def selftest_wait_timeout(workspace: "Workspace", stream=None) -> None:
    """asd_selftest_wait_timeout: a bounded wait on a barrier nothing signals (about one second); the
    workspace's error word then reads ASD_ERR_TIMEOUT."""
    _check("asd_selftest_wait_timeout", load().asd_selftest_wait_timeout(workspace.ptr, workspace.nbytes,
                                                                         _stream(stream)))


def make_ledger(B: int, budget: float, spent: float = 0.0, device="cuda") -> torch.Tensor:
    led = torch.empty(B, 2, dtype=torch.float32, device=device)
    led[:, 0] = budget
    led[:, 1] = spent
    return led


def alloc_outputs(B: int, K: int, device="cuda", with_rows: bool = True, stream=None) -> dict:
    with _torch_on(stream):
        out = {
            "accepted_len": torch.empty(B, dtype=torch.int32, device=device),
            "committed": torch.empty(B, K + 1, dtype=torch.int32, device=device),
            "recovery": torch.empty(B, dtype=torch.int32, device=device),
            "status": torch.empty(B, dtype=torch.int32, device=device),
        }
        if with_rows:
            out["row_argmax"] = torch.empty(B, K + 1, dtype=torch.int32, device=device)
            out["row_regret"] = torch.empty(B, K, dtype=torch.float32, device=device)
    return out


def _shape(logits: torch.Tensor, draft: torch.Tensor):
    if logits.dim() != 3 or not logits.is_cuda or not logits.is_contiguous():
        raise ValueError("logits must be a contiguous CUDA tensor [B, K+1, V]")
    B, K1, V = logits.shape
    K = K1 - 1
    if draft.shape != (B, K) or draft.dtype != torch.int32 or not draft.is_contiguous():
        raise ValueError("draft must be a contiguous int32 tensor [B, K]")
    return B, K, V


def verify(logits: torch.Tensor, draft: torch.Tensor, ledger: torch.Tensor, gate: float, cap: int,
           workspace: Workspace | None = None, out: dict | None = None, stream=None, resident: bool = False) -> dict:
    """asd_verify: ASD verification of a batch of draft blocks; updates ``ledger`` in place.

    ``resident=True`` passes ASD_RESIDENT_INPUTS: no kernel still running or queued ahead on the stream
    writes ``logits`` or ``draft``, so the row stage may stream them while the previous kernel finishes.
    """
    B, K, V = _shape(logits, draft)
    if ledger.shape != (B, 2) or ledger.dtype != torch.float32 or not ledger.is_contiguous():
        raise ValueError("ledger must be a contiguous float32 tensor [B, 2] of (budget, spent)")
    code = _dtype_code(logits)
    ws = workspace or Workspace(B, K, V, code, logits.device, stream)
    o = out or alloc_outputs(B, K, logits.device, stream=stream)
    rc = load().asd_verify(_ptr(logits), code | _flag(resident), B, K, V, _ptr(draft), _ptr(ledger), float(gate),
                           int(cap),
                           _ptr(o["accepted_len"]), _ptr(o["committed"]), _ptr(o["recovery"]),
                           _ptr(o.get("row_argmax")), _ptr(o.get("row_regret")), _ptr(o.get("status")),
                           ws.ptr, ws.nbytes, _stream(stream))
    _check("asd_verify", rc)
    return o


def verify_noalloc(logits: torch.Tensor, draft: torch.Tensor, ledger: torch.Tensor, gate: float, cap: int,
                   out: dict | None = None, stream=None, resident: bool = False) -> dict:
    """asd_verify_noalloc: asd_verify with the library's fixed scratch instead of a workspace.

    For callers that may not allocate device memory while verifying. Calls that
    may overlap on the GPU share that scratch and must be ordered on one stream.
    """
    B, K, V = _shape(logits, draft)
    if ledger.shape != (B, 2) or ledger.dtype != torch.float32 or not ledger.is_contiguous():
        raise ValueError("ledger must be a contiguous float32 tensor [B, 2] of (budget, spent)")
    o = out or alloc_outputs(B, K, logits.device, stream=stream)
    rc = load().asd_verify_noalloc(_ptr(logits), _dtype_code(logits) | _flag(resident), B, K, V, _ptr(draft),
                                   _ptr(ledger),
                                   float(gate), int(cap), _ptr(o["accepted_len"]), _ptr(o["committed"]),
                                   _ptr(o["recovery"]), _ptr(o.get("row_argmax")), _ptr(o.get("row_regret")),
                                   _ptr(o.get("status")), _stream(stream))
    _check("asd_verify_noalloc", rc)
    return o


def verify_strict(logits: torch.Tensor, draft: torch.Tensor, workspace: Workspace | None = None,
                  out: dict | None = None, stream=None, resident: bool = False) -> dict:
    """asd_verify_strict: strict greedy verification (Eq. 2)."""
    B, K, V = _shape(logits, draft)
    code = _dtype_code(logits)
    ws = workspace or Workspace(B, K, V, code, logits.device, stream)
    o = out or alloc_outputs(B, K, logits.device, stream=stream)
    rc = load().asd_verify_strict(_ptr(logits), code | _flag(resident), B, K, V, _ptr(draft),
                                  _ptr(o["accepted_len"]), _ptr(o["committed"]), _ptr(o["recovery"]),
                                  _ptr(o.get("row_argmax")), _ptr(o.get("row_regret")), _ptr(o.get("status")),
                                  ws.ptr, ws.nbytes, _stream(stream))
    _check("asd_verify_strict", rc)
    return o


_aliases: dict = {}
_ALIAS_CACHE = 64  # the most recently used pinned buffers keep their looked-up device address


def _alias(t: torch.Tensor) -> int:
    key = (t.data_ptr(), t.numel() * t.element_size())
    addr = _aliases.pop(key, None)
    if addr is None:
        addr = host_alias(t)
    _aliases[key] = addr  # re-inserted: dicts keep insertion order, so the oldest entry is first
    while len(_aliases) > _ALIAS_CACHE:
        _aliases.pop(next(iter(_aliases)))
    return addr


def verify_from_host(logits_host: torch.Tensor, draft_host: torch.Tensor, ledger: torch.Tensor, gate: float,
                     cap: int, workspace: Workspace, out: dict, host_out: dict, stream=None,
                     resident: bool = False) -> dict:
    """End-to-end step from pinned host buffers: verify reading them in place, copy the results out.

    The kernels read the pinned logits and drafts through their device aliases
    (asd_host_alias), so the host-to-device transfer is the verify's own
    stream of reads over the host link, with no separate copy; the ledger stays
    on the device (the request state carried between rounds); the per-request
    results are copied back to pinned host tensors, asynchronously on ``stream``.
    """
    if logits_host.dim() != 3 or not logits_host.is_pinned() or not draft_host.is_pinned():
        raise ValueError("verify_from_host needs pinned host logits [B, K+1, V] and drafts [B, K]")
    B, K1, V = logits_host.shape
    K = K1 - 1
    code = _dtype_code(logits_host)
    rc = load().asd_verify(_alias(logits_host), code | _flag(resident), B, K, V, _alias(draft_host), _ptr(ledger),
                           float(gate),
                           int(cap), _ptr(out["accepted_len"]), _ptr(out["committed"]), _ptr(out["recovery"]),
                           _ptr(out.get("row_argmax")), _ptr(out.get("row_regret")), _ptr(out.get("status")),
                           workspace.ptr, workspace.nbytes, _stream(stream))
    _check("asd_verify", rc)
    with _torch_on(stream):
        for k in ("accepted_len", "committed", "recovery"):
            host_out[k].copy_(out[k], non_blocking=True)
    return host_out


def lmhead_workspace(B: int, K: int, V: int, H: int, device=None, stream=None) -> Workspace:
    n = ctypes.c_size_t(0)
    _check("asd_lmhead_workspace_size", load().asd_lmhead_workspace_size(B, K, V, H, ctypes.byref(n)))
    ws = Workspace.__new__(Workspace)
    ws.nbytes = n.value
    with _torch_on(stream):
        ws.buffer = torch.empty(ws.nbytes, dtype=torch.uint8, device=device or "cuda")
    _check("asd_workspace_init", load().asd_workspace_init(ws.buffer.data_ptr(), ws.nbytes, _stream(stream)))
    return ws


def _lm_shapes(hidden: torch.Tensor, weight: torch.Tensor):
    for name, t in (("hidden", hidden), ("weight", weight)):
        if t.dtype != torch.bfloat16 or t.dim() != 2 or not t.is_cuda or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous 2-D bf16 CUDA tensor")
    if hidden.shape[1] != weight.shape[1]:
        raise ValueError("hidden and weight must share the hidden size H")
    return hidden.shape[0], weight.shape[0], hidden.shape[1]


def lmhead_verify(hidden: torch.Tensor, weight: torch.Tensor, draft: torch.Tensor, ledger: torch.Tensor,
                  gate: float, cap: int, workspace: Workspace | None = None, out: dict | None = None,
                  stream=None) -> dict:
    """asd_lmhead_verify: logits = hidden @ weight.T on the tensor cores, reduced on chip, then Alg. 1."""
    T, V, H = _lm_shapes(hidden, weight)
    B, K = draft.shape
    if T != B * (K + 1):
        raise ValueError("hidden must hold B*(K+1) rows")
    ws = workspace or lmhead_workspace(B, K, V, H, hidden.device, stream)
    o = out or alloc_outputs(B, K, hidden.device, stream=stream)
    if "row_top" not in o:
        with _torch_on(stream):
            o["row_top"] = torch.empty(B, K + 1, dtype=torch.float32, device=hidden.device)
    rc = load().asd_lmhead_verify(_ptr(hidden), _ptr(weight), H, B, K, V, _ptr(draft), _ptr(ledger), float(gate),
                                  int(cap), _ptr(o["accepted_len"]), _ptr(o["committed"]), _ptr(o["recovery"]),
                                  _ptr(o.get("row_argmax")), _ptr(o.get("row_regret")), _ptr(o.get("row_top")),
                                  _ptr(o.get("status")), ws.ptr, ws.nbytes, _stream(stream))
    _check("asd_lmhead_verify", rc)
    return o


def lmhead_partials(hidden: torch.Tensor, weight_shard: torch.Tensor, draft: torch.Tensor, v_offset: int, V: int,
                    workspace: Workspace | None = None, out: torch.Tensor | None = None,
                    stream=None) -> torch.Tensor:
    """asd_lmhead_partials: one vocabulary shard of the fused LM-head verify, as int32 [B*(K+1), 6] partials.

    weight_shard [Vs, H] holds rows v_offset .. v_offset+Vs-1 of the LM-head weight; draft holds global ids.
    """
    T, Vs, H = _lm_shapes(hidden, weight_shard)
    B, K = draft.shape
    if T != B * (K + 1):
        raise ValueError("hidden must hold B*(K+1) rows")
    ws = workspace or lmhead_workspace(B, K, Vs, H, hidden.device, stream)
    with _torch_on(stream):
        o = out if out is not None else torch.empty(T, PARTIAL_WORDS, dtype=torch.int32, device=hidden.device)
    _check("asd_lmhead_partials", load().asd_lmhead_partials(_ptr(hidden), _ptr(weight_shard), H, B, K, Vs,
                                                             int(v_offset), int(V), _ptr(draft), _ptr(o), ws.ptr,
                                                             ws.nbytes, _stream(stream)))
    return o


def lmhead_logits(hidden: torch.Tensor, weight: torch.Tensor, out: torch.Tensor | None = None,
                  stream=None) -> torch.Tensor:
    """asd_lmhead_logits: the same tensor-core GEMM, writing the fp32 logits [T, V]."""
    T, V, H = _lm_shapes(hidden, weight)
    with _torch_on(stream):
        o = out if out is not None else torch.empty(T, V, dtype=torch.float32, device=hidden.device)
    _check("asd_lmhead_logits", load().asd_lmhead_logits(_ptr(hidden), _ptr(weight), H, T, V, _ptr(o),
                                                         _stream(stream)))
    return o


def blocks_workspace(nblk: int, B: int, K: int, V: int, dtype: int, device=None, stream=None) -> Workspace:
    n = ctypes.c_size_t(0)
    _check("asd_blocks_workspace_size", load().asd_blocks_workspace_size(nblk, B, K, V, dtype, ctypes.byref(n)))
    ws = Workspace.__new__(Workspace)
    ws.nbytes = n.value
    with _torch_on(stream):
        ws.buffer = torch.empty(max(ws.nbytes, 1), dtype=torch.uint8, device=device or "cuda")
    _check("asd_workspace_init", load().asd_workspace_init(ws.buffer.data_ptr(), ws.nbytes, _stream(stream)))
    return ws


def verify_blocks(logits: torch.Tensor, draft: torch.Tensor, ledger: torch.Tensor, gate: float, cap: int,
                  workspace: Workspace | None = None, out: dict | None = None, stream=None,
                  resident: bool = False) -> dict:
    """asd_verify_blocks: nblk sequential blocks of the same requests in one call.

    logits [nblk, B, K+1, V], draft [nblk, B, K], ledger [B, 2]; outputs carry a
    leading nblk dimension.
    """
    if logits.dim() != 4 or not logits.is_cuda or not logits.is_contiguous():
        raise ValueError("logits must be a contiguous CUDA tensor [nblk, B, K+1, V]")
    nblk, B, K1, V = logits.shape
    K = K1 - 1
    if draft.shape != (nblk, B, K) or draft.dtype != torch.int32 or not draft.is_contiguous():
        raise ValueError("draft must be a contiguous int32 tensor [nblk, B, K]")
    if ledger.shape != (B, 2) or ledger.dtype != torch.float32 or not ledger.is_contiguous():
        raise ValueError("ledger must be a contiguous float32 tensor [B, 2] of (budget, spent)")
    code = _dtype_code(logits)
    ws = workspace or blocks_workspace(nblk, B, K, V, code, logits.device, stream)
    if out is None:
        flat = alloc_outputs(nblk * B, K, logits.device, stream=stream)
        out = {k: v.view(nblk, B, *v.shape[1:]) for k, v in flat.items()}
    rc = load().asd_verify_blocks(_ptr(logits), code | _flag(resident), nblk, B, K, V, _ptr(draft), _ptr(ledger),
                                  float(gate),
                                  int(cap), _ptr(out["accepted_len"]), _ptr(out["committed"]), _ptr(out["recovery"]),
                                  _ptr(out.get("row_argmax")), _ptr(out.get("row_regret")), _ptr(out.get("status")),
                                  ws.ptr, ws.nbytes, _stream(stream))
    _check("asd_verify_blocks", rc)
    return out


def opportunity(row_argmax: torch.Tensor, draft: torch.Tensor, row_regret: torch.Tensor, taus, ps,
                status: torch.Tensor | None = None, counts: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """asd_opportunity: Eq. 4 counts over the block-requests' row outputs (accumulated into ``counts``).

    Returns the int64 counts tensor [len(taus) * len(ps) + 1] (the last entry is |M|).
    """
    import numpy as _np
    n, K1 = row_argmax.shape[0], row_argmax.shape[-1]
    tau = _np.ascontiguousarray(taus, dtype=_np.float32)
    pv = _np.ascontiguousarray(ps, dtype=_np.int32)
    if counts is None:
        with _torch_on(stream):
            counts = torch.zeros(len(tau) * len(pv) + 1, dtype=torch.int64, device=row_argmax.device)
    rc = load().asd_opportunity(_ptr(row_argmax), _ptr(draft), _ptr(row_regret), _ptr(status), n, K1 - 1,
                                tau.ctypes.data, len(tau), pv.ctypes.data, len(pv), _ptr(counts), _stream(stream))
    _check("asd_opportunity", rc)
    return counts


PARTIAL_WORDS = 6  # asd_partial: uint64 key, float top, float draft_logit, uint32 flags, uint32 reserved


def shard_partials(logits: torch.Tensor, draft: torch.Tensor, v_offset: int, V: int,
                   workspace: Workspace | None = None, out: torch.Tensor | None = None, stream=None,
                   resident: bool = False) -> torch.Tensor:
    """asd_shard_partials: one vocabulary shard's per-row partials, as int32 [B*(K+1), 6] (asd_partial).

    logits [B, K+1, Vs] hold vocabulary entries v_offset .. v_offset+Vs-1 of V; draft holds global ids.
    """
    B, K, Vs = _shape(logits, draft)
    code = _dtype_code(logits)
    ws = workspace or Workspace(B, K, Vs, code, logits.device, stream)
    with _torch_on(stream):
        o = out if out is not None else torch.empty(B * (K + 1), PARTIAL_WORDS, dtype=torch.int32,
                                                    device=logits.device)
    rc = load().asd_shard_partials(_ptr(logits), code | _flag(resident), B, K, Vs, int(v_offset), int(V), _ptr(draft),
                                   _ptr(o),
                                   ws.ptr, ws.nbytes, _stream(stream))
    _check("asd_shard_partials", rc)
    return o


def shard_combine(partials: torch.Tensor, draft: torch.Tensor, ledger: torch.Tensor, gate: float, cap: int, V: int,
                  out: dict | None = None, stream=None) -> dict:
    """asd_shard_combine: partials [S, B*(K+1), 6] of all shards -> the outputs of asd_verify."""
    S, R, words = partials.shape
    B, K = draft.shape
    if words != PARTIAL_WORDS or R != B * (K + 1) or partials.dtype != torch.int32 or not partials.is_contiguous():
        raise ValueError("partials must be a contiguous int32 tensor [S, B*(K+1), 6]")
    o = out or alloc_outputs(B, K, partials.device, stream=stream)
    rc = load().asd_shard_combine(_ptr(partials), S, B, K, int(V), _ptr(draft), _ptr(ledger), float(gate), int(cap),
                                  _ptr(o["accepted_len"]), _ptr(o["committed"]), _ptr(o["recovery"]),
                                  _ptr(o.get("row_argmax")), _ptr(o.get("row_regret")), _ptr(o.get("status")),
                                  _stream(stream))
    _check("asd_shard_combine", rc)
    return o


def allgather_partials(part: torch.Tensor, group=None) -> torch.Tensor:
    """The exchange step of tensor-parallel verification: every rank's [B*(K+1), 6] partials -> [S, ...]."""
    import torch.distributed as dist
    world = dist.get_world_size(group)
    parts = [torch.empty_like(part) for _ in range(world)]
    dist.all_gather(parts, part.contiguous(), group=group)
    return torch.stack(parts).contiguous()


def commit(accepted_len: torch.Tensor, committed: torch.Tensor, pending: int = 1, kv_len: torch.Tensor | None = None,
           tokens: torch.Tensor | None = None, token_len: torch.Tensor | None = None,
           status: torch.Tensor | None = None, stream=None) -> None:
    """asd_commit: append the emitted tokens to the history and advance the KV length (in place)."""
    B, K1 = committed.shape
    max_tokens = tokens.shape[1] if tokens is not None else 0
    rc = load().asd_commit(B, K1 - 1, _ptr(accepted_len), _ptr(committed), int(pending), _ptr(kv_len), _ptr(tokens),
                           _ptr(token_len), max_tokens, _ptr(status), _stream(stream))
    _check("asd_commit", rc)


# ---------------------------------------------------------------- the cache side of a verified block

class _Cache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("dtype", ctypes.c_int), ("layers", ctypes.c_int),
                ("pages", ctypes.c_int), ("page_size", ctypes.c_int), ("heads", ctypes.c_int),
                ("head_dim", ctypes.c_int), ("layer_stride", ctypes.c_int64), ("page_stride", ctypes.c_int64),
                ("token_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64), ("page_table", ctypes.c_void_p),
                ("B", ctypes.c_int), ("table_width", ctypes.c_int)]


_CACHE_DTYPES = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}


class KVCache:
    """A paged key/value cache (asd_kv_cache) over the caller's tensors.

    k, v        [layers, pages, page_size, heads, head_dim], or without the first dimension for one layer; float32,
                bfloat16 or float16, the last dimension contiguous, any strides otherwise (the same for both): a
                [pages, heads, page_size, head_dim] cache is passed as its ``transpose(-3, -2)``.
    page_table  int32 [B, table_width]: slot s of request b is place s % page_size of page
                page_table[b, s // page_size].
    """

    def __init__(self, k: torch.Tensor, v: torch.Tensor, page_table: torch.Tensor):
        if k.dim() == 4 and v.dim() == 4:
            k, v = k.unsqueeze(0), v.unsqueeze(0)
        if k.dim() != 5 or k.shape != v.shape or k.stride() != v.stride() or k.dtype != v.dtype:
            raise ValueError("k and v must be [layers, pages, page_size, heads, head_dim] alike, strides included")
        if k.dtype not in _CACHE_DTYPES:
            raise TypeError(f"a cache holds float32, bfloat16 or float16, got {k.dtype}")
        if k.stride(4) != 1 and k.shape[4] > 1:
            raise ValueError("the cache's last dimension must be contiguous")
        if page_table.dim() != 2 or page_table.dtype != torch.int32 or not page_table.is_contiguous():
            raise ValueError("page_table must be a contiguous int32 tensor [B, table_width]")
        if not (k.is_cuda and k.device == v.device == page_table.device):
            raise ValueError("k, v and page_table must be on one CUDA device")
        self.k, self.v, self.page_table = k, v, page_table
        self.dtype, self.device, self.index = k.dtype, k.device, k.get_device()
        self.layers, self.pages, self.page_size, self.heads, self.head_dim = k.shape
        self.B, self.table_width = page_table.shape
        s = k.stride()
        self._c = _Cache(k.data_ptr(), v.data_ptr(), _CACHE_DTYPES[k.dtype], self.layers, self.pages, self.page_size,
                         self.heads, self.head_dim, s[0], s[1], s[2], s[3], page_table.data_ptr(), self.B,
                         self.table_width)
        self._ref = ctypes.addressof(self._c)


# The arguments of asd_append and asd_attention as they lie in memory. One packed block and a call of three arguments:
# as 31 arguments of a ctypes call asd_append took 3.2 us of host time, packed 0.8.
_APPEND = struct.Struct("4P 9q 3P 2P 2P P 6i f i")
_ATTENTION = struct.Struct("3P 3q 3P P P N 3i f")
_I32 = torch.int32


def _check_heads(name: str, t: torch.Tensor, cache: KVCache, shape: tuple) -> tuple:
    """The strides of a [B, T, heads, head_dim] tensor of the cache's type."""
    st = t.stride()
    if t.shape != shape or t.dtype is not cache.dtype or t.get_device() != cache.index or \
            (st[3] != 1 and shape[3] > 1):
        raise ValueError(f"{name} must be a {list(shape)} tensor of the cache's type and device, its last dimension "
                         "contiguous")
    return st


def _check_vector(name: str, t: torch.Tensor, cache: KVCache, shape: tuple, dtype: torch.dtype = _I32) -> int:
    if t.dtype is not dtype or t.shape != shape or t.get_device() != cache.index or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor {list(shape)} on the cache's device")
    return t.data_ptr()


def kv_append(k: torch.Tensor, v: torch.Tensor, cache: KVCache, kv_len: torch.Tensor, layer: int = 0,
              q: torch.Tensor | None = None, q_out: torch.Tensor | None = None,
              positions: torch.Tensor | None = None, new_len: torch.Tensor | None = None,
              cos: torch.Tensor | None = None, sin: torch.Tensor | None = None, interleaved: bool = False,
              q_norm: torch.Tensor | None = None, k_norm: torch.Tensor | None = None, eps: float = 1e-6,
              status: torch.Tensor | None = None, stream=None) -> torch.Tensor | None:
    """asd_kv_append: norm and rotate the new tokens' keys (and queries), append keys and values to one layer.

    k, v [B, T, heads, D] and q [B, T, q_heads, D] may be strided views of a fused projection's rows. cos, sin
    [positions, rot_dim / 2] float32. Returns ``q_out`` (allocated on ``stream`` and zeroed if not given), or None
    without queries.
    """
    B, D = cache.B, cache.head_dim
    T = k.shape[1] if k.dim() == 4 else -1
    shape = (B, T, cache.heads, D)
    ks = _check_heads("k", k, cache, shape)
    vs = _check_heads("v", v, cache, shape)
    if q is None:
        qs, q_heads, qp, op = (0, 0, 0), 0, 0, 0
    else:
        q_heads = q.shape[2] if q.dim() == 4 else -1
        shape = (B, T, q_heads, D)
        qs = _check_heads("q", q, cache, shape)
        if q_out is None:
            with _torch_on(stream):
                q_out = torch.zeros(shape, dtype=q.dtype, device=q.device)
        op, qp = _check_vector("q_out", q_out, cache, shape, cache.dtype), q.data_ptr()
    one = (B,)
    cp = sp = table = rot = 0
    if cos is not None or sin is not None:
        if cos is None or sin is None or cos.dim() != 2:
            raise ValueError("cos and sin must be float32 tensors [positions, rot_dim / 2], both or neither")
        shape = cos.shape
        table, rot = shape[0], 2 * shape[1]
        cp = _check_vector("cos", cos, cache, shape, torch.float32)
        sp = _check_vector("sin", sin, cache, shape, torch.float32)
    args = _APPEND.pack(
        k.data_ptr(), v.data_ptr(), qp, op, ks[0], ks[1], ks[2], vs[0], vs[1], vs[2], qs[0], qs[1], qs[2],
        _check_vector("kv_len", kv_len, cache, one),
        0 if new_len is None else _check_vector("new_len", new_len, cache, one),
        0 if positions is None else _check_vector("positions", positions, cache, (B, T)), cp, sp,
        0 if q_norm is None else _check_vector("q_norm", q_norm, cache, (D,), cache.dtype),
        0 if k_norm is None else _check_vector("k_norm", k_norm, cache, (D,), cache.dtype),
        0 if status is None else _check_vector("status", status, cache, one), layer, T, q_heads, rot, table,
        1 if interleaved else 0, eps, 0)
    rc = load().asd_kv_append(cache._ref, args, _stream(stream))
    if rc:
        raise AsdError("asd_kv_append", rc)
    return None if q is None else q_out


def attention_workspace(cache: KVCache, T: int, q_heads: int, stream=None) -> Workspace:
    """A workspace for tree_attention with up to T tokens per request (asd_attention_workspace_size)."""
    n = ctypes.c_size_t(0)
    _check("asd_attention_workspace_size",
           load().asd_attention_workspace_size(cache._ref, T, q_heads, ctypes.byref(n)))
    ws = Workspace.__new__(Workspace)
    ws.nbytes = n.value
    with _torch_on(stream):
        ws.buffer = torch.empty(ws.nbytes, dtype=torch.uint8, device=cache.device)
    _check("asd_workspace_init", load().asd_workspace_init(ws.buffer.data_ptr(), ws.nbytes, _stream(stream)))
    return ws


def tree_mask(parents: torch.Tensor) -> torch.Tensor:
    """Trees as tree_attention takes them: parents int [B, T] (node t's parent, < t, or -1 for a root) -> int32
    [B, T, ceil(T / 32)], bit u of row t set where u is t itself or one of its ancestors."""
    B, T = parents.shape
    at = torch.arange(T, device=parents.device)
    if bool((parents >= at).any()) or bool((parents < -1).any()):
        raise ValueError("a node's parent must come before it (or be -1)")
    sees = torch.eye(T, dtype=torch.bool, device=parents.device).expand(B, T, T).clone()
    rows = torch.arange(B, device=parents.device)
    for t in range(1, T):
        p = parents[:, t].long()
        sees[:, t] |= sees[rows, p.clamp(min=0)] & (p >= 0)[:, None]
    words = (T + 31) // 32
    bits = torch.zeros(B, T, words * 32, dtype=torch.int64, device=parents.device)
    bits[:, :, :T] = sees.long()
    w = (bits.view(B, T, words, 32) << torch.arange(32, device=parents.device)).sum(-1)
    return (w - ((w >> 31) << 32)).to(torch.int32).contiguous()


def tree_attention(q: torch.Tensor, cache: KVCache, kv_len: torch.Tensor, layer: int = 0,
                   tree_mask: torch.Tensor | None = None, new_len: torch.Tensor | None = None,
                   scale: float | None = None, workspace: Workspace | None = None, out: dict | None = None,
                   status: torch.Tensor | None = None, stream=None) -> dict:
    """asd_tree_attention: the newest T tokens of every request against its context and their own ancestors.

    q [B, T, q_heads, D] (any strides, last dimension contiguous); ``tree_mask`` int32 [B, T, ceil(T / 32)] or None
    for a chain; ``scale`` defaults to 1 / sqrt(D). Returns {"out": [B, T, q_heads, D], "lse": float32 [B, T, q_heads]};
    an ``out`` dict without "lse" leaves it out. Outputs and a workspace that are not given are allocated on ``stream``.
    """
    B, D = cache.B, cache.head_dim
    T, q_heads = q.shape[1:3] if q.dim() == 4 else (-1, -1)
    shape, rows = (B, T, q_heads, D), (B, T, q_heads)
    qs = _check_heads("q", q, cache, shape)
    if out is None:
        with _torch_on(stream):
            out = {"out": torch.empty(shape, dtype=q.dtype, device=q.device),
                   "lse": torch.empty(rows, dtype=torch.float32, device=q.device)}
    lse = out.get("lse")
    ws = workspace or attention_workspace(cache, T, q_heads, stream)
    args = _ATTENTION.pack(
        q.data_ptr(), _check_vector("out", out["out"], cache, shape, cache.dtype),
        0 if lse is None else _check_vector("lse", lse, cache, rows, torch.float32), qs[0], qs[1], qs[2],
        _check_vector("kv_len", kv_len, cache, (B,)),
        0 if new_len is None else _check_vector("new_len", new_len, cache, (B,)),
        0 if tree_mask is None else _check_vector("tree_mask", tree_mask, cache, (B, T, (T + 31) // 32)),
        0 if status is None else _check_vector("status", status, cache, (B,)), ws.buffer.data_ptr(), ws.nbytes, layer,
        T, q_heads, D ** -0.5 if scale is None else scale)
    rc = load().asd_tree_attention(cache._ref, args, _stream(stream))
    if rc:
        raise AsdError("asd_tree_attention", rc)
    return out


def kv_compact(cache: KVCache, kv_len: torch.Tensor, path: torch.Tensor, path_len: torch.Tensor,
               status: torch.Tensor | None = None, stream=None) -> None:
    """asd_kv_compact: move a verified path's keys and values next to the context, in every layer (in place).

    path int32 [B, P], ascending tree nodes with path[b, i] >= i; path_len int32 [B].
    """
    B = cache.B
    P = path.shape[1] if path.dim() == 2 else -1
    rc = load().asd_kv_compact(cache._ref, P, _check_vector("kv_len", kv_len, cache, (B,)),
                               _check_vector("path", path, cache, (B, P)),
                               _check_vector("path_len", path_len, cache, (B,)),
                               None if status is None else _check_vector("status", status, cache, (B,)),
                               _stream(stream))
    if rc:
        raise AsdError("asd_kv_compact", rc)


# asd_weigh and asd_evict as they lie in memory
_WEIGH = struct.Struct("2P 3q 2P 3P P d f 5i")
_EVICT = struct.Struct("6P 4i")


def kv_weigh(q: torch.Tensor, lse: torch.Tensor, cache: KVCache, kv_len: torch.Tensor, weight: torch.Tensor | None,
             layer: int = 0, decay: float = 1.0, new_len: torch.Tensor | None = None,
             path: torch.Tensor | None = None, scale: float | None = None, out: torch.Tensor | None = None,
             status: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """asd_kv_weigh: add to every cached slot's weight what the rows of a pass gave it.

    q [B, T, q_heads, D] and lse [B, T, q_heads] as tree_attention took and left them; weight float32 [B, heads,
    width], one layer's, is written in place or to ``out`` (``None`` with ``decay=0`` and ``out``). Row i of a request
    is token i, or token ``path[b, i]`` of int32 [B, rows], and sees the new slots kv_len .. kv_len + i; ``new_len``
    int32 [B] counts a request's rows. A call that gave up waiting shows in ``status`` and in ``weigh_error()``.
    """
    B, D = cache.B, cache.head_dim
    T, q_heads = q.shape[1:3] if q.dim() == 4 else (-1, -1)
    qs = _check_heads("q", q, cache, (B, T, q_heads, D))
    if out is None:
        out = weight
    if out is None:
        raise ValueError("kv_weigh needs a weight tensor or out")
    width = out.shape[2] if out.dim() == 3 else -1
    shape = (B, cache.heads, width)
    rows = T
    if path is not None:
        rows = path.shape[1] if path.dim() == 2 else -1
    args = _WEIGH.pack(
        q.data_ptr(), _check_vector("lse", lse, cache, (B, T, q_heads), torch.float32), qs[0], qs[1], qs[2],
        0 if weight is None else _check_vector("weight", weight, cache, shape, torch.float32),
        _check_vector("out", out, cache, shape, torch.float32), _check_vector("kv_len", kv_len, cache, (B,)),
        0 if new_len is None else _check_vector("new_len", new_len, cache, (B,)),
        0 if path is None else _check_vector("path", path, cache, (B, rows)),
        0 if status is None else _check_vector("status", status, cache, (B,)), D ** -0.5 if scale is None else scale,
        decay, layer, T, rows, q_heads, width)
    rc = load().asd_kv_weigh(cache._ref, args, _stream_at(stream, cache.index))
    if rc:
        raise AsdError("asd_kv_weigh", rc)
    return out


def weigh_error(stream=None) -> int:
    """asd_weigh_error: whether a kv_weigh on the current device has given up a wait since the last time.

    0, or 9 (ASD_ERR_TIMEOUT): weights that it was to write may be missing. Synchronises the stream.
    """
    word = ctypes.c_int(0)
    rc = load().asd_weigh_error(ctypes.byref(word), _stream(stream))
    if rc:
        raise AsdError("asd_weigh_error", rc)
    return word.value


def kv_evict(cache: KVCache, kv_len: torch.Tensor, weight: torch.Tensor, keep: torch.Tensor, first: int = 0,
             last: int = 0, out: torch.Tensor | None = None, new_len: torch.Tensor | None = None,
             status: torch.Tensor | None = None, stream=None, numbers: torch.Tensor | None = None,
             tokens: torch.Tensor | None = None) -> torch.Tensor:
    """asd_kv_evict: cut every request's cache to ``keep[b]`` slots, in every layer and in place.

    weight float32 [layers, B, heads, width] (or without the first dimension for one layer), moved with the slots in
    place or to ``out``. The first ``first`` and the last ``last`` slots stay. Pages that two requests' tables share are
    not for this: each would move the other's slots. Returns the new lengths, int32 [B] (``new_len``, allocated on
    ``stream`` if not given; not ``kv_len`` itself).

    The last slots are the newest tokens only where at least ``last`` tokens were appended since the last eviction. A
    loop that evicts more often passes ``numbers`` int32, of weight's shape, filled with -1 for each new request, and
    ``tokens`` int32 [B], how many the request's cache has been given in all (asd_kv_evict_numbered): the newest
    ``last`` tokens stay wherever they lie, and ``numbers`` says afterwards which token a slot holds.
    """
    B = cache.B
    one = (B,)
    shape = (cache.layers, B, cache.heads, weight.shape[-1] if weight.dim() else -1)
    if weight.dim() == 3 and cache.layers == 1:
        shape = shape[1:]
    to = weight if out is None else out
    if new_len is None:
        with _torch_on(stream):
            new_len = torch.empty(one, dtype=_I32, device=cache.device)
    args = _EVICT.pack(_check_vector("weight", weight, cache, shape, torch.float32),
                       _check_vector("out", to, cache, shape, torch.float32),
                       _check_vector("kv_len", kv_len, cache, one), _check_vector("new_len", new_len, cache, one),
                       _check_vector("keep", keep, cache, one),
                       0 if status is None else _check_vector("status", status, cache, one), first, last, shape[-1], 0)
    if numbers is None and tokens is None:
        rc = load().asd_kv_evict(cache._ref, args, _stream_at(stream, cache.index))
    elif numbers is None or tokens is None:
        raise ValueError("numbers and tokens go together")
    else:
        rc = load().asd_kv_evict_numbered(cache._ref, args, _check_vector("numbers", numbers, cache, shape),
                                          _check_vector("tokens", tokens, cache, one),
                                          _stream_at(stream, cache.index))
    if rc:
        raise AsdError("asd_kv_evict", rc)
    return new_len


# ---------------------------------------------------------------- logits under rules

_RULES = struct.Struct("6P 2q 2i")           # asd_token_rules
_RULES_BLOCK = struct.Struct("10P N 2i f i")  # asd_rules_block


class TokenRules:
    """What a batch's requests know of their tokens, and their penalties (asd_token_rules).

    marks       int32 [B, ceil(V / 32)]: bit v % 32 of word v / 32 set where token v has a record
    records     int32 [B, V, 2]: (TOKEN_PROMPT if in the prompt | times said, the bits of a float32 bias)
    repetition, frequency, presence  float32 [B] or None (no such penalty)

    The tensors stay the caller's, who writes new values into them (calls keep to the tensors given here); tokens_record
    and tokens_bias write the first two. ``TokenRules.empty(B, V)`` makes them, ``clear(b)`` empties a request's row for
    its next user.
    """

    def __init__(self, marks: torch.Tensor, records: torch.Tensor, repetition: torch.Tensor | None = None,
                 frequency: torch.Tensor | None = None, presence: torch.Tensor | None = None):
        if records.dim() != 3 or records.shape[2] != 2 or records.dtype is not _I32 or not records.is_contiguous():
            raise ValueError("records must be a contiguous int32 tensor [B, V, 2]")
        B, V = records.shape[:2]
        words = (V + 31) // 32
        if marks.shape != (B, words) or marks.dtype is not _I32 or not marks.is_contiguous():
            raise ValueError("marks must be a contiguous int32 tensor [B, ceil(V / 32)]")
        if not (records.is_cuda and marks.device == records.device):
            raise ValueError("marks and records must be on one CUDA device")
        for name, t in (("repetition", repetition), ("frequency", frequency), ("presence", presence)):
            if t is not None and (t.shape != (B,) or t.dtype is not torch.float32 or not t.is_contiguous() or
                                  t.device != records.device):
                raise ValueError(f"{name} must be a contiguous float32 tensor [B] on the records' device")
        self.marks, self.records = marks, records
        self.repetition, self.frequency, self.presence = repetition, frequency, presence
        self.B, self.V, self.words = B, V, words
        self.device, self.index = records.device, records.get_device()
        self._head = (marks.data_ptr(), records.data_ptr(), _ptr(repetition) or 0, _ptr(frequency) or 0,
                      _ptr(presence) or 0)
        self._plain = _RULES.pack(*self._head, 0, 0, 0, B, V)

    @classmethod
    def empty(cls, B: int, V: int, repetition: torch.Tensor | None = None, frequency: torch.Tensor | None = None,
              presence: torch.Tensor | None = None, device="cuda", stream=None) -> "TokenRules":
        with _torch_on(stream):
            marks = torch.zeros(B, (V + 31) // 32, dtype=_I32, device=device)
            records = torch.zeros(B, V, 2, dtype=_I32, device=device)
        return cls(marks, records, repetition, frequency, presence)

    def clear(self, b: int, stream=None) -> None:
        """Forget what is known of request b's tokens."""
        with _torch_on(stream):
            self.marks[b].zero_()
            self.records[b].zero_()

    def _pack(self, allow: torch.Tensor | None, rows: int) -> bytes:
        if allow is None:
            return self._plain
        strides = allow.stride()
        if allow.shape != (self.B, rows, self.words) or allow.dtype is not _I32 or allow.get_device() != self.index or \
                (strides[2] != 1 and self.words > 1):
            raise ValueError(f"allow must be an int32 tensor {[self.B, rows, self.words]} on the rules' device, its "
                             "last dimension contiguous")
        return _RULES.pack(*self._head, allow.data_ptr(), strides[0], strides[1], self.B, self.V)


def _check_rules(rules: TokenRules, name: str, t: torch.Tensor, shape: tuple, dtype: torch.dtype = _I32) -> int:
    if t.dtype is not dtype or t.shape != shape or t.get_device() != rules.index or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor {list(shape)} on the rules' device")
    return t.data_ptr()


def rules_verify(logits: torch.Tensor, draft: torch.Tensor, ledger: torch.Tensor | None, gate: float, cap: int,
                 rules: TokenRules, allow: torch.Tensor | None = None, workspace: Workspace | None = None,
                 out: dict | None = None, stream=None, flag_empty: bool = False) -> dict:
    """asd_rules_verify: ``verify`` of the logits under the rules (``verify_strict`` with ``ledger=None``).

    logits [B, K+1, V] float32 or bfloat16; row j counts the drafts before it. ``allow`` int32 [B, K+1, ceil(V / 32)]:
    a bit a token that the grammar lets come (strides of 0 for masks that several rows share). Workspaces are verify's.
    A draft that may not come (changed logit -inf) is never accepted. ``flag_empty``: a request whose recovery token
    stands for a row in which no token may come (its 0 means nothing then) has STATUS_EMPTY_ROW in its status.
    """
    shape, index = logits.shape, rules.index
    if len(shape) != 3 or shape[0] != rules.B or shape[2] != rules.V or logits.get_device() != index or \
            not logits.is_contiguous():
        raise ValueError(f"logits must be a contiguous [{rules.B}, K+1, {rules.V}] tensor on the rules' device")
    B, K = shape[0], shape[1] - 1
    code = _dtype_code(logits)
    xp = _check_rules(rules, "draft", draft, (B, K))
    lp = 0 if ledger is None else _check_rules(rules, "ledger", ledger, (B, 2), torch.float32)
    packed = rules._plain if allow is None else rules._pack(allow, K + 1)
    ws = workspace or Workspace(B, K, rules.V, code, logits.device, stream)
    o = out or alloc_outputs(B, K, logits.device, stream=stream)
    argmax, regret, status = o.get("row_argmax"), o.get("row_regret"), o.get("status")
    block = _RULES_BLOCK.pack(
        logits.data_ptr(), xp, lp, o["accepted_len"].data_ptr(), o["committed"].data_ptr(), o["recovery"].data_ptr(),
        0 if argmax is None else argmax.data_ptr(), 0 if regret is None else regret.data_ptr(),
        0 if status is None else status.data_ptr(), ws.buffer.data_ptr(), ws.nbytes,
        code | FLAG_EMPTY_ROWS if flag_empty else code, K, gate, cap)
    rc = load().asd_rules_verify(packed, block, _stream_at(stream, index))
    if rc:
        raise AsdError("asd_rules_verify", rc)
    return o


def rules_logits(logits: torch.Tensor, draft: torch.Tensor | None, rules: TokenRules,
                 allow: torch.Tensor | None = None, out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """asd_rules_logits: the logits [B, rows, V] under the rules, in ``out`` (which may be ``logits`` itself).

    draft int32 [B, rows - 1], or None where no row continues drafts; ``allow`` as in rules_verify.
    """
    if logits.dim() != 3 or logits.shape[0] != rules.B or logits.shape[2] != rules.V:
        raise ValueError(f"logits must be [{rules.B}, rows, {rules.V}] like the rules")
    shape = tuple(logits.shape)
    rows = shape[1]
    code = _dtype_code(logits)
    zp = _check_rules(rules, "logits", logits, logits.shape, logits.dtype)
    xp = None if draft is None else _check_rules(rules, "draft", draft, (rules.B, rows - 1))
    packed = rules._pack(allow, rows)
    if out is None:
        with _torch_on(stream):
            out = torch.empty(shape, dtype=logits.dtype, device=logits.device)
    rc = load().asd_rules_logits(packed, zp, code, rows, xp, _check_rules(rules, "out", out, shape, logits.dtype),
                                 _stream_at(stream, rules.index))
    if rc:
        raise AsdError("asd_rules_logits", rc)
    return out


def tokens_record(tokens: torch.Tensor, rules: TokenRules, prompt: bool = False,
                  token_len: torch.Tensor | None = None, status: torch.Tensor | None = None, stream=None) -> None:
    """asd_tokens_record: add int32 tokens [B, n] to the records, as said or as the prompt's; negative ids are skipped.

    ``verify``'s "committed" can be passed as it is; ``token_len`` int32 [B] says how many of the n a request has.
    """
    n = tokens.shape[1] if tokens.dim() == 2 else -1
    one = (rules.B,)
    rc = load().asd_tokens_record(rules._plain, _check_rules(rules, "tokens", tokens, (rules.B, n)), n,
                                  None if token_len is None else _check_rules(rules, "token_len", token_len, one),
                                  int(bool(prompt)),
                                  None if status is None else _check_rules(rules, "status", status, one),
                                  _stream_at(stream, rules.index))
    if rc:
        raise AsdError("asd_tokens_record", rc)


def tokens_bias(ids: torch.Tensor, bias: torch.Tensor, rules: TokenRules, length: torch.Tensor | None = None,
                status: torch.Tensor | None = None, stream=None) -> None:
    """asd_tokens_bias: set the bias of int32 ids [B, n] to float32 values [B, n]; the later one of an id counts."""
    n = ids.shape[1] if ids.dim() == 2 else -1
    one = (rules.B,)
    rc = load().asd_tokens_bias(rules._plain, _check_rules(rules, "ids", ids, (rules.B, n)),
                                _check_rules(rules, "bias", bias, (rules.B, n), torch.float32), n,
                                None if length is None else _check_rules(rules, "length", length, one),
                                None if status is None else _check_rules(rules, "status", status, one),
                                _stream_at(stream, rules.index))
    if rc:
        raise AsdError("asd_tokens_bias", rc)
