"""Python binding of libcachespec.so: the same entry points, argument marshalling only.

Every step of the draft-and-verify path runs in the library's CUDA kernels;
this module checks tensor dtypes, shapes and devices, passes raw device
pointers and the current CUDA stream through ctypes, and turns a non-OK
status into an exception.  It never computes any part of the method and has
no CPU fallback: if the library is missing, every call raises.  The calls
of a step go through the compiled module ``_marshal``, which does the same
checks and passes on what it does not take to the code here.
"""
from __future__ import annotations

import contextlib
import ctypes
import importlib.machinery
import importlib.util
import os
import threading
from typing import NamedTuple

import torch

from . import build as _build

CS_OK, CS_ERR_INVALID_ARG, CS_ERR_UNSUPPORTED, CS_ERR_CUDA, CS_ERR_WORKSPACE = range(5)
CS_F32, CS_BF16 = 0, 1
CS_DEVICE_WAIT_TIMEOUT = 1   # device status bit: a bounded wait inside a kernel gave up
STATUS_NAMES = {0: "CS_OK", 1: "CS_ERR_INVALID_ARG", 2: "CS_ERR_UNSUPPORTED", 3: "CS_ERR_CUDA",
                4: "CS_ERR_WORKSPACE"}
EXPORTED_SYMBOLS = ("cs_abi_version", "cs_last_error", "cs_verify_attention_workspace_bytes",
                    "cs_verify_attention", "cs_spec_accept_workspace_bytes", "cs_spec_accept",
                    "cs_read_device_status", "cs_verify_attention_noalloc", "cs_verify_attention_noalloc_status",
                    "cs_sample_workspace_bytes",
                    "cs_sample", "cs_kv_append", "cs_kv_commit", "cs_route_workspace_bytes",
                    "cs_route_norms", "cs_route", "cs_tree_verify_attention_workspace_bytes",
                    "cs_tree_verify_attention", "cs_tree_accept_workspace_bytes", "cs_tree_accept",
                    "cs_kv_commit_tree", "cs_selftest_wait_timeout",
                    "cs_packed_kv_append", "cs_packed_kv_read", "cs_packed_verify_attention_workspace_bytes",
                    "cs_packed_verify_attention", "cs_kv_fork_workspace_bytes", "cs_kv_fork", "cs_kv_release",
                    "cs_kv_compact_workspace_bytes", "cs_kv_compact", "cs_logprobs", "cs_kv_fork_more",
                    "cs_kv_compact_more", "cs_rope_kv_append", "cs_packed_rope_kv_append",
                    "cs_chunk_attention_workspace_bytes", "cs_chunk_attention")
CS_MAX_TOP = 32
CS_MAX_PAGE_POOLS = 128


class RouteDims(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("n_groups", ctypes.c_int32), ("dim", ctypes.c_int32)]


class AttnDims(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("n_q_heads", ctypes.c_int32),
                ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("max_pages_per_seq", ctypes.c_int32),
                ("num_pages", ctypes.c_int32), ("sm_scale", ctypes.c_float)]


class AcceptDims(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("vocab", ctypes.c_int32),
                ("logit_dtype", ctypes.c_int32)]


class PackedPoolPtrs(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("k_codes", "k_scales", "v_codes", "v_scales", "k_head_scale",
                                               "v_head_scale")]


class PageDims(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int32), ("max_pages_per_seq", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("num_pages", ctypes.c_int32)]


class PagePool(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("page_bytes", ctypes.c_size_t)]


class LogprobDims(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int32), ("vocab", ctypes.c_int32), ("logit_dtype", ctypes.c_int32),
                ("n_top", ctypes.c_int32), ("row_stride", ctypes.c_int64)]


class RopeDims(ctypes.Structure):
    _fields_ = [("tokens", ctypes.c_int32), ("rot_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32),
                ("n_positions", ctypes.c_int32), ("norm_eps", ctypes.c_float), ("q_stride", ctypes.c_int64),
                ("k_stride", ctypes.c_int64), ("v_stride", ctypes.c_int64), ("q_out_stride", ctypes.c_int64)]


class PackedPool(NamedTuple):
    """A K/V cache in 4 bits a value: codes uint8 [P, Hkv, ps, 64] (two dims a byte, the even one in the low four
    bits), scales float8_e4m3fn [P, Hkv, ps, 8] (one for 16 dims) and, optionally, fp32 [Hkv] scales of the heads.
    See include/cachespec.h."""
    k_codes: torch.Tensor
    k_scales: torch.Tensor
    v_codes: torch.Tensor
    v_scales: torch.Tensor
    k_head_scale: torch.Tensor | None = None
    v_head_scale: torch.Tensor | None = None


class CacheSpecError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {message}")
        self.status = status


_lib = None
_lock = threading.Lock()


def library_path() -> str:
    return _build.LIB


def load_library(path: str | None = None):
    """Load libcachespec.so (built in-tree by ``__graft_entry__.build()``).  Raises if absent."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    with _lock:
        if _lib is not None and path is None:
            return _lib
        p = path or _build.LIB
        if not os.path.exists(p):
            raise RuntimeError(f"libcachespec.so not found at {p}; build it with "
                               "`python -c 'import __graft_entry__ as g; g.build()'`")
        lib = ctypes.CDLL(p)
        vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
        lib.cs_abi_version.restype = i32
        lib.cs_last_error.restype = ctypes.c_char_p
        lib.cs_verify_attention_workspace_bytes.restype = sz
        lib.cs_verify_attention_workspace_bytes.argtypes = [ctypes.POINTER(AttnDims), i32]
        lib.cs_verify_attention.restype = ctypes.c_int
        lib.cs_verify_attention.argtypes = [ctypes.POINTER(AttnDims), vp, vp, vp, vp, vp, i32, vp,
                                            vp, sz, vp]
        lib.cs_spec_accept_workspace_bytes.restype = sz
        lib.cs_spec_accept_workspace_bytes.argtypes = [ctypes.POINTER(AcceptDims), i32]
        lib.cs_spec_accept.restype = ctypes.c_int
        lib.cs_spec_accept.argtypes = [ctypes.POINTER(AcceptDims), vp, vp, vp, vp, i32,
                                       ctypes.c_float, vp, vp, vp, sz, vp]
        lib.cs_verify_attention_noalloc.restype = ctypes.c_int
        lib.cs_verify_attention_noalloc.argtypes = [ctypes.POINTER(AttnDims), vp, vp, vp, vp, vp,
                                                    i32, vp, vp]
        lib.cs_verify_attention_noalloc_status.restype = ctypes.c_int
        lib.cs_verify_attention_noalloc_status.argtypes = [ctypes.POINTER(ctypes.c_int32), vp]
        lib.cs_read_device_status.restype = ctypes.c_int
        lib.cs_read_device_status.argtypes = [vp, ctypes.POINTER(ctypes.c_int32), vp]
        lib.cs_selftest_wait_timeout.restype = ctypes.c_int
        lib.cs_selftest_wait_timeout.argtypes = [vp, vp]
        lib.cs_kv_append.restype = ctypes.c_int
        lib.cs_kv_append.argtypes = [ctypes.POINTER(AttnDims), vp, vp, vp, vp, vp, vp, i32, vp]
        lib.cs_kv_commit.restype = ctypes.c_int
        lib.cs_kv_commit.argtypes = [i32, vp, vp, i32, vp]
        lib.cs_route_workspace_bytes.restype = sz
        lib.cs_route_workspace_bytes.argtypes = [ctypes.POINTER(RouteDims)]
        lib.cs_route_norms.restype = ctypes.c_int
        lib.cs_route_norms.argtypes = [i32, i32, vp, vp, vp]
        lib.cs_route.restype = ctypes.c_int
        lib.cs_route.argtypes = [ctypes.POINTER(RouteDims), vp, vp, vp, ctypes.c_float, vp, vp, vp, vp, sz, vp]
        lib.cs_sample_workspace_bytes.restype = sz
        lib.cs_sample_workspace_bytes.argtypes = [ctypes.POINTER(AcceptDims)]
        lib.cs_sample.restype = ctypes.c_int
        lib.cs_sample.argtypes = [ctypes.POINTER(AcceptDims), vp, vp, ctypes.c_float, vp, vp, sz, vp]
        lib.cs_tree_verify_attention_workspace_bytes.restype = sz
        lib.cs_tree_verify_attention_workspace_bytes.argtypes = [ctypes.POINTER(AttnDims), i32]
        lib.cs_tree_verify_attention.restype = ctypes.c_int
        lib.cs_tree_verify_attention.argtypes = [ctypes.POINTER(AttnDims), vp, vp, vp, vp, vp, vp, i32, vp,
                                                 vp, sz, vp]
        lib.cs_tree_accept_workspace_bytes.restype = sz
        lib.cs_tree_accept_workspace_bytes.argtypes = [ctypes.POINTER(AcceptDims), i32]
        lib.cs_tree_accept.restype = ctypes.c_int
        lib.cs_tree_accept.argtypes = [ctypes.POINTER(AcceptDims), vp, vp, vp, vp, vp, i32, ctypes.c_float,
                                       vp, vp, vp, vp, sz, vp]
        lib.cs_packed_kv_append.restype = ctypes.c_int
        lib.cs_packed_kv_append.argtypes = [ctypes.POINTER(AttnDims), ctypes.POINTER(PackedPoolPtrs), vp, vp, vp, vp, i32,
                                            vp]
        lib.cs_packed_kv_read.restype = ctypes.c_int
        lib.cs_packed_kv_read.argtypes = [ctypes.POINTER(AttnDims), ctypes.POINTER(PackedPoolPtrs), vp, vp, i32, vp, vp, vp]
        lib.cs_packed_verify_attention_workspace_bytes.restype = sz
        lib.cs_packed_verify_attention_workspace_bytes.argtypes = [ctypes.POINTER(AttnDims), i32]
        lib.cs_packed_verify_attention.restype = ctypes.c_int
        lib.cs_packed_verify_attention.argtypes = [ctypes.POINTER(AttnDims), vp, ctypes.POINTER(PackedPoolPtrs), vp, vp, i32,
                                                   vp, vp, sz, vp]
        lib.cs_kv_fork_workspace_bytes.restype = sz
        lib.cs_kv_fork_workspace_bytes.argtypes = [ctypes.POINTER(PageDims), i32]
        lib.cs_kv_fork.restype = ctypes.c_int
        lib.cs_kv_fork.argtypes = [ctypes.POINTER(PageDims), ctypes.POINTER(PagePool), i32, vp, vp, vp, vp, vp, i32, i32, vp,
                                   vp, sz, vp]
        lib.cs_kv_release.restype = ctypes.c_int
        lib.cs_kv_release.argtypes = [ctypes.POINTER(PageDims), vp, vp, vp, vp, vp, i32, vp]
        lib.cs_kv_compact_workspace_bytes.restype = sz
        lib.cs_kv_compact_workspace_bytes.argtypes = [ctypes.POINTER(PageDims)]
        lib.cs_kv_compact.restype = ctypes.c_int
        lib.cs_kv_compact.argtypes = [ctypes.POINTER(PageDims), ctypes.POINTER(PagePool), i32, vp, vp, vp, vp, sz, vp]
        lib.cs_kv_fork_more.restype = ctypes.c_int
        lib.cs_kv_fork_more.argtypes = [ctypes.POINTER(PageDims), ctypes.POINTER(PagePool), i32, i32, vp, sz, vp]
        lib.cs_kv_compact_more.restype = ctypes.c_int
        lib.cs_kv_compact_more.argtypes = [ctypes.POINTER(PageDims), ctypes.POINTER(PagePool), i32, vp, sz, vp]
        lib.cs_logprobs.restype = ctypes.c_int
        lib.cs_logprobs.argtypes = [ctypes.POINTER(LogprobDims), vp, vp, ctypes.c_float, vp, vp, vp, vp, vp]
        lib.cs_rope_kv_append.restype = ctypes.c_int
        lib.cs_rope_kv_append.argtypes = [ctypes.POINTER(AttnDims), ctypes.POINTER(RopeDims), *[vp] * 14]
        lib.cs_packed_rope_kv_append.restype = ctypes.c_int
        lib.cs_packed_rope_kv_append.argtypes = [ctypes.POINTER(AttnDims), ctypes.POINTER(RopeDims), *[vp] * 8,
                                                 ctypes.POINTER(PackedPoolPtrs), *[vp] * 4]
        lib.cs_chunk_attention_workspace_bytes.restype = sz
        lib.cs_chunk_attention_workspace_bytes.argtypes = [ctypes.POINTER(AttnDims), i32]
        lib.cs_chunk_attention.restype = ctypes.c_int
        lib.cs_chunk_attention.argtypes = [ctypes.POINTER(AttnDims), vp, ctypes.c_int64, i32, vp, vp, vp, vp, vp, vp, vp,
                                           sz, vp]
        lib.cs_kv_commit_tree.restype = ctypes.c_int
        lib.cs_kv_commit_tree.argtypes = [ctypes.POINTER(AttnDims), vp, vp, vp, vp, vp, vp, i32, vp]
        if path is None:
            _lib = lib
        return lib


_fast = None


def _load_fast():
    """The compiled marshalling module, beside the library.  Raises if absent."""
    global _fast
    load_library()
    with _lock:
        if _fast is None:
            if not os.path.exists(_build.MARSHAL):
                raise RuntimeError(f"{os.path.basename(_build.MARSHAL)} not found at {_build.MARSHAL}; build it with "
                                   "`python -c 'import __graft_entry__ as g; g.build()'`")
            name = __package__ + "._marshal"
            loader = importlib.machinery.ExtensionFileLoader(name, _build.MARSHAL)
            mod = importlib.util.module_from_spec(importlib.util.spec_from_file_location(name, _build.MARSHAL,
                                                                                         loader=loader))
            loader.exec_module(mod)
            mod.use_workspaces(lambda kind, index, n, stream: _workspace_of(kind, torch.device("cuda", index), n, stream))
            _fast = mod
    return _fast


def _done(r):
    """A result of the marshalling module; a status (an int) raises."""
    if type(r) is int:
        _check(load_library(), r)
    return r


def _check(lib, status: int) -> None:
    if status != CS_OK:
        raise CacheSpecError(status, lib.cs_last_error().decode(errors="replace"))


def _ptr(t: torch.Tensor | None) -> int | None:
    return None if t is None else t.data_ptr()


# The current stream's handle without a torch.cuda.Stream object around it
# (2 us a call less on the host).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(device: torch.device) -> int:
    if _raw_stream is not None and device.index is not None:
        return _raw_stream(device.index)
    return torch.cuda.current_stream(device).cuda_stream


def _need(t: torch.Tensor, name: str, dtype: torch.dtype, ndim: int, device) -> None:
    if (isinstance(t, torch.Tensor) and t.dtype is dtype and t.dim() == ndim and t.is_cuda and t.is_contiguous()
            and (device is None or t.device == device)):
        return
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.dim() != ndim:
        raise ValueError(f"{name} must have {ndim} dims, got shape {tuple(t.shape)}")
    if not t.is_cuda or (device is not None and t.device != device):
        raise ValueError(f"{name} must live on {device or 'a CUDA device'}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


def attn_dims(q: torch.Tensor, k_pages: torch.Tensor, page_table: torch.Tensor,
              sm_scale: float = 0.0) -> AttnDims:
    B, _, Hq, D = q.shape
    P, Hkv, ps, _ = k_pages.shape
    return AttnDims(B, Hq, Hkv, D, ps, page_table.shape[1], P, float(sm_scale))


# Workspaces handed out by this module, one per (kind, device, stream, size): the
# kernels leave a workspace ready for the next call, so calls ordered on one
# stream may share it, and calls on two streams may not.  They stay for the
# process's life (a captured graph holds their addresses).
_workspaces: dict = {}
_WITH_STATUS = ("attn", "tree_attn", "route", "chunk_attn")   # whose first word has to start at zero
_WITH_COUNTS = ("chunk_attn",)                                # and words that results depend on


def _made_on(stream: int, device):
    """The context in which a new workspace's memory, and its zero fill, are ordered with the calls on ``stream``."""
    if device.type != "cuda" or stream == _stream(device):
        return contextlib.nullcontext()
    if stream in (0, 1):   # the legacy default stream's two handles
        return torch.cuda.stream(torch.cuda.default_stream(device))
    return torch.cuda.stream(torch.cuda.ExternalStream(stream, device=device))


def _workspace_of(kind: str, device, n: int, stream: int | None = None):
    """(workspace, whether it is the stream's own)"""
    device = torch.device(device)   # "cuda:0", "cuda" and the device itself are one key
    if device.index is None and device.type == "cuda":
        device = torch.device("cuda", torch.cuda.current_device())
    here = _stream(device) if device.type == "cuda" else 0
    if stream is None:
        stream = here
    else:   # as ctypes takes it
        stream = (stream if isinstance(stream, ctypes.c_void_p) else ctypes.c_void_p(stream)).value or 0
    key = (kind, device, stream, n)
    ws = _workspaces.get(key)
    if ws is not None:
        return ws, True
    with _made_on(stream, device):
        captured = kind in _WITH_STATUS and device.type == "cuda" and torch.cuda.is_current_stream_capturing()
        if captured:
            # a zero fill would become a part of the graph, so a captured call takes
            # the workspace of the calls before the capture (with whose stream the
            # graph's replays have to be ordered)
            for (k, d, _, m), ws in list(_workspaces.items()):
                if (k, d, m) == (kind, device, n):
                    return ws, False
        ws = (torch.zeros if kind in _WITH_STATUS else torch.empty)(max(n, 256), dtype=torch.uint8, device=device)
    if captured and kind in _WITH_COUNTS:
        return ws, False   # the fill is the graph's: for nobody else is this memory zero
    return _workspaces.setdefault(key, ws), True


def _cached_workspace(kind: str, device, n: int, stream: int | None = None) -> torch.Tensor:
    return _workspace_of(kind, device, n, stream)[0]


def verify_attention_workspace(dims: AttnDims, n_draft: int, device) -> torch.Tensor:
    """The default workspace of the current stream's calls."""
    n = load_library().cs_verify_attention_workspace_bytes(ctypes.byref(dims), int(n_draft))
    return _cached_workspace("attn", device, n)


def cs_verify_attention_workspace_bytes(q, k_pages, page_table, n_draft, sm_scale=0.0) -> int:
    lib = load_library()
    d = attn_dims(q, k_pages, page_table, sm_scale)
    return int(lib.cs_verify_attention_workspace_bytes(ctypes.byref(d), int(n_draft)))


def cs_verify_attention(q, k_pages, v_pages, page_table, ctx_lens, n_draft, out=None,
                        workspace=None, sm_scale: float = 0.0, stream: int | None = None):
    """Verify attention; returns ``out`` (bf16 [B, k+1, Hq, D]).  See include/cachespec.h."""
    r = (_fast or _load_fast()).verify_attention(q, k_pages, v_pages, page_table, ctx_lens, n_draft, out, workspace,
                                                 sm_scale, stream)
    if r is not None:
        return _done(r)
    lib = load_library()
    dev = q.device
    _need(q, "q", torch.bfloat16, 4, dev)
    _need(k_pages, "k_pages", torch.bfloat16, 4, dev)
    _need(v_pages, "v_pages", torch.bfloat16, 4, dev)
    _need(page_table, "page_table", torch.int32, 2, dev)
    _need(ctx_lens, "ctx_lens", torch.int32, 1, dev)
    if v_pages.shape != k_pages.shape:
        raise ValueError("k_pages and v_pages must have the same shape")
    if q.shape[1] != n_draft + 1:
        raise ValueError(f"q has {q.shape[1]} rows per request, n_draft+1 = {n_draft + 1}")
    d = attn_dims(q, k_pages, page_table, sm_scale)
    if out is None:
        out = torch.empty_like(q)
    else:
        _need(out, "out", torch.bfloat16, 4, dev)
    if workspace is None:
        workspace = _cached_workspace("attn", dev, lib.cs_verify_attention_workspace_bytes(ctypes.byref(d), int(n_draft)),
                                      stream)
    st = lib.cs_verify_attention(ctypes.byref(d), q.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(),
                                 page_table.data_ptr(), ctx_lens.data_ptr(), int(n_draft), out.data_ptr(),
                                 workspace.data_ptr(), workspace.nbytes,
                                 _stream(dev) if stream is None else stream)
    if st:
        _check(lib, st)
    return out


def spec_accept_workspace(dims: AcceptDims, n_draft: int, device) -> torch.Tensor:
    """The default workspace of the current stream's calls."""
    n = load_library().cs_spec_accept_workspace_bytes(ctypes.byref(dims), int(n_draft))
    return _cached_workspace("accept", device, n)


def cs_spec_accept(target_logits, draft_logits, draft_tokens, uniforms, temperature,
                   out_tokens=None, out_n_accepted=None, workspace=None,
                   stream: int | None = None):
    """Speculative acceptance; returns (out_tokens [B, k+1], n_accepted [B]).  See include/cachespec.h."""
    r = (_fast or _load_fast()).spec_accept(target_logits, draft_logits, draft_tokens, uniforms, temperature, out_tokens,
                                            out_n_accepted, workspace, stream)
    if r is not None:
        return _done(r)
    lib = load_library()
    dev = target_logits.device
    if target_logits.dtype not in (torch.float32, torch.bfloat16):
        raise TypeError("logits must be float32 or bfloat16")
    dtype = target_logits.dtype
    _need(target_logits, "target_logits", dtype, 3, dev)
    B, rows, V = target_logits.shape
    k = rows - 1
    if draft_logits is not None:
        _need(draft_logits, "draft_logits", dtype, 3, dev)
        if tuple(draft_logits.shape) != (B, k, V):
            raise ValueError(f"draft_logits must be [{B}, {k}, {V}]")
    _need(draft_tokens, "draft_tokens", torch.int32, 2, dev)
    _need(uniforms, "uniforms", torch.float32, 2, dev)
    if out_tokens is None:
        out_tokens = draft_tokens.new_empty((B, k + 1))
    else:
        _need(out_tokens, "out_tokens", torch.int32, 2, dev)
    if out_n_accepted is None:
        out_n_accepted = draft_tokens.new_empty((B,))
    else:
        _need(out_n_accepted, "out_n_accepted", torch.int32, 1, dev)
    d = AcceptDims(B, V, CS_F32 if dtype == torch.float32 else CS_BF16)
    if workspace is None:
        workspace = _cached_workspace("accept", dev, lib.cs_spec_accept_workspace_bytes(ctypes.byref(d), int(k)), stream)
    st = lib.cs_spec_accept(ctypes.byref(d), target_logits.data_ptr(), _ptr(draft_logits),
                            draft_tokens.data_ptr(), uniforms.data_ptr(), int(k), float(temperature),
                            out_tokens.data_ptr(), out_n_accepted.data_ptr(), workspace.data_ptr(),
                            workspace.nbytes, _stream(dev) if stream is None else stream)
    if st:
        _check(lib, st)
    return out_tokens, out_n_accepted


def cs_kv_append(new_k, new_v, k_pages, v_pages, page_table, ctx_lens, stream: int | None = None):
    """Append the K/V rows of the newest positions into the page pools (in place).
    new_k / new_v bf16 [B, n_new, Hkv, D]; pools [P, Hkv, ps, D].  See include/cachespec.h."""
    r = (_fast or _load_fast()).kv_append(new_k, new_v, k_pages, v_pages, page_table, ctx_lens, stream)
    if r is not None:
        _done(r)
        return
    lib = load_library()
    dev = k_pages.device
    _need(new_k, "new_k", torch.bfloat16, 4, dev)
    _need(new_v, "new_v", torch.bfloat16, 4, dev)
    _need(k_pages, "k_pages", torch.bfloat16, 4, dev)
    _need(v_pages, "v_pages", torch.bfloat16, 4, dev)
    _need(page_table, "page_table", torch.int32, 2, dev)
    _need(ctx_lens, "ctx_lens", torch.int32, 1, dev)
    B, n_new, Hkv, D = new_k.shape
    P, Hkv2, ps, D2 = k_pages.shape
    if tuple(new_v.shape) != tuple(new_k.shape) or Hkv2 != Hkv or D2 != D or k_pages.shape != v_pages.shape:
        raise ValueError("new rows and pools do not match")
    d = AttnDims(B, Hkv, Hkv, D, ps, page_table.shape[1], P, 0.0)
    st = lib.cs_kv_append(ctypes.byref(d), new_k.data_ptr(), new_v.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(),
                          page_table.data_ptr(), ctx_lens.data_ptr(), int(n_new),
                          _stream(dev) if stream is None else stream)
    if st:
        _check(lib, st)


def cs_kv_commit(ctx_lens, n_accepted, n_draft: int, stream: int | None = None):
    """Keep the accepted prefix: ctx_lens <- max(0, ctx_lens - k + n_accepted), in place."""
    r = (_fast or _load_fast()).kv_commit(ctx_lens, n_accepted, n_draft, stream)
    if r is not None:
        _done(r)
        return
    lib = load_library()
    dev = ctx_lens.device
    _need(ctx_lens, "ctx_lens", torch.int32, 1, dev)
    _need(n_accepted, "n_accepted", torch.int32, 1, dev)
    st = lib.cs_kv_commit(int(ctx_lens.shape[0]), ctx_lens.data_ptr(), n_accepted.data_ptr(), int(n_draft),
                          _stream(dev) if stream is None else stream)
    if st:
        _check(lib, st)


def cs_route_norms(centroids, inv_norms=None, stream: int | None = None):
    """Inverse L2 norms of the group centroids (bf16 [N, d]); returns fp32 [N]."""
    lib = load_library()
    dev = centroids.device
    _need(centroids, "centroids", torch.bfloat16, 2, dev)
    N, d = centroids.shape
    if inv_norms is None:
        inv_norms = torch.empty((N,), dtype=torch.float32, device=dev)
    _need(inv_norms, "inv_norms", torch.float32, 1, dev)
    st = lib.cs_route_norms(int(N), int(d), centroids.data_ptr() if N else None, inv_norms.data_ptr() if N else None,
                            _stream(dev) if stream is None else stream)
    if st:
        _check(lib, st)
    return inv_norms


def cs_route(emb, centroids, inv_norms, tau, out_group=None, out_best=None, out_score=None, workspace=None,
             stream: int | None = None):
    """Batched semantic routing; returns (group [B], best [B], score [B]).  See include/cachespec.h."""
    if out_group is None and out_best is None and out_score is None:
        r = (_fast or _load_fast()).route(emb, centroids, inv_norms, tau, workspace, stream)
        if r is not None:
            return _done(r)
    lib = load_library()
    dev = emb.device
    _need(emb, "emb", torch.bfloat16, 2, dev)
    _need(centroids, "centroids", torch.bfloat16, 2, dev)
    _need(inv_norms, "inv_norms", torch.float32, 1, dev)
    B, d = emb.shape
    N = centroids.shape[0]
    if N and centroids.shape[1] != d:
        raise ValueError("emb and centroids differ in width")
    out_group = inv_norms.new_empty((B,), dtype=torch.int32) if out_group is None else out_group
    out_best = inv_norms.new_empty((B,), dtype=torch.int32) if out_best is None else out_best
    out_score = inv_norms.new_empty((B,)) if out_score is None else out_score
    dims = RouteDims(B, N, d)
    if workspace is None:
        workspace = _cached_workspace("route", dev, lib.cs_route_workspace_bytes(ctypes.byref(dims)), stream)
    st = lib.cs_route(ctypes.byref(dims), emb.data_ptr(), centroids.data_ptr() if N else None,
                      inv_norms.data_ptr() if N else None,
                      float(tau), out_group.data_ptr(), out_best.data_ptr(), out_score.data_ptr(), workspace.data_ptr(),
                      workspace.nbytes, _stream(dev) if stream is None else stream)
    if st:
        _check(lib, st)
    return out_group, out_best, out_score


def cs_sample(logits, uniforms, temperature, out_tokens=None, workspace=None,
              stream: int | None = None):
    """Draft-side sampling, one token per row of ``logits`` [B, V]; returns out_tokens [B].
    See include/cachespec.h."""
    r = (_fast or _load_fast()).sample(logits, uniforms, temperature, out_tokens, workspace, stream)
    if r is not None:
        return _done(r)
    lib = load_library()
    dev = logits.device
    if logits.dtype not in (torch.float32, torch.bfloat16):
        raise TypeError("logits must be float32 or bfloat16")
    _need(logits, "logits", logits.dtype, 2, dev)
    B, V = logits.shape
    _need(uniforms, "uniforms", torch.float32, 1, dev)
    if out_tokens is None:
        out_tokens = uniforms.new_empty((B,), dtype=torch.int32)
    else:
        _need(out_tokens, "out_tokens", torch.int32, 1, dev)
    d = AcceptDims(B, V, CS_F32 if logits.dtype == torch.float32 else CS_BF16)
    if workspace is None:
        workspace = _cached_workspace("sample", dev, lib.cs_sample_workspace_bytes(ctypes.byref(d)), stream)
    st = lib.cs_sample(ctypes.byref(d), logits.data_ptr(), uniforms.data_ptr(), float(temperature),
                       out_tokens.data_ptr(),
                       workspace.data_ptr(), workspace.nbytes,
                       _stream(dev) if stream is None else stream)
    if st:
        _check(lib, st)
    return out_tokens


def cs_tree_verify_attention(q, k_pages, v_pages, page_table, ctx_lens, parents, out=None, workspace=None,
                             sm_scale: float = 0.0, stream: int | None = None):
    """Token-tree verify attention; q / out bf16 [B, n, Hq, D], parents int32 [B, n].
    Returns ``out``.  See include/cachespec.h."""
    r = (_fast or _load_fast()).tree_verify_attention(q, k_pages, v_pages, page_table, ctx_lens, parents, out, workspace,
                                                      sm_scale, stream)
    if r is not None:
        return _done(r)
    lib = load_library()
    dev = q.device
    _need(q, "q", torch.bfloat16, 4, dev)
    _need(k_pages, "k_pages", torch.bfloat16, 4, dev)
    _need(v_pages, "v_pages", torch.bfloat16, 4, dev)
    _need(page_table, "page_table", torch.int32, 2, dev)
    _need(ctx_lens, "ctx_lens", torch.int32, 1, dev)
    _need(parents, "parents", torch.int32, 2, dev)
    if v_pages.shape != k_pages.shape:
        raise ValueError("k_pages and v_pages must have the same shape")
    B, n = q.shape[0], q.shape[1]
    if tuple(parents.shape) != (B, n):
        raise ValueError(f"parents must be [{B}, {n}]")
    d = attn_dims(q, k_pages, page_table, sm_scale)
    if out is None:
        out = torch.empty_like(q)
    else:
        _need(out, "out", torch.bfloat16, 4, dev)
    if workspace is None:
        workspace = _cached_workspace("tree_attn", dev,
                                      lib.cs_tree_verify_attention_workspace_bytes(ctypes.byref(d), int(n)), stream)
    st = lib.cs_tree_verify_attention(ctypes.byref(d), q.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(),
                                      page_table.data_ptr(), ctx_lens.data_ptr(), parents.data_ptr(), int(n),
                                      out.data_ptr(), workspace.data_ptr(), workspace.nbytes,
                                      _stream(dev) if stream is None else stream)
    if st:
        _check(lib, st)
    return out


def cs_tree_accept(target_logits, draft_logits, parents, node_tokens, uniforms, temperature, out_tokens=None,
                   out_path=None, out_n_accepted=None, workspace=None, stream: int | None = None):
    """Token-tree acceptance walk; target / draft logits [B, n, V], parents / node_tokens int32 [B, n],
    uniforms fp32 [B, n].  Returns (tokens [B, n], path [B, n], n_accepted [B]).  See include/cachespec.h."""
    r = (_fast or _load_fast()).tree_accept(target_logits, draft_logits, parents, node_tokens, uniforms, temperature,
                                            out_tokens, out_path, out_n_accepted, workspace, stream)
    if r is not None:
        return _done(r)
    lib = load_library()
    dev = target_logits.device
    if target_logits.dtype not in (torch.float32, torch.bfloat16):
        raise TypeError("logits must be float32 or bfloat16")
    dtype = target_logits.dtype
    _need(target_logits, "target_logits", dtype, 3, dev)
    B, n, V = target_logits.shape
    if draft_logits is not None:
        _need(draft_logits, "draft_logits", dtype, 3, dev)
        if tuple(draft_logits.shape) != (B, n, V):
            raise ValueError(f"draft_logits must be [{B}, {n}, {V}]")
    for name, t in (("parents", parents), ("node_tokens", node_tokens)):
        _need(t, name, torch.int32, 2, dev)
        if tuple(t.shape) != (B, n):
            raise ValueError(f"{name} must be [{B}, {n}]")
    _need(uniforms, "uniforms", torch.float32, 2, dev)
    if out_tokens is None:
        out_tokens = parents.new_empty((B, n))
    else:
        _need(out_tokens, "out_tokens", torch.int32, 2, dev)
    if out_path is None:
        out_path = parents.new_empty((B, n))
    else:
        _need(out_path, "out_path", torch.int32, 2, dev)
    if out_n_accepted is None:
        out_n_accepted = parents.new_empty((B,))
    else:
        _need(out_n_accepted, "out_n_accepted", torch.int32, 1, dev)
    d = AcceptDims(B, V, CS_F32 if dtype == torch.float32 else CS_BF16)
    if workspace is None:
        workspace = _cached_workspace("tree_accept", dev, lib.cs_tree_accept_workspace_bytes(ctypes.byref(d), int(n)),
                                      stream)
    st = lib.cs_tree_accept(ctypes.byref(d), target_logits.data_ptr(), _ptr(draft_logits), parents.data_ptr(),
                            node_tokens.data_ptr(), uniforms.data_ptr(), int(n), float(temperature),
                            out_tokens.data_ptr(),
                            out_path.data_ptr(), out_n_accepted.data_ptr(), workspace.data_ptr(),
                            workspace.nbytes, _stream(dev) if stream is None else stream)
    if st:
        _check(lib, st)
    return out_tokens, out_path, out_n_accepted


def cs_kv_commit_tree(k_pages, v_pages, page_table, ctx_lens, path, n_accepted, stream: int | None = None):
    """Move the accepted tree path's K/V rows next to the root and shorten ctx_lens (in place);
    path int32 [B, n] and n_accepted [B] as returned by cs_tree_accept."""
    r = (_fast or _load_fast()).kv_commit_tree(k_pages, v_pages, page_table, ctx_lens, path, n_accepted, stream)
    if r is not None:
        _done(r)
        return
    lib = load_library()
    dev = k_pages.device
    _need(k_pages, "k_pages", torch.bfloat16, 4, dev)
    _need(v_pages, "v_pages", torch.bfloat16, 4, dev)
    _need(page_table, "page_table", torch.int32, 2, dev)
    _need(ctx_lens, "ctx_lens", torch.int32, 1, dev)
    _need(path, "path", torch.int32, 2, dev)
    _need(n_accepted, "n_accepted", torch.int32, 1, dev)
    if k_pages.shape != v_pages.shape:
        raise ValueError("k_pages and v_pages must have the same shape")
    P, Hkv, ps, D = k_pages.shape
    B, n = path.shape
    d = AttnDims(B, Hkv, Hkv, D, ps, page_table.shape[1], P, 0.0)
    st = lib.cs_kv_commit_tree(ctypes.byref(d), k_pages.data_ptr(), v_pages.data_ptr(), page_table.data_ptr(),
                               ctx_lens.data_ptr(), path.data_ptr(), n_accepted.data_ptr(), int(n),
                               _stream(dev) if stream is None else stream)
    if st:
        _check(lib, st)


def packed_pool(num_pages: int, n_kv_heads: int, page_size: int, device, k_head_scale=None,
                v_head_scale=None) -> PackedPool:
    """An empty (all zero) packed cache of ``num_pages`` pages."""
    def zeros(width, dtype):
        return torch.zeros((num_pages, n_kv_heads, page_size, width), dtype=dtype, device=device)
    return PackedPool(zeros(64, torch.uint8), zeros(8, torch.float8_e4m3fn), zeros(64, torch.uint8),
                      zeros(8, torch.float8_e4m3fn), k_head_scale, v_head_scale)


def _packed(pool: PackedPool, dev):
    """The pool's pointers, after the checks, and its geometry (P, Hkv, ps)."""
    pool = PackedPool(*pool)
    _need(pool.k_codes, "k_codes", torch.uint8, 4, dev)
    P, Hkv, ps, width = pool.k_codes.shape
    if width != 64:
        raise ValueError(f"k_codes must be [P, Hkv, ps, 64], got {tuple(pool.k_codes.shape)}")
    _need(pool.v_codes, "v_codes", torch.uint8, 4, dev)
    if pool.v_codes.shape != pool.k_codes.shape:
        raise ValueError("k_codes and v_codes must have the same shape")
    for name in ("k_scales", "v_scales"):
        t = getattr(pool, name)
        _need(t, name, torch.float8_e4m3fn, 4, dev)
        if tuple(t.shape) != (P, Hkv, ps, 8):
            raise ValueError(f"{name} must be [{P}, {Hkv}, {ps}, 8], got {tuple(t.shape)}")
    for name in ("k_head_scale", "v_head_scale"):
        t = getattr(pool, name)
        if t is not None:
            _need(t, name, torch.float32, 1, dev)
            if t.shape[0] != Hkv:
                raise ValueError(f"{name} must be [{Hkv}], got {tuple(t.shape)}")
    return PackedPoolPtrs(*(_ptr(t) for t in pool)), (P, Hkv, ps)


def _rows_of(page_table, ctx_lens, B: int, dev) -> None:
    _need(page_table, "page_table", torch.int32, 2, dev)
    _need(ctx_lens, "ctx_lens", torch.int32, 1, dev)
    if page_table.shape[0] != B or ctx_lens.shape[0] != B:
        raise ValueError(f"page_table and ctx_lens must have {B} rows")


def cs_packed_kv_append(new_k, new_v, pool, page_table, ctx_lens, stream: int | None = None):
    """Quantise the K/V rows of the newest positions into a packed cache (in place).
    new_k / new_v bf16 [B, n_new, Hkv, 128]; ``pool`` a PackedPool.  See include/cachespec.h."""
    r = (_fast or _load_fast()).packed_kv_append(new_k, new_v, pool, page_table, ctx_lens, stream)
    if r is not None:
        _done(r)
        return
    lib = load_library()
    _need(new_k, "new_k", torch.bfloat16, 4, None)
    dev = new_k.device
    _need(new_v, "new_v", torch.bfloat16, 4, dev)
    ptrs, (P, Hkv, ps) = _packed(pool, dev)
    B, n_new, H, D = new_k.shape
    if new_v.shape != new_k.shape or H != Hkv or D != 128:
        raise ValueError("new rows and pool do not match")
    _rows_of(page_table, ctx_lens, B, dev)
    d = AttnDims(B, Hkv, Hkv, D, ps, page_table.shape[1], P, 0.0)
    st = lib.cs_packed_kv_append(ctypes.byref(d), ctypes.byref(ptrs), new_k.data_ptr(), new_v.data_ptr(),
                                 page_table.data_ptr(), ctx_lens.data_ptr(), int(n_new),
                                 _stream(dev) if stream is None else stream)
    if st:
        _check(lib, st)


def cs_packed_kv_read(pool, page_table, ctx_lens, n_rows: int, stream: int | None = None):
    """The newest ``n_rows`` rows of every request from a packed cache; returns (k, v), bf16 [B, n_rows, Hkv, 128]."""
    r = (_fast or _load_fast()).packed_kv_read(pool, page_table, ctx_lens, n_rows, stream)
    if r is not None:
        return _done(r)
    lib = load_library()
    dev = page_table.device
    ptrs, (P, Hkv, ps) = _packed(pool, dev)
    B = page_table.shape[0]
    _rows_of(page_table, ctx_lens, B, dev)
    out = [torch.empty((B, max(int(n_rows), 0), Hkv, 128), dtype=torch.bfloat16, device=dev) for _ in range(2)]
    d = AttnDims(B, Hkv, Hkv, 128, ps, page_table.shape[1], P, 0.0)
    st = lib.cs_packed_kv_read(ctypes.byref(d), ctypes.byref(ptrs), page_table.data_ptr(), ctx_lens.data_ptr(),
                               int(n_rows), out[0].data_ptr(), out[1].data_ptr(),
                               _stream(dev) if stream is None else stream)
    if st:
        _check(lib, st)
    return tuple(out)


def packed_attn_dims(q: torch.Tensor, pool: PackedPool, page_table: torch.Tensor, sm_scale: float = 0.0) -> AttnDims:
    return attn_dims(q, pool[0], page_table, sm_scale)


def packed_verify_attention_workspace(dims: AttnDims, n_draft: int, device, stream: int | None = None) -> torch.Tensor:
    """The default workspace of the (current) stream's calls of cs_packed_verify_attention with these dims: after one,
    cs_read_device_status of it tells whether it finished normally."""
    n = load_library().cs_packed_verify_attention_workspace_bytes(ctypes.byref(dims), int(n_draft))
    return _cached_workspace("packed_attn", device, n, stream)


def cs_packed_verify_attention(q, pool, page_table, ctx_lens, n_draft, out=None, workspace=None, sm_scale: float = 0.0,
                               stream: int | None = None):
    """Verify attention over a packed cache, ``n_draft`` in [0, 16]; returns ``out`` (bf16 [B, k+1, Hq, 128]).
    See include/cachespec.h."""
    r = (_fast or _load_fast()).packed_verify_attention(q, pool, page_table, ctx_lens, n_draft, out, workspace, sm_scale,
                                                        stream)
    if r is not None:
        return _done(r)
    lib = load_library()
    _need(q, "q", torch.bfloat16, 4, None)
    dev = q.device
    ptrs, (P, Hkv, ps) = _packed(pool, dev)
    B, R, Hq, D = q.shape
    if R != n_draft + 1:
        raise ValueError(f"q has {R} rows per request, n_draft+1 = {n_draft + 1}")
    _rows_of(page_table, ctx_lens, B, dev)
    d = AttnDims(B, Hq, Hkv, D, ps, page_table.shape[1], P, float(sm_scale))
    if out is None:
        out = torch.empty_like(q)
    else:
        _need(out, "out", torch.bfloat16, 4, dev)
        if out.shape != q.shape:
            raise ValueError("out must have the shape of q")
    if workspace is None:
        n = lib.cs_packed_verify_attention_workspace_bytes(ctypes.byref(d), int(n_draft))
        workspace = _cached_workspace("packed_attn", dev, n, stream)
    st = lib.cs_packed_verify_attention(ctypes.byref(d), q.data_ptr(), ctypes.byref(ptrs), page_table.data_ptr(),
                                        ctx_lens.data_ptr(), int(n_draft), out.data_ptr(), workspace.data_ptr(),
                                        workspace.nbytes, _stream(dev) if stream is None else stream)
    if st:
        _check(lib, st)
    return out


def _token_rows(t: torch.Tensor, name: str, dev) -> int:
    """Checks rows of heads [T, H, 128], a token's heads side by side; returns the stride from token to token."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.dtype != torch.bfloat16:
        raise TypeError(f"{name} must be {torch.bfloat16}, got {t.dtype}")
    if t.dim() != 3 or t.shape[2] != 128:
        raise ValueError(f"{name} must be [tokens, heads, 128], got shape {tuple(t.shape)}")
    if not t.is_cuda or (dev is not None and t.device != dev):
        raise ValueError(f"{name} must live on {dev or 'a CUDA device'}")
    T, H, D = t.shape
    if T and H and (t.stride(2) != 1 or (H > 1 and t.stride(1) != D)):
        raise ValueError(f"the heads of a token of {name} must lie together")
    if T <= 1 or H == 0:
        return H * D
    if t.stride(0) < H * D or t.stride(0) % 8:
        raise ValueError(f"the tokens of {name} must lie a multiple of 8 elements apart, at least {H * D}")
    return t.stride(0)


def _ragged(page_table, ctx_lens, q_starts, T: int, dev) -> int:
    """Checks the arrays of a batch whose requests have rows of their own; returns the number of requests."""
    _need(ctx_lens, "ctx_lens", torch.int32, 1, dev)
    B = ctx_lens.shape[0]
    _rows_of(page_table, ctx_lens, B, dev)
    if q_starts is not None:
        _need(q_starts, "q_starts", torch.int32, 1, dev)
        if q_starts.shape[0] != B + 1:
            raise ValueError(f"q_starts must be [{B + 1}]")
    elif T % max(B, 1):
        raise ValueError(f"{T} tokens of {B} requests without q_starts")
    return B


def _rope_call(q, new_k, new_v, cos_sin, page_table, ctx_lens, q_starts, positions, q_norm, k_norm, norm_eps, interleaved,
               q_out, Hkv: int, ps: int, P: int, dev):
    """The checks of the two rotated appends; returns (dims, rope dims, q_out)."""
    k_stride, v_stride = _token_rows(new_k, "new_k", dev), _token_rows(new_v, "new_v", dev)
    T, H, D = new_k.shape
    if new_v.shape != new_k.shape or H != Hkv:
        raise ValueError("new rows and pools do not match")
    q_stride = out_stride = 0
    if q is not None:
        q_stride = _token_rows(q, "q", dev)
        if q.shape[0] != T:
            raise ValueError(f"q has {q.shape[0]} tokens, new_k {T}")
        if q_out is None:
            q_out = q.new_empty(q.shape)
        out_stride = _token_rows(q_out, "q_out", dev)
        if q_out.shape != q.shape:
            raise ValueError("q_out must have the shape of q")
    elif q_out is not None:
        raise ValueError("q_out without q")
    _need(cos_sin, "cos_sin", torch.float32, 2, dev)
    B = _ragged(page_table, ctx_lens, q_starts, T, dev)
    if positions is not None:
        _need(positions, "positions", torch.int32, 1, dev)
        if positions.shape[0] != T:
            raise ValueError(f"positions must be [{T}]")
    for name, t in (("q_norm", q_norm), ("k_norm", k_norm)):
        if t is not None:
            _need(t, name, torch.bfloat16, 1, dev)
            if t.shape[0] != D:
                raise ValueError(f"{name} must be [{D}]")
    return (AttnDims(B, Hkv if q is None else q.shape[1], Hkv, D, ps, page_table.shape[1], P, 0.0),
            RopeDims(T, cos_sin.shape[1], int(bool(interleaved)), cos_sin.shape[0], float(norm_eps), q_stride, k_stride,
                     v_stride, out_stride), q_out)


def cs_rope_kv_append(q, new_k, new_v, cos_sin, k_pages, v_pages, page_table, ctx_lens, q_starts=None, positions=None,
                      q_norm=None, k_norm=None, norm_eps: float = 1e-6, interleaved: bool = False, q_out=None,
                      stream: int | None = None):
    """Turn the queries and keys of new tokens by their positions and append keys and values to the page pools (in
    place).  q bf16 [tokens, Hq, 128] or None, new_k / new_v [tokens, Hkv, 128], whose tokens may lie apart; request b's
    are the rows q_starts[b] .. q_starts[b+1] - 1 (None: as many each).  cos_sin fp32 [positions, rot_dim]: it has to
    reach every position, for a token past it is left out, in silence, its key, value and query unwritten.  Returns
    q_out (where it is made here, rows of tokens left out and of no request hold anything).  See
    include/cachespec.h."""
    r = (_fast or _load_fast()).rope_kv_append(q, new_k, new_v, cos_sin, k_pages, v_pages, page_table, ctx_lens, q_starts,
                                               positions, q_norm, k_norm, norm_eps, interleaved, q_out, stream)
    if r is not None:
        return None if r is True else _done(r)
    lib = load_library()
    _need(k_pages, "k_pages", torch.bfloat16, 4, None)
    dev = k_pages.device
    _need(v_pages, "v_pages", torch.bfloat16, 4, dev)
    P, Hkv, ps, D = k_pages.shape
    if v_pages.shape != k_pages.shape or D != 128:
        raise ValueError("k_pages and v_pages must have the same shape [P, Hkv, ps, 128]")
    d, r, q_out = _rope_call(q, new_k, new_v, cos_sin, page_table, ctx_lens, q_starts, positions, q_norm, k_norm,
                             norm_eps, interleaved, q_out, Hkv, ps, P, dev)
    with torch.cuda.device(dev):
        st = lib.cs_rope_kv_append(ctypes.byref(d), ctypes.byref(r), _ptr(q), new_k.data_ptr(), new_v.data_ptr(),
                                   cos_sin.data_ptr(), _ptr(positions), _ptr(q_norm), _ptr(k_norm), _ptr(q_out),
                                   k_pages.data_ptr(), v_pages.data_ptr(), page_table.data_ptr(), ctx_lens.data_ptr(),
                                   _ptr(q_starts), _stream(dev) if stream is None else stream)
    if st:
        _check(lib, st)
    return q_out


def cs_packed_rope_kv_append(q, new_k, new_v, cos_sin, pool, page_table, ctx_lens, q_starts=None, positions=None,
                             q_norm=None, k_norm=None, norm_eps: float = 1e-6, interleaved: bool = False, q_out=None,
                             stream: int | None = None):
    """cs_rope_kv_append into a packed cache; ``pool`` a PackedPool.  Returns q_out.  See include/cachespec.h."""
    r = (_fast or _load_fast()).packed_rope_kv_append(q, new_k, new_v, cos_sin, pool, page_table, ctx_lens, q_starts,
                                                      positions, q_norm, k_norm, norm_eps, interleaved, q_out, stream)
    if r is not None:
        return None if r is True else _done(r)
    lib = load_library()
    _need(pool[0], "k_codes", torch.uint8, 4, None)
    dev = pool[0].device
    ptrs, (P, Hkv, ps) = _packed(pool, dev)
    d, r, q_out = _rope_call(q, new_k, new_v, cos_sin, page_table, ctx_lens, q_starts, positions, q_norm, k_norm,
                             norm_eps, interleaved, q_out, Hkv, ps, P, dev)
    with torch.cuda.device(dev):
        st = lib.cs_packed_rope_kv_append(ctypes.byref(d), ctypes.byref(r), _ptr(q), new_k.data_ptr(), new_v.data_ptr(),
                                          cos_sin.data_ptr(), _ptr(positions), _ptr(q_norm), _ptr(k_norm), _ptr(q_out),
                                          ctypes.byref(ptrs), page_table.data_ptr(), ctx_lens.data_ptr(), _ptr(q_starts),
                                          _stream(dev) if stream is None else stream)
    if st:
        _check(lib, st)
    return q_out


def chunk_attn_dims(q: torch.Tensor, k_pages: torch.Tensor, page_table: torch.Tensor, sm_scale: float = 0.0) -> AttnDims:
    P, Hkv, ps, D = k_pages.shape
    return AttnDims(page_table.shape[0], q.shape[1], Hkv, D, ps, page_table.shape[1], P, float(sm_scale))


def _chunk_workspace_bytes(lib, d: AttnDims, tokens: int) -> int:
    """Of the default workspace: what 256 tokens need, which is what all larger calls do, so that a stream has one
    for whatever calls, and one call before a capture has made it for all calls in it."""
    return max(lib.cs_chunk_attention_workspace_bytes(ctypes.byref(d), t) for t in (tokens, 256))


def chunk_attention_workspace(dims: AttnDims, tokens: int, device, stream: int | None = None) -> torch.Tensor:
    """The default workspace of the (current) stream's calls of cs_chunk_attention: after one, cs_read_device_status of
    it tells whether it finished normally."""
    return _cached_workspace("chunk_attn", device, _chunk_workspace_bytes(load_library(), dims, int(tokens)), stream)


def cs_chunk_attention(q, k_pages, v_pages, page_table, ctx_lens, q_starts=None, out=None, workspace=None,
                       sm_scale: float = 0.0, stream: int | None = None):
    """Attention of every request's newest tokens over the paged cache, causal among them.  q bf16 [tokens, Hq, 128],
    whose tokens may lie apart; request b's are the rows q_starts[b] .. q_starts[b+1] - 1 (None: as many each).
    Returns ``out`` (bf16 [tokens, Hq, 128]; rows of no request stay as they are: anything, where it is made here).
    See include/cachespec.h."""
    r = (_fast or _load_fast()).chunk_attention(q, k_pages, v_pages, page_table, ctx_lens, q_starts, out, workspace,
                                                sm_scale, stream)
    if r is not None:
        return _done(r)
    lib = load_library()
    q_stride = _token_rows(q, "q", None)
    dev = q.device
    _need(k_pages, "k_pages", torch.bfloat16, 4, dev)
    _need(v_pages, "v_pages", torch.bfloat16, 4, dev)
    if v_pages.shape != k_pages.shape:
        raise ValueError("k_pages and v_pages must have the same shape")
    _ragged(page_table, ctx_lens, q_starts, q.shape[0], dev)
    d = chunk_attn_dims(q, k_pages, page_table, sm_scale)
    if out is None:
        out = q.new_empty(q.shape)
    else:
        _need(out, "out", torch.bfloat16, 3, dev)
        if out.shape != q.shape:
            raise ValueError("out must have the shape of q")
    T = q.shape[0]
    with torch.cuda.device(dev):
        if workspace is None:
            workspace = _cached_workspace("chunk_attn", dev, _chunk_workspace_bytes(lib, d, int(T)), stream)
        st = lib.cs_chunk_attention(ctypes.byref(d), q.data_ptr(), q_stride, int(T), k_pages.data_ptr(),
                                    v_pages.data_ptr(), page_table.data_ptr(), ctx_lens.data_ptr(), _ptr(q_starts),
                                    out.data_ptr(), workspace.data_ptr(), workspace.nbytes,
                                    _stream(dev) if stream is None else stream)
    if st:
        _check(lib, st)
    return out


def _page_call(page_table, ctx_lens, ref_counts, page_size, dev) -> PageDims:
    _need(page_table, "page_table", torch.int32, 2, dev)
    _need(ref_counts, "ref_counts", torch.int32, 1, dev)
    R, cols = page_table.shape
    if ctx_lens is not None:
        _need(ctx_lens, "ctx_lens", torch.int32, 1, dev)
        if ctx_lens.shape[0] != R:
            raise ValueError(f"ctx_lens must be [{R}]")
    return PageDims(R, cols, int(page_size), ref_counts.shape[0])


def _page_pools(pools, P: int, dev):
    pools = [t for t in pools if t is not None]
    for i, t in enumerate(pools):
        _need(t, f"pools[{i}]", t.dtype, t.dim(), dev)
        if t.dim() < 2 or t.shape[0] != P:
            raise ValueError(f"pools[{i}] must be [{P}, ...], a page a row, got {tuple(t.shape)}")
    return (PagePool * len(pools))(*((t.data_ptr(), t.nbytes // max(P, 1)) for t in pools)), len(pools)


def cs_kv_fork(pools, page_table, ctx_lens, ref_counts, src, dst, page_size: int, room: int = 0, workspace=None,
               stream: int | None = None):
    """Rows ``dst`` of the page table become copies of rows ``src`` (-1: empty rows) that share their full pages,
    with room for ``room`` more tokens each; table, lengths and counts change in place.  ``pools``: the cache's
    tensors, each [P, ...].  Returns int32 [n]: 1 where there were enough free pages.  See include/cachespec.h."""
    r = (_fast or _load_fast()).kv_fork(pools, page_table, ctx_lens, ref_counts, src, dst, page_size, room, workspace, stream)
    if r is not None:
        return _done(r)
    lib = load_library()
    dev = page_table.device
    d = _page_call(page_table, ctx_lens, ref_counts, page_size, dev)
    arr, n_pools = _page_pools(pools, d.num_pages, dev)
    _need(src, "src", torch.int32, 1, dev)
    _need(dst, "dst", torch.int32, 1, dev)
    n = src.shape[0]
    if dst.shape[0] != n:
        raise ValueError("src and dst must have the same length")
    out = src.new_empty((n,))
    if workspace is None:
        workspace = _cached_workspace("fork", dev, lib.cs_kv_fork_workspace_bytes(ctypes.byref(d), int(n)), stream)
    st = lib.cs_kv_fork(ctypes.byref(d), arr, n_pools, page_table.data_ptr(), ctx_lens.data_ptr(),
                        ref_counts.data_ptr(), src.data_ptr(), dst.data_ptr(), int(n), int(room), out.data_ptr(),
                        workspace.data_ptr(), workspace.nbytes, _stream(dev) if stream is None else stream)
    if st:
        _check(lib, st)
    return out


def cs_kv_fork_more(pools, page_table, ref_counts, n: int, workspace=None, stream: int | None = None):
    """The page copies of the fork of ``n`` rows before, in further pools: a cache of more than CS_MAX_PAGE_POOLS
    tensors goes through cs_kv_fork with the first of them and through this with the others, up to that many a call.
    ``workspace`` is that call's (None: the stream's default one, as there).  See include/cachespec.h."""
    lib = load_library()
    dev = page_table.device
    d = _page_call(page_table, None, ref_counts, 1, dev)
    arr, n_pools = _page_pools(pools, d.num_pages, dev)
    if workspace is None:
        workspace = _cached_workspace("fork", dev, lib.cs_kv_fork_workspace_bytes(ctypes.byref(d), int(n)), stream)
    st = lib.cs_kv_fork_more(ctypes.byref(d), arr, n_pools, int(n), workspace.data_ptr(), workspace.nbytes,
                             _stream(dev) if stream is None else stream)
    if st:
        _check(lib, st)


def cs_kv_release(page_table, ctx_lens, ref_counts, rows, keep_lens, page_size: int, stream: int | None = None):
    """Rows ``rows`` keep the pages of their first ``keep_lens`` tokens and give the others back (in place)."""
    r = (_fast or _load_fast()).kv_release(page_table, ctx_lens, ref_counts, rows, keep_lens, page_size, stream)
    if r is not None:
        _done(r)
        return
    lib = load_library()
    dev = page_table.device
    d = _page_call(page_table, ctx_lens, ref_counts, page_size, dev)
    _need(rows, "rows", torch.int32, 1, dev)
    _need(keep_lens, "keep_lens", torch.int32, 1, dev)
    if rows.shape != keep_lens.shape:
        raise ValueError("rows and keep_lens must have the same length")
    st = lib.cs_kv_release(ctypes.byref(d), page_table.data_ptr(), ctx_lens.data_ptr(), ref_counts.data_ptr(),
                           rows.data_ptr(), keep_lens.data_ptr(), int(rows.shape[0]),
                           _stream(dev) if stream is None else stream)
    if st:
        _check(lib, st)


def cs_kv_compact(pools, page_table, ref_counts, workspace=None, stream: int | None = None):
    """Moves the pages in use to the lowest ids; pools, table and counts change in place.
    Returns int32 [1]: how many pages are in use.  See include/cachespec.h."""
    r = (_fast or _load_fast()).kv_compact(pools, page_table, ref_counts, workspace, stream)
    if r is not None:
        return _done(r)
    lib = load_library()
    dev = page_table.device
    d = _page_call(page_table, None, ref_counts, 1, dev)
    arr, n_pools = _page_pools(pools, d.num_pages, dev)
    out = ref_counts.new_empty((1,))
    if workspace is None:
        workspace = _cached_workspace("compact", dev, lib.cs_kv_compact_workspace_bytes(ctypes.byref(d)), stream)
    st = lib.cs_kv_compact(ctypes.byref(d), arr, n_pools, page_table.data_ptr(), ref_counts.data_ptr(),
                           out.data_ptr(), workspace.data_ptr(), workspace.nbytes,
                           _stream(dev) if stream is None else stream)
    if st:
        _check(lib, st)
    return out


def cs_kv_compact_more(pools, page_table, ref_counts, workspace=None, stream: int | None = None):
    """The page copies of the compaction before, in further pools (as cs_kv_fork_more those of a fork)."""
    lib = load_library()
    dev = page_table.device
    d = _page_call(page_table, None, ref_counts, 1, dev)
    arr, n_pools = _page_pools(pools, d.num_pages, dev)
    if workspace is None:
        workspace = _cached_workspace("compact", dev, lib.cs_kv_compact_workspace_bytes(ctypes.byref(d)), stream)
    st = lib.cs_kv_compact_more(ctypes.byref(d), arr, n_pools, workspace.data_ptr(), workspace.nbytes,
                                _stream(dev) if stream is None else stream)
    if st:
        _check(lib, st)


def cs_logprobs(logits, tokens, temperature: float = 1.0, n_top: int = 0, stream: int | None = None):
    """Log probabilities of ``tokens`` (int32 [N]; negative: the row is skipped) under ``logits`` [N, V], whose rows
    may lie apart.  Returns (logprob [N], entropy [N], top tokens [N, n_top], their log probabilities [N, n_top]).
    See include/cachespec.h."""
    r = (_fast or _load_fast()).logprobs(logits, tokens, temperature, n_top, stream)
    if r is not None:
        return _done(r)
    lib = load_library()
    if not isinstance(logits, torch.Tensor):
        raise TypeError("logits must be a torch.Tensor")
    if logits.dtype not in (torch.float32, torch.bfloat16):
        raise TypeError("logits must be float32 or bfloat16")
    if logits.dim() != 2:
        raise ValueError(f"logits must have 2 dims, got shape {tuple(logits.shape)}")
    if not logits.is_cuda:
        raise ValueError("logits must live on a CUDA device")
    N, V = logits.shape
    if V > 1 and logits.stride(1) != 1:
        raise ValueError("the logits of a row must be contiguous")
    dev = logits.device
    _need(tokens, "tokens", torch.int32, 1, dev)
    if tokens.shape[0] != N:
        raise ValueError(f"tokens must be [{N}]")
    top = max(int(n_top), 0)
    lp, entropy = (torch.empty((N,), dtype=torch.float32, device=dev) for _ in range(2))
    top_tokens = tokens.new_empty((N, top))
    top_lp = lp.new_empty((N, top))
    d = LogprobDims(N, V, CS_F32 if logits.dtype == torch.float32 else CS_BF16, int(n_top),
                    logits.stride(0) if N > 1 else V)
    st = lib.cs_logprobs(ctypes.byref(d), logits.data_ptr(), tokens.data_ptr(), float(temperature), lp.data_ptr(),
                         entropy.data_ptr(), top_tokens.data_ptr(), top_lp.data_ptr(),
                         _stream(dev) if stream is None else stream)
    if st:
        _check(lib, st)
    return lp, entropy, top_tokens, top_lp


def cs_verify_attention_noalloc(q, k_pages, v_pages, page_table, ctx_lens, n_draft, out=None,
                                sm_scale: float = 0.0, stream: int | None = None):
    """Verify attention without a workspace, for callers that cannot allocate device
    memory (the library's own fixed scratch is used; see include/cachespec.h)."""
    lib = load_library()
    dev = q.device
    _need(q, "q", torch.bfloat16, 4, dev)
    _need(k_pages, "k_pages", torch.bfloat16, 4, dev)
    _need(v_pages, "v_pages", torch.bfloat16, 4, dev)
    _need(page_table, "page_table", torch.int32, 2, dev)
    _need(ctx_lens, "ctx_lens", torch.int32, 1, dev)
    d = attn_dims(q, k_pages, page_table, sm_scale)
    if out is None:
        out = torch.empty_like(q)
    else:
        _need(out, "out", torch.bfloat16, 4, dev)
    st = lib.cs_verify_attention_noalloc(ctypes.byref(d), q.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(),
                                         page_table.data_ptr(), ctx_lens.data_ptr(), int(n_draft), out.data_ptr(),
                                         _stream(dev) if stream is None else stream)
    if st:
        _check(lib, st)
    return out


def cs_selftest_wait_timeout(workspace: torch.Tensor, stream: int | None = None) -> None:
    """Runs the kernels' bounded wait on a barrier nothing completes (about one
    second); it sets CS_DEVICE_WAIT_TIMEOUT in the workspace's status word."""
    lib = load_library()
    _check(lib, lib.cs_selftest_wait_timeout(_ptr(workspace),
                                             _stream(workspace.device) if stream is None else stream))


def cs_read_device_status(workspace: torch.Tensor, stream: int | None = None) -> int:
    """Status word of a verify-attention workspace, packed attention's among them (synchronises the stream)."""
    lib = load_library()
    v = ctypes.c_int32(0)
    _check(lib, lib.cs_read_device_status(_ptr(workspace), ctypes.byref(v),
                                          _stream(workspace.device) if stream is None else stream))
    return int(v.value)


def cs_verify_attention_noalloc_status(device=None, stream: int | None = None) -> int:
    """Status word of the allocation-free entry point on the current device: the
    CS_DEVICE_* bits of its latest call (synchronises the stream)."""
    lib = load_library()
    dev = torch.device("cuda", torch.cuda.current_device()) if device is None else torch.device(device)
    v = ctypes.c_int32(0)
    _check(lib, lib.cs_verify_attention_noalloc_status(ctypes.byref(v), _stream(dev) if stream is None else stream))
    return int(v.value)
