"""Python binding of the serving operators (ctypes; argument marshalling
only).  include/lumen_attn.h states what each computes: block tables and slot
maps, the 4-bit cache's append and read-back, decode attention over it, and
causal attention over packed prompts.

Each function has the name of the C entry point it calls; the prepare_* twins
check the arguments once and return a kvckpt.PreparedCall.
"""
from __future__ import annotations

import ctypes
import os
import re
from typing import Optional

import torch

from . import kvckpt as _kv
from .workloads import CacheShape, NHD

HEADER = os.path.join(os.path.dirname(_kv.HEADER), "lumen_attn.h")

LUMEN_ATTN_BF16 = 0
LUMEN_ATTN_FP16 = 1
LUMEN_ATTN_MAX_REQS = 4096  # include/lumen_attn.h
LUMEN_ATTN_MAX_TOKENS = 134217728  # include/lumen_attn.h
LUMEN_ATTN_MAX_STRIDE = 16777216  # include/lumen_attn.h
LUMEN_ATTN_KV4_MAX = 6848  # include/lumen_attn.h

_DTYPES = {torch.bfloat16: LUMEN_ATTN_BF16, torch.float16: LUMEN_ATTN_FP16}


class lumen_attn_rows(ctypes.Structure):
    _fields_ = [("d_base", ctypes.c_void_p),
                ("token_stride", ctypes.c_int64),
                ("head_stride", ctypes.c_int64)]


def exported_names():
    """Entry points declared in include/lumen_attn.h."""
    with open(HEADER) as f:
        text = f.read()
    return sorted(set(re.findall(r"\b(lumen_attn_\w+)\s*\(", text)))


_BOUND = None


def _lib():
    global _BOUND
    lib = _kv.load_library()
    if _BOUND is lib:
        return lib
    p, i32, i64, sz, f32 = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64,
                            ctypes.c_size_t, ctypes.c_float)
    lay = ctypes.POINTER(_kv.lumen_kv_layout)
    rows = ctypes.POINTER(lumen_attn_rows)
    sigs = {
        "lumen_attn_slots": (ctypes.c_int,
                             [p, p, p, i32, p, i32, i32, i64, p, p, i64, p,
                              i64, p, p, p, p, p]),
        "lumen_attn_append4": (ctypes.c_int,
                               [lay, i32, p, rows, rows, i32, p, i64, p, p]),
        "lumen_attn_read4": (ctypes.c_int,
                             [lay, i32, p, p, i64, rows, rows, i32, p, p]),
        "lumen_attn_decode4_workspace_bytes": (sz, [lay, i32, i32]),
        "lumen_attn_decode4": (ctypes.c_int,
                               [lay, i32, p, p, i32, p, i32, rows, i32, i32,
                                f32, p, p, sz, p, p]),
        "lumen_attn_prompt": (ctypes.c_int,
                              [rows, rows, rows, i32, p, p, i32, i64, i64,
                               i32, i32, i32, f32, p, p, sz, p, p]),
        "lumen_attn_prompt_workspace_bytes": (sz, [i32, i64, i64, i32, i32,
                                                   i32]),
    }
    for name, (res, args) in sigs.items():
        f = getattr(lib, name)
        f.restype, f.argtypes = res, args
    _BOUND = lib
    return lib


# ------------------------------------------------------------ marshalling

def row_bytes4(head_dim: int) -> int:
    """Bytes of a 4-bit row of head_dim elements."""
    return head_dim // 2 + 16


def cache_shape4(num_layers: int, num_kv_heads: int, head_dim: int,
                 block_size: int, order: str = NHD) -> CacheShape:
    """The cache shape of a 4-bit cache for a model of this head_dim: one-byte
    elements, D/2 + 16 of them a row.  The checkpoint calls take it too."""
    if head_dim not in (64, 128, 256):
        raise ValueError(f"head_dim {head_dim}: 64, 128 or 256 are supported")
    return CacheShape(num_layers, num_kv_heads, row_bytes4(head_dim),
                      block_size, order, 1)


def head_dim4(shape) -> int:
    """The model's head_dim of a 4-bit cache shape."""
    return 2 * (shape.head_dim - 16)


def _rows(t: torch.Tensor, what: str, heads: int, head_dim: int):
    """lumen_attn_rows of a [tokens, heads, head_dim] tensor, which may be
    strided over tokens and heads."""
    if t.dim() != 3 or t.shape[1] != heads or t.shape[2] != head_dim:
        raise ValueError(f"{what} must be [tokens, {heads}, {head_dim}], got "
                         f"{tuple(t.shape)}")
    d = t.get_device()
    if d < 0:
        raise ValueError(f"{what} must be a device tensor")
    if d != _kv._current_device():
        raise ValueError(f"{what} is on cuda:{d}, the current device is "
                         f"cuda:{torch.cuda.current_device()}")
    if t.numel() and t.stride(2) != 1:
        raise ValueError(f"{what}: a head's elements must be contiguous")
    # a stride over a dimension of one entry is never taken
    return lumen_attn_rows(t.data_ptr(),
                           t.stride(0) if t.shape[0] > 1 else 0,
                           t.stride(1) if t.shape[1] > 1 else 0)


def _dtype(t: torch.Tensor, *others) -> int:
    if t.dtype not in _DTYPES:
        raise ValueError(f"{t.dtype}: bfloat16 or float16 are supported")
    for o in others:
        if o.dtype != t.dtype:
            raise ValueError("tensors of one call must have one dtype")
    return _DTYPES[t.dtype]


def _out(t: torch.Tensor, like_shape, dtype, what: str = "out") -> int:
    if tuple(t.shape) != tuple(like_shape) or t.dtype != dtype:
        raise ValueError(f"{what} must be {tuple(like_shape)} of {dtype}")
    return _kv._dev(t, what)


def _status(status: torch.Tensor) -> int:
    if status.numel() != 1:
        raise ValueError("status must be one int32 element")
    return _kv._dev(status, "status", torch.int32)


def _scale(scale: Optional[float], head_dim: int) -> float:
    return float(head_dim) ** -0.5 if scale is None else float(scale)


def _call(name: str, args: tuple, stream) -> None:
    _kv._check(getattr(_lib(), name)(*args, _kv._stream_handle(stream)), name)


def _prepared(name: str, args: tuple, keep: tuple) -> "_kv.PreparedCall":
    _lib()
    return _kv.PreparedCall(name, args, (args, keep))


# ------------------------------------------------------------- entry points

def _slots_args(start, end, block_tables, block_size, num_blocks, free,
                free_count, slots, cu, lens, free_left, status, have):
    i32, i64 = torch.int32, torch.int64
    R = start.numel()
    for t, what in ((end, "end"), (lens, "lens"), (have, "have")):
        if t is not None and t.numel() != R:
            raise ValueError(f"{what} must have one entry per request")
    if cu.numel() != R + 1:
        raise ValueError("cu must have num_reqs + 1 entries")
    if free_count.numel() != 1 or free_left.numel() != 1:
        raise ValueError("free_count and free_left are one int64 element")
    _kv._check_tables(block_tables, R)
    # an empty tensor has no address, which would say that no map is wanted
    into = None if slots is None else (_kv._dev(slots, "slots", i64) or
                                       free_left.data_ptr())
    return (_kv._dev(start, "start", i32), _kv._dev(end, "end", i32),
            None if have is None else _kv._dev(have, "have", i32), R,
            _kv._dev(block_tables, "block_tables", i32),
            block_tables.shape[1], int(block_size), int(num_blocks),
            _kv._dev(free, "free", i32),
            _kv._dev(free_count, "free_count", i64), free.numel(),
            into,
            0 if slots is None else slots.numel(),
            _kv._dev(cu, "cu", i32), _kv._dev(lens, "lens", i32),
            _kv._dev(free_left, "free_left", i64), _status(status))


def lumen_attn_slots(start: torch.Tensor, end: torch.Tensor,
                     block_tables: torch.Tensor, block_size: int,
                     num_blocks: int, free: torch.Tensor,
                     free_count: torch.Tensor, slots: Optional[torch.Tensor],
                     cu: torch.Tensor, lens: torch.Tensor,
                     free_left: torch.Tensor, status: torch.Tensor,
                     have: Optional[torch.Tensor] = None,
                     stream: Optional[torch.cuda.Stream] = None) -> None:
    """Pages for the tokens [start, end) of every request, taken from the end
    of the free list into block_tables, and the slot of each packed token
    (slots None: no slot map)."""
    _call("lumen_attn_slots",
          _slots_args(start, end, block_tables, block_size, num_blocks, free,
                      free_count, slots, cu, lens, free_left, status, have),
          stream)


def prepare_slots(start, end, block_tables, block_size, num_blocks, free,
                  free_count, slots, cu, lens, free_left, status,
                  have=None) -> "_kv.PreparedCall":
    """lumen_attn_slots with its arguments checked once; see PreparedCall."""
    args = _slots_args(start, end, block_tables, block_size, num_blocks, free,
                       free_count, slots, cu, lens, free_left, status, have)
    return _prepared("lumen_attn_slots", args,
                     (start, end, block_tables, free, free_count, slots, cu,
                      lens, free_left, status, have))


def _kv4_args(shape, num_blocks, layer, cache, k, v, slots, status):
    """(layout, layer, cache, k rows, v rows, dtype, slots, tokens, status)"""
    D = head_dim4(shape)
    _kv._check_cache(shape, num_blocks, cache, "cache")
    T = slots.numel()
    for t, what in ((k, "k"), (v, "v")):
        if t.shape[0] != T:
            raise ValueError(f"{what} must have one row per slot")
    return (ctypes.byref(_kv.layout(shape, num_blocks)), int(layer),
            _kv._dev(cache, "cache"),
            ctypes.byref(_rows(k, "k", shape.num_kv_heads, D)),
            ctypes.byref(_rows(v, "v", shape.num_kv_heads, D)), _dtype(k, v),
            _kv._dev(slots, "slots", torch.int64), T, _status(status))


def lumen_attn_append4(shape, num_blocks: int, layer: int,
                       cache: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                       slots: torch.Tensor, status: torch.Tensor,
                       stream: Optional[torch.cuda.Stream] = None) -> None:
    """Quantise k and v [tokens, H, D] into their slots of one layer of the
    4-bit cache."""
    _call("lumen_attn_append4",
          _kv4_args(shape, num_blocks, layer, cache, k, v, slots, status),
          stream)


def prepare_append4(shape, num_blocks, layer, cache, k, v, slots,
                    status) -> "_kv.PreparedCall":
    """lumen_attn_append4 with its arguments checked once."""
    return _prepared("lumen_attn_append4",
                     _kv4_args(shape, num_blocks, layer, cache, k, v, slots,
                               status), (cache, k, v, slots, status))


def _read4_args(shape, num_blocks, layer, cache, slots, k, v, status):
    a = _kv4_args(shape, num_blocks, layer, cache, k, v, slots, status)
    return (a[0], a[1], a[2], a[6], a[7], a[3], a[4], a[5], a[8])


def lumen_attn_read4(shape, num_blocks: int, layer: int, cache: torch.Tensor,
                     slots: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                     status: torch.Tensor,
                     stream: Optional[torch.cuda.Stream] = None) -> None:
    """Write the values of the tokens in `slots` of one layer of the 4-bit
    cache to k and v [tokens, H, D]."""
    _call("lumen_attn_read4",
          _read4_args(shape, num_blocks, layer, cache, slots, k, v, status),
          stream)


def prepare_read4(shape, num_blocks, layer, cache, slots, k, v,
                  status) -> "_kv.PreparedCall":
    """lumen_attn_read4 with its arguments checked once."""
    return _prepared("lumen_attn_read4",
                     _read4_args(shape, num_blocks, layer, cache, slots, k, v,
                                 status), (cache, slots, k, v, status))


def lumen_attn_decode4_workspace_bytes(shape, num_reqs: int,
                                       num_q_heads: int) -> int:
    return int(_lib().lumen_attn_decode4_workspace_bytes(
        ctypes.byref(_kv.layout(shape, 1)), int(num_reqs), int(num_q_heads)))


def new_decode4_workspace(shape, num_reqs: int, num_q_heads: int,
                          device=None) -> torch.Tensor:
    """Workspace for decode4 calls of up to num_reqs requests."""
    n = lumen_attn_decode4_workspace_bytes(shape, num_reqs, num_q_heads)
    return torch.empty(max(n, 16), dtype=torch.uint8, device=device or "cuda")


def _decode4_args(shape, num_blocks, layer, cache, block_tables, lens, q, out,
                  workspace, status, scale):
    D = head_dim4(shape)
    _kv._check_cache(shape, num_blocks, cache, "cache")
    R = lens.numel()
    _kv._check_tables(block_tables, R)
    if q.dim() != 3 or q.shape[0] != R:
        raise ValueError("q must be [num_reqs, num_q_heads, head_dim]")
    return (ctypes.byref(_kv.layout(shape, num_blocks)), int(layer),
            _kv._dev(cache, "cache"),
            _kv._dev(block_tables, "block_tables", torch.int32),
            block_tables.shape[1], _kv._dev(lens, "lens", torch.int32), R,
            ctypes.byref(_rows(q, "q", q.shape[1], D)), _dtype(q),
            q.shape[1], _scale(scale, D), _out(out, q.shape, q.dtype),
            _kv._dev(workspace, "workspace"), _kv._nbytes(workspace),
            _status(status))


def lumen_attn_decode4(shape, num_blocks: int, layer: int,
                       cache: torch.Tensor, block_tables: torch.Tensor,
                       lens: torch.Tensor, q: torch.Tensor,
                       out: torch.Tensor, workspace: torch.Tensor,
                       status: torch.Tensor, scale: Optional[float] = None,
                       stream: Optional[torch.cuda.Stream] = None) -> None:
    """Attention of one token per request, q [R, Hq, D], over one layer of
    the 4-bit cache into out (scale None: D ** -0.5)."""
    _call("lumen_attn_decode4",
          _decode4_args(shape, num_blocks, layer, cache, block_tables, lens,
                        q, out, workspace, status, scale), stream)


def prepare_decode4(shape, num_blocks, layer, cache, block_tables, lens, q,
                    out, workspace, status,
                    scale=None) -> "_kv.PreparedCall":
    """lumen_attn_decode4 with its arguments checked once."""
    return _prepared("lumen_attn_decode4",
                     _decode4_args(shape, num_blocks, layer, cache,
                                   block_tables, lens, q, out, workspace,
                                   status, scale),
                     (cache, block_tables, lens, q, out, workspace, status))


def lumen_attn_prompt_workspace_bytes(num_seqs: int, num_q_tokens: int,
                                      num_k_tokens: int, num_q_heads: int,
                                      num_kv_heads: int,
                                      head_dim: int) -> int:
    return int(_lib().lumen_attn_prompt_workspace_bytes(
        num_seqs, num_q_tokens, num_k_tokens, num_q_heads, num_kv_heads,
        head_dim))


def new_prompt_workspace(q: torch.Tensor, k: torch.Tensor,
                         num_seqs: int) -> Optional[torch.Tensor]:
    """Workspace for prompt calls of these sizes; None where they take
    none."""
    n = lumen_attn_prompt_workspace_bytes(num_seqs, q.shape[0], k.shape[0],
                                          q.shape[1], k.shape[1], q.shape[2])
    return torch.empty(n, dtype=torch.uint8, device=q.device) if n else None


def _prompt_args(q, k, v, out, cu_q, status, cu_k, scale, workspace):
    if q.dim() != 3 or k.dim() != 3:
        raise ValueError("q, k and v are [tokens, heads, head_dim]")
    D, H = q.shape[2], k.shape[1]
    if tuple(v.shape) != tuple(k.shape):
        raise ValueError("k and v differ in shape")
    if cu_k is None and k.shape[0] != q.shape[0]:
        raise ValueError("without cu_k, k must have q's tokens")
    if cu_q.numel() < 1 or (cu_k is not None and
                            cu_k.numel() != cu_q.numel()):
        raise ValueError("cu_q and cu_k have num_seqs + 1 entries")
    return (ctypes.byref(_rows(q, "q", q.shape[1], D)),
            ctypes.byref(_rows(k, "k", H, D)),
            ctypes.byref(_rows(v, "v", H, D)), _dtype(q, k, v),
            _kv._dev(cu_q, "cu_q", torch.int32),
            None if cu_k is None else _kv._dev(cu_k, "cu_k", torch.int32),
            cu_q.numel() - 1, q.shape[0], k.shape[0], q.shape[1], H, D,
            _scale(scale, D), _out(out, q.shape, q.dtype),
            None if workspace is None else _kv._dev(workspace, "workspace"),
            0 if workspace is None else _kv._nbytes(workspace),
            _status(status))


def _own_workspace(q, k, cu_q, workspace):
    """The caller's workspace, or one of the call's own."""
    if workspace is None and q.is_cuda and k.dim() == q.dim() == 3:
        return new_prompt_workspace(q, k, cu_q.numel() - 1)
    return workspace


def lumen_attn_prompt(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                      out: torch.Tensor, cu_q: torch.Tensor,
                      status: torch.Tensor,
                      cu_k: Optional[torch.Tensor] = None,
                      scale: Optional[float] = None,
                      workspace: Optional[torch.Tensor] = None,
                      stream: Optional[torch.cuda.Stream] = None) -> None:
    """Causal attention over packed sequences, q [Tq, Hq, D], k and v
    [Tk, H, D], into out [Tq, Hq, D] (cu_k None: the keys are the queries'
    own tokens).  workspace None: one is allocated for the call, on the
    stream it runs on."""
    if stream is not None and workspace is None:
        with torch.cuda.stream(stream):
            workspace = _own_workspace(q, k, cu_q, None)
    workspace = _own_workspace(q, k, cu_q, workspace)
    _call("lumen_attn_prompt",
          _prompt_args(q, k, v, out, cu_q, status, cu_k, scale, workspace),
          stream)


class _OwnWorkspaceCall(_kv.PreparedCall):
    """A prepared call with a workspace that no one else holds: a stream it
    runs on is recorded, so that the memory is not given away while that
    stream still uses it, whenever the object goes."""
    __slots__ = ("_workspace", "_home")

    def __init__(self, name: str, args: tuple, keep: tuple, workspace):
        _lib()
        super().__init__(name, args, (args, keep))
        self._workspace = workspace
        self._home = _kv._stream_handle(None)  # the allocation's

    def __call__(self, stream: Optional[torch.cuda.Stream] = None) -> None:
        super().__call__(stream)
        if _kv._stream_handle(stream) != self._home:
            self._workspace.record_stream(stream or
                                          torch.cuda.current_stream())


def prepare_prompt(q, k, v, out, cu_q, status, cu_k=None, scale=None,
                   workspace=None) -> "_kv.PreparedCall":
    """lumen_attn_prompt with its arguments checked once; workspace None: one
    is allocated and kept, on the current stream, so the object must not be in
    flight twice at a time, and a graph that holds its calls needs it alive."""
    own = workspace is None
    workspace = _own_workspace(q, k, cu_q, workspace)
    args = _prompt_args(q, k, v, out, cu_q, status, cu_k, scale, workspace)
    keep = (q, k, v, out, cu_q, status, cu_k, workspace)
    if own and workspace is not None:
        return _OwnWorkspaceCall("lumen_attn_prompt", args, keep, workspace)
    return _prepared("lumen_attn_prompt", args, keep)
