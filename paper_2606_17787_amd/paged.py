"""Python binding of the operators of 16-bit paged caches (ctypes; argument
marshalling only).  include/lumen_paged.h states what each computes: K and V into
their slots, attention of new tokens over a paged cache, the weights that places
gather, eviction down to a budget, and pages given back.

Each function has the name of the C entry point it calls; the prepare_* twins
check the arguments once and return a kvckpt.PreparedCall.
"""
from __future__ import annotations

import ctypes
import os
import re
from typing import Optional

import torch

from . import attn as _attn
from . import kvckpt as _kv
from .workloads import CacheShape, NHD

HEADER = os.path.join(os.path.dirname(_kv.HEADER), "lumen_paged.h")

LUMEN_PAGED_MAX_ROWS = 1073741824  # include/lumen_paged.h
LUMEN_PAGED_MAX_PLACES = 1048576  # include/lumen_paged.h


def exported_names():
    """Entry points declared in include/lumen_paged.h."""
    with open(HEADER) as f:
        text = f.read()
    return sorted(set(re.findall(r"\b(lumen_paged_\w+)\s*\(", text)))


_BOUND = None


def _lib():
    global _BOUND
    lib = _kv.load_library()
    if _BOUND is lib:
        return lib
    p, i32, i64, sz, f32 = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64,
                            ctypes.c_size_t, ctypes.c_float)
    lay = ctypes.POINTER(_kv.lumen_kv_layout)
    rows = ctypes.POINTER(_attn.lumen_attn_rows)
    sigs = {
        "lumen_paged_append": (ctypes.c_int,
                               [lay, i32, p, rows, rows, p, p, i64, p, p, p]),
        "lumen_paged_attend_workspace_bytes": (sz, [lay, i32, i32, i64, i32,
                                                    i32]),
        "lumen_paged_attend": (ctypes.c_int,
                               [lay, i32, p, p, i32, p, p, i32, rows, i64,
                                i32, i32, i32, f32, p, p, p, sz, p, p]),
        "lumen_paged_weigh_workspace_bytes": (sz, [lay, i32, i32, i64, i32,
                                                   i32]),
        "lumen_paged_weigh": (ctypes.c_int,
                              [lay, i32, p, p, i32, p, p, i32, rows, i64, i32,
                               i32, i32, f32, p, p, p, sz, p, p]),
        "lumen_paged_evict_workspace_bytes": (sz, [lay, i32, i32, i32]),
        "lumen_paged_evict": (ctypes.c_int,
                              [lay, i32, i32, p, p, p, i32, p, p, p, i32, i32,
                               p, p, sz, p, p]),
        "lumen_paged_release": (ctypes.c_int,
                                [p, p, i32, p, i32, i32, i64, p, p, i64, p, p,
                                 p]),
    }
    for name, (res, args) in sigs.items():
        f = getattr(lib, name)
        f.restype, f.argtypes = res, args
    _BOUND = lib
    return lib


# ------------------------------------------------------------ marshalling

def ledger_dims(shape, num_blocks: int):
    """Dimensions of a cache's ledger, int32 (the weights are the bits of
    float32): layers, (weights, positions), blocks, heads, slots of a block."""
    return (shape.num_layers, 2, int(num_blocks), shape.num_kv_heads,
            shape.block_size)


def new_ledger(shape, num_blocks: int, device=None) -> torch.Tensor:
    """A ledger for a cache; append starts the places that it fills."""
    return torch.zeros(ledger_dims(shape, num_blocks), dtype=torch.int32,
                       device=device or "cuda")


def weights_of(ledger: torch.Tensor) -> torch.Tensor:
    """The ledger's weights [layers, blocks, heads, block_size], a view."""
    return ledger[:, 0].view(torch.float32)


def positions_of(ledger: torch.Tensor) -> torch.Tensor:
    """The ledger's positions [layers, blocks, heads, block_size], a view."""
    return ledger[:, 1]


def ledger_shape(shape) -> CacheShape:
    """The ledger as a cache of the checkpoint calls, a page a token: they take
    it with this shape, the same block tables and ranges counted in pages."""
    words = shape.num_kv_heads * shape.block_size
    if words % 4:
        raise ValueError(f"{shape.num_kv_heads} heads of {shape.block_size} "
                         "slots: a page must hold a multiple of 4 words")
    return CacheShape(shape.num_layers, 1, words, 1, NHD, 4)


def _check_ledger(shape, num_blocks: int, ledger: torch.Tensor) -> int:
    if tuple(ledger.shape) != ledger_dims(shape, num_blocks):
        raise ValueError(f"ledger must be {ledger_dims(shape, num_blocks)}, "
                         f"got {tuple(ledger.shape)}")
    return _kv._dev(ledger, "ledger", torch.int32)


def _call(name: str, args: tuple, stream) -> None:
    _kv._check(getattr(_lib(), name)(*args, _kv._stream_handle(stream)), name)


def _prepared(name: str, args: tuple, keep: tuple) -> "_kv.PreparedCall":
    _lib()
    return _kv.PreparedCall(name, args, (args, keep))


# ------------------------------------------------------------- entry points

def _append_args(shape, num_blocks, layer, cache, k, v, slots, status, ledger,
                 positions):
    _kv._check_cache(shape, num_blocks, cache, "cache")
    T = slots.numel()
    for t, what in ((k, "k"), (v, "v")):
        if t.shape[0] != T:
            raise ValueError(f"{what} must have one row per slot")
        if t.dtype != cache.dtype:
            raise ValueError(f"{what} must be {cache.dtype}, as the cache")
    if (ledger is None) != (positions is None):
        raise ValueError("ledger and positions come together")
    if positions is not None and positions.numel() != T:
        raise ValueError("positions must have one entry per slot")
    H, D = shape.num_kv_heads, shape.head_dim
    return (ctypes.byref(_kv.layout(shape, num_blocks)), int(layer),
            _kv._dev(cache, "cache"), ctypes.byref(_attn._rows(k, "k", H, D)),
            ctypes.byref(_attn._rows(v, "v", H, D)),
            _kv._dev(slots, "slots", torch.int64),
            None if positions is None else
            _kv._dev(positions, "positions", torch.int32), T,
            None if ledger is None else
            _check_ledger(shape, num_blocks, ledger),
            _attn._status(status))


def lumen_paged_append(shape, num_blocks: int, layer: int,
                       cache: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                       slots: torch.Tensor, status: torch.Tensor,
                       ledger: Optional[torch.Tensor] = None,
                       positions: Optional[torch.Tensor] = None,
                       stream: Optional[torch.cuda.Stream] = None) -> None:
    """Copy k and v [tokens, H, D] into their slots of one layer; with a ledger,
    start their places there with weight 0 and the tokens' positions (int32)."""
    _call("lumen_paged_append",
          _append_args(shape, num_blocks, layer, cache, k, v, slots, status,
                       ledger, positions), stream)


def prepare_append(shape, num_blocks, layer, cache, k, v, slots, status,
                   ledger=None, positions=None) -> "_kv.PreparedCall":
    """lumen_paged_append with its arguments checked once."""
    return _prepared("lumen_paged_append",
                     _append_args(shape, num_blocks, layer, cache, k, v, slots,
                                  status, ledger, positions),
                     (cache, k, v, slots, status, ledger, positions))


def _workspace_bytes(name, shape, bt_cols, num_reqs, num_tokens, max_new,
                     num_q_heads):
    return int(getattr(_lib(), name)(
        ctypes.byref(_kv.layout(shape, 1)), int(bt_cols), int(num_reqs),
        int(num_tokens), int(max_new), int(num_q_heads)))


def lumen_paged_attend_workspace_bytes(shape, bt_cols: int, num_reqs: int,
                                       num_tokens: int, max_new: int,
                                       num_q_heads: int) -> int:
    return _workspace_bytes("lumen_paged_attend_workspace_bytes", shape,
                            bt_cols, num_reqs, num_tokens, max_new,
                            num_q_heads)


def lumen_paged_weigh_workspace_bytes(shape, bt_cols: int, num_reqs: int,
                                      num_tokens: int, max_new: int,
                                      num_q_heads: int) -> int:
    return _workspace_bytes("lumen_paged_weigh_workspace_bytes", shape,
                            bt_cols, num_reqs, num_tokens, max_new,
                            num_q_heads)


def _most_new(q, max_new) -> int:
    return q.shape[0] if max_new is None else int(max_new)


def _new_workspace(name, shape, block_tables, lens, q, max_new):
    if q.dim() != 3 or block_tables.dim() != 2 or not q.is_cuda:
        return None
    n = _workspace_bytes(name, shape, block_tables.shape[1], lens.numel(),
                         q.shape[0], _most_new(q, max_new), q.shape[1])
    return torch.empty(n, dtype=torch.uint8, device=q.device) if n else None


def new_attend_workspace(shape, block_tables, lens, q,
                         max_new=None) -> Optional[torch.Tensor]:
    """Workspace for attend calls of these sizes; None where they take none."""
    return _new_workspace("lumen_paged_attend_workspace_bytes", shape,
                          block_tables, lens, q, max_new)


def new_weigh_workspace(shape, block_tables, lens, q,
                        max_new=None) -> Optional[torch.Tensor]:
    """Workspace for weigh calls of these sizes: None, at present they take none."""
    return _new_workspace("lumen_paged_weigh_workspace_bytes", shape,
                          block_tables, lens, q, max_new)


def _query_args(shape, num_blocks, layer, cache, block_tables, lens, cu, q,
                max_new, scale):
    _kv._check_cache(shape, num_blocks, cache, "cache")
    R = lens.numel()
    _kv._check_tables(block_tables, R)
    if cu.numel() != R + 1:
        raise ValueError("cu must have num_reqs + 1 entries")
    if q.dim() != 3:
        raise ValueError("q must be [tokens, num_q_heads, head_dim]")
    if q.dtype != cache.dtype:
        raise ValueError(f"q must be {cache.dtype}, as the cache")
    return (ctypes.byref(_kv.layout(shape, num_blocks)), int(layer),
            _kv._dev(cache, "cache"),
            _kv._dev(block_tables, "block_tables", torch.int32),
            block_tables.shape[1], _kv._dev(lens, "lens", torch.int32),
            _kv._dev(cu, "cu", torch.int32), R,
            ctypes.byref(_attn._rows(q, "q", q.shape[1], shape.head_dim)),
            q.shape[0], _most_new(q, max_new), _attn._dtype(q), q.shape[1],
            _attn._scale(scale, shape.head_dim))


def _lse(lse: torch.Tensor, q: torch.Tensor) -> int:
    if tuple(lse.shape) != tuple(q.shape[:2]):
        raise ValueError(f"lse must be {tuple(q.shape[:2])}")
    return _kv._dev(lse, "lse", torch.float32)


def _ws(workspace):
    if workspace is None:
        return None, 0
    return _kv._dev(workspace, "workspace"), _kv._nbytes(workspace)


def _attend_args(shape, num_blocks, layer, cache, block_tables, lens, cu, q,
                 out, status, max_new, lse, scale, workspace):
    return _query_args(shape, num_blocks, layer, cache, block_tables, lens, cu,
                       q, max_new, scale) + (
        _attn._out(out, q.shape, q.dtype),
        None if lse is None else _lse(lse, q), *_ws(workspace),
        _attn._status(status))


def _own_workspace(stream, workspace, *sizes):
    """The caller's workspace, or one of the attend call's own, on its stream."""
    if workspace is not None:
        return workspace
    if stream is None:
        return new_attend_workspace(*sizes)
    with torch.cuda.stream(stream):
        return new_attend_workspace(*sizes)


def lumen_paged_attend(shape, num_blocks: int, layer: int,
                       cache: torch.Tensor, block_tables: torch.Tensor,
                       lens: torch.Tensor, cu: torch.Tensor, q: torch.Tensor,
                       out: torch.Tensor, status: torch.Tensor,
                       max_new: Optional[int] = None,
                       lse: Optional[torch.Tensor] = None,
                       scale: Optional[float] = None,
                       workspace: Optional[torch.Tensor] = None,
                       stream: Optional[torch.cuda.Stream] = None) -> None:
    """Attention of each request's new tokens, q [tokens, Hq, D] packed by cu,
    over its lens places of one layer of the cache (the new tokens' own are the
    last), into out and lse (float32 [tokens, Hq]; None: not wanted).  max_new:
    at least the most new tokens of a request (None: all).  scale None:
    D ** -0.5.  workspace None: one is allocated for the call, on the stream it
    runs on."""
    workspace = _own_workspace(stream, workspace, shape, block_tables, lens, q,
                               max_new)
    _call("lumen_paged_attend",
          _attend_args(shape, num_blocks, layer, cache, block_tables, lens, cu,
                       q, out, status, max_new, lse, scale, workspace), stream)


def prepare_attend(shape, num_blocks, layer, cache, block_tables, lens, cu, q,
                   out, status, max_new=None, lse=None, scale=None,
                   workspace=None) -> "_kv.PreparedCall":
    """lumen_paged_attend with its arguments checked once; workspace None: one
    is allocated and kept, on the current stream, so the object must not be in
    flight twice at a time, and a graph that holds its calls needs it alive."""
    ws = _own_workspace(None, workspace, shape, block_tables, lens, q, max_new)
    args = _attend_args(shape, num_blocks, layer, cache, block_tables, lens,
                        cu, q, out, status, max_new, lse, scale, ws)
    keep = (cache, block_tables, lens, cu, q, out, status, lse, ws)
    if workspace is None and ws is not None:
        _lib()
        return _attn._OwnWorkspaceCall("lumen_paged_attend", args, keep, ws)
    return _prepared("lumen_paged_attend", args, keep)


def _weigh_args(shape, num_blocks, layer, cache, block_tables, lens, cu, q,
                lse, ledger, status, max_new, scale, workspace):
    return _query_args(shape, num_blocks, layer, cache, block_tables, lens, cu,
                       q, max_new, scale) + (
        _lse(lse, q), _check_ledger(shape, num_blocks, ledger),
        *_ws(workspace), _attn._status(status))


def lumen_paged_weigh(shape, num_blocks: int, layer: int, cache: torch.Tensor,
                      block_tables: torch.Tensor, lens: torch.Tensor,
                      cu: torch.Tensor, q: torch.Tensor, lse: torch.Tensor,
                      ledger: torch.Tensor, status: torch.Tensor,
                      max_new: Optional[int] = None,
                      scale: Optional[float] = None,
                      workspace: Optional[torch.Tensor] = None,
                      stream: Optional[torch.cuda.Stream] = None) -> None:
    """Add the attention weights of each request's last tokens, q and lse as
    attend had and gave them (or the last ones of each request alone, with a cu
    of their own), to the places that they see in the ledger.  max_new, at least
    the most tokens of a request, chooses the form: None stands for all tokens of
    the call, and costs a batch of single tokens up to three times their time.  No
    workspace is needed."""
    _call("lumen_paged_weigh",
          _weigh_args(shape, num_blocks, layer, cache, block_tables, lens, cu,
                      q, lse, ledger, status, max_new, scale, workspace),
          stream)


def prepare_weigh(shape, num_blocks, layer, cache, block_tables, lens, cu, q,
                  lse, ledger, status, max_new=None, scale=None,
                  workspace=None) -> "_kv.PreparedCall":
    """lumen_paged_weigh with its arguments checked once."""
    return _prepared("lumen_paged_weigh",
                     _weigh_args(shape, num_blocks, layer, cache, block_tables,
                                 lens, cu, q, lse, ledger, status, max_new,
                                 scale, workspace),
                     (cache, block_tables, lens, cu, q, lse, ledger, status,
                      workspace))


def lumen_paged_evict_workspace_bytes(shape, num_layers: int, bt_cols: int,
                                      num_reqs: int) -> int:
    return int(_lib().lumen_paged_evict_workspace_bytes(
        ctypes.byref(_kv.layout(shape, 1)), int(num_layers), int(bt_cols),
        int(num_reqs)))


def new_evict_workspace(shape, num_reqs: int, bt_cols: int, device=None,
                        num_layers: Optional[int] = None) -> torch.Tensor:
    """Workspace for evict calls over num_layers layers (None: all)."""
    n = lumen_paged_evict_workspace_bytes(
        shape, shape.num_layers if num_layers is None else num_layers, bt_cols,
        num_reqs)
    return torch.empty(max(n, 16), dtype=torch.uint8, device=device or "cuda")


def _evict_args(shape, num_blocks, cache, ledger, block_tables, lens, keep,
                recent_from, left, workspace, status, sinks, first_layer,
                num_layers):
    _kv._check_cache(shape, num_blocks, cache, "cache")
    R, i32 = lens.numel(), torch.int32
    _kv._check_tables(block_tables, R)
    for t, what in ((keep, "keep"), (recent_from, "recent_from"),
                    (left, "left")):
        if t.numel() != R:
            raise ValueError(f"{what} must have one entry per request")
    if num_layers is None:
        num_layers = shape.num_layers - int(first_layer)
    return (ctypes.byref(_kv.layout(shape, num_blocks)), int(first_layer),
            int(num_layers), _kv._dev(cache, "cache"),
            _check_ledger(shape, num_blocks, ledger),
            _kv._dev(block_tables, "block_tables", i32),
            block_tables.shape[1], _kv._dev(lens, "lens", i32),
            _kv._dev(keep, "keep", i32),
            _kv._dev(recent_from, "recent_from", i32), int(sinks), R,
            _kv._dev(left, "left", i32), *_ws(workspace),
            _attn._status(status))


def lumen_paged_evict(shape, num_blocks: int, cache: torch.Tensor,
                      ledger: torch.Tensor, block_tables: torch.Tensor,
                      lens: torch.Tensor, keep: torch.Tensor,
                      recent_from: torch.Tensor, left: torch.Tensor,
                      workspace: torch.Tensor, status: torch.Tensor,
                      sinks: int = 0, first_layer: int = 0,
                      num_layers: Optional[int] = None,
                      stream: Optional[torch.cuda.Stream] = None) -> None:
    """Hold every request to keep places in each layer (num_layers None: all
    from first_layer on) and head: the positions under `sinks` and from
    recent_from on first, then those that gathered the most weight.  left
    becomes the requests' new numbers of places."""
    _call("lumen_paged_evict",
          _evict_args(shape, num_blocks, cache, ledger, block_tables, lens,
                      keep, recent_from, left, workspace, status, sinks,
                      first_layer, num_layers), stream)


def prepare_evict(shape, num_blocks, cache, ledger, block_tables, lens, keep,
                  recent_from, left, workspace, status, sinks=0, first_layer=0,
                  num_layers=None) -> "_kv.PreparedCall":
    """lumen_paged_evict with its arguments checked once."""
    return _prepared("lumen_paged_evict",
                     _evict_args(shape, num_blocks, cache, ledger,
                                 block_tables, lens, keep, recent_from, left,
                                 workspace, status, sinks, first_layer,
                                 num_layers),
                     (cache, ledger, block_tables, lens, keep, recent_from,
                      left, workspace, status))


def _release_args(lens, have, block_tables, block_size, num_blocks, free,
                  free_count, free_now, status):
    i32, i64 = torch.int32, torch.int64
    R = lens.numel()
    if have.numel() != R:
        raise ValueError("have must have one entry per request")
    if free_count.numel() != 1 or free_now.numel() != 1:
        raise ValueError("free_count and free_now are one int64 element")
    _kv._check_tables(block_tables, R)
    return (_kv._dev(lens, "lens", i32), _kv._dev(have, "have", i32), R,
            _kv._dev(block_tables, "block_tables", i32),
            block_tables.shape[1], int(block_size), int(num_blocks),
            _kv._dev(free, "free", i32),
            _kv._dev(free_count, "free_count", i64), free.numel(),
            _kv._dev(free_now, "free_now", i64), _attn._status(status))


def lumen_paged_release(lens: torch.Tensor, have: torch.Tensor,
                        block_tables: torch.Tensor, block_size: int,
                        num_blocks: int, free: torch.Tensor,
                        free_count: torch.Tensor, free_now: torch.Tensor,
                        status: torch.Tensor,
                        stream: Optional[torch.cuda.Stream] = None) -> None:
    """The pages behind every request's first lens places, up to those of its
    first have, go behind the free list's free_count blocks."""
    _call("lumen_paged_release",
          _release_args(lens, have, block_tables, block_size, num_blocks, free,
                        free_count, free_now, status), stream)


def prepare_release(lens, have, block_tables, block_size, num_blocks, free,
                    free_count, free_now, status) -> "_kv.PreparedCall":
    """lumen_paged_release with its arguments checked once."""
    return _prepared("lumen_paged_release",
                     _release_args(lens, have, block_tables, block_size,
                                   num_blocks, free, free_count, free_now,
                                   status),
                     (lens, have, block_tables, free, free_count, free_now,
                      status))
