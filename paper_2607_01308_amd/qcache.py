"""Serving a merged cache from 8-bit pages: the binding of cm_qcache_tables,
cm_qcache_write and cm_qcache_attention (include/cmerge.h). ServingCache (serving.py)
strings them together for a set of requests.

A cache holds, for each layer and K/V, pages of B tokens of every head: codes
[L, 2, P, H, B, d] in float8_e4m3fn and scales [L, 2, P, H] in float32, one scale for a
page and a head; a stored value is code * scale. Every call enqueues its work on one
stream (the `stream` argument, else the current one), marks the tensors it was given as
in use there and does not wait: lengths, tables and slots stay on the device."""

from __future__ import annotations

import ctypes
from contextlib import nullcontext
from dataclasses import dataclass
from typing import Dict, Optional, Sequence

import torch

from . import _cabi as C
from .binding import _DTYPES

CODES = torch.float8_e4m3fn


class QCache:
    """An 8-bit paged cache over tensors of the caller: codes [L, 2, P, H, B, d]
    (float8_e4m3fn or uint8) and scales [L, 2, P, H] (float32), both contiguous and on
    one GPU."""

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor):
        if codes.dim() != 6 or codes.shape[1] != 2 or not codes.is_contiguous():
            raise ValueError("codes must be a contiguous [L, 2, P, H, B, d] tensor")
        if codes.dtype is not CODES and codes.dtype is not torch.uint8:
            raise TypeError(f"codes must be float8_e4m3fn or uint8, got {codes.dtype}")
        if scales.dtype is not torch.float32:
            raise TypeError(f"scales must be float32, got {scales.dtype}")
        if scales.shape != codes.shape[:4] or not scales.is_contiguous():
            raise ValueError(f"scales must be a contiguous {list(codes.shape[:4])} tensor")
        if not codes.is_cuda or scales.device != codes.device:
            raise ValueError("codes and scales must live on one GPU")
        self.codes, self.scales = codes, scales
        self.device = codes.device
        self.L, _, self.P, self.H, self.B, self.d = codes.shape
        self.struct = C.CmQcache(self.L, self.H, self.d, self.B, self.P, codes.data_ptr(),
                                 scales.data_ptr())

    @classmethod
    def empty(cls, L: int, H: int, d: int, pages: int, block: int = 16,
              device="cuda") -> "QCache":
        """A cache of zeros."""
        codes = torch.zeros((L, 2, pages, H, block, d), dtype=torch.uint8, device=device)
        return cls(codes.view(CODES), torch.zeros((L, 2, pages, H), device=device))

    def __repr__(self) -> str:
        return (f"QCache(L={self.L}, H={self.H}, d={self.d}, pages={self.P}, block={self.B}, "
                f"device={self.device})")


def _made_on(stream):
    """Where tensors that a call makes are allocated: on the stream it enqueues on."""
    return nullcontext() if stream is None else torch.cuda.stream(stream)


def _use(stream, device, *tensors):
    """The stream a call enqueues on and whether its GPU is the current one, with the tensors
    its kernels read and write marked as in use there: their memory must not go to another
    tensor before that work has finished, whichever stream they were allocated on."""
    if stream is None:
        stream = torch.cuda.current_stream(device.index)
    elif stream.device != device:
        raise ValueError(f"the stream is of {stream.device}, the tensors live on {device}")
    for t in tensors:
        if t is not None:
            t.record_stream(stream)
    return stream, device.index == torch.cuda.current_device()


def _call(here: bool, device, f, *args) -> int:
    """f(*args) with `device` as the current GPU (here: it is): the library enqueues there, and a
    GPU's default stream has the same handle as any other's."""
    if here:
        return f(*args)
    with torch.cuda.device(device):
        return f(*args)


def _int32(x: int, name: str) -> int:
    """A number that the library takes in 32 bits (ctypes would cut it to them)."""
    if not -2 ** 31 <= x < 2 ** 31:
        raise ValueError(f"{name} must be a number of 32 bits, got {x}")
    return x


def _check(t: torch.Tensor, name: str, dtype, device, shape=None) -> torch.Tensor:
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.device != device:
        raise ValueError(f"{name} must live on {device}, got {t.device}")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{name} must have shape {list(shape)}, got {list(t.shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t


@dataclass
class QCacheStep:
    """What cm_qcache_tables makes of a step, on the device: slots [tokens] int64, rows
    [n + 1] and lens [n] int32, info [4] int64 (status, tokens, pages taken, longest
    length)."""
    slots: torch.Tensor
    rows: torch.Tensor
    lens: torch.Tensor
    info: torch.Tensor

    def check(self) -> "QCacheStep":
        """Waits for the step and raises if it was refused (nothing was written then)."""
        status, tokens, pages, longest = self.info.tolist()
        if status != C.CM_OK:
            raise C.CmError(status, "cm_qcache_tables",
                            f"the step was refused: {tokens} new tokens, {pages} pages needed, "
                            f"longest request {longest} tokens (a length is negative, the new "
                            "tokens are not as many as given, a table row is too short or the "
                            "free list is)")
        return self


def qcache_tables(pages: int, block: int, held: torch.Tensor, new: torch.Tensor,
                  free: torch.Tensor, table: torch.Tensor, tokens: int,
                  stream=None) -> QCacheStep:
    """cm_qcache_tables: the table rows [n, width] (in place), slots, rows and lengths
    of a step in which request r, holding held[r] tokens, brings new[r] more; free: the
    page ids to take from, in order; tokens: the sum of new."""
    dev = table.device
    if table.dim() != 2:
        raise ValueError("table must be [n, width]")
    n, width = table.shape
    i32 = torch.int32
    _check(table, "table", i32, dev)
    _check(held, "held", i32, dev, (n,))
    _check(new, "new", i32, dev, (n,))
    _check(free, "free", i32, dev)
    with _made_on(stream):
        step = QCacheStep(torch.empty(tokens, dtype=torch.int64, device=dev),
                          torch.empty(n + 1, dtype=i32, device=dev),
                          torch.empty(n, dtype=i32, device=dev),
                          torch.empty(4, dtype=torch.int64, device=dev))
    s, here = _use(stream, dev, held, new, free, table)
    C.check(_call(here, dev, C.lib().cm_qcache_tables,
                  pages, _int32(block, "block"), n, held.data_ptr(), new.data_ptr(), free.data_ptr(), free.numel(),
                  table.data_ptr(), width, tokens, step.slots.data_ptr(), step.rows.data_ptr(),
                  step.lens.data_ptr(), step.info.data_ptr(), s.cuda_stream), "cm_qcache_tables")
    return step


def check_rows(x: torch.Tensor, name: str, device) -> None:
    """What cm_qcache_write needs of rows [tokens, H, d] beside their shape and type."""
    if x.device != device:
        raise ValueError(f"{name} must live on {device}, got {x.device}")
    if x.stride(2) != 1:
        raise ValueError(f"the last dimension of {name} must be contiguous")
    if x.numel() and (x.data_ptr() % 16 or any(x.shape[i] > 1 and x.stride(i) * x.element_size() % 16
                                               for i in (0, 1))):
        raise ValueError(f"{name} must be 16-byte aligned, and its strides multiples of 16 bytes")


def _rows(x: torch.Tensor, name: str, cache: QCache, tokens: int):
    """The layers of x and its rows as the library takes them."""
    shape, stride = x.shape, x.stride()
    if len(shape) == 3:
        shape, stride = (1, *shape), (0, *stride)
    if len(shape) != 4 or shape[1:] != (tokens, cache.H, cache.d):
        raise ValueError(f"{name} must be [layers, {tokens}, {cache.H}, {cache.d}], got "
                         f"{list(x.shape)}")
    if x.device != cache.device:
        raise ValueError(f"{name} must live on {cache.device}")
    if stride[3] != 1:
        raise ValueError(f"the last dimension of {name} must be contiguous")
    return shape[0], C.CmQrows(x.data_ptr(), *stride[:3])


def qcache_write(cache: QCache, layer: int, k: torch.Tensor, v: torch.Tensor,
                 slots: torch.Tensor, stream=None) -> None:
    """cm_qcache_write: rows k and v, [tokens, H, d] of one layer or [layers, tokens, H, d]
    of the layers from `layer` on, into their slots. Strides are free but for the last
    dimension, in multiples of 16 bytes."""
    tokens = slots.numel()
    _check(slots, "slots", torch.int64, cache.device)
    layers, kr = _rows(k, "k", cache, tokens)
    v_layers, vr = _rows(v, "v", cache, tokens)
    if k.dtype not in _DTYPES or v.dtype is not k.dtype:
        raise TypeError(f"k and v must both be bfloat16 or float32, got {k.dtype} and {v.dtype}")
    if layers != v_layers:
        raise ValueError("k and v must have the same layers")
    s, here = _use(stream, cache.device, cache.codes, cache.scales, k, v, slots)
    C.check(_call(here, cache.device, C.lib().cm_qcache_write, ctypes.byref(cache.struct),
                  _int32(layer, "layer"), layers, _DTYPES[k.dtype], ctypes.byref(kr), ctypes.byref(vr), tokens,
                  slots.data_ptr(), s.cuda_stream), "cm_qcache_write")


_WS: Dict[tuple, torch.Tensor] = {}
_NONE = torch.empty(0, dtype=torch.uint8)


def _workspace(cache: QCache, step: C.CmQattention, size: str) -> torch.Tensor:
    """Scratch for a call, allocated on the current stream."""
    need = ctypes.c_size_t(0)
    C.check(getattr(C.lib(), size)(ctypes.byref(cache.struct), ctypes.byref(step),
                                   ctypes.byref(need)), size)
    ws = torch.empty(need.value, dtype=torch.uint8, device=cache.device)
    # the calls count in it, and leave their counters at zero
    ws[:C.CM_QCACHE_COUNTER_BYTES].zero_()
    return ws


def release_qcache_workspace() -> None:
    _WS.clear()


def _attention_step(cache: QCache, q, table, lens, rows, max_rows, scale, window, out, lse, stream):
    """The checked arguments of an attention call as the library takes them, with out and lse."""
    dev = cache.device
    if q.dim() != 3 or q.shape[2] != cache.d:
        raise ValueError(f"q must be [rows, q_heads, {cache.d}], got {list(q.shape)}")
    if q.dtype not in _DTYPES:
        raise TypeError(f"unsupported dtype {q.dtype} (bfloat16 or float32)")
    if q.device != dev:
        raise ValueError(f"q must live on {dev}")
    n_rows, q_heads, d = q.shape
    if q.stride(2) != 1:
        raise ValueError("the last dimension of q must be contiguous")
    if table.dim() != 2:
        raise ValueError("table must be [n, width]")
    n, width = table.shape
    _check(table, "table", torch.int32, dev)
    _check(lens, "lens", torch.int32, dev, (n,))
    if rows is not None:
        _check(rows, "rows", torch.int32, dev, (n + 1,))
    if max_rows is None:
        max_rows = 1 if rows is None else n_rows
    if out is None or lse is None:
        with _made_on(stream):
            if out is None:
                out = torch.empty((n_rows, q_heads, d), dtype=q.dtype, device=dev)
            if lse is None:
                lse = torch.empty((n_rows, q_heads), dtype=torch.float32, device=dev)
    if out.shape != q.shape or out.dtype is not q.dtype or out.device != dev or out.stride(2) != 1:
        raise ValueError("out must have q's shape, type and device and a contiguous last dimension")
    _check(lse, "lse", torch.float32, dev, (n_rows, q_heads))
    step = C.CmQattention(
        n, q_heads, _DTYPES[q.dtype], _int32(window, "window"), n_rows, _int32(max_rows, "max_rows"),
        d ** -0.5 if scale is None else scale, q.data_ptr(), q.stride(0), q.stride(1),
        out.data_ptr(), out.stride(0), out.stride(1), lse.data_ptr(),
        None if rows is None else rows.data_ptr(), lens.data_ptr(), table.data_ptr(), width)
    return step, out, lse


def qcache_attention(cache: QCache, layer: int, q: torch.Tensor, table: torch.Tensor,
                     lens: torch.Tensor, rows: Optional[torch.Tensor] = None,
                     max_rows: Optional[int] = None, scale: Optional[float] = None,
                     window: int = 0, out: Optional[torch.Tensor] = None,
                     lse: Optional[torch.Tensor] = None, stream=None):
    """cm_qcache_attention: queries q [rows, q_heads, d] over one layer of the cache;
    returns (out, lse). table [n, width], lens [n]: each request's pages and tokens, the
    step's own included; rows [n + 1]: where each request's query rows begin (None: one
    row for each request); max_rows: the most rows of a request (default: all of them,
    or 1 without rows; the host does not see rows, so a decoding step that gives rows and
    not max_rows goes the slower way of prompts); scale: of the scores (default
    d ** -0.5); window: positions that a query sees, itself included (0: all up to its
    own). out: q's shape and type; lse [rows, q_heads] float32 (made if not given)."""
    step, out, lse = _attention_step(cache, q, table, lens, rows, max_rows, scale, window, out, lse,
                                     stream)
    s, here = _use(stream, cache.device, cache.codes, cache.scales, q, table, lens, rows, out, lse)
    with _made_on(None if stream is None and here else s):
        C.check(_attention(cache, layer, step, s), "cm_qcache_attention")
    return out, lse


def _attention(cache: QCache, layer: int, step: C.CmQattention, s, call: str = "cm_qcache_attention",
               more: tuple = ()) -> int:
    """The call on s, which is the current stream; more: arguments of it after the step.

    Scratch is cached for (device, stream), so calls on two streams never share it, and
    replaced by a larger one where it is too small. A call that is being captured gets
    scratch of its graph's own memory, whose counters every replay clears: what is cached may
    be replaced while the graph still refers to it."""
    capturing = torch.cuda.is_current_stream_capturing()
    key = (cache.device, s.cuda_stream)
    layer = _int32(layer, "layer")
    size = call + "_size"
    ws = _workspace(cache, step, size) if capturing else _WS.get(key, _NONE)
    args = ctypes.byref(cache.struct), layer, ctypes.byref(step), *more
    f = getattr(C.lib(), call)
    status = f(*args, ws.data_ptr(), ws.numel(), s.cuda_stream)
    if status == C.CM_EWORKSPACE and not capturing:
        ws = _WS[key] = _workspace(cache, step, size)
        status = f(*args, ws.data_ptr(), ws.numel(), s.cuda_stream)
    return status
