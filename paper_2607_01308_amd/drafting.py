"""Decoding with drafted tokens over the 8-bit paged cache: the binding of cm_norm_rotate,
cm_qcache_tree, cm_qcache_tree_attention, cm_verify_drafts, cm_qcache_keep and
cm_qcache_copy (include/cmerge.h). ServingCache (serving.py) strings them together.

As in qcache.py, every call enqueues its work on one stream (the `stream` argument, else
the current one), marks the tensors it was given as in use there and does not wait."""

from __future__ import annotations

import ctypes
import functools
from dataclasses import dataclass
from typing import Optional

import torch

from . import _cabi as C
from .binding import _DTYPES, _STYLES
from .qcache import _WS, QCache, _attention, _attention_step, _call, _check, _int32, _made_on, _use


def _heads(x: torch.Tensor, out: Optional[torch.Tensor], weight: Optional[torch.Tensor], name: str,
           device, tokens: int, d: int, dtype, stream):
    """The heads of x as the library takes them, and where their results go."""
    if x.dim() != 3 or x.shape[0] != tokens or x.shape[2] != d:
        raise ValueError(f"{name} must be [{tokens}, heads, {d}], got {list(x.shape)}")
    if x.dtype is not dtype:
        raise TypeError(f"q and k must both be bfloat16 or float32, got {x.dtype}")
    if x.device != device:
        raise ValueError(f"{name} must live on {device}, got {x.device}")
    if out is None and stream is None:
        out = x.new_empty(x.shape)
    elif out is None:
        with _made_on(stream):
            out = x.new_empty(x.shape)
    elif out.shape != x.shape or out.dtype is not dtype or out.device != device:
        raise ValueError(f"{name}_out must have {name}'s shape, type and device")
    if x.stride(2) != 1 or out.stride(2) != 1:
        raise ValueError(f"the last dimension of {name} and of its results must be contiguous")
    if weight is not None:
        if weight.dtype not in _DTYPES:
            raise TypeError(f"{name}_weight must be bfloat16 or float32, got {weight.dtype}")
        _check(weight, f"{name}_weight", weight.dtype, device, (d,))
    rows = C.CmHeadRows(x.data_ptr(), x.stride(0), x.stride(1), out.data_ptr(), out.stride(0),
                        out.stride(1), None if weight is None else weight.data_ptr(),
                        0 if weight is None else _DTYPES[weight.dtype], x.shape[1])
    return out, rows


def norm_rotate(q: torch.Tensor, k: Optional[torch.Tensor], positions: torch.Tensor, rope_base: float,
                style: str = "half", q_weight: Optional[torch.Tensor] = None,
                k_weight: Optional[torch.Tensor] = None, eps: float = 1e-6,
                q_out: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None, stream=None):
    """cm_norm_rotate: queries q [tokens, q_heads, d] and keys k [tokens, heads, d] (or None),
    each head divided by its root mean square and multiplied by its weight [d] (None: not
    normalised), then rotated for positions [tokens] (int32); returns (q_out, k_out), made if not
    given, which may be q and k themselves. Strides are free but for the last dimension, in
    multiples of 16 bytes: q and k may be parts of one projection's output."""
    if q.dim() != 3:
        raise ValueError(f"q must be [tokens, heads, d], got {list(q.shape)}")
    if q.dtype not in _DTYPES:
        raise TypeError(f"unsupported dtype {q.dtype} (bfloat16 or float32)")
    if style not in _STYLES:
        raise ValueError(f"style must be one of {sorted(_STYLES)}, got {style!r}")
    dev, (tokens, _, d) = q.device, q.shape
    if not q.is_cuda:
        raise ValueError("q must live on a GPU")
    _check(positions, "positions", torch.int32, dev, (tokens,))
    given = q_out, k_out
    q_out, qr = _heads(q, q_out, q_weight, "q", dev, tokens, d, q.dtype, stream)
    kr = None
    if k is not None:
        k_out, kr = _heads(k, k_out, k_weight, "k", dev, tokens, d, q.dtype, stream)
    elif k_out is not None or k_weight is not None:
        raise ValueError("k_out and k_weight need k")
    s, here = _use(stream, dev, q, k, positions, q_weight, k_weight, *given)
    rope = C.CmRope(base=float(rope_base), style=_STYLES[style], reserved=0)
    C.check(_call(here, dev, C.lib().cm_norm_rotate, d, _DTYPES[q.dtype], tokens, positions.data_ptr(),
                  ctypes.byref(rope), eps, ctypes.byref(qr), None if kr is None else ctypes.byref(kr),
                  s.cuda_stream), "cm_norm_rotate")
    return q_out, k_out


@dataclass
class QCacheTree:
    """What the attention of a step of drafted nodes needs, on the device: masks [tokens, words] int64
    (bit j % 64 of word j / 64: the row sees node j of its request), positions [tokens] int32, the
    window that they were made for; info [n] int32: the requests' status."""
    masks: Optional[torch.Tensor]
    positions: torch.Tensor
    window: int = 0
    info: Optional[torch.Tensor] = None

    def check(self) -> "QCacheTree":
        """Waits for the step and raises if a request's rows, nodes or parents were not as they have
        to be."""
        if self.info is not None:
            bad = [r for r, status in enumerate(self.info.tolist()) if status != C.CM_OK]
            if bad:
                raise C.CmError(C.CM_EINVAL, "cm_qcache_tree",
                                f"requests {bad[:8]}: too many nodes or too few tokens, a parent that is "
                                "no earlier node, or rows that do not lie in the step")
        return self


def qcache_tree(parents: Optional[torch.Tensor], rows: torch.Tensor, lens: torch.Tensor, tokens: int,
                max_rows: int, window: int = 0, masks: bool = True, stream=None) -> QCacheTree:
    """cm_qcache_tree: masks and positions of a step of `tokens` nodes, at most max_rows of a request.
    parents [tokens] int32: the node that each hangs on, counted within its request, -1 for node 0
    (None: chains); rows [n + 1], lens [n]: as qcache_tables gives them; window: positions that a node
    sees, itself included (0: all); masks: False for positions alone."""
    dev, n = lens.device, lens.numel()
    if not lens.is_cuda:
        raise ValueError("lens must live on a GPU")
    _check(lens, "lens", torch.int32, dev, (n,))
    _check(rows, "rows", torch.int32, dev, (n + 1,))
    if parents is not None:
        _check(parents, "parents", torch.int32, dev, (tokens,))
    words = -(-_int32(max(max_rows, 1), "max_rows") // 64) if masks else 0
    window = _int32(window, "window")
    with _made_on(stream):
        out = QCacheTree(torch.empty((tokens, words), dtype=torch.int64, device=dev) if masks else None,
                         torch.empty(tokens, dtype=torch.int32, device=dev), window,
                         torch.empty(n, dtype=torch.int32, device=dev))
    s, here = _use(stream, dev, parents, rows, lens)
    C.check(_call(here, dev, C.lib().cm_qcache_tree, n, tokens,
                  None if parents is None else parents.data_ptr(), rows.data_ptr(), lens.data_ptr(), window,
                  words, out.masks.data_ptr() if masks else None, out.positions.data_ptr(),
                  out.info.data_ptr(), s.cuda_stream), "cm_qcache_tree")
    return out


def qcache_tree_attention(cache: QCache, layer: int, q: torch.Tensor, table: torch.Tensor,
                          lens: torch.Tensor, rows: Optional[torch.Tensor], tree: QCacheTree,
                          max_rows: Optional[int] = None, scale: Optional[float] = None,
                          out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                          stream=None):
    """cm_qcache_tree_attention: queries q [rows, q_heads, d] of drafted nodes over one layer of the
    cache; returns (out, lse). Each sees its request's context, the tokens before the nodes, and the
    nodes that its mask has (tree.masks, with tree.positions where tree.window is not 0). Other
    arguments as qcache_attention."""
    dev, masks = cache.device, tree.masks
    step, out, lse = _attention_step(cache, q, table, lens, rows, max_rows, scale, tree.window, out, lse,
                                     stream)
    if masks is None or masks.dim() != 2:
        raise ValueError("tree.masks must be [rows, words]")
    _check(masks, "tree.masks", torch.int64, dev, (q.shape[0], masks.shape[1]))
    _check(tree.positions, "tree.positions", torch.int32, dev, (q.shape[0],))
    of = C.CmQtree(masks.data_ptr(), masks.shape[1], tree.positions.data_ptr())
    s, here = _use(stream, dev, cache.codes, cache.scales, q, table, lens, rows, masks, tree.positions, out,
                   lse)
    with _made_on(None if stream is None and here else s):
        C.check(_attention(cache, layer, step, s, "cm_qcache_tree_attention", (ctypes.byref(of),)),
                "cm_qcache_tree_attention")
    return out, lse


@dataclass
class Verified:
    """What cm_verify_drafts decides, on the device: path [tokens] int32 (at a request's rows its
    accepted nodes in order, 0 first, -1 behind them), counts [n] int32 (how many), tokens [n]
    int64 (the token sampled after them; -1 for a request without nodes)."""
    path: torch.Tensor
    counts: torch.Tensor
    tokens: torch.Tensor


def _probabilities(x: torch.Tensor, name: str, device, tokens: int):
    if x.dim() != 2 or x.shape[0] != tokens:
        raise ValueError(f"{name} must be [{tokens}, vocabulary], got {list(x.shape)}")
    if x.dtype not in _DTYPES:
        raise TypeError(f"{name} must be bfloat16 or float32, got {x.dtype}")
    if x.device != device:
        raise ValueError(f"{name} must live on {device}, got {x.device}")
    if x.stride(1) != 1 and x.shape[1] > 1:
        raise ValueError(f"the last dimension of {name} must be contiguous")


def verify_drafts(probs: torch.Tensor, drafts: torch.Tensor, parents: torch.Tensor, rows: torch.Tensor,
                  accept: torch.Tensor, sample: torch.Tensor,
                  draft_probs: Optional[torch.Tensor] = None, stream=None) -> Verified:
    """cm_verify_drafts: which drafted nodes the target accepts, and the token after them. probs
    [tokens, vocabulary] (bfloat16 or float32): the target's probabilities of the token after each node;
    drafts [tokens] int64 the nodes' tokens, parents [tokens] int32 the node that each hangs on, counted
    within its request (-1: node 0), rows [n + 1] int32 where each request's nodes begin; accept [tokens] and
    sample [n] float32: numbers in [0, 1). draft_probs: the probabilities that each node's children
    were sampled from (None: the drafts were not sampled)."""
    if drafts.dim() != 1 or rows.dim() != 1 or rows.numel() < 2:
        raise ValueError("drafts must be [tokens] and rows [n + 1]")
    dev, tokens, n = rows.device, drafts.numel(), rows.numel() - 1
    if not rows.is_cuda:
        raise ValueError("rows must live on a GPU")
    _check(rows, "rows", torch.int32, dev)
    _check(drafts, "drafts", torch.int64, dev)
    _check(parents, "parents", torch.int32, dev, (tokens,))
    _check(accept, "accept", torch.float32, dev, (tokens,))
    _check(sample, "sample", torch.float32, dev, (n,))
    _probabilities(probs, "probs", dev, tokens)
    if draft_probs is not None:
        _probabilities(draft_probs, "draft_probs", dev, tokens)
        if draft_probs.shape != probs.shape or draft_probs.dtype is not probs.dtype:
            raise ValueError("draft_probs must have the shape and type of probs")
    with _made_on(stream):
        out = Verified(torch.empty(tokens, dtype=torch.int32, device=dev),
                       torch.empty(n, dtype=torch.int32, device=dev),
                       torch.empty(n, dtype=torch.int64, device=dev))
    step = C.CmDrafts(n, _DTYPES[probs.dtype], tokens, probs.shape[1], probs.data_ptr(), probs.stride(0),
                      None if draft_probs is None else draft_probs.data_ptr(),
                      0 if draft_probs is None else draft_probs.stride(0), drafts.data_ptr(),
                      parents.data_ptr(), rows.data_ptr(), accept.data_ptr(), sample.data_ptr(),
                      out.path.data_ptr(), out.counts.data_ptr(), out.tokens.data_ptr())
    s, here = _use(stream, dev, probs, draft_probs, drafts, parents, rows, accept, sample)
    with _made_on(None if stream is None and here else s):
        ws = _verify_workspace(step, dev, s)
        if ws is not None:
            step.workspace, step.workspace_bytes = ws.data_ptr(), ws.numel()
        C.check(C.lib().cm_verify_drafts(ctypes.byref(step), s.cuda_stream), "cm_verify_drafts")
    return out


@functools.lru_cache(maxsize=256)
def _verify_bytes(dev, n: int, dtype: int, vocabulary: int) -> int:
    """The workspace of these sizes on the current GPU, dev."""
    need = ctypes.c_size_t(0)
    step = C.CmDrafts(n=n, dtype=dtype, vocabulary=vocabulary)
    C.check(C.lib().cm_verify_drafts_size(ctypes.byref(step), ctypes.byref(need)), "cm_verify_drafts_size")
    return need.value


def _verify_workspace(step: C.CmDrafts, dev, s) -> Optional[torch.Tensor]:
    """Zeros for a call on s, the current stream; kept as the attention's scratch is."""
    need = _verify_bytes(dev, step.n, step.dtype, step.vocabulary)
    if need == 0:
        return None
    capturing = torch.cuda.is_current_stream_capturing()
    key = (dev, s.cuda_stream, "cm_verify_drafts")
    ws = None if capturing else _WS.get(key)
    if ws is None or ws.numel() < need:
        ws = torch.zeros(need, dtype=torch.uint8, device=dev)
        if not capturing:
            _WS[key] = ws
    return ws


@dataclass
class QCacheKept:
    """What cm_qcache_keep leaves, on the device: lens [n] int32, info [2] int64 (status, pages
    freed)."""
    lens: torch.Tensor
    info: torch.Tensor

    def check(self) -> "QCacheKept":
        """Waits for the step and raises if something of it was not as it has to be."""
        status, pages = self.info.tolist()
        if status != C.CM_OK:
            raise C.CmError(status, "cm_qcache_keep",
                            f"{pages} pages freed; a request's rows, length, count or path is not as it "
                            "has to be, or the tensor of freed pages is too short")
        return self


def qcache_keep(cache: QCache, table: torch.Tensor, lens: torch.Tensor, rows: torch.Tensor,
                path: torch.Tensor, counts: torch.Tensor, freed: Optional[torch.Tensor] = None,
                stream=None) -> QCacheKept:
    """cm_qcache_keep: of each request's nodes the first counts[r] of path (as verify_drafts gives
    them) stay and move to the front of the nodes' places, in every layer; returns the lengths then.
    table [n, width], lens [n], rows [n + 1]: as the step had them; freed (int32): takes the pages
    that the others leave, in order, entries past them left as they are."""
    dev = cache.device
    if table.dim() != 2:
        raise ValueError("table must be [n, width]")
    n, width = table.shape
    i32 = torch.int32
    _check(table, "table", i32, dev)
    _check(lens, "lens", i32, dev, (n,))
    _check(rows, "rows", i32, dev, (n + 1,))
    _check(counts, "counts", i32, dev, (n,))
    if path.dim() != 1:
        raise ValueError("path must be [tokens]")
    _check(path, "path", i32, dev)
    with _made_on(stream):
        if freed is None:
            freed = torch.empty(path.numel() // cache.B + n, dtype=i32, device=dev)
        out = QCacheKept(torch.empty(n, dtype=i32, device=dev),
                         torch.empty(2, dtype=torch.int64, device=dev))
    _check(freed, "freed", i32, dev)
    step = C.CmQkeep(n, path.numel(), table.data_ptr(), width, lens.data_ptr(), rows.data_ptr(),
                     path.data_ptr(), counts.data_ptr(), out.lens.data_ptr(), freed.data_ptr(),
                     freed.numel(), out.info.data_ptr())
    s, here = _use(stream, dev, cache.codes, cache.scales, table, lens, rows, path, counts, freed)
    C.check(_call(here, dev, C.lib().cm_qcache_keep, ctypes.byref(cache.struct), ctypes.byref(step),
                  s.cuda_stream), "cm_qcache_keep")
    return out


def qcache_copy(cache: QCache, src: torch.Tensor, dst: torch.Tensor, layer: int = 0,
                layers: Optional[int] = None, stream=None) -> None:
    """cm_qcache_copy: pages src [n] to dst [n] (int32), codes and scales, of `layers` layers from `layer`
    on (default: all that follow). No destination is another one, nor a source."""
    if src.dim() != 1:
        raise ValueError("src must be [n]")
    _check(src, "src", torch.int32, cache.device)
    _check(dst, "dst", torch.int32, cache.device, src.shape)
    s, here = _use(stream, cache.device, cache.codes, cache.scales, src, dst)
    C.check(_call(here, cache.device, C.lib().cm_qcache_copy, ctypes.byref(cache.struct),
                  _int32(layer, "layer"), _int32(cache.L - layer if layers is None else layers, "layers"),
                  src.numel(), src.data_ptr(), dst.data_ptr(), s.cuda_stream), "cm_qcache_copy")
