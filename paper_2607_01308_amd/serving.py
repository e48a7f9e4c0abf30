"""ServingCache: requests served from an 8-bit paged cache, step after step. It strings
qcache_tables, qcache_write and qcache_attention together and keeps what they need
between steps: the block table, the lengths and the free pages, on the device. The host
follows with numbers alone, so no call waits for the device.

    sc = ServingCache(QCache.empty(L, H, d, pages), places=8, max_len=32768)
    sc.load(0, render_deliveries(...).cache)      # a merged cache into place 0
    step = sc.extend([1, 0, 0, 0, 0, 0, 0, 0])    # one token more for it
    for layer in range(L):
        sc.write(layer, k, v, step)               # the new tokens' K and V, [tokens, H, d]
        out, lse = sc.attend(layer, q, step)      # their queries, [tokens, q_heads, d]
    sc.release(0)                                 # its pages are free again"""

from __future__ import annotations

from dataclasses import dataclass
from typing import List, Optional, Sequence

import torch

from .binding import _DTYPES
from .qcache import (QCache, QCacheStep, _made_on, _use, check_rows, qcache_attention,
                     qcache_tables, qcache_write)


@dataclass
class ServingStep:
    """A step of ServingCache.extend: the new tokens of all places, place after place.
    tables: slots, rows and lengths on the device; tokens: how many; max_rows: the most of
    one place."""
    tables: QCacheStep
    tokens: int
    max_rows: int


class ServingCache:
    """`places` requests at a time, of at most max_len tokens each, in the pages of
    `cache` (all of them: what they held is lost). Calls enqueue on one stream (`stream`,
    else the current one); a caller that changes streams between calls orders them.

    The lengths and the free pages move on with each extend, load and release on the host, so
    these are not captured into a HIP graph, whose replays would deal out the same pages
    again; write and attend of a step may be."""

    def __init__(self, cache: QCache, places: int, max_len: int):
        if places < 1 or max_len < 1:
            raise ValueError("places and max_len must be at least 1")
        self.cache, self.places, self.max_len = cache, int(places), int(max_len)
        self.lengths: List[int] = [0] * self.places       # tokens of each place
        dev, i32 = cache.device, torch.int32
        self.table = torch.zeros((self.places, -(-max_len // cache.B)), dtype=i32, device=dev)
        self._held = torch.zeros(self.places, dtype=i32, device=dev)
        # free pages: places _head .. _tail of a buffer of twice as many as there are
        self._free = torch.empty(2 * cache.P, dtype=i32, device=dev)
        torch.arange(cache.P, dtype=i32, device=dev, out=self._free[:cache.P])
        self._head, self._tail = 0, cache.P
        self._new: Optional[tuple] = None                 # the last step's new lengths

    @property
    def free_pages(self) -> int:
        return self._tail - self._head

    def _refuse_capture(self, what: str, stream) -> None:
        if not self._held.is_cuda:
            return
        s, here = _use(stream, self._held.device)
        with _made_on(None if stream is None and here else s):
            if torch.cuda.is_current_stream_capturing():
                raise RuntimeError(f"{what} cannot be captured into a graph: its replays would not "
                                   "move on")

    def _pages(self, tokens: int) -> int:
        return -(-tokens // self.cache.B)

    def extend(self, new: Sequence[int], stream=None) -> ServingStep:
        """Room for new[r] more tokens in each place r. The step is refused, and nothing
        changed, if a place would grow beyond max_len or the free pages do not suffice."""
        self._refuse_capture("extend", stream)
        new = tuple(int(x) for x in new)
        if len(new) != self.places or min(new) < 0:
            raise ValueError(f"new must be {self.places} numbers >= 0, got {list(new)}")
        after = [a + b for a, b in zip(self.lengths, new)]
        if max(after) > self.max_len:
            raise ValueError(f"a place would hold {max(after)} tokens, more than {self.max_len}")
        need = sum(self._pages(b) - self._pages(a) for a, b in zip(self.lengths, after))
        if need > self.free_pages:
            raise RuntimeError(f"the step needs {need} pages, {self.free_pages} are free")
        with _made_on(stream):
            if self._new is None or self._new[0] != new:
                host = torch.tensor(new, dtype=torch.int32, pin_memory=self._held.is_cuda)
                self._new = (new, host.to(self._held.device, non_blocking=True), host)
        free = self._free[self._head:self._tail]
        tables = qcache_tables(self.cache.P, self.cache.B, self._held, self._new[1], free,
                               self.table, sum(new), stream)
        self._head += need
        self._held, self.lengths = tables.lens, after
        return ServingStep(tables, sum(new), max(new))

    def release(self, place: int, stream=None) -> None:
        """Empties a place; its pages are free again, after the work enqueued so far."""
        if not 0 <= place < self.places:
            raise ValueError(f"place must be in [0, {self.places}), got {place}")
        self._refuse_capture("release", stream)
        pages = self._pages(self.lengths[place])
        if pages == 0:
            return
        if self._held.is_cuda:
            _use(stream, self._held.device, self._free, self._held, self.table)
        with _made_on(stream):
            if self._tail + pages > self._free.numel():
                left = self._free[self._head:self._tail].clone()
                self._free[:left.numel()] = left
                self._head, self._tail = 0, left.numel()
            self._free[self._tail:self._tail + pages] = self.table[place, :pages]
            self._held = self._held.clone()               # (a step may still be read)
            self._held[place:place + 1].zero_()
        self._tail += pages
        self.lengths[place] = 0

    def write(self, layer: int, k: torch.Tensor, v: torch.Tensor, step: ServingStep,
              stream=None) -> None:
        """qcache_write of the step's rows, [tokens, H, d], or of several layers from `layer`
        on, [layers, tokens, H, d]."""
        qcache_write(self.cache, layer, k, v, step.tables.slots, stream)

    def attend(self, layer: int, q: torch.Tensor, step: ServingStep,
               scale: Optional[float] = None, window: int = 0,
               out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
               stream=None):
        """qcache_attention of the step's queries, [tokens, q_heads, d], each over its place's
        tokens up to its own; returns (out, lse)."""
        return qcache_attention(self.cache, layer, q, self.table, step.tables.lens,
                                rows=step.tables.rows, max_rows=step.max_rows, scale=scale,
                                window=window, out=out, lse=lse, stream=stream)

    def load(self, place: int, layers: Sequence, stream=None) -> ServingStep:
        """Appends a merged cache to a place: per layer (K, V), each [1, H, T, d], as the
        renders return it. One write for a cache that is one buffer, else one for each
        layer. A cache that cannot be written is refused, and nothing changed.

        The tokens come after those that the place holds, but K is written as it is: a merged
        cache's keys are rotated for positions from 0, so queries rotated for the place's
        positions see it right in an empty place alone."""
        if not 0 <= place < self.places:
            raise ValueError(f"place must be in [0, {self.places}), got {place}")
        H, d = self.cache.H, self.cache.d
        if len(layers) != self.cache.L:
            raise ValueError(f"the cache has {self.cache.L} layers, got {len(layers)}")
        T = layers[0][0].shape[2]
        for K, V in layers:
            if K.shape != (1, H, T, d) or V.shape != (1, H, T, d):
                raise ValueError(f"K and V must be [1, {H}, {T}, {d}], got {list(K.shape)} and "
                                 f"{list(V.shape)}")
            if K.dtype not in _DTYPES or V.dtype is not K.dtype:
                raise TypeError(f"K and V must both be bfloat16 or float32, got {K.dtype} and "
                                f"{V.dtype}")
            for x, name in ((K, "K"), (V, "V")):
                check_rows(x[0].transpose(0, 1), name, self.cache.device)
        before = self._head, self._held, self.lengths
        step = self.extend([T if r == place else 0 for r in range(self.places)], stream)
        try:
            k, v = (_one_buffer([pair[i] for pair in layers]) for i in (0, 1))
            if k is not None and v is not None:
                self.write(0, k, v, step, stream)
            else:
                for layer, (K, V) in enumerate(layers):
                    self.write(layer, K[0].transpose(0, 1), V[0].transpose(0, 1), step, stream)
        except Exception:
            # (the table's entries past a place's tokens and their pages are dealt again)
            self._head, self._held, self.lengths = before
            raise
        return step


def _one_buffer(xs: Sequence[torch.Tensor]) -> Optional[torch.Tensor]:
    """Tensors [1, H, T, d] at equal distances in one buffer as one [len(xs), T, H, d]."""
    x = xs[0]
    step = xs[1].storage_offset() - x.storage_offset() if len(xs) > 1 else 0
    base = x.untyped_storage().data_ptr()
    for i, y in enumerate(xs):
        if (y.untyped_storage().data_ptr() != base or y.stride() != x.stride()
                or y.dtype is not x.dtype or step < 0
                or y.storage_offset() != x.storage_offset() + i * step):
            return None
    _, H, T, d = x.shape
    return x.as_strided((len(xs), T, H, d), (step, x.stride(2), x.stride(1), x.stride(3)))
