"""ServingCache: requests served from an 8-bit paged cache, step after step. It strings
qcache_tables, qcache_write and qcache_attention together, and for drafted tokens
qcache_tree, qcache_tree_attention, qcache_keep and qcache_copy, and keeps what they need
between steps: the block table, the lengths and the free pages, on the device. The host
follows with numbers alone, so no call waits for the device.

    sc = ServingCache(QCache.empty(L, H, d, pages), places=8, max_len=32768)
    sc.load(0, render_deliveries(...).cache)      # a merged cache into place 0
    step = sc.extend([1, 0, 0, 0, 0, 0, 0, 0])    # one token more for it
    for layer in range(L):
        sc.write(layer, k, v, step)               # the new tokens' K and V, [tokens, H, d]
        out, lse = sc.attend(layer, q, step)      # their queries, [tokens, q_heads, d]
    sc.release(0)                                 # its pages are free again

A step of drafted tokens brings each place a tree, of which the target accepts a path:

    sc.fork(0, 1)                                 # place 1 goes on from place 0's tokens
    step = sc.draft([[-1, 0, 0, 1], [-1, 0], ...])           # each node's parent
    q, k = norm_rotate(q, k, sc.positions(step), rope_base, q_weight=.., k_weight=..)
    sc.write(layer, k, v, step)
    out, lse = sc.attend(layer, q, step)
    done = verify_drafts(probs, drafts, step.parents, step.tables.rows, accept, sample)
    sc.accept(step, done.path, done.counts.tolist())         # the others' pages are free again"""

from __future__ import annotations

from dataclasses import dataclass
from typing import List, Optional, Sequence, Tuple

import torch

from ._cabi import CM_DRAFT_MAX_NODES
from .binding import _DTYPES
from .drafting import QCacheKept, QCacheTree, qcache_copy, qcache_keep, qcache_tree, qcache_tree_attention
from .qcache import (QCache, QCacheStep, _made_on, _use, check_rows, qcache_attention,
                     qcache_tables, qcache_write)


@dataclass
class ServingStep:
    """A step of ServingCache.extend: the new tokens of all places, place after place.
    tables: slots, rows and lengths on the device; tokens: how many; max_rows: the most of
    one place; new: how many of each. Of ServingCache.draft also the nodes' parents [tokens] int32 and
    their tree, on the device."""
    tables: QCacheStep
    tokens: int
    max_rows: int
    new: Tuple[int, ...] = ()
    parents: Optional[torch.Tensor] = None
    tree: Optional[QCacheTree] = None


@dataclass
class _Shared:
    """Pages that several places hold, as consecutive entries of their tables."""
    pages: int
    places: int


class ServingCache:
    """`places` requests at a time, of at most max_len tokens each, in the pages of
    `cache` (all of them: what they held is lost). Calls enqueue on one stream (`stream`,
    else the current one); a caller that changes streams between calls orders them.

    The lengths and the free pages move on with each extend, draft, accept, fork, load and
    release on the host, so these are not captured into a HIP graph, whose replays would deal
    out the same pages again; write, attend and positions of a step may be."""

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
        self._parents: Optional[tuple] = None             # the last drafted step's parents
        # what each place shares with others: the first entries of its table
        self._shared: List[List[_Shared]] = [[] for _ in range(self.places)]

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
        return ServingStep(tables, sum(new), max(new), new)

    def draft(self, parents: Sequence[Sequence[int]], window: int = 0, stream=None) -> ServingStep:
        """Room for a tree of drafted tokens in each place r: parents[r][i] is the node that node i
        hangs on, -1 for node 0, the token that was sampled last (no nodes: nothing for that
        place). window: positions that a node sees, itself included (0: all). The step is refused, and
        nothing changed, where extend would refuse it."""
        self._refuse_capture("draft", stream)
        parents = tuple(tuple(int(x) for x in tree) for tree in parents)
        if len(parents) != self.places:
            raise ValueError(f"parents must be of {self.places} places, got {len(parents)}")
        for r, tree in enumerate(parents):
            if len(tree) > CM_DRAFT_MAX_NODES:
                raise ValueError(f"place {r} has {len(tree)} nodes, more than {CM_DRAFT_MAX_NODES}")
            if any(not 0 <= p < i for i, p in enumerate(tree) if i) or tree[:1] not in ((), (-1,)):
                raise ValueError(f"place {r}: node 0 hangs on -1, every other on an earlier one, got "
                                 f"{list(tree)}")
        if not 0 <= window < 2 ** 31:
            raise ValueError(f"window must be in [0, 2^31), got {window}")
        before = self._head, self._held, self.lengths
        step = self.extend([len(tree) for tree in parents], stream)
        try:
            if self._parents is None or self._parents[0] != parents:
                self._parents = (parents, *self._upload([p for tree in parents for p in tree], stream))
            elif self._held.is_cuda:
                _use(stream, self._held.device, self._parents[1])
            step.parents = self._parents[1]
            step.tree = qcache_tree(step.parents, step.tables.rows, step.tables.lens, step.tokens,
                                    step.max_rows, window, stream=stream)
        except Exception:
            # (as in load: the pages are dealt again)
            self._head, self._held, self.lengths = before
            raise
        return step

    def _upload(self, numbers: Sequence[int], stream):
        """The numbers as int32 on the device, and the host memory that they come from."""
        with _made_on(stream):
            host = torch.tensor(numbers, dtype=torch.int32, pin_memory=self._held.is_cuda)
            return host.to(self._held.device, non_blocking=True), host

    def positions(self, step: ServingStep, stream=None) -> torch.Tensor:
        """The positions of a step's tokens [tokens] int32: of drafted ones those of their trees."""
        if step.tree is not None:
            return step.tree.positions
        return qcache_tree(None, step.tables.rows, step.tables.lens, step.tokens, step.max_rows,
                           masks=False, stream=stream).positions

    def accept(self, step: ServingStep, path: torch.Tensor, counts: Sequence[int], stream=None) -> QCacheKept:
        """Of the nodes of a drafted step, the last one, the first counts[r] of place r's path (as
        verify_drafts gives it) stay, and their K and V move to the front; the others' pages are
        free again. The path stays on the device: check() of what this returns waits and raises where one
        was not ascending within the nodes, of whose place nothing has moved then."""
        self._refuse_capture("accept", stream)
        counts = tuple(int(x) for x in counts)
        if step.tables.lens is not self._held:
            raise ValueError("accept is of the last step, and once; nothing may come between")
        if len(counts) != self.places or any(not 0 <= k <= c for k, c in zip(counts, step.new)):
            raise ValueError(f"counts must be of {self.places} places, each at most its nodes "
                             f"{list(step.new)}, got {list(counts)}")
        after = [a - c + k for a, c, k in zip(self.lengths, step.new, counts)]
        pages = sum(self._pages(a) - self._pages(b) for a, b in zip(self.lengths, after))
        if path.numel() != step.tokens:
            raise ValueError(f"path must be [{step.tokens}], got {list(path.shape)}")
        on_device, _host = self._upload(counts, stream)
        self._room(pages, stream)
        kept = qcache_keep(self.cache, self.table, step.tables.lens, step.tables.rows, path, on_device,
                           self._free[self._tail:self._tail + pages], stream)
        self._tail += pages
        self._held, self.lengths = kept.lens, after
        return kept

    def fork(self, place: int, to: int, stream=None) -> None:
        """The empty place `to` goes on from the tokens of `place`: both hold the same full pages,
        which are free again when the last of their places is released, and `to` a copy of a page
        that is not full, as far as it is written when the call comes to run: a step's K and V go in before
        it is forked."""
        for x in (place, to):
            if not 0 <= x < self.places:
                raise ValueError(f"place must be in [0, {self.places}), got {x}")
        if self.lengths[to] or to == place:
            raise ValueError(f"place {to} is not empty")
        self._refuse_capture("fork", stream)
        full, part = divmod(self.lengths[place], self.cache.B)
        if part and self.free_pages < 1:
            raise RuntimeError("the fork needs a page, none is free")
        if self._held.is_cuda:
            _use(stream, self._held.device, self._free, self._held, self.table)
        with _made_on(stream):
            page = self._free[self._head:self._head + 1]
            if part:
                qcache_copy(self.cache, self.table[place, full:full + 1], page, stream=stream)
                self.table[to, full:full + 1] = page
            self.table[to, :full] = self.table[place, :full]
            self._held = self._held.clone()               # (a step may still be read)
            self._held[to] = self._held[place]
        self._head += part > 0
        own = full - sum(run.pages for run in self._shared[place])
        if own:
            self._shared[place].append(_Shared(own, 1))
        for run in self._shared[place]:
            run.places += 1
        self._shared[to] = list(self._shared[place])
        self.lengths[to] = self.lengths[place]

    def _room(self, pages: int, stream) -> None:
        """Room for `pages` more behind the free ones."""
        if self._tail + pages <= self._free.numel():
            return
        if self._held.is_cuda:
            _use(stream, self._held.device, self._free)
        with _made_on(stream):
            left = self._free[self._head:self._tail].clone()
            self._free[:left.numel()] = left
        self._head, self._tail = 0, left.numel()

    def release(self, place: int, stream=None) -> None:
        """Empties a place; its pages are free again, after the work enqueued so far (what it shares
        with other places when the last of them is released)."""
        if not 0 <= place < self.places:
            raise ValueError(f"place must be in [0, {self.places}), got {place}")
        self._refuse_capture("release", stream)
        pages = self._pages(self.lengths[place])
        if pages == 0:
            return
        if self._held.is_cuda:
            _use(stream, self._held.device, self._free, self._held, self.table)
        # the table's entries whose pages nobody else holds
        runs, at = [], 0
        for run in self._shared[place]:
            if run.places == 1:
                runs.append((at, at + run.pages))
            at += run.pages
        runs.append((at, pages))
        self._room(pages, stream)
        tail = self._tail
        with _made_on(stream):
            held = self._held.clone()                     # (a step may still be read)
            held[place:place + 1].zero_()
            for a, b in runs:
                self._free[tail:tail + b - a] = self.table[place, a:b]
                tail += b - a
        # (nothing fails from here on)
        for run in self._shared[place]:
            run.places -= 1
        self._shared[place] = []
        self._tail, self._held = tail, held
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
        tokens up to its own; of a drafted step qcache_tree_attention, each over its place's tokens
        before the step and its ancestors (the window is draft's); returns (out, lse)."""
        if step.tree is not None:
            if window not in (0, step.tree.window):
                raise ValueError(f"the step was drafted for a window of {step.tree.window}, not {window}")
            return qcache_tree_attention(self.cache, layer, q, self.table, step.tables.lens,
                                         step.tables.rows, step.tree, max_rows=step.max_rows, scale=scale,
                                         out=out, lse=lse, stream=stream)
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
