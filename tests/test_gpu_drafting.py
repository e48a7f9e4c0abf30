"""Decoding with drafted tokens as it is used: places forked from one context draft trees step after
step, through norm_rotate, ServingCache's writes and attention, verify_drafts and accept. Pages are
followed exactly (tests/draft_ref.py, tests/qcache_ref.py), attention within its bounds."""

import os
import runpy

import numpy as np
import pytest
import torch

import draft_ref as ref
import paper_2607_01308_amd as cm
import qcache_ref
from test_gpu_keep import same_codes
from test_gpu_tree import check

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
ROOT = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..")


def values(*shape, seed, dtype):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


@pytest.mark.parametrize("dtype,d,B,H,G,window,own_stream", [
    (BF16, 128, 16, 2, 4, 0, False), (F32, 64, 32, 1, 3, 40, False), (BF16, 256, 64, 1, 2, 0, True)])
def test_drafted_steps(dtype, d, B, H, G, window, own_stream):
    rng = np.random.default_rng(d)
    L, places, V, steps = 2, 4, 500, 6
    stream = torch.cuda.Stream() if own_stream else None
    with torch.cuda.stream(stream):
        sc = cm.ServingCache(cm.QCache.empty(L, H, d, 60, B), places, 40 * B)
        codes = sc.cache.codes.view(torch.uint8).cpu().numpy().copy()
        scales = sc.cache.scales.cpu().numpy().copy()
        qw, kw = values(d, seed=1, dtype=dtype), values(d, seed=2, dtype=dtype)

        def layers(step, seed):
            """A step's projections through all layers; K and V as they are written."""
            pos = sc.positions(step)
            for l in range(L):
                x = values(step.tokens, (G + 2) * H, d, seed=seed + l, dtype=dtype)
                q, k, v = x.split((H * G, H, H), 1)
                q, k = cm.norm_rotate(q, k, pos, 1e6, q_weight=qw, k_weight=kw)
                sc.write(l, k, v, step)
                for w, y in enumerate((k, v)):
                    qcache_ref.write(codes[l, w], scales[l, w], y.double().cpu().numpy(), step.tables.slots.tolist())
                yield l, q, sc.attend(l, q, step, window=0 if step.tree is not None else window)

        # a context in place 0, that the others go on from
        for _ in layers(sc.extend([3 * B + 5, 0, 0, 0]), 100):
            pass
        for r in range(1, places):
            sc.fork(0, r)
            for l in range(L):
                old, new = int(sc.table[0, 3]), int(sc.table[r, 3])
                codes[l, :, new], scales[l, :, new] = codes[l, :, old], scales[l, :, old]
        kept = 0
        for n in range(steps):
            trees = [ref.random_tree(rng, int(rng.integers(1, 20)), 3) for _ in range(places)]
            if n == 2:
                trees[1] = []
            if n == 4:
                sc.release(2)
                sc.fork(3, 2)
                full, part = divmod(sc.lengths[3], B)
                if part:
                    for l in range(L):
                        old, new = int(sc.table[3, full]), int(sc.table[2, full])
                        codes[l, :, new], scales[l, :, new] = codes[l, :, old], scales[l, :, old]
            held = list(sc.lengths)
            step = sc.draft(trees, window=window)
            step.tables.check()
            step.tree.check()
            counts = [len(t) for t in trees]
            assert sc.lengths == [a + b for a, b in zip(held, counts)] == step.tables.lens.tolist()
            sees, positions = [], []
            for t, a in zip(trees, held):
                s, p = ref.tree(t, a, window)
                sees, positions = sees + s, positions + p
            assert sc.positions(step).tolist() == positions
            table = sc.table.cpu().numpy()
            for l, q, got in layers(step, 1000 * (n + 1)):
                assert np.array_equal(sc.cache.scales[l].cpu().numpy(), scales[l])
                assert same_codes(sc.cache.codes[l].view(torch.uint8).cpu().numpy(), codes[l])
                check(q, sc.cache.codes, sc.cache.scales, l, table, sc.lengths, counts, sees, positions, window, got=got)
            probs = torch.softmax(2 * values(step.tokens, V, seed=n, dtype=F32), 1).to(dtype)
            drafts = torch.multinomial(probs.float(), 1)[:, 0]
            u, s = torch.rand(step.tokens, device="cuda") * 0.5, torch.rand(places, device="cuda")
            done = cm.verify_drafts(probs, drafts, step.parents, step.tables.rows, u, s, draft_probs=probs)
            rows = step.tables.rows.tolist()
            path, accepted, tokens = ref.verify(probs.float().cpu().numpy(), drafts.tolist(), step.parents.tolist(), rows,
                                                u.tolist(), s.tolist(), probs.float().cpu().numpy())
            assert done.path.tolist() == path and done.counts.tolist() == accepted and done.tokens.tolist() == tokens
            free = sc.free_pages
            sc.accept(step, done.path, done.counts.tolist())
            lens, freed = ref.keep(codes, scales, table, step.tables.lens.tolist(), rows, path, accepted)
            assert sc.lengths == lens == sc._held.tolist() and sc.free_pages == free + len(freed)
            assert sc._free[sc._tail - len(freed):sc._tail].tolist() == freed
            assert np.array_equal(sc.cache.scales.cpu().numpy(), scales)
            assert same_codes(sc.cache.codes.view(torch.uint8).cpu().numpy(), codes)
            kept += sum(accepted)
        assert kept > 2 * places                         # (more than one node of a tree, now and then)
        # and one token more by a plain step
        step = sc.extend([1] * places)
        table = sc.table.cpu().numpy()
        for l, q, got in layers(step, 9000):
            out, lse, A, X = qcache_ref.attend(q.double().cpu(), codes[l], scales[l], table, sc.lengths, list(range(places + 1)), window)
            bound, _ = ref.attend_bounds(dtype, d, max(sc.lengths), out, A, X)
            assert bool(((got[0].double().cpu() - out).abs() <= bound).all())
        for r in range(places):
            sc.release(r)
        assert sc.free_pages == 60
        if stream is not None:
            torch.cuda.current_stream().synchronize()


def test_drafted_layers_are_captured():
    """A drafted step's layers replayed from a graph, with other drafts' K and V each time; steps, accepts and
    forks are refused there."""
    H, G, d, B = 2, 2, 64, 16
    sc, twin = (cm.ServingCache(cm.QCache.empty(1, H, d, 20, B), 2, 100) for _ in range(2))
    x = values(33, H, d, seed=1, dtype=BF16)
    for s in (sc, twin):
        s.write(0, x, x, s.extend([30, 3]))
    trees = [[-1, 0, 0, 1], [-1, 0]]
    one, two = sc.draft(trees), twin.draft(trees)
    k, q = values(6, H, d, seed=2, dtype=BF16), values(6, H * G, d, seed=3, dtype=BF16)
    w = values(d, seed=4, dtype=BF16)
    out, lse = torch.empty_like(q), torch.empty((6, H * G), device="cuda")
    rotated = torch.empty_like(q), torch.empty_like(k)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cm.norm_rotate(q, k, one.tree.positions, 1e4, q_weight=w, k_weight=w, q_out=rotated[0], k_out=rotated[1])
        sc.write(0, rotated[1], k, one)
        sc.attend(0, rotated[0], one, out=out, lse=lse)
        for call in (lambda: sc.draft(trees), lambda: sc.accept(one, one.parents, [1, 1]), lambda: sc.fork(0, 1)):
            with pytest.raises((RuntimeError, ValueError), match="captured|not empty"):
                call()
    for n in range(3):
        k.copy_(values(6, H, d, seed=10 + n, dtype=BF16))
        q.copy_(values(6, H * G, d, seed=20 + n, dtype=BF16))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        a, b = cm.norm_rotate(q, k, twin.positions(two), 1e4, q_weight=w, k_weight=w)
        twin.write(0, b, k, two)
        want = twin.attend(0, a, two)
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


def test_nothing_drafted():
    sc = cm.ServingCache(cm.QCache.empty(1, 1, 64, 8, 16), 2, 64)
    sc.extend([5, 0])
    step = sc.draft([[], []])
    assert (step.tokens, step.max_rows) == (0, 0)
    q = torch.empty((0, 2, 64), device="cuda", dtype=BF16)
    assert sc.attend(0, q, step)[0].shape == (0, 2, 64)
    sc.write(0, q[:, :1], q[:, :1], step)
    done = cm.verify_drafts(torch.empty((0, 9), device="cuda"), torch.empty(0, dtype=torch.int64, device="cuda"),
                            step.parents, step.tables.rows, torch.empty(0, device="cuda"), torch.rand(2, device="cuda"))
    assert done.counts.tolist() == [0, 0] and done.tokens.tolist() == [-1, -1]
    sc.accept(step, done.path, done.counts.tolist())
    assert sc.lengths == [5, 0] == sc._held.tolist() and sc.free_pages == 7
