"""ServingCache's bookkeeping of drafted steps and forks, on the CPU: the library's tables, kept tokens
and copies are plain ones over a stand-in cache that holds one number for each token."""

import numpy as np
import pytest
import torch

import draft_ref
from paper_2607_01308_amd import serving
from paper_2607_01308_amd.drafting import QCacheKept, QCacheTree
from test_serving import FakeCache, plain  # noqa: F401


@pytest.fixture
def numbers(plain, monkeypatch):  # noqa: F811
    """Stand-ins that work on cache.tokens [P, B]."""

    def tree(parents, rows, lens, tokens, max_rows, window=0, masks=True, stream=None):
        out = []
        for r, T in enumerate(lens.tolist()):
            a, b = int(rows[r]), int(rows[r + 1])
            mine = list(range(-1, b - a - 1)) if parents is None else parents[a:b].tolist()
            out += draft_ref.tree(mine, T - (b - a), window)[1]
        return QCacheTree(torch.zeros((tokens, 1), dtype=torch.int64) if masks else None,
                          torch.tensor(out, dtype=torch.int32), window)

    def keep(cache, table, lens, rows, path, counts, freed, stream=None):
        out, pages = [], []
        B = cache.B
        for r, T in enumerate(lens.tolist()):
            a, c, k = int(rows[r]), int(rows[r + 1] - rows[r]), int(counts[r])
            held = T - c
            come = [cache.tokens[int(table[r, (held + p) // B]), (held + p) % B].item()
                    for p in path[a:a + k].tolist()]
            for i, x in enumerate(come):
                cache.tokens[int(table[r, (held + i) // B]), (held + i) % B] = x
            out.append(held + k)
            pages += table[r, -(-out[-1] // B):-(-T // B)].tolist()
        assert len(pages) == len(freed)
        freed.copy_(torch.tensor(pages, dtype=torch.int32))
        return QCacheKept(torch.tensor(out, dtype=torch.int32), torch.tensor([0, len(pages)]))

    def copy(cache, src, dst, layer=0, layers=None, stream=None):
        cache.tokens[dst.long()] = cache.tokens[src.long()]

    monkeypatch.setattr(serving, "qcache_tree", tree)
    monkeypatch.setattr(serving, "qcache_keep", keep)
    monkeypatch.setattr(serving, "qcache_copy", copy)


def cache_of(P, B, places, max_len):
    fake = FakeCache(P, B)
    fake.tokens = torch.full((P, B), -1, dtype=torch.int64)
    return serving.ServingCache(fake, places, max_len)


def check(sc, want):
    """Every place holds its tokens; every page is free or held, as often as forks say."""
    B, holders = sc.cache.B, {}
    for r, tokens in enumerate(want):
        assert sc.lengths[r] == len(tokens) == int(sc._held[r])
        got = [int(sc.cache.tokens[int(sc.table[r, t // B]), t % B]) for t in range(len(tokens))]
        assert got == tokens
        for j, p in enumerate(sc.table[r, :-(-len(tokens) // B)].tolist()):
            holders.setdefault(p, set()).add(r)
            # a page that is not full is nobody else's
            if (j + 1) * B > len(tokens):
                assert holders[p] == {r}
    free = sc._free[sc._head:sc._tail].tolist()
    assert sorted(free + list(holders)) == list(range(sc.cache.P))
    assert sc.free_pages == len(free)


@pytest.mark.parametrize("seed,P,B,places", [(0, 60, 16, 4), (1, 20, 16, 3), (2, 200, 32, 8), (3, 33, 16, 2)])
def test_places_draft_fork_and_go(numbers, seed, P, B, places):
    rng = np.random.default_rng(seed)
    sc = cache_of(P, B, places, P * B)
    want = [[] for _ in range(places)]
    forks = accepted = 0
    for number in range(400):
        kind = rng.random()
        before = (list(sc.lengths), sc.free_pages)
        if kind < 0.15:
            r = int(rng.integers(places))
            sc.release(r)
            want[r] = []
        elif kind < 0.3:
            a, b = (int(x) for x in rng.integers(0, places, size=2))
            if a != b and rng.random() < 0.7:
                sc.release(b)
                want[b] = []
                before = (list(sc.lengths), sc.free_pages)
            try:
                sc.fork(a, b)
            except (ValueError, RuntimeError):
                assert before == (sc.lengths, sc.free_pages)
                continue
            want[b] = list(want[a])
            forks += len(want[a]) > B
        else:
            trees = [draft_ref.random_tree(rng, int(rng.integers(0, 40)), 3) if rng.random() < 0.6 else []
                     for _ in range(places)]
            drafted = kind < 0.8
            try:
                step = sc.draft(trees) if drafted else sc.extend([len(t) for t in trees])
            except (ValueError, RuntimeError):
                assert before == (sc.lengths, sc.free_pages)
                continue
            fresh = [[1000 * number + 100 * r + i for i in range(len(t))] for r, t in enumerate(trees)]
            ids = [x for t in fresh for x in t]
            for slot, x in zip(step.tables.slots.tolist(), ids):
                sc.cache.tokens[slot // B, slot % B] = x
            if not drafted:
                assert sc.positions(step).tolist() == [len(w) + i for w, t in zip(want, fresh) for i in range(len(t))]
                want = [w + t for w, t in zip(want, fresh)]
            else:
                path, counts = [], []
                for r, t in enumerate(trees):
                    up = sorted(draft_ref.ancestors(t)[int(rng.integers(len(t)))]) if t else []
                    counts.append(int(rng.integers(0, len(up) + 1)) if rng.random() < 0.3 else len(up))
                    path += up + [-1] * (len(t) - len(up))
                    want[r] = want[r] + [fresh[r][i] for i in up[:counts[-1]]]
                depth = [len(a) - 1 for t in trees for a in draft_ref.ancestors(t)]
                at = [before[0][r] for r, t in enumerate(trees) for _ in t]
                assert sc.positions(step).tolist() == [a + e for a, e in zip(at, depth)]
                check_refused(sc, step, path, counts)
                sc.accept(step, torch.tensor(path, dtype=torch.int32), counts)
                with pytest.raises(ValueError, match="last step"):
                    sc.accept(step, torch.tensor(path, dtype=torch.int32), counts)
                accepted += sum(counts)
        check(sc, want)
    assert forks > 3 and accepted > 100


def check_refused(sc, step, path, counts):
    before = (list(sc.lengths), sc.free_pages, sc._held)
    path = torch.tensor(path, dtype=torch.int32)
    for bad in (counts[:-1], [-1] + counts[1:], [step.new[0] + 1] + counts[1:]):
        with pytest.raises(ValueError, match="counts"):
            sc.accept(step, path, bad)
    with pytest.raises(ValueError, match="path"):
        sc.accept(step, torch.zeros(step.tokens + 1, dtype=torch.int32), counts)
    assert before[:2] == (sc.lengths, sc.free_pages) and before[2] is sc._held


def test_refusals(numbers):
    sc = cache_of(10, 16, 3, 64)
    sc.extend([20, 0, 3])
    before = (list(sc.lengths), sc.free_pages)
    for trees, match in (([[-1]], "3 places"), ([[0], [], []], "place 0"), ([[], [-1, 1], []], "place 1"),
                         ([[], [-1, 0, -1], []], "place 1"), ([[], [], [-1, 0, 5]], "place 2"),
                         ([[-1] + [0] * 1024, [], []], "1025 nodes"), ([[-1] + [0] * 50, [], []], "would hold 71")):
        with pytest.raises(ValueError, match=match):
            sc.draft(trees)
    with pytest.raises(ValueError, match="window"):
        sc.draft([[-1], [], []], window=-1)
    with pytest.raises(ValueError, match="not empty"):
        sc.fork(0, 2)
    with pytest.raises(ValueError, match="not empty"):
        sc.fork(1, 1)
    for a, b in ((3, 1), (0, -1)):
        with pytest.raises(ValueError, match="place must be"):
            sc.fork(a, b)
    assert before == (sc.lengths, sc.free_pages)
    step = sc.draft([[-1, 0], [], []], window=7)
    with pytest.raises(ValueError, match="window of 7"):
        sc.attend(0, torch.zeros((2, 2, 64)), step, window=8)
    sc.extend([0, 0, 1])
    with pytest.raises(ValueError, match="last step"):
        sc.accept(step, torch.zeros(2, dtype=torch.int32), [1, 0, 0])
    # a fork of a place whose last page is not full, with no page free
    sc = cache_of(3, 16, 2, 64)
    sc.extend([40, 0])
    with pytest.raises(RuntimeError, match="none is free"):
        sc.fork(0, 1)
    # of full pages none is needed
    sc.extend([8, 0])
    sc.fork(0, 1)
    assert sc.lengths == [48, 48] and sc.free_pages == 0
    sc.release(0)
    assert sc.free_pages == 0
    sc.release(1)
    assert sc.free_pages == 3


def test_forks_of_forks(numbers):
    """Pages are free when the last of their places goes, in whatever order."""
    for order in ([0, 1, 2, 3], [3, 2, 1, 0], [1, 3, 0, 2]):
        sc = cache_of(40, 16, 4, 200)
        sc.extend([40, 0, 0, 0])                         # two full pages
        sc.fork(0, 1)
        sc.extend([0, 60, 0, 0])                         # place 1: six full pages, two of them place 0's
        sc.fork(1, 2)
        sc.fork(0, 3)
        sc.extend([5, 5, 5, 5])
        shared, held = sc.free_pages, [45, 105, 105, 45]
        assert sc.lengths == held
        # 2 + 4 shared; each place's own: 1, 1, 1, 1
        assert shared == 40 - 6 - 4
        for n, r in enumerate(order):
            sc.release(r)
            left = set(order[n + 1:])
            pages = (2 if left else 0) + (4 if left & {1, 2} else 0) + len(left)
            assert sc.free_pages == 40 - pages
        assert sorted(sc._free[sc._head:sc._tail].tolist()) == list(range(40))
