"""ServingCache's own bookkeeping, on the CPU: the library's tables are the plain ones
(tests/qcache_ref.py), the cache is a stand-in."""

import numpy as np
import pytest
import torch

import qcache_ref as ref
from paper_2607_01308_amd import serving
from paper_2607_01308_amd.qcache import QCacheStep


class FakeCache:
    def __init__(self, P, B, L=2, H=2, d=64):
        self.P, self.B, self.L, self.H, self.d = P, B, L, H, d
        self.device = torch.device("cpu")


@pytest.fixture
def plain(monkeypatch):
    """qcache_tables on the CPU; the calls it got."""
    calls = []

    def tables(pages, block, held, new, free, table, tokens, stream=None):
        got = ref.tables(pages, block, held.tolist(), new.tolist(), free.tolist(), table.numpy())
        assert got is not None and sum(new.tolist()) == tokens
        table.copy_(torch.from_numpy(got[0]))
        calls.append((held.clone(), new.clone(), got[4]))
        return QCacheStep(torch.tensor(got[1], dtype=torch.int64),
                          torch.tensor(got[2], dtype=torch.int32),
                          torch.tensor(got[3], dtype=torch.int32),
                          torch.tensor([0, tokens, got[4], max(got[3])]))

    monkeypatch.setattr(serving, "qcache_tables", tables)
    return calls


@pytest.mark.parametrize("seed,P,B,places", [(0, 40, 16, 4), (1, 7, 32, 3), (2, 200, 16, 9), (3, 1, 16, 1)])
def test_pages_are_dealt_once(plain, seed, P, B, places):
    rng = np.random.default_rng(seed)
    sc = serving.ServingCache(FakeCache(P, B), places, P * B)
    for _ in range(300):
        if rng.random() < 0.3:
            sc.release(int(rng.integers(places)))
        else:
            new = [int(rng.integers(0, 3 * B)) if rng.random() < 0.5 else 0 for _ in range(places)]
            before = (list(sc.lengths), sc.free_pages, sc.table.clone())
            try:
                step = sc.extend(new)
            except (RuntimeError, ValueError):
                assert before[:2] == (sc.lengths, sc.free_pages)
                assert torch.equal(before[2], sc.table)
                continue
            assert plain[-1][0].tolist() == before[0] and plain[-1][1].tolist() == new
            assert before[1] - sc.free_pages == plain[-1][2]
            assert (step.tokens, step.max_rows) == (sum(new), max(new))
        used = [int(p) for r in range(places) for p in sc.table[r, :-(-sc.lengths[r] // B)]]
        free = sc._free[sc._head:sc._tail].tolist()
        assert sorted(used + free) == list(range(P))
        assert sc._held.tolist() == sc.lengths


def test_layers_of_one_buffer():
    one = torch.arange(3 * 2 * 2 * 10 * 4.).view(3, 2, 1, 2, 10, 4)
    ks = [one[l, 0, :, :, :7] for l in range(3)]
    got = serving._one_buffer(ks)
    assert got is not None
    assert torch.equal(got, torch.stack([k[0].transpose(0, 1) for k in ks]))
    assert serving._one_buffer([k.clone() for k in ks]) is None
    assert serving._one_buffer([ks[0], ks[2], ks[1]]) is None
    assert serving._one_buffer([ks[0], ks[1], ks[1]]) is None
    assert serving._one_buffer([ks[0]]) is not None
    assert serving._one_buffer([ks[0], one[1, 0, :, :, :7].double()]) is None


class Writes:
    """qcache_write that refuses the `bad`-th call."""
    def __init__(self, bad):
        self.bad, self.calls = bad, 0

    def __call__(self, cache, layer, k, v, slots, stream=None):
        self.calls += 1
        if self.calls == self.bad:
            raise RuntimeError("no")


def state(sc):
    return (list(sc.lengths), sc.free_pages, sc._held.tolist(), sc._free[sc._head:sc._tail].tolist())


def test_caches_that_cannot_be_written_are_refused_before(plain, monkeypatch):
    """Nothing is taken for K and V whose last dimension is strided, that are misaligned or whose
    strides are, or that live elsewhere."""
    sc = serving.ServingCache(FakeCache(9, 16), 2, 64)
    writes = Writes(0)
    monkeypatch.setattr(serving, "qcache_write", writes)
    sc.extend([17, 3])
    before = state(sc)
    good = torch.zeros((1, 2, 5, 64))
    flat = torch.zeros(1 + 2 * 5 * 64)
    for bad in (torch.zeros((1, 2, 5, 128))[..., ::2],               # strided
                flat[1:].view(1, 2, 5, 64),                          # a base that is not aligned
                torch.zeros((1, 2, 5, 65))[..., :64],                # rows that are not
                torch.zeros((1, 2, 5, 64), device="meta")):          # another device
        for pair in ((good, bad), (bad, good)):
            with pytest.raises(ValueError, match="K|V"):
                sc.load(1, [(good, good), pair])
            assert state(sc) == before and writes.calls == 0
    sc.load(1, [(good, good)] * 2)
    assert sc.lengths == [17, 8]


@pytest.mark.parametrize("bad", [1, 2])
def test_a_write_that_fails_gives_the_pages_back(plain, monkeypatch, bad):
    sc = serving.ServingCache(FakeCache(9, 16), 2, 64)
    sc.extend([17, 3])
    before = state(sc)
    monkeypatch.setattr(serving, "qcache_write", Writes(bad))
    layers = [(torch.zeros((1, 2, 40, 64)), torch.zeros((1, 2, 40, 64))) for _ in range(2)]
    with pytest.raises(RuntimeError, match="no"):
        sc.load(1, layers)
    assert state(sc) == before
    sc.load(1, layers)                                   # the same pages again
    assert sc.lengths == [17, 43] and plain[-1][2] == 2
    used = [int(p) for r in range(2) for p in sc.table[r, :-(-sc.lengths[r] // 16)]]
    assert sorted(used + sc._free[sc._head:sc._tail].tolist()) == list(range(9))


@pytest.mark.parametrize("max_len", [1, 15, 16, 17, 70])
def test_places_do_not_grow_beyond_their_length(plain, max_len):
    """To the token, also where the last page has room for more."""
    sc = serving.ServingCache(FakeCache(20, 16), 2, max_len)
    sc.extend([max_len, 0])
    for new in ([1, 0], [0, max_len + 1]):
        before = state(sc)
        with pytest.raises(ValueError, match=f"would hold {max_len + 1} tokens"):
            sc.extend(new)
        assert state(sc) == before
    sc.extend([0, max_len])
    assert sc.lengths == [max_len, max_len]


def test_one_token_of_unaligned_rows_is_loaded(plain, monkeypatch):
    sc = serving.ServingCache(FakeCache(9, 16, L=1, H=1), 1, 64)
    monkeypatch.setattr(serving, "qcache_write", Writes(0))
    sc.load(0, [(torch.zeros(67).as_strided((1, 1, 1, 64), (67, 67, 67, 1)),) * 2])
    assert sc.lengths == [1]
