"""Accepted nodes moved within the 8-bit cache (qcache_keep) and pages copied (qcache_copy) on the GPU:
codes, scales, lengths and freed pages exactly (tests/draft_ref.py)."""

import numpy as np
import pytest
import torch

import draft_ref as ref
import paper_2607_01308_amd as cm
from paper_2607_01308_amd import _cabi as C
from test_gpu_qcache import deal, ints

pytestmark = pytest.mark.gpu


def cache_of(L, P, H, B, d, seed, power=True):
    """Every code and scales of several powers of two (or of any size); NaN codes among them."""
    rng = np.random.default_rng(seed)
    codes = rng.integers(0, 256, size=(L, 2, P, H, B, d), dtype=np.uint8)
    scales = np.exp2(rng.integers(-9, 3, size=(L, 2, P, H))).astype(np.float32)
    if not power:
        scales *= rng.uniform(1, 2, size=scales.shape).astype(np.float32)
    codes[rng.random(codes.shape[:4])[..., None, None] * np.ones(codes.shape) < 0.3] &= 0x7B
    cache = cm.QCache(torch.tensor(codes, device="cuda"), torch.tensor(scales, device="cuda"))
    return cache, codes, scales


def same_codes(got, want):
    """Equal, NaN of either sign being one."""
    got, want = np.array(got), np.array(want)
    got[(got & 0x7F) == 0x7F] = want[(want & 0x7F) == 0x7F] = 0x7F
    return np.array_equal(got, want)


def paths(rng, new, kept):
    path = []
    for c, k in zip(new, kept):
        some = [0] + sorted(int(x) for x in 1 + rng.permutation(c - 1)[:k - 1]) if k else []
        path += some + [-1] * (c - len(some))
    return path


def run(cache, codes, scales, table, lens, rows, path, counts, power=True):
    freed = torch.full((64,), -7, dtype=torch.int32, device="cuda")
    got = cm.qcache_keep(cache, ints(table), ints(lens), ints(rows), ints(path), ints(counts), freed=freed)
    out, pages = ref.keep(codes, scales, table, lens, rows, path, counts)
    got.check()
    assert got.lens.tolist() == out
    assert got.info.tolist() == [0, len(pages)]
    assert freed.tolist() == pages + [-7] * (64 - len(pages))
    assert np.array_equal(cache.scales.cpu().numpy(), scales)
    assert same_codes(cache.codes.cpu().numpy(), codes)


@pytest.mark.parametrize("power", [True, False])
@pytest.mark.parametrize("L,H,B,d", [(2, 2, 16, 128), (1, 3, 32, 64), (3, 1, 64, 256), (1, 2, 128, 64),
                                     (5, 1, 16, 64), (1, 1, 128, 256)])
def test_paths(L, H, B, d, power):
    """Contexts that end anywhere in a page, nodes over several pages, none to all of them kept."""
    rng = np.random.default_rng(L + B + d)
    held = [0, 1, B - 1, B, B + 3, 2 * B - 5, 5, 37]
    new = [1, 2 * B + 3, 5, B, 64, 31, 7, 3]
    kept = [1, B + 9, 0, B, 20, 30, 7, 1]
    lens = [a + b for a, b in zip(held, new)]
    table, P = deal(lens, B, seed=B)
    cache, codes, scales = cache_of(L, P, H, B, d, seed=d, power=power)
    rows = [0] + [int(x) for x in np.cumsum(new)]
    run(cache, codes, scales, table, lens, rows, paths(rng, new, kept), kept)


@pytest.mark.parametrize("seed", range(6))
def test_many_requests(seed):
    rng = np.random.default_rng(seed)
    B, n = 16, [1, 3, 40, 200, 17, 64][seed]
    held = [int(x) for x in rng.integers(0, 60, size=n)]
    new = [int(x) for x in rng.integers(1, 20, size=n)]
    kept = [int(rng.integers(0, c + 1)) for c in new]
    lens = [a + b for a, b in zip(held, new)]
    table, P = deal(lens, B, seed=seed)
    cache, codes, scales = cache_of(1, P, 1, B, 64, seed=seed)
    rows = [0] + [int(x) for x in np.cumsum(new)]
    path = paths(rng, new, kept)
    freed = torch.full((n + sum(new),), -7, dtype=torch.int32, device="cuda")
    got = cm.qcache_keep(cache, ints(table), ints(lens), ints(rows), ints(path), ints(kept), freed=freed)
    out, pages = ref.keep(codes, scales, table, lens, rows, path, kept)
    assert got.check().lens.tolist() == out and freed.tolist()[:len(pages)] == pages
    assert np.array_equal(cache.scales.cpu().numpy(), scales)
    assert same_codes(cache.codes.cpu().numpy(), codes)


def test_chains_change_nothing():
    """A path of 0, 1, 2, .. leaves every byte; a second call with the lengths then moves nothing either."""
    lens, new, kept = [70, 33, 20], [9, 33, 4], [4, 33, 0]
    table, P = deal(lens, 16)
    cache, codes, scales = cache_of(2, P, 2, 16, 128, seed=3)
    path = [0, 1, 2, 3, -1, -1, -1, -1, -1] + list(range(33)) + [-1] * 4
    run(cache, codes.copy(), scales.copy(), table, lens, [0, 9, 42, 46], path, kept)
    assert np.array_equal(cache.codes.cpu().numpy(), codes)
    assert np.array_equal(cache.scales.cpu().numpy(), scales)


def test_pages_that_are_not_there():
    """Entries outside the pool: rows that come from them or go to them stay as they are."""
    rng = np.random.default_rng(4)
    lens, new, kept = [50, 80], [30, 40], [20, 33]
    table, P = deal(lens, 16, seed=2)
    cache, codes, scales = cache_of(1, P, 2, 16, 64, seed=6)
    table[0, 2], table[1, 3], table[1, 4] = -1, P, 2 ** 31 - 1
    run(cache, codes, scales, table, lens, [0, 30, 70], paths(rng, new, kept), kept)


def test_what_is_not_as_said():
    """Such a request's rows are not moved; lengths and pages go by its counts."""
    B, lens, rows = 16, [40, 40, 40], [0, 20, 40, 60]
    table, P = deal(lens, B, seed=5)
    good = list(range(0, 20, 2)) + [-1] * 10
    for first, counts, held in (
            ([0, 2, 2] + [-1] * 17, [3, 10, 10], 23),                # not ascending
            ([1, 0] + [-1] * 18, [2, 10, 10], 22),
            ([0, 20] + [-1] * 18, [2, 10, 10], 22),                  # past the nodes
            ([0, 3, -1] + [-1] * 17, [3, 10, 10], 23),               # shorter than its count
            (good, [-1, 10, 10], 20), (good, [21, 10, 10], 40),      # counts outside the nodes
    ):
        cache, codes, scales = cache_of(1, P, 1, B, 64, seed=1)
        freed = torch.full((20,), -7, dtype=torch.int32, device="cuda")
        got = cm.qcache_keep(cache, ints(table), ints(lens), ints(rows), ints(first + good + good),
                             ints(counts), freed=freed)
        want = codes.copy(), scales.copy()
        ref.keep(*want, table[1:], lens[1:], [0, 20, 40], good + good, [10, 10])
        assert got.info.tolist()[0] == C.CM_EINVAL and got.lens.tolist() == [held, 30, 30]
        pages = [int(table[0, j]) for j in range(-(-held // B), 3)]
        pages += [int(table[1, 2]), int(table[2, 2])]
        assert freed.tolist() == pages + [-7] * (20 - len(pages))
        assert same_codes(cache.codes.cpu().numpy(), want[0])
        assert np.array_equal(cache.scales.cpu().numpy(), want[1])
        with pytest.raises(cm.CmError, match="not as it has to be"):
            got.check()
    # rows out of order, lengths shorter than the nodes or longer than the table's rows
    for lens2, rows2, out in (([40, 40, 40], [0, 30, 20, 60], [20, 40, 10]),
                              ([5, 40, 40], rows, [0, 30, 30]), ([40, 2 ** 31 - 1, 40], rows, [30, 2 ** 31 - 11, 30])):
        cache, codes, scales = cache_of(1, P, 1, B, 64, seed=1)
        got = cm.qcache_keep(cache, ints(table), ints(lens2), ints(rows2), ints(good * 3), ints([10, 10, 10]))
        assert got.info.tolist()[0] == C.CM_EINVAL and got.lens.tolist() == out
    # freed pages: too few places, none at all
    cache, codes, scales = cache_of(1, P, 1, B, 64, seed=1)
    freed = torch.full((2,), -7, dtype=torch.int32, device="cuda")
    got = cm.qcache_keep(cache, ints(table), ints(lens), ints(rows), ints(good * 3), ints([10, 10, 10]), freed=freed)
    assert got.info.tolist() == [C.CM_EINVAL, 3] and freed.tolist() == [int(table[0, 2]), int(table[1, 2])]


def test_a_graph_and_another_stream():
    rng = np.random.default_rng(7)
    lens, new, kept = [70, 33], [30, 20], [12, 9]
    table, P = deal(lens, 16)
    args = [ints(table), ints(lens), ints([0, 30, 50]), ints([0] * 50), ints(kept)]
    cache, codes, scales = cache_of(2, P, 2, 16, 128, seed=3)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = cm.qcache_keep(cache, *args)
    for n in range(3):
        path = paths(rng, new, kept)
        args[3].copy_(ints(path))
        torch.cuda.synchronize()
        if n < 2:
            graph.replay()
        else:
            got = cm.qcache_keep(cache, *args, stream=side)
        torch.cuda.synchronize()
        out, _ = ref.keep(codes, scales, table, lens, [0, 30, 50], path, kept)
        assert got.lens.tolist() == out
        assert np.array_equal(cache.scales.cpu().numpy(), scales)
        assert same_codes(cache.codes.cpu().numpy(), codes)


@pytest.mark.parametrize("L,H,B,d,n", [(3, 2, 16, 64, 1), (1, 1, 16, 64, 40), (2, 8, 16, 128, 9),
                                       (1, 3, 128, 256, 5), (2, 5, 64, 128, 3)])
def test_copies(L, H, B, d, n):
    P = 2 * n + 4
    cache, codes, scales = cache_of(L, P, H, B, d, seed=n)
    order = np.random.default_rng(n).permutation(P)
    src, dst = order[:n].tolist(), order[n:2 * n].tolist()
    src[n // 2] = src[0]                                 # one page to several places
    pairs = list(zip(src, dst)) + [(order[2 * n], order[2 * n])]
    bad = [(-1, order[2 * n + 1]), (order[0], P), (P, order[2 * n + 1]), (order[1], -1)]
    every = pairs + bad
    for first, layers in ((0, None), (L - 1, None), (0, 1)):
        cm.qcache_copy(cache, ints([a for a, _ in every]), ints([b for _, b in every]), first, layers)
        upto = L if layers is None else first + layers
        for a, b in pairs:
            codes[first:upto, :, b] = codes[first:upto, :, a]
            scales[first:upto, :, b] = scales[first:upto, :, a]
        assert np.array_equal(cache.codes.cpu().numpy(), codes)
        assert np.array_equal(cache.scales.cpu().numpy(), scales)
    cm.qcache_copy(cache, ints([]), ints([]))
