"""The 8-bit cache's attention where its arguments reach their ends (more rows than are computed, a
scale of 0, the widest windows and groups, strides that are not used), against 64-bit results
(tests/qcache_ref.py)."""

import numpy as np
import pytest
import torch

import paper_2607_01308_amd as cm
from test_gpu_qcache import BF16, F32, check_attention, deal, filled, ints, queries

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("H,G,d,B,window,ends,most", [
    (2, 1, 64, 16, 0, [10, 14, 29, 32], 4),              # few rows of a request are computed
    (1, 4, 128, 32, 0, [10, 14, 29, 32], 4),
    (2, 2, 256, 16, 20, [3, 12, 12, 17], 6),
    (1, 2, 128, 16, 0, [70, 90, 300, 340], 40),          # many
    (2, 4, 64, 32, 33, [70, 90, 300, 340], 40),
    (1, 1, 256, 64, 0, [500, 640, 650, 700], 130),
])
def test_more_rows_than_are_computed(dtype, H, G, d, B, window, ends, most):
    """A request's rows past max_rows and past the queries' end are not computed; the others stand at
    the positions that the request's true number of rows gives them."""
    starts, n_rows = [0] + ends[:-1], ends[-1] - 1       # the last request's end lies past the queries
    counts = [b - a for a, b in zip(starts, ends)]
    lens = [c + 3 + 50 * r for r, c in enumerate(counts)]
    lens[1] = max(counts[1] - 2, 1)                      # its first rows stand before its first token
    table, P = deal(lens, B, seed=d)
    codes, scales = filled(P, H, B, d, seed=d + B)
    q = queries(n_rows, H * G, d, dtype, seed=most)
    out = torch.full_like(q, 7.0)
    lse = torch.full((n_rows, H * G), 7.0, device="cuda")
    cm.qcache_attention(cm.QCache(codes, scales), 0, q, ints(table), ints(lens), rows=ints([0] + ends),
                        max_rows=most, window=window, out=out, lse=lse)
    done = [min(c, most, max(n_rows - a, 0)) for a, c in zip(starts, counts)]
    at = torch.tensor(np.concatenate([np.arange(a, a + m) for a, m in zip(starts, done)]),
                      device="cuda")
    # the last row computed sees as many tokens less as rows come after it
    seen = [t - (c - m) for t, c, m in zip(lens, counts, done)]
    check_attention(q[at], codes, scales, 0, table, seen, done, window=window,
                    got=(out[at], lse[at]))
    others = torch.ones(n_rows, dtype=torch.bool, device="cuda")
    others[at] = False
    assert bool((out[others] == 7).all()) and bool((lse[others] == 7).all())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("H,G,d,B,window", [(2, 2, 128, 16, 0), (1, 4, 64, 32, 50), (1, 1, 256, 64, 0)])
def test_scale_of_zero(dtype, H, G, d, B, window):
    """All weights are equal: the mean of the values that a row sees, lse the logarithm of their
    number; the same from the kernel for few rows and the one for many."""
    lens, counts = [300, 77, 140, 90], [1, 3, 97, 40]
    table, P = deal(lens, B, seed=1)
    table[2, 1] = -1                                     # an evicted page
    codes, scales = filled(P, H, B, d, seed=d)
    q = queries(sum(counts), H * G, d, dtype, seed=d)
    for scale in (0.0, -0.0, 1e-45):
        check_attention(q, codes, scales, 0, table, lens, counts, window=window, scale=scale)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("H,G,d", [(1, 1, 64), (2, 1, 128), (1, 1, 256)])
def test_the_widest_windows(dtype, H, G, d):
    """Windows up to the greatest that a caller can give, also for rows that stand before their
    request's first token: the same as none."""
    lens, counts, B = [5, 5, 0, 300], [9, 40, 3, 130], 16
    table, P = deal(lens, B, seed=2)
    codes, scales = filled(P, H, B, d, seed=d)
    q = queries(sum(counts), H * G, d, dtype, seed=d)
    none = check_attention(q, codes, scales, 0, table, lens, counts)
    for window in (2 ** 31 - 1, 2 ** 31 - 30, 2 ** 30):
        got = check_attention(q, codes, scales, 0, table, lens, counts, window=window)
        assert torch.equal(got[0], none[0]) and torch.equal(got[1], none[1])


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_one_token_of_unaligned_rows(dtype):
    """Dimensions of size 1 with strides that are no multiple of 16 bytes."""
    H, d, B = 1, 64, 16
    k, v, q = (queries(1, 1, d, dtype, seed=i).expand(3, 1, d) for i in range(3))
    odd = [torch.empty((3, 67), dtype=dtype, device="cuda") for _ in range(4)]
    for to, x in zip(odd, (k, v, q)):
        to[0, :64] = x[0, 0]
    k, v, q, out = (x[:1, None, :64].as_strided((1, 1, d), (67, 67, 1)) for x in odd)
    cache = cm.QCache.empty(1, H, d, 2, B)
    table, one = ints([[1]]), ints([1])
    cm.qcache_write(cache, 0, k, v, torch.tensor([B], device="cuda"))
    _, lse = cm.qcache_attention(cache, 0, q, table, one, out=out)
    same = cm.QCache.empty(1, H, d, 2, B)
    cm.qcache_write(same, 0, k.clone().view(1, 1, d), v.clone().view(1, 1, d),
                    torch.tensor([B], device="cuda"))
    assert torch.equal(same.codes.view(torch.uint8), cache.codes.view(torch.uint8))
    want = cm.qcache_attention(same, 0, q.clone().view(1, 1, d), table, one)
    assert torch.equal(want[0], out) and torch.equal(want[1], lse)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("H,G,d,B,counts", [
    (2, 17, 64, 16, [1, 1, 1, 1]), (1, 32, 128, 16, [1, 0, 1, 1]), (1, 64, 128, 32, [1, 1, 2, 1]),
    (2, 64, 256, 16, [1, 1, 0, 1]), (1, 48, 64, 64, [3, 1, 17, 0])])
def test_wide_groups(dtype, H, G, d, B, counts):
    """17 to 64 query heads for a KV head: a decoding step's row is more than a tile of 16."""
    lens = [700, 1, 33, 5000]
    table, P = deal(lens, B, seed=G)
    codes, scales = filled(P, H, B, d, seed=G)
    q = queries(sum(counts), H * G, d, dtype, seed=G)
    for window in (0, 100):
        check_attention(q, codes, scales, 0, table, lens, counts, window=window, device="cuda")
