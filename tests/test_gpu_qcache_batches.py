"""The 8-bit cache's attention over batches of many requests against 64-bit results: short ones
beside long ones, requests without rows, and more row tiles than are ever cut."""

import numpy as np
import pytest
import torch

import paper_2607_01308_amd as cm
from test_gpu_qcache import BF16, F32, check_attention, deal, filled, ints, queries

pytestmark = pytest.mark.gpu

SHORT = [0, 1, 2, 31, 32, 33, 64, 127, 129, 255, 256, 257, 300, 511, 512, 513, 640]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d,B,H,G,n,window,rows", [
    (128, 16, 2, 4, 700, 0, 1), (64, 32, 8, 3, 300, 0, 1), (256, 64, 4, 1, 250, 0, 1),
    (128, 16, 4, 2, 500, 100, 2), (64, 16, 1, 16, 1024, 0, 1), (256, 16, 8, 2, 120, 33, 5)])
def test_short_requests_beside_long_ones(dtype, d, B, H, G, n, window, rows):
    rng = np.random.default_rng(n + d)
    lens = [int(x) for x in rng.choice(SHORT, n)]
    for r in rng.choice(n, 3, replace=False):
        lens[r] = int(rng.integers(2000, 5000))
    counts = [int(x) for x in rng.choice([0, 1, rows], n)]
    table, P = deal(lens, B, seed=n)
    codes, scales = filled(P, H, B, d, seed=n)
    q = queries(sum(counts), H * G, d, dtype, seed=n)
    check_attention(q, codes, scales, 0, table, lens, counts, window=window, device="cuda")


@pytest.mark.parametrize("dtype,d", [(BF16, 128), (F32, 128), (BF16, 256)])
@pytest.mark.parametrize("counts", [[900, 3, 40, 411, 1], [17] * 60 + [700]])
def test_prompts_longer_than_what_a_workgroup_has_to_do(dtype, d, counts):
    """More row tiles than workgroups that run together, some of them far longer than the others."""
    H, G, B = 8, 4, 16
    held = [0, 3000, 7, 1500, 40] if len(counts) == 5 else [5] * 60 + [2500]
    lens = [a + b for a, b in zip(held, counts)]
    table, P = deal(lens, B, seed=d)
    codes, scales = filled(P, H, B, d, seed=d)
    q = queries(sum(counts), H * G, d, dtype, seed=d)
    check_attention(q, codes, scales, 0, table, lens, counts, device="cuda")


def test_more_row_tiles_than_are_cut():
    """So many tiles that no place is kept for partial results: long requests go uncut."""
    H, G, d, B, n, each = 64, 1, 64, 16, 1010, 20
    lens = [20 + r % 17 for r in range(n)]
    lens[400] = 3001
    table, P = deal(lens, B, seed=3)
    codes, scales = filled(P, H, B, d, seed=3)
    q = queries(n * each, H * G, d, BF16, seed=3)
    rows = ints(np.arange(n + 1) * each)
    out, lse = cm.qcache_attention(cm.QCache(codes, scales), 0, q, ints(table), ints(lens), rows=rows,
                                   max_rows=each)
    for some in ([0, 1, 2], [399, 400, 401], [n - 1]):
        at = np.concatenate([np.arange(r * each, (r + 1) * each) for r in some])
        i = torch.tensor(at, device="cuda")
        check_attention(q[i], codes, scales, 0, table[some], [lens[r] for r in some],
                        [each] * len(some), got=(out[i], lse[i]), device="cuda")


def test_a_long_request_among_more_row_tiles_than_run_together():
    """It is cut, however many tiles there are beside it."""
    H, G, d, B, n, each = 64, 1, 64, 16, 1010, 20
    lens = [20 + r % 17 for r in range(n)]
    lens[400] = 30001
    table, P = deal(lens, B, seed=4)
    codes, scales = filled(P, H, B, d, seed=4)
    q = queries(n * each, H * G, d, BF16, seed=4)
    rows = ints(np.arange(n + 1) * each)
    out, lse = cm.qcache_attention(cm.QCache(codes, scales), 0, q, ints(table), ints(lens), rows=rows,
                                   max_rows=each)
    for some in ([0, 1, 2], [399, 400, 401], [n - 1]):
        at = np.concatenate([np.arange(r * each, (r + 1) * each) for r in some])
        i = torch.tensor(at, device="cuda")
        check_attention(q[i], codes, scales, 0, table[some], [lens[r] for r in some],
                        [each] * len(some), got=(out[i], lse[i]), device="cuda")
