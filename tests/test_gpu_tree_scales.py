"""Tree attention over pages whose scale is not finite, or next to the greatest number: rows that do not see
them are as they would be without, rows that see one that is not finite are NaN."""

import numpy as np
import pytest
import torch

import draft_ref as ref
import paper_2607_01308_amd as cm
from test_gpu_qcache import deal, filled, ints, queries
from test_gpu_tree import check, forest, packed, seen

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
NAN, INF = float("nan"), float("inf")
SHAPES = [(64, 16, 2, 1), (128, 16, 1, 4), (256, 64, 1, 2), (64, 128, 1, 16)]


def places(B, spread=0):
    """Three requests of 40 nodes or fewer, and of each the table's entries that some rows see and some do
    not: the second half of the nodes of requests 0 and 1, seen by every other row, and with a window the
    first page of request 2. (Nodes lie behind their context's last full page.)"""
    held, counts = [2 * B, 4 * B + spread * B, 9 * B], [40 * B // 16, 2 * B, 5]
    lens = [a + b for a, b in zip(held, counts)]
    sees = []
    for c in counts:
        for i in range(c):
            up = {j for j in range(min(i + 1, B))}
            if i % 2:
                up |= {j for j in range(B, c) if j % 3 != 1}
            sees.append(up)
    positions = [h + min(i, 3 * B) for h, c in zip(held, counts) for i in range(c)]
    odd = [(0, held[0] // B + 1), (1, held[1] // B + 1)]
    touched = [i % 2 == 1 and c > B for c in counts for i in range(c)]
    return lens, counts, sees, positions, odd, touched


def run(q, codes, scales, table, lens, counts, sees, positions, window=0):
    at = [0] + [int(x) for x in np.cumsum(counts)]
    tree = cm.QCacheTree(packed(sees, -(-max(counts) // 64)), ints(positions), window)
    return cm.qcache_tree_attention(cm.QCache(codes, scales), 0, q, ints(table), ints(lens), ints(at), tree,
                                    max_rows=max(counts))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("kv,value", [(0, NAN), (0, INF), (1, NAN), (1, INF)])
@pytest.mark.parametrize("d,B,H,G", SHAPES)
def test_scales_that_are_not_finite(dtype, kv, value, d, B, H, G):
    """Of nodes that every other row sees."""
    lens, counts, sees, positions, odd, touched = places(B)
    table, P = deal(lens, B, seed=d)
    codes, scales = filled(P, H, B, d, seed=d + B)
    q = queries(sum(counts), H * G, d, dtype, seed=d)
    clean = run(q, codes, scales, table, lens, counts, sees, positions)
    for r, entry in odd:
        scales[0, kv, int(table[r, entry])] = value
    got = run(q, codes, scales, table, lens, counts, sees, positions)
    assert any(touched) and not all(touched)
    rows = None if value != value else [not x for x in touched]
    check(q, codes, scales, 0, table, lens, counts, sees, positions, got=got, rows=rows)
    touched = torch.tensor(touched, device="cuda")
    if kv == 1:                                              # (scores, and what they are relative to, are the same)
        assert torch.equal(got[0][~touched], clean[0][~touched])
        assert torch.equal(got[1], clean[1]) and bool(torch.isfinite(got[1]).all())
    assert bool(torch.isnan(got[0][touched]).all()) and bool(torch.isnan(got[1][touched]).all()) == (kv == 0)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("value", [NAN, INF])
@pytest.mark.parametrize("spread", [0, 300])
def test_pages_before_the_window_and_of_nobody(dtype, value, spread):
    """Pages that no row sees, or that the window hides from all but some: in one range of the context and
    in many."""
    d, B, H, G, window = 128, 16, 2, 2, 50
    lens, counts, sees, positions, _, _ = places(B, spread)
    table, P = deal(lens, B, seed=3)
    codes, scales = filled(P, H, B, d, seed=4)
    q = queries(sum(counts), H * G, d, dtype, seed=5)
    clean = run(q, codes, scales, table, lens, counts, sees, positions, window)
    used = {int(p) for r, T in enumerate(lens) for p in table[r, :-(-T // B)]}
    for p in set(range(P)) - used:
        scales[0, :, p] = value
    for r, T in enumerate(lens):
        held = T - counts[r]
        for p in table[r, :max(0, held - window + 1) // B]:
            scales[0, :, int(p)] = value
    got = run(q, codes, scales, table, lens, counts, sees, positions, window)
    assert torch.equal(got[0], clean[0]) and torch.equal(got[1], clean[1])
    # of a page whose last token is the first that request 2's first row sees: that row alone
    held = lens[2] - counts[2]
    assert (held - window + 1) % B == B - 1 and positions[-5:] == [held + i for i in range(5)]
    for kv in (0, 1):
        some = scales.clone()
        some[0, kv, int(table[2, (held - window + 1) // B])] = value
        got = run(q, codes, some, table, lens, counts, sees, positions, window)
        assert bool(torch.isnan(got[0][-5]).all()) and bool(torch.isnan(got[1][-5]).all()) == (kv == 0)
        others = torch.arange(len(q), device="cuda") != len(q) - 5
        if kv == 1:
            assert torch.equal(got[0][others], clean[0][others])
        check(q, codes, some, 0, table, lens, counts, sees, positions, window, got=got, rows=others.tolist())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("power", [110, 118, 119, 120, 121])
@pytest.mark.parametrize("d,B,H,G", SHAPES[:3])
def test_scales_next_to_the_greatest_number(dtype, power, d, B, H, G):
    """V scales of 2^110 to 2^121. The least codes are seen right: a sum of weights, each up to 2^8 (they are
    relative to an earlier maximum), times at most 160 values of 1.5 * 2^(121 - 1 - 9) stays below 2^127.
    The greatest codes, whose products do not, leave the rows alone that do not see them."""
    lens, counts, sees, positions, odd, touched = places(B)
    table, P = deal(lens, B, seed=d)
    codes, scales = filled(P, H, B, d, seed=d + B)
    raw = codes.view(torch.uint8)
    q = queries(sum(counts), H * G, d, dtype, seed=d)
    clean = run(q, codes, scales, table, lens, counts, sees, positions)
    least = 1 + 0x80 * (torch.arange(B * d, device="cuda") % 3 == 0).to(torch.uint8).view(B, d)
    for r, entry in odd:
        page = int(table[r, entry])
        scales[0, 1, page] = 1.5 * 2.0 ** (power - 1)
        raw[0, 1, page] = least
    got = check(q, codes, scales, 0, table, lens, counts, sees, positions)
    touched = torch.tensor(touched, device="cuda")
    assert torch.equal(got[0][~touched], clean[0][~touched])
    for r, entry in odd:
        raw[0, 1, int(table[r, entry])] = 0x7E
        scales[0, 1, int(table[r, entry])] = 1.5 * 2.0 ** (power + 6)
    got = run(q, codes, scales, table, lens, counts, sees, positions)
    assert torch.equal(got[0][~touched], clean[0][~touched]) and torch.equal(got[1][~touched], clean[1][~touched])
