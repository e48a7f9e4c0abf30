"""How many bits the 8-bit cache's attention holds (tests/qcache_precision.py): decoding steps and
prompts, batches and long contexts, against 64-bit results within what the roundings allow."""

import numpy as np
import pytest
import torch

import paper_2607_01308_amd as cm
import qcache_precision as bits
from test_gpu_qcache import BF16, F32, deal, filled, ints, queries

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d,B,H,G,lens,counts,window", [
    (64, 32, 1, 2, [70000], [1], 0),                              # one long context, few rows
    (128, 16, 2, 4, [20011], [3], 0),
    (128, 16, 8, 4, list(range(100, 4100, 127)), [1] * 32, 0),    # a decoding batch
    (256, 64, 2, 4, list(range(30, 3000, 211)), [1] * 15, 700),
    (64, 16, 4, 1, [500] * 70, [1] * 70, 0),                      # short ones, a wave each
    (128, 16, 2, 4, [4000, 2500, 900], [300, 77, 900], 0),        # prompts and questions
    (64, 32, 2, 2, [3000, 2000], [1000, 33], 500),
    (256, 32, 1, 3, [2000, 1500], [500, 20], 0),
    (128, 16, 2, 4, [6000, 2000, 40, 3000], [400, 1, 2, 1], 0),   # a prompt beside decoding requests
])
def test_bits_of_the_output(dtype, d, B, H, G, lens, counts, window):
    table, P = deal(lens, B, seed=d)
    codes, scales = filled(P, H, B, d, seed=G + d)
    q = queries(sum(counts), H * G, d, dtype, seed=d)
    rows = [0] + [int(x) for x in np.cumsum(counts)]
    got = cm.qcache_attention(cm.QCache(codes, scales), 0, q, ints(table), ints(lens), rows=ints(rows),
                              max_rows=max(counts), window=window)
    want = bits.attend(q, codes[0].view(torch.uint8), scales[0], table, lens, counts, window)
    far = bits.check(got, dtype, max(lens), *want)
    assert max(far) <= 1, f"out, lse: {far} of what is allowed"


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("counts", [[1] * 64, [64]])
def test_bits_of_the_queries(d, counts):
    """Equal elements of a query over equal codes: lse is their product."""
    B, H = 16, 1
    lens = [33] * len(counts) if len(counts) > 1 else [200]
    table, P = deal(lens, B)
    codes, scales = filled(P, H, B, d, seed=1)
    codes.view(torch.uint8)[0, 0] = 0x3C                 # K: 1.5 everywhere
    scales[0, 0] = 2.0 ** -3
    a = bits.lined_up(d, 64, d).cuda()
    q = a[:, None, None].expand(64, 1, d).contiguous()
    rows = [0] + [int(x) for x in np.cumsum(counts)]
    _, lse = cm.qcache_attention(cm.QCache(codes, scales), 0, q, ints(table), ints(lens),
                                 rows=ints(rows), max_rows=max(counts), scale=1.0)
    seen = torch.tensor([t - c + i + 1 for t, c in zip(lens, counts) for i in range(c)], device="cuda")
    want = a.double() * (d * 1.5 / 8) + seen.double().log()
    assert float(((lse[:, 0].double() - want) / want).abs().max()) <= bits.LINED_UP


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("counts", [[1] * 64, [64]])
def test_bits_of_the_weights(d, counts):
    """One token scores more than the others, all values are equal: the output is that value."""
    B, H = 16, 1
    lens = [250] * len(counts) if len(counts) > 1 else [250 + 64]
    table, P = deal(lens, B)
    codes, scales = filled(P, H, B, d, seed=1)
    raw = codes.view(torch.uint8)
    raw[0, 0] = 0x38                                     # K: 1 everywhere
    for r in range(len(lens)):
        raw[0, 0, int(table[r, 0]), :, 3] = 0x3C         # 1.5 in one token
    scales[0, 0] = 1.0 / d
    raw[0, 1] = 0x3A                                     # V: 1.25 * 1.375
    scales[0, 1] = 1.375
    a = bits.lined_up(d, 64, d + 1).cuda()
    q = a[:, None, None].expand(64, 1, d).contiguous()
    rows = [0] + [int(x) for x in np.cumsum(counts)]
    out, _ = cm.qcache_attention(cm.QCache(codes, scales), 0, q, ints(table), ints(lens),
                                 rows=ints(rows), max_rows=max(counts), scale=1.0)
    value = 1.25 * 1.375
    assert float((out.double() / value - 1).abs().max()) <= bits.LINED_UP


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d,B,H,G,lens,counts", [
    (128, 16, 2, 4, [4000, 900, 2000], [300, 200, 40]),
    (64, 32, 1, 2, [2500, 700], [500, 33]),
    (256, 64, 1, 4, [3000, 1000], [100, 20]),
    (128, 16, 1, 4, [16000], [4]),
])
def test_bits_of_flat_weights(dtype, d, B, H, G, lens, counts):
    """Scores that differ little: no token has more than a small part of a row's sum."""
    table, P = deal(lens, B, seed=d)
    codes, scales = filled(P, H, B, d, seed=G + d)
    q = queries(sum(counts), H * G, d, dtype, seed=d, spread=0.25)
    rows = [0] + [int(x) for x in np.cumsum(counts)]
    got = cm.qcache_attention(cm.QCache(codes, scales), 0, q, ints(table), ints(lens), rows=ints(rows),
                              max_rows=max(counts))
    want = bits.attend(q, codes[0].view(torch.uint8), scales[0], table, lens, counts)
    far = bits.check(got, dtype, max(lens), *want)
    assert max(far) <= 1, f"out, lse: {far} of what is allowed"
