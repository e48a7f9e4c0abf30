"""That the tolerances of tests/qcache_precision.py tell the attention's arithmetic from one that
holds fewer bits or loses tokens: the mistakes are made in the 64-bit attention, on the CPU."""

import numpy as np
import pytest
import torch

import qcache_precision as bits

BF16, F32 = torch.bfloat16, torch.float32


def case(T, count, d, dtype, G=2, B=16, seed=0):
    g = torch.Generator().manual_seed(seed)
    P = -(-T // B)
    x = torch.randn((2, P, 1, B, d), generator=g)
    scales = torch.exp2(torch.ceil(torch.log2(x.abs().amax((-2, -1)) / 448)))
    codes = (x / scales[..., None, None]).to(torch.float8_e4m3fn).view(torch.uint8)
    q = torch.randn((count, G, d), generator=g).to(dtype)
    table = np.random.default_rng(seed).permutation(P)[None]
    return q, codes, scales, table, [T], [count]


def result(dtype, args, **mistake):
    out, lse, _, _ = bits.attend(*args, **mistake)
    return out.to(dtype), lse.float()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,count,d", [(3000, 40, 64), (900, 5, 128), (20000, 1, 128), (70000, 1, 64)])
def test_bits_of_the_output(dtype, T, count, d):
    args = case(T, count, d, dtype)
    want = bits.attend(*args)
    held = 2 if dtype is BF16 else 3
    far = bits.check(result(dtype, args, weights=lambda e: bits.terms(e, held)), dtype, T, *want)
    assert max(far) <= 1
    # weights of fewer terms
    far = bits.check(result(dtype, args, weights=lambda e: bits.terms(e, 1)), dtype, T, *want)
    assert far[0] > 1.2

    def lost(v, at=T // 2):
        v = v.clone()
        v[:, at:at + 128] = 0
        return v

    def moved(v, at=T // 2):
        return torch.cat((v[:, :at], v[:, at:at + 128].flip(1), v[:, at + 128:]), 1)

    for values in (lost, moved):
        far = bits.check(result(dtype, args, values=values), dtype, T, *want)
        assert far[0] > 2


def test_errors_that_add_up():
    a = bits.lined_up(128, 64, 128).double()
    assert float(((bits.terms(a, 3) - a) / a).abs().max()) < bits.LINED_UP / 16
    assert float(((bits.terms(a, 2) - a) / a).abs().max()) > 2 * bits.LINED_UP
    # the weights of test_bits_of_the_weights
    for d in (64, 128, 256):
        p = torch.exp(-0.5 * bits.lined_up(d, 64, d + 1).double())
        for held, far in ((3, False), (2, True)):
            t = bits.terms(p, held)
            e = ((1 + 249 * t) / (1 + 249 * p) - 1).abs().max()
            assert bool(e > 2 * bits.LINED_UP) == far
