"""Norms of queries and keys with the rotation (norm_rotate) on the GPU against 64 bits, within what
its roundings allow (tests/draft_ref.py)."""

import pytest
import torch

import draft_ref as ref
import paper_2607_01308_amd as cm

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def values(*shape, seed, dtype, spread=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * spread).to(dtype)


def check(x, got, positions, base, style, weight, eps=1e-6):
    w = None if weight is None else weight.double().cpu()
    want, size = ref.norm_rotate(x.double().cpu(), positions, base, style, w, eps)
    off = (got.double().cpu() - want).abs()
    bound = ref.norm_rotate_bound(got.dtype, want, size, positions, w is not None)
    assert bool((off <= bound).all()), f"{float((off / bound).max())} of the bound"


POSITIONS = [0, 1, 2, 7, 100, 4095, 65537, 260_001, 1 << 20, -1, -300, 5, 6]


@pytest.mark.parametrize("style", ["half", "interleaved"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("dtype,wtype", [(BF16, BF16), (BF16, F32), (F32, F32), (F32, BF16)])
def test_heads_of_one_projection(style, d, dtype, wtype):
    """q and k as parts of a projection's output, odd numbers of heads and tokens."""
    T, Hq, Hk = len(POSITIONS), 7, 3
    x = values(T, Hq + 2 * Hk, d, seed=d, dtype=dtype, spread=2.5)
    q, k, v = x.split((Hq, Hk, Hk), 1)
    qw, kw = (values(d, seed=s, dtype=wtype) + 1 for s in (1, 2))
    pos = torch.tensor(POSITIONS, dtype=torch.int32, device="cuda")
    before = x.clone()
    got = cm.norm_rotate(q, k, pos, 1e6, style=style, q_weight=qw, k_weight=kw)
    check(q, got[0], POSITIONS, 1e6, style, qw)
    check(k, got[1], POSITIONS, 1e6, style, kw)
    assert torch.equal(x, before)
    # in place: the same, and the values behind them as they were
    again = cm.norm_rotate(q, k, pos, 1e6, style=style, q_weight=qw, k_weight=kw, q_out=q, k_out=k)
    assert again[0] is q and torch.equal(q, got[0]) and torch.equal(k, got[1])
    assert torch.equal(v, before[:, Hq + Hk:])


@pytest.mark.parametrize("at", [1, 3, 7])
@pytest.mark.parametrize("d", [64, 256])
@pytest.mark.parametrize("dtype,wtype", [(BF16, BF16), (BF16, F32), (F32, F32), (F32, BF16)])
def test_weights_at_any_address(dtype, wtype, d, at):
    """Weights that begin anywhere in a tensor, with nothing of it behind them."""
    q, k = values(5, 3, d, seed=d, dtype=dtype), values(5, 2, d, seed=d + 1, dtype=dtype)
    positions = [3, 0, 70_000, 12, 9]
    pos = torch.tensor(positions, dtype=torch.int32, device="cuda")
    w = values(at + d, seed=at, dtype=wtype)[at:]
    got = cm.norm_rotate(q, k, pos, 1e4, q_weight=w, k_weight=w)
    check(q, got[0], positions, 1e4, "half", w)
    check(k, got[1], positions, 1e4, "half", w)


@pytest.mark.parametrize("T", [0, 1, 2, 63, 700, 9000])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_any_number_of_tokens(T, dtype):
    q, k = values(T, 3, 64, seed=T, dtype=dtype), values(T, 1, 64, seed=T + 1, dtype=dtype)
    positions = [(37 * i) % 20011 for i in range(T)]
    pos = torch.tensor(positions, dtype=torch.int32, device="cuda")
    w = values(64, seed=3, dtype=dtype)
    got = cm.norm_rotate(q, k, pos, 1e4, q_weight=w, k_weight=w)
    assert got[0].shape == q.shape and got[1].shape == k.shape
    check(q, got[0], positions, 1e4, "half", w)
    check(k, got[1], positions, 1e4, "half", w)


@pytest.mark.parametrize("heads", [1, 4, 9, 40, 129])
def test_rotation_alone_and_queries_alone(heads):
    """Without weights nothing is normalised; without k there are queries alone."""
    q = values(11, heads, 128, seed=heads, dtype=F32)
    positions = list(range(1000, 1011))
    pos = torch.tensor(positions, dtype=torch.int32, device="cuda")
    got, none = cm.norm_rotate(q, None, pos, 5e5, style="interleaved")
    assert none is None
    check(q, got, positions, 5e5, "interleaved", None)
    k = values(11, heads, 128, seed=heads + 1, dtype=F32)
    w = values(128, seed=5, dtype=F32)
    a, b = cm.norm_rotate(q, k, pos, 5e5, style="interleaved", k_weight=w)
    assert torch.equal(a, got)
    check(k, b, positions, 5e5, "interleaved", w)


def test_strides():
    """Heads before tokens, as a render lays a cache out; results into a strided buffer."""
    x = values(2, 5, 33, 128, seed=1, dtype=BF16)
    q, k = x[0].transpose(0, 1), x[1].transpose(0, 1)
    out = torch.full((33, 12, 128), 7.0, device="cuda", dtype=BF16)
    positions = [3 * i for i in range(33)]
    pos = torch.tensor(positions, dtype=torch.int32, device="cuda")
    w = values(128, seed=2, dtype=BF16)
    a, b = cm.norm_rotate(q, k, pos, 1e6, q_weight=w, k_weight=w, q_out=out[:, 1:6], k_out=out[:, 7:])
    check(q, out[:, 1:6], positions, 1e6, "half", w)
    check(k, out[:, 7:], positions, 1e6, "half", w)
    assert bool((out[:, 0] == 7).all()) and bool((out[:, 6] == 7).all())
    # a single token's stride may be anything
    one = torch.empty(5 * 128 + 8, device="cuda", dtype=BF16)[:640].as_strided((1, 5, 128), (3, 128, 1))
    one.copy_(q[:1])
    got, _ = cm.norm_rotate(one, None, pos[:1], 1e6, q_weight=w)
    check(one, got, positions[:1], 1e6, "half", w)


def test_rows_of_zeros_and_of_no_numbers():
    """A row of zeros stays one; what is not finite stays in its own row."""
    q = values(4, 3, 64, seed=1, dtype=F32)
    q[0, 1] = 0
    q[1, 2, 5] = float("nan")
    q[2, 0, 7] = float("inf")
    w = values(64, seed=2, dtype=F32)
    positions = [9, 10, 11, 12]
    pos = torch.tensor(positions, dtype=torch.int32, device="cuda")
    got, _ = cm.norm_rotate(q, None, pos, 1e4, q_weight=w)
    assert bool((got[0, 1] == 0).all())
    assert bool(torch.isnan(got[1, 2]).all())
    bad = torch.isnan(got[2, 0])
    assert bad[7] and bad[39] and int(bad.sum()) == 2 and bool((got[2, 0][~bad] == 0).all())
    q[1, 2], q[2, 0], w2 = 1, 1, w
    clean, _ = cm.norm_rotate(q, None, pos, 1e4, q_weight=w2)
    keep = torch.ones((4, 3), dtype=torch.bool, device="cuda")
    keep[1, 2] = keep[2, 0] = False
    assert torch.equal(got[keep], clean[keep])
    check(q, clean, positions, 1e4, "half", w)


def test_another_stream_and_a_graph():
    q, k = values(40, 8, 128, seed=1, dtype=BF16), values(40, 2, 128, seed=2, dtype=BF16)
    w = values(128, seed=3, dtype=BF16)
    pos = torch.arange(40, dtype=torch.int32, device="cuda")
    want = cm.norm_rotate(q, k, pos, 1e6, q_weight=w, k_weight=w)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = cm.norm_rotate(q, k, pos, 1e6, q_weight=w, k_weight=w, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    outs = torch.empty_like(q), torch.empty_like(k)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cm.norm_rotate(q, k, pos, 1e6, q_weight=w, k_weight=w, q_out=outs[0], k_out=outs[1])
    for n in range(3):
        q.copy_(values(40, 8, 128, seed=10 + n, dtype=BF16))
        pos.add_(100)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = cm.norm_rotate(q, k, pos, 1e6, q_weight=w, k_weight=w)
        assert torch.equal(outs[0], want[0]) and torch.equal(outs[1], want[1])
