"""What of ServingCache can be captured into a HIP graph: a step's write and attention, replayed with
eager work between the replays; the steps themselves are refused."""

import pytest
import torch

import paper_2607_01308_amd as cm
from test_gpu_serving import BF16, rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("own_stream", [False, True])
def test_steps_are_not_captured(own_stream):
    sc = cm.ServingCache(cm.QCache.empty(1, 2, 64, 20), 2, 200)
    K = torch.zeros((1, 2, 1, 64), device="cuda", dtype=BF16)
    for _ in range(2):
        sc.extend([1, 0])                                # (the lengths of a step, on the device)
        sc.extend([0, 1])
    sc.load(1, [(K, K)])
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    before = (list(sc.lengths), sc.free_pages, sc._held)
    x = torch.zeros(4, device="cuda")
    graph = torch.cuda.CUDAGraph()
    stream = side if own_stream else None
    with torch.cuda.graph(graph, stream=side):
        x += 1
        for call in (lambda: sc.extend([0, 1], stream), lambda: sc.release(0, stream),
                     lambda: sc.load(1, [(K, K)], stream)):
            with pytest.raises(RuntimeError, match="captured"):
                call()
    assert (sc.lengths, sc.free_pages) == before[:2] and sc._held is before[2]
    for n in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert x.tolist() == [float(n + 1)] * 4
    sc.extend([3, 3])
    assert sc.lengths == [5, 6]


def test_a_steps_layers_are_captured():
    L, H, G, d = 2, 2, 2, 64
    sc = cm.ServingCache(cm.QCache.empty(L, H, d, 40), 2, 200)
    twin = cm.ServingCache(cm.QCache.empty(L, H, d, 40), 2, 200)
    k, q = rows(37, H, d, BF16, 1), rows(37, H * G, d, BF16, 2)
    for s in (sc, twin):
        step = s.extend([30, 7])
        for l in range(L):
            s.write(l, k, k, step)
    one, two = sc.extend([1, 1]), twin.extend([1, 1])
    k, q = k[:2].clone(), q[:2].clone()
    outs = [(torch.zeros_like(q), torch.zeros((2, H * G), device="cuda")) for _ in range(L)]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        for l in range(L):
            sc.write(l, k, k, one)
            sc.attend(l, q, one, out=outs[l][0], lse=outs[l][1])
    for n in range(4):
        k.copy_(rows(2, H, d, BF16, 10 + n))
        q.copy_(rows(2, H * G, d, BF16, 20 + n))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for l in range(L):
            twin.write(l, k, k, two)
            got = twin.attend(l, q, two)
            assert torch.equal(got[0], outs[l][0]) and torch.equal(got[1], outs[l][1]), (n, l)
