"""The scratch of the 8-bit cache's attention: a captured call's own, whatever the stream's
becomes afterwards, and steps whose rows lie over one another, which must stay inside it."""

import ctypes

import numpy as np
import pytest
import torch

import paper_2607_01308_amd as cm
from paper_2607_01308_amd import _cabi as C
from test_gpu_qcache import BF16, check_attention, deal, filled, ints, queries

pytestmark = pytest.mark.gpu


def test_a_captured_call_keeps_its_scratch():
    """Captured with no call before it on that stream; between the replays the stream's eager calls
    need more scratch than there was, release it and fill what was free."""
    B, H, G, d = 16, 2, 4, 128
    cm.release_qcache_workspace()
    lens, counts = [3000, 700, 41], [1, 9, 40]
    table, P = deal(lens, B)
    codes, scales = filled(P, H, B, d, seed=5)
    cache = cm.QCache(codes, scales)
    rows = ints([0] + list(np.cumsum(counts)))
    q = queries(sum(counts), H * G, d, BF16, seed=5)
    t, ln = ints(table), ints(lens)
    side = torch.cuda.Stream()
    out, lse = torch.zeros_like(q), torch.zeros((q.shape[0], H * G), device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        cm.qcache_attention(cache, 0, q, t, ln, rows=rows, max_rows=max(counts), out=out, lse=lse)
    many = queries(3000, H * G, d, BF16, seed=6)
    for turn in range(4):
        q.copy_(queries(sum(counts), H * G, d, BF16, seed=7 + turn))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        check_attention(q, codes, scales, 0, table, lens, counts, got=(out, lse))
        with torch.cuda.stream(side):                     # eager work on the captured stream
            got = cm.qcache_attention(cache, 0, q, t, ln, rows=rows, max_rows=max(counts))
            assert torch.equal(got[0], out) and torch.equal(got[1], lse)
            cm.qcache_attention(cache, 0, many, t, ints([3000, 0, 0]), rows=ints([0, 3000, 3000, 3000]),
                                max_rows=3000)
        side.synchronize()
        cm.release_qcache_workspace()
        junk = [torch.full((1 << 22,), 0x5A, dtype=torch.uint8, device="cuda") for _ in range(8)]
        del junk


@pytest.mark.parametrize("n,each", [(6, 40), (300, 200), (1000, 64)])
def test_rows_over_one_another_stay_inside_the_workspace(n, each):
    """Every other request is given the same rows: more row tiles than the workspace has places
    for. Nothing is written outside it and the next step is right."""
    B, H, G, d = 16, 1, 4, 64
    lens = [300] * n
    table, P = deal([300], B)
    table = np.repeat(table, n, 0)
    codes, scales = filled(P, H, B, d, seed=n)
    cache = cm.QCache(codes, scales)
    q = queries(each, H * G, d, BF16, seed=n)
    t, ln = ints(table), ints(lens)
    out, lse = torch.zeros_like(q), torch.zeros((each, H * G), device="cuda")

    def call(rows, ws, need):
        step = C.CmQattention(n, H * G, C.CM_BF16, 0, each, each, d ** -0.5, q.data_ptr(), q.stride(0),
                              q.stride(1), out.data_ptr(), out.stride(0), out.stride(1), lse.data_ptr(),
                              rows.data_ptr(), ln.data_ptr(), t.data_ptr(), t.shape[1])
        f = C.lib().cm_qcache_attention_size
        C.check(f(ctypes.byref(cache.struct), ctypes.byref(step), ctypes.byref(need)), "size")
        if ws is not None:
            C.check(C.lib().cm_qcache_attention(ctypes.byref(cache.struct), 0, ctypes.byref(step),
                                                ws.data_ptr(), need.value,
                                                torch.cuda.current_stream().cuda_stream), "attention")

    need = ctypes.c_size_t(0)
    over = ints([0 if r % 2 == 0 else each for r in range(n + 1)])
    call(over, None, need)
    guard = 1 << 20
    ws = torch.full((need.value + guard,), 0xC3, dtype=torch.uint8, device="cuda")
    ws[:C.CM_QCACHE_COUNTER_BYTES].zero_()
    call(over, ws, need)
    torch.cuda.synchronize()
    assert bool((ws[need.value:] == 0xC3).all())
    assert bool((ws[:C.CM_QCACHE_COUNTER_BYTES] == 0).all())
    # the rows dealt to one request alone
    rows = ints([0] + [each] * n)
    call(rows, ws, need)
    counts = [each] + [0] * (n - 1)
    check_attention(q, codes, scales, 0, table, lens, counts, got=(out, lse))
    assert bool((ws[need.value:] == 0xC3).all())
