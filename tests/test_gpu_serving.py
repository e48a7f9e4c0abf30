"""ServingCache on the GPU: steps of places that come, grow and go, the pages' contents
exactly and attention within its bounds (tests/qcache_ref.py), and the example that
serves merged caches."""

import os
import runpy

import numpy as np
import pytest
import torch

import paper_2607_01308_amd as cm
import qcache_ref as ref
import synth
from test_gpu_qcache import check_attention, queries

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
ROOT = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..")


def rows(T, H, d, dtype, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn((T, H, d), generator=g, device="cuda").to(dtype)


def contents(cache):
    return cache.codes.view(torch.uint8).cpu().numpy().copy(), cache.scales.cpu().numpy().copy()


@pytest.mark.parametrize("dtype,d,B,H,G", [(BF16, 128, 16, 2, 4), (F32, 64, 32, 1, 3),
                                           (BF16, 256, 64, 1, 2)])
def test_places_come_grow_and_go(dtype, d, B, H, G):
    """Steps of prompts, questions and single tokens in which places are emptied and filled
    again until the free pages have gone round more than once."""
    rng = np.random.default_rng(d + B)
    L, places, max_len, P = 2, 5, 40 * B, 60
    sc = cm.ServingCache(cm.QCache.empty(L, H, d, P, B), places, max_len)
    assert sc.free_pages == P
    codes, scales = contents(sc.cache)
    given = i = 0
    while given <= 2 * P:
        new = []
        for r in range(places):
            kind = rng.integers(0, 4)
            want = int([0, 1, rng.integers(2, 30), rng.integers(30, 8 * B)][kind])
            new.append(min(want, max_len - sc.lengths[r]))
        while sum(-(-(a + b) // B) for a, b in zip(sc.lengths, new)) > P:
            place = int(np.argmax([a + b for a, b in zip(sc.lengths, new)]))
            sc.release(place)
            new[place] = min(new[place], 3)
        held, free = list(sc.lengths), sc.free_pages
        step = sc.extend(new)
        step.tables.check()
        table = sc.table.cpu().numpy()
        # no page belongs to two places, and the free ones are the others
        used = [int(p) for r in range(places) for p in table[r, :-(-sc.lengths[r] // B)]]
        assert len(set(used)) == len(used) and len(used) + sc.free_pages == P
        given += free - sc.free_pages
        assert sc.lengths == [a + b for a, b in zip(held, new)] == step.tables.lens.tolist()
        slots = [int(table[r, p // B]) * B + p % B
                 for r in range(places) for p in range(held[r], held[r] + new[r])]
        assert step.tables.slots.tolist() == slots
        k, v = (torch.stack([rows(sum(new), H, d, dtype, 100 * i + 10 * w + l) for l in range(L)])
                for w in range(2))
        if i % 2:
            sc.write(0, k, v, step)
        else:
            for l in range(L):
                sc.write(l, k[l], v[l], step)
        for l in range(L):
            for w, x in enumerate((k, v)):
                ref.write(codes[l, w], scales[l, w], x[l].double().cpu().numpy(), slots)
        got = contents(sc.cache)
        assert np.array_equal(got[1], scales)
        assert np.array_equal(got[0], codes)
        q = queries(sum(new), H * G, d, dtype, seed=i)
        for l in range(L):
            got = sc.attend(l, q, step, window=0 if i % 3 else 2 * B + 1)
            check_attention(q, sc.cache.codes, sc.cache.scales, l, table, sc.lengths, new,
                            window=0 if i % 3 else 2 * B + 1, got=got)
        i += 1


def test_merged_cache_into_pages():
    """A render's cache, one buffer, by one write; the same layers apart, by one each."""
    w = synth.custom(lengths=(150, 90, 161), deliveries=(0, 1, 2, 1), dtype="bfloat16", d=128,
                     L=3, H=2)
    res = cm.render_deliveries(synth.make_deliveries(w, synth.make_fragments(w, device="cuda")),
                               w.routing_layer, w.rope_base)
    caches = [cm.ServingCache(cm.QCache.empty(3, 2, 128, 64), 2, 480) for _ in range(2)]
    apart = [(K.clone(), V.clone()) for K, V in res.cache]
    for sc, layers in zip(caches, (res.cache, apart)):
        sc.load(1, layers)
        assert sc.lengths == [0, res.T_out]
    one, other = (contents(sc.cache) for sc in caches)
    assert np.array_equal(one[0], other[0]) and np.array_equal(one[1], other[1])
    # values: each within half a step of 3 bits of its own, or of its page's least step
    sc = caches[0]
    table = sc.table.cpu().numpy()
    for l, (K, V) in enumerate(res.cache):
        for x, code, scale in zip((K, V), ref.E4M3[one[0][l]], one[1][l]):
            x = x[0].double().cpu().numpy()
            for t in range(res.T_out):
                page = int(table[1, t // 16])
                y = code[page, :, t % 16] * scale[page][:, None]
                bound = np.maximum(np.abs(x[:, t]) * 2.0 ** -4, scale[page][:, None] * 2.0 ** -10)
                assert (np.abs(y - x[:, t]) <= bound).all()


def test_two_streams():
    """A cache used on a stream of its own, while another stream's tensors come and go."""
    side = torch.cuda.Stream()
    out = []
    for stream in (None, side):
        if stream is not None:
            side.wait_stream(torch.cuda.current_stream())
        sc = cm.ServingCache(cm.QCache.empty(1, 2, 64, 20), 2, 128)
        k, q = rows(40, 2, 64, BF16, 1), rows(40, 6, 64, BF16, 2)
        if stream is not None:
            side.wait_stream(torch.cuda.current_stream())
        for n in range(3):
            step = sc.extend([30, 10], stream=stream)
            sc.write(0, k, k, step, stream=stream)
            got = sc.attend(0, q, step, stream=stream)
            junk = torch.full((1 << 16,), float("nan"), device="cuda")
            del junk
            if n == 1:
                sc.release(0, stream=stream)
        if stream is not None:
            torch.cuda.current_stream().wait_stream(side)
        out.append([x.clone() for x in got])
    assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1])


def test_refusals_change_nothing():
    sc = cm.ServingCache(cm.QCache.empty(2, 2, 64, 6), 2, 64)
    sc.extend([17, 0])
    state = (list(sc.lengths), sc.free_pages)
    for new in ([1], [1, -1], [1, 2, 3]):
        with pytest.raises(ValueError, match="new must be"):
            sc.extend(new)
    with pytest.raises(ValueError, match="would hold 65"):
        sc.extend([48, 0])
    with pytest.raises(RuntimeError, match="needs 5 pages, 4 are free"):
        sc.extend([40, 33])
    with pytest.raises(ValueError, match="place"):
        sc.release(2)
    K = torch.zeros((1, 2, 5, 64), device="cuda", dtype=BF16)
    with pytest.raises(ValueError, match="2 layers"):
        sc.load(1, [(K, K)])
    with pytest.raises(ValueError, match="K and V must be"):
        sc.load(1, [(K, K), (K, K[:, :, :4])])
    with pytest.raises(TypeError, match="bfloat16 or float32"):
        sc.load(1, [(K.half(), K.half())] * 2)
    with pytest.raises(ValueError, match="place"):
        sc.load(-1, [(K, K)] * 2)
    assert (list(sc.lengths), sc.free_pages) == state
    sc.release(1)                                        # (an empty place: nothing to do)
    sc.load(1, [(K, K)] * 2)
    assert sc.lengths == [17, 5] and sc.free_pages == 3


def test_example_serves_merged_caches():
    """The example at a small size. What 8 bits cost: values are off by 2^-4 of themselves at most,
    0.026 in the mean square, scores by as much times their spread of about 2; the outputs' errors are
    sums with the same weights as the outputs, so 0.06 of their norm, for the worst
    of the heads three times that."""
    main = runpy.run_path(os.path.join(ROOT, "examples", "serve_merged.py"))["main"]
    got = main(agents=3, steps=8, question=9, lengths=(100, 60, 75), L=2, H=2)
    assert got["free_pages"] == got["pages"]
    assert 0 < got["relative_error"] < 0.2
