"""Drafted trees over the 8-bit paged cache on the GPU: masks and positions exactly, attention against
64 bits within what its roundings allow (tests/draft_ref.py)."""

import numpy as np
import pytest
import torch

import draft_ref as ref
import paper_2607_01308_amd as cm
from paper_2607_01308_amd import _cabi as C
from test_gpu_qcache import deal, filled, ints, queries

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def packed(sees, words):
    """Masks of sets of nodes; bits past the words are left out."""
    out = np.zeros((len(sees), words), dtype=np.uint64)
    for i, s in enumerate(sees):
        for j in s:
            if j < 64 * words:
                out[i, j // 64] |= np.uint64(1) << np.uint64(j % 64)
    return torch.tensor(out.view(np.int64), device="cuda")


def forest(counts, branch, seed):
    rng = np.random.default_rng(seed)
    return [ref.random_tree(rng, c, branch) for c in counts]


def seen(trees, lens, window):
    sees, positions = [], []
    for parents, T in zip(trees, lens):
        s, p = ref.tree(parents, T - len(parents), window)
        sees += s
        positions += p
    return sees, positions


def check(q, codes, scales, layer, table, lens, counts, sees, positions, window=0, scale=None, got=None,
          device="cpu", words=None, max_rows=None, rows=None):
    at = [0] + [int(x) for x in np.cumsum(counts)]
    if got is None:
        words = words or max(1, -(-max(counts) // 64))
        tree = cm.QCacheTree(packed(sees, words), ints(positions), window)
        got = cm.qcache_tree_attention(cm.QCache(codes, scales), layer, q, ints(table), ints(lens),
                                       ints(at), tree, max_rows=max_rows or max(max(counts), 1), scale=scale)
    out, lse, A, X = ref.attend(q.double().to(device), codes[layer].view(torch.uint8).to(device),
                                scales[layer].to(device), table, lens, at, sees, positions, window, scale,
                                device)
    bo, bl = ref.attend_bounds(q.dtype, q.shape[2], max(max(lens), 1), out, A, X)
    go, gl = got[0].double().to(device), got[1].double().to(device)
    keep = torch.ones(len(q), dtype=torch.bool, device=device) if rows is None else torch.tensor(rows, device=device)
    go, gl, out, lse, bo, bl = (x[keep] for x in (go, gl, out, lse, bo, bl))
    nan = torch.isnan(out)
    assert torch.equal(torch.isnan(go), nan), "NaN in other places"
    assert torch.equal(torch.isnan(gl), torch.isnan(lse))
    none = lse == -np.inf
    assert torch.equal(gl == -np.inf, none) and bool((go[none] == 0).all())
    fin = torch.isfinite(lse)
    worst = ((go - out).abs() / bo)[~nan]
    assert worst.numel() == 0 or float(worst.max()) <= 1, f"out: {float(worst.max())} of its bound"
    worst = ((gl - lse).abs() / bl)[fin]
    assert worst.numel() == 0 or float(worst.max()) <= 1, f"lse: {float(worst.max())} of its bound"
    return got


# ------------------------------------------------------------------ masks and positions

@pytest.mark.parametrize("window", [0, 1, 3, 70])
@pytest.mark.parametrize("branch", [1, 2, 5])
def test_masks_and_positions(window, branch):
    counts = [1, 64, 0, 65, 7, 130, 1000, 2]
    lens = [1, 64, 5, 300, 1000, 131, 1000, 2]
    trees = forest(counts, branch, seed=branch)
    sees, positions = seen(trees, lens, window)
    rows = [0] + [int(x) for x in np.cumsum(counts)]
    parents = [p for t in trees for p in t]
    got = cm.qcache_tree(ints(parents), ints(rows), ints(lens), rows[-1], 1000, window).check()
    assert got.positions.tolist() == positions
    assert torch.equal(got.masks, packed(sees, 16)) and got.window == window
    alone = cm.qcache_tree(ints(parents), ints(rows), ints(lens), rows[-1], 1000, window, masks=False)
    assert alone.masks is None and alone.positions.tolist() == positions
    if branch == 1:
        chain = cm.qcache_tree(None, ints(rows), ints(lens), rows[-1], 1000, window).check()
        assert torch.equal(chain.masks, got.masks) and chain.positions.tolist() == positions


def test_positions_of_prompts():
    """Chains of any length without masks; with masks they are refused."""
    counts, lens = [5000, 1, 70000], [5000, 9, 70500]
    rows = [0] + [int(x) for x in np.cumsum(counts)]
    got = cm.qcache_tree(None, ints(rows), ints(lens), rows[-1], 70000, masks=False).check()
    assert got.positions.tolist() == [T - c + i for c, T in zip(counts, lens) for i in range(c)]
    got = cm.qcache_tree(None, ints(rows), ints(lens), rows[-1], 1024)
    assert got.info.tolist() == [C.CM_EINVAL, 0, C.CM_EINVAL]
    assert bool((got.masks[:5000] == 0).all()) and got.masks[5000].tolist() == [1] + [0] * 15


def test_trees_that_are_not_as_said():
    counts, lens = [6, 6, 6, 3], [10, 10, 4, 3]
    rows = [0, 6, 12, 18, 21]
    parents = [-1, 0, 1, 3, 9, 2] + [-2, 0, 0, 1, 2 ** 31 - 1, 4] + [-1, 0, 1, 2, 3, 4] + [-1, 0, 0]
    got = cm.qcache_tree(ints(parents), ints(rows), ints(lens), 21, 6)
    assert got.info.tolist() == [C.CM_EINVAL, C.CM_EINVAL, C.CM_EINVAL, 0]
    fixed = [[-1, 0, 1, -1, -1, 2], [-1, 0, 0, 1, -1, 4], [-1, 0, 1, 2, 3, 4], [-1, 0, 0]]
    sees, positions = seen(fixed, lens, 0)
    assert got.positions.tolist() == positions and torch.equal(got.masks, packed(sees, 1))
    with pytest.raises(cm.CmError, match=r"\[0, 1, 2\]"):
        got.check()
    # rows that do not lie in the step: nothing is written for them
    tree = cm.qcache_tree(ints(parents), ints([0, 6, 5, 30, 21]), ints(lens), 21, 6)
    assert tree.info.tolist()[1:] == [C.CM_EINVAL] * 3
    assert tree.positions.tolist()[:6] == positions[:6]


# ------------------------------------------------------------------ attention

SHAPES = [(64, 16, 2, 1), (128, 16, 2, 4), (128, 32, 1, 7), (256, 64, 1, 2), (64, 128, 1, 16),
          (256, 128, 1, 3), (128, 64, 3, 5)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("window", [0, 1, 40, 300])
@pytest.mark.parametrize("d,B,H,G", SHAPES)
def test_ragged_trees(dtype, window, d, B, H, G):
    """Trees of one node to 40 over contexts of none to 1200 tokens, which end anywhere in a page."""
    counts = [1, 2, 16, 17, 0, 40, 3, 33, 8, 5]
    held = [0, 0, 16, 31, 7, 129, 1200, 33, 500, 64]
    lens = [a + b for a, b in zip(held, counts)]
    table, P = deal(lens, B, seed=B)
    codes, scales = filled(P, H, B, d, seed=d + B + G, spread=1.5, layers=2)
    sees, positions = seen(forest(counts, 3, seed=G), lens, window)
    q = queries(sum(counts), H * G, d, dtype, seed=G)
    check(q, codes, scales, 1, table, lens, counts, sees, positions, window)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("most", [1, 3, 4, 8, 9, 16, 100, 300])
def test_any_number_of_nodes(dtype, most):
    """Row tiles of 16, 32 and 64, one and many of them, masks of one word and several."""
    counts = [most, 1, max(1, most // 2), most]
    lens = [most, 700, most + 60, most + 333]
    table, P = deal(lens, 16, seed=most)
    codes, scales = filled(P, 2, 16, 64, seed=most)
    sees, positions = seen(forest(counts, 4, seed=most), lens, 0)
    q = queries(sum(counts), 8, 64, dtype, seed=most)
    check(q, codes, scales, 0, table, lens, counts, sees, positions)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,c,d,B,G,window", [(20011, 16, 128, 16, 4, 0), (70000, 5, 64, 32, 2, 0),
                                              (33333, 9, 256, 16, 8, 9000), (40001, 33, 128, 128, 4, 0)])
def test_long_axis(dtype, T, c, d, B, G, window):
    """One long context: many ranges, joined."""
    table, P = deal([T], B, seed=T)
    codes, scales = filled(P, 1, B, d, seed=T)
    sees, positions = seen(forest([c], 3, seed=T), [T], window)
    q = queries(c, G, d, dtype, seed=T)
    check(q, codes, scales, 0, table, [T], [c], sees, positions, window, device="cuda")


@pytest.mark.parametrize("n", [2, 63, 65, 300, 1024])
def test_many_requests(n):
    rng = np.random.default_rng(n)
    counts = [int(x) for x in rng.integers(0, 7, size=n)]
    lens = [c + int(x) for c, x in zip(counts, rng.integers(0, 90, size=n))]
    table, P = deal(lens, 16, seed=n)
    codes, scales = filled(P, 1, 16, 64, seed=n)
    sees, positions = seen(forest(counts, 2, seed=n), lens, 0)
    q = queries(sum(counts), 3, 64, BF16, seed=n)
    check(q, codes, scales, 0, table, lens, counts, sees, positions)


@pytest.mark.parametrize("longest", [100, 2500])
@pytest.mark.parametrize("n", [3, 40, 63, 64, 90])
def test_ranges_of_many_tiles(n, longest):
    """Eight heads leave 64 workgroups for a head: fewer and more tiles than those, which begin with them
    or anywhere, short ones of one range and long ones of several."""
    rng = np.random.default_rng(n + longest)
    counts = [int(x) for x in rng.integers(0, 4, size=n)]
    lens = [c + int(x) for c, x in zip(counts, rng.integers(0, longest, size=n))]
    lens[0], counts[1] = 8 * longest, 1
    counts[0] = 3
    lens[1] = 1
    table, P = deal(lens, 32, seed=n)
    codes, scales = filled(P, 8, 32, 64, seed=n)
    sees, positions = seen(forest(counts, 2, seed=n), lens, 0)
    q = queries(sum(counts), 8, 64, BF16, seed=n)
    check(q, codes, scales, 0, table, lens, counts, sees, positions, device="cuda")


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_a_chain_is_causal(dtype):
    """A chain of nodes sees what the causal attention's rows see."""
    counts, lens = [5, 1, 30, 12], [5, 90, 400, 77]
    table, P = deal(lens, 16)
    codes, scales = filled(P, 2, 16, 128, seed=1)
    q = queries(sum(counts), 8, 128, dtype, seed=2)
    rows = ints([0] + [int(x) for x in np.cumsum(counts)])
    cache = cm.QCache(codes, scales)
    for window in (0, 9):
        tree = cm.qcache_tree(None, rows, ints(lens), sum(counts), 30, window).check()
        got = cm.qcache_tree_attention(cache, 0, q, ints(table), ints(lens), rows, tree, max_rows=30)
        sees, positions = seen([list(range(-1, c - 1)) for c in counts], lens, window)
        check(q, codes, scales, 0, table, lens, counts, sees, positions, window, got=got)
        want = cm.qcache_attention(cache, 0, q, ints(table), ints(lens), rows=rows, max_rows=30, window=window)
        off = 2.0 ** -6 if dtype == BF16 else 2.0 ** -15
        assert float((got[0].double() - want[0].double()).abs().max()) < off * 4
    # one row a request: rows left out
    one = cm.QCacheTree(torch.ones((4, 1), dtype=torch.int64, device="cuda"), ints([t - 1 for t in lens]))
    got = cm.qcache_tree_attention(cache, 0, q[:4], ints(table), ints(lens), None, one)
    check(q[:4], codes, scales, 0, table, lens, [1] * 4, [{0}] * 4, [t - 1 for t in lens], got=got)


def test_masks_that_are_no_trees():
    """Rows that see nothing of their own, nothing at all, later nodes, or nodes that there are not."""
    counts, held = [5, 5, 70, 3], [0, 40, 100, 17]
    lens = [a + b for a, b in zip(held, counts)]
    rng = np.random.default_rng(5)
    sees = [{int(x) for x in rng.integers(0, c, size=rng.integers(0, c + 1))} for c in counts for _ in range(c)]
    sees[0] = sees[3] = sees[6] = set()
    table, P = deal(lens, 16)
    codes, scales = filled(P, 1, 16, 64, seed=3)
    q = queries(sum(counts), 2, 64, F32, seed=4)
    positions = [h + i for h, c in zip(held, counts) for i in range(c)]
    got = check(q, codes, scales, 0, table, lens, counts, sees, positions)
    assert bool((got[0][0] == 0).all()) and bool((got[1][3] == -np.inf).all())
    # bits of nodes that there are not change nothing
    masks = packed(sees, 3)
    at = [0] + [int(x) for x in np.cumsum(counts)]
    for r, c in enumerate(counts):
        masks[at[r]:at[r + 1], 2] = -1
        if c < 64:
            masks[at[r]:at[r + 1], 0] |= -1 << c
            masks[at[r]:at[r + 1], 1] = -1
        else:
            masks[at[r]:at[r + 1], 1] |= -1 << (c - 64)
    again = cm.qcache_tree_attention(cm.QCache(codes, scales), 0, q, ints(table), ints(lens), ints(at),
                                     cm.QCacheTree(masks, ints(positions)), max_rows=70)
    assert torch.equal(again[0], got[0]) and torch.equal(again[1], got[1])
    # words that there are not hide their nodes
    short = [{j for j in s if j < 64} for s in sees]
    check(q, codes, scales, 0, table, lens, counts, short, positions, words=1)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_what_a_row_does_not_see_has_no_effect(dtype):
    """NaN codes of K and V at nodes and pages that some rows see and others do not."""
    counts, held, B = [9, 20], [37, 100], 16
    lens = [a + b for a, b in zip(held, counts)]
    table, P = deal(lens, B)
    codes, scales = filled(P, 2, B, 128, seed=6)
    raw = codes.view(torch.uint8)
    trees = forest(counts, 2, seed=7)
    sees, positions = seen(trees, lens, 0)
    q = queries(29, 8, 128, dtype, seed=8)

    def put(kv, r, place, code):
        raw[0, kv, int(table[r, place // B]), :, place % B, 5:7] = code

    put(0, 0, held[0] + 4, 0x7F)
    put(1, 0, held[0] + 6, 0xFF)
    put(1, 1, held[1] + 11, 0x7F)
    put(0, 1, held[1] + 3, 0xFF)
    check(q, codes, scales, 0, table, lens, counts, sees, positions)
    # behind the last token and in a page that is not there
    put(1, 0, lens[0], 0x7F)
    put(0, 0, lens[0], 0x7F)
    gone = table.copy()
    gone[1, 2] = -1
    gone[0, 1] = P
    check(q, codes, scales, 0, gone, lens, counts, sees, positions)
    # and a window that begins behind them
    put(1, 1, 20, 0x7F)
    sees, positions = seen(trees, lens, 60)
    check(q, codes, scales, 0, table, lens, counts, sees, positions, 60)


def test_scales_of_any_size():
    """Pages whose scales differ by 2^40, scores of a thousand, a softmax scale that is 0 or negative."""
    counts, lens = [12, 30], [300, 95]
    table, P = deal(lens, 32)
    codes, scales = filled(P, 2, 32, 64, seed=9)
    g = torch.Generator(device="cuda")
    g.manual_seed(10)
    scales = scales * torch.exp2(torch.randint(-20, 20, scales.shape, generator=g, device="cuda").float())
    scales[:, 0] = 2.0 ** -6                              # (K's: scores within what bounds can say)
    sees, positions = seen(forest(counts, 3, seed=1), lens, 0)
    for dtype in (BF16, F32):
        q = queries(42, 4, 64, dtype, seed=11)
        for scale in (None, 0.0, -0.3, 2.0):
            check(q, codes, scales, 0, table, lens, counts, sees, positions, scale=scale)


def test_rows_left_out():
    """max_rows below a request's nodes: the others' rows; rows behind the last request and requests whose
    rows are not in order leave out and lse as they were."""
    counts, lens = [20, 6, 40], [50, 200, 90]
    table, P = deal(lens, 16)
    codes, scales = filled(P, 2, 16, 64, seed=12)
    sees, positions = seen(forest(counts, 3, seed=2), lens, 0)
    q = queries(66, 4, 64, BF16, seed=13)
    cache = cm.QCache(codes, scales)

    def run(rows, max_rows):
        out, lse = torch.full_like(q, 7.0), torch.full((66, 4), 7.0, device="cuda")
        return cm.qcache_tree_attention(cache, 0, q, ints(table), ints(lens), ints(rows),
                                        cm.QCacheTree(packed(sees, 1), ints(positions)), max_rows=max_rows,
                                        out=out, lse=lse)

    inside = [i < 10 for c in counts for i in range(c)]
    got = run([0, 20, 26, 66], 10)
    check(q, codes, scales, 0, table, lens, counts, sees, positions, got=got, rows=inside)
    left = ~torch.tensor(inside, device="cuda")
    assert bool((got[0][left] == 7).all()) and bool((got[1][left] == 7).all())
    for rows in ([0, 20, 26, 26], [0, 20, 26, 67], [0, 20, 26, 5]):
        got = run(rows, 40)
        check(q, codes, scales, 0, table, lens, counts, sees, positions, got=got, rows=[i < 26 for i in range(66)])
        assert bool((got[0][26:] == 7).all()) and bool((got[1][26:] == 7).all())


def test_fewer_tokens_than_nodes():
    """Nodes whose place would lie before the first token have none; lengths below 0 and beyond the
    table's rows count as 0 and as those."""
    counts, lens = [8, 5, 4], [3, 0, 90]
    table, P = deal(lens, 16)
    codes, scales = filled(P, 1, 16, 64, seed=14)
    trees = forest(counts, 2, seed=3)
    sees, positions = seen(trees, lens, 0)
    q = queries(17, 3, 64, F32, seed=15)
    got = check(q, codes, scales, 0, table, lens, counts, sees, positions)
    tree = cm.QCacheTree(packed(sees, 1), ints(positions))
    for other in ([3, -7, 90], [3, 0, 90]):
        again = cm.qcache_tree_attention(cm.QCache(codes, scales), 0, q, ints(table), ints(other),
                                         ints([0, 8, 13, 17]), tree, max_rows=8)
        assert torch.equal(again[0], got[0]) and torch.equal(again[1], got[1])
    width = table.shape[1]
    far = cm.qcache_tree_attention(cm.QCache(codes, scales), 0, q, ints(table), ints([3, 0, 2 ** 31 - 1]),
                                   ints([0, 8, 13, 17]), tree, max_rows=8)
    full = [3, 0, width * 16]
    sees, positions = seen(trees, full, 0)
    check(q, codes, scales, 0, table, full, counts, sees, positions, got=far)


def test_strides_streams_and_repeats():
    """Queries of one projection, outputs in a wider buffer, another stream: the same bits; a call that
    is repeated gives them again."""
    counts, lens = [16, 9, 25], [4000, 700, 60]
    table, P = deal(lens, 16)
    codes, scales = filled(P, 2, 16, 128, seed=16)
    sees, positions = seen(forest(counts, 3, seed=4), lens, 0)
    wide = queries(50, 12, 128, BF16, seed=17)
    q = wide[:, :8]
    got = check(q, codes, scales, 0, table, lens, counts, sees, positions)
    tree = cm.QCacheTree(packed(sees, 1), ints(positions))
    args = cm.QCache(codes, scales), 0, q, ints(table), ints(lens), ints([0, 16, 25, 50]), tree
    out = torch.full((50, 9, 160), 7.0, device="cuda", dtype=BF16)
    again = cm.qcache_tree_attention(*args, max_rows=25, out=out[:, :8, 16:144])
    assert torch.equal(out[:, :8, 16:144], got[0]) and torch.equal(again[1], got[1])
    assert bool((out[:, 8] == 7).all()) and bool((out[..., :16] == 7).all())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        other = cm.qcache_tree_attention(*args, max_rows=25, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(other[0], got[0]) and torch.equal(other[1], got[1])
    # not knowing max_rows changes how rows are grouped, not what they are
    check(q, codes, scales, 0, table, lens, counts, sees, positions, got=cm.qcache_tree_attention(*args))


def test_two_graphs_and_eager_calls():
    """Captured calls of two graphs, replayed in turn with eager calls of other shapes between them."""
    counts, lens = [16, 16], [3000, 2000]
    table, P = deal(lens, 16)
    codes, scales = filled(P, 2, 16, 128, seed=18, layers=2)
    sees, positions = seen(forest(counts, 3, seed=5), lens, 0)
    tree = cm.QCacheTree(packed(sees, 1), ints(positions))
    cache = cm.QCache(codes, scales)
    q = queries(32, 8, 128, BF16, seed=19)
    rows, t, n = ints([0, 16, 32]), ints(table), ints(lens)
    graphs, outs = [], []
    for layer in range(2):
        out = torch.empty_like(q), torch.empty((32, 8), device="cuda")
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            cm.qcache_tree_attention(cache, layer, q, t, n, rows, tree, max_rows=16, out=out[0], lse=out[1])
        graphs.append(graph)
        outs.append(out)
    for step in range(4):
        q.copy_(queries(32, 8, 128, BF16, seed=20 + step))
        torch.cuda.synchronize()
        for layer in (0, 1, 0):
            graphs[layer].replay()
            cm.qcache_attention(cache, layer, q[:2], t, n)
        torch.cuda.synchronize()
        for layer in range(2):
            want = cm.qcache_tree_attention(cache, layer, q, t, n, rows, tree, max_rows=16)
            assert torch.equal(want[0], outs[layer][0]) and torch.equal(want[1], outs[layer][1])


def test_binding_refusals():
    table, P = deal([40], 16)
    codes, scales = filled(P, 2, 16, 64, seed=1)
    cache, q = cm.QCache(codes, scales), queries(4, 4, 64, BF16, seed=1)
    one = torch.ones((4, 1), dtype=torch.int64, device="cuda")
    pos, rows, lens, t = ints([36, 37, 38, 39]), ints([0, 4]), ints([40]), ints(table)
    for tree, kind in ((cm.QCacheTree(None, pos), ValueError), (cm.QCacheTree(one[:3], pos), ValueError),
                       (cm.QCacheTree(one.int(), pos), TypeError), (cm.QCacheTree(one, pos.long()), TypeError),
                       (cm.QCacheTree(one, pos[:2]), ValueError), (cm.QCacheTree(one.cpu(), pos), ValueError),
                       (cm.QCacheTree(one, pos, -1), cm.CmError),
                       (cm.QCacheTree(one.expand(4, 17).contiguous(), pos), cm.CmError)):
        with pytest.raises(kind):
            cm.qcache_tree_attention(cache, 0, q, t, lens, rows, tree)
    with pytest.raises(cm.CmError, match="words"):
        cm.qcache_tree(ints([-1, 0, 1, 2]), rows, lens, 4, 1025)
    with pytest.raises(TypeError):
        cm.qcache_tree(torch.zeros(4, device="cuda"), rows, lens, 4, 4)
    with pytest.raises(ValueError):
        cm.qcache_tree(ints([-1, 0, 1]), rows, lens, 4, 4)
