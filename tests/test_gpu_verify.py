"""Verification of drafted tokens (verify_drafts) on the GPU: accepted nodes and sampled tokens are
those of a walk in 64 bits (tests/draft_ref.py)."""

import ctypes

import numpy as np
import pytest
import torch

import draft_ref as ref
import paper_2607_01308_amd as cm
from paper_2607_01308_amd import _cabi as C

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def case(counts, V, branch, dtype, sampled, seed, spread=2.0):
    """Trees of the counts with drafts from their parents' draft probabilities, which are the target's
    disturbed."""
    rng = np.random.default_rng(seed)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    parents = [p for c in counts for p in ref.random_tree(rng, c, branch)]
    rows = [0] + [int(x) for x in np.cumsum(counts)]
    T = rows[-1]
    x = spread * torch.randn((T, V), generator=g, device="cuda")
    p = torch.softmax(x, 1).to(dtype)
    q = torch.softmax(x + torch.randn((T, V), generator=g, device="cuda"), 1).to(dtype)
    of = [a + max(parents[i], 0) for a, b in zip(rows[:-1], rows[1:]) for i in range(a, b)]
    drafts = torch.multinomial(q.float(), 1, generator=g)[:, 0]
    drafts = torch.stack([torch.multinomial(q[i].float(), 1, generator=g)[0] for i in of]) if T else drafts
    u, s = rng.random(T).astype(np.float32), rng.random(len(counts)).astype(np.float32)
    return dict(probs=p, drafts=drafts, parents=parents, rows=rows, accept=u, sample=s,
                draft_probs=q if sampled else None)


def check(c):
    i32 = dict(dtype=torch.int32, device="cuda")
    got = cm.verify_drafts(c["probs"], c["drafts"], torch.tensor(c["parents"], **i32),
                           torch.tensor(c["rows"], **i32), torch.tensor(c["accept"], device="cuda"),
                           torch.tensor(c["sample"], device="cuda"), draft_probs=c["draft_probs"])
    host = {k: None if c[k] is None else c[k].float().cpu().numpy() for k in ("probs", "draft_probs")}
    path, counts, tokens = ref.verify(host["probs"], c["drafts"].tolist(), c["parents"], c["rows"],
                                      c["accept"], c["sample"], host["draft_probs"])
    assert got.counts.tolist() == counts
    assert got.path.tolist() == path
    assert got.tokens.tolist() == tokens
    return path, counts, tokens


@pytest.mark.parametrize("sampled", [True, False])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("V", [1, 2, 7, 8, 9, 100, 511, 513, 4097, 8191, 8200, 65537])
def test_vocabularies(V, dtype, sampled):
    """Trees of one node to 23 over vocabularies whose rows begin at any element and end anywhere
    in a load."""
    got = check(case([1, 5, 0, 23, 2, 8], V, 3, dtype, sampled, seed=V))
    assert got[1][2] == 0 and got[2][2] == -1


@pytest.mark.parametrize("sampled", [True, False])
@pytest.mark.parametrize("branch", [1, 2, 6, 70])
@pytest.mark.parametrize("counts", [[64, 65, 130], [1024], [3] * 90])
def test_trees(counts, branch, sampled):
    path, got, _ = check(case(counts, 300, branch, F32, sampled, seed=branch + len(counts), spread=1.0))
    if sampled and branch < 70 and len(counts) == 90:    # (p alone is 1 in 300: few are accepted)
        assert {1, 2} <= set(got)                        # some drafts accepted, some not


@pytest.mark.parametrize("sampled", [True, False])
def test_random_numbers_at_their_ends(sampled):
    """u = 0 accepts what has any probability; s = 0 and the greatest number below 1 give the first and the
    last token that may be sampled."""
    below = np.float32(1) - np.float32(2.0 ** -24)
    for u, s in ((0.0, 0.0), (0.0, below), (below, 0.0), (below, below)):
        c = case([6, 1, 9], 777, 2, F32, sampled, seed=5)
        c["probs"][:, :3] = 0
        c["probs"][:, -2:] = 0
        c["accept"][:], c["sample"][:] = u, s
        _, counts, tokens = check(c)
        if u == 0:
            assert counts[0] > 1
        assert all(3 <= t < 775 for t in tokens)


def test_equal_probabilities_accept_every_draft():
    """p = q: u q < p for every u below 1."""
    c = case([12, 30], 1000, 1, F32, True, seed=8)
    c["draft_probs"] = c["probs"].clone()
    _, counts, _ = check(c)
    assert counts == [12, 30]


def test_certain_targets():
    """Rows with one token: a draft of that token is accepted, another never; the token sampled is
    it."""
    for sampled in (True, False):
        c = case([8, 8, 8], 500, 3, F32, sampled, seed=9)
        c["probs"].zero_()
        c["probs"][:, 123] = 1
        c["drafts"][:] = 77
        c["drafts"][9:12] = 123
        _, counts, tokens = check(c)
        assert counts[0] == counts[2] == 1 and counts[1] > 1 and tokens == [123] * 3


def test_what_is_no_probability():
    """Negative, infinite and NaN entries count as none, rows without any give -1, tokens outside the
    vocabulary are never accepted, a token drafted twice is out after the first rejection."""
    for sampled in (True, False):
        c = case([9, 9, 9, 9], 130, 3, F32, sampled, seed=10)
        p = c["probs"]
        p[:, 5] = float("nan")
        p[:, 6] = float("inf")
        p[:, 7] = -1.0
        if sampled:
            c["draft_probs"][:, 8] = float("nan")
            c["draft_probs"][:, 9] = -0.5
        p[18:27] = 0
        p[20, 4] = float("nan")
        c["drafts"][1], c["drafts"][2] = -1, 130
        c["drafts"][28:] = int(c["drafts"][28])
        c["accept"][:] = 0.5
        _, counts, tokens = check(c)
        assert tokens[2] == -1 and counts[2] == 1


def test_nothing_left_samples_the_row_itself():
    """p below q everywhere and every draft rejected: what is left of p is nothing."""
    c = case([2], 64, 1, F32, True, seed=11)
    c["draft_probs"][:] = 1.0
    c["accept"][:] = 0.999
    _, counts, _ = check(c)
    assert counts == [1]


def test_rows_of_wider_buffers_and_rows_of_nobody():
    c = case([4, 7], 99, 2, BF16, True, seed=12)
    wide = torch.full((11, 250), float("nan"), device="cuda", dtype=BF16)
    wide[:, 3:102], wide[:, 110:209] = c["probs"], c["draft_probs"]
    c["probs"], c["draft_probs"] = wide[:, 3:102], wide[:, 110:209]
    check(c)
    # the same with rows behind the last request: their path stays as it is, which nobody sees here,
    # and none of their numbers is read
    i32 = dict(dtype=torch.int32, device="cuda")
    got = cm.verify_drafts(c["probs"], c["drafts"], torch.tensor(c["parents"], **i32),
                           torch.tensor([0, 4, 4], **i32), torch.tensor(c["accept"], device="cuda"),
                           torch.tensor(c["sample"], device="cuda"), draft_probs=c["draft_probs"])
    assert got.counts.tolist()[1] == 0 and got.tokens.tolist()[1] == -1


def test_rows_that_are_not_as_said():
    """Rows out of order or outside the step, parents that are no earlier node, too many nodes: no
    request reads or writes beyond its own."""
    c = case([6, 6, 6], 50, 2, F32, False, seed=13)
    i32 = dict(dtype=torch.int32, device="cuda")
    args = (torch.tensor(c["accept"], device="cuda"), torch.tensor(c["sample"], device="cuda"))
    for rows in ([0, -3, 12, 18], [0, 6, 5, 18], [0, 6, 12, 99], [-5, 6, 12, 18]):
        got = cm.verify_drafts(c["probs"], c["drafts"], torch.tensor(c["parents"], **i32),
                               torch.tensor(rows, **i32), *args)
        for r in range(3):
            bad = not 0 <= rows[r] <= rows[r + 1] <= 18
            if bad:
                assert got.counts[r] == 0 and got.tokens[r] == -1
    parents = torch.tensor(c["parents"], **i32)
    parents[1:] = torch.tensor([1, 2, 9, -7, 2 ** 31 - 1] + [5] * 12, **i32)
    got = cm.verify_drafts(c["probs"], c["drafts"], parents, torch.tensor([0, 6, 12, 18], **i32), *args)
    assert got.counts.tolist() == [1, 1, 1]
    T = 1025
    probs = torch.ones((T, 4), device="cuda")
    got = cm.verify_drafts(probs, torch.zeros(T, dtype=torch.int64, device="cuda"),
                           torch.arange(-1, T - 1, **i32), torch.tensor([0, T], **i32),
                           torch.zeros(T, device="cuda"), torch.zeros(1, device="cuda"))
    assert got.counts.tolist() == [0] and got.tokens.tolist() == [-1] and bool((got.path == -1).all())


def test_samples_follow_the_target():
    """Whatever the drafts are sampled from, the first token after node 0 is distributed as the target's
    row: 4096 requests of one drafted child, shares within 5 standard deviations."""
    n, V = 1024, 5
    total = torch.zeros(V)
    p = torch.tensor([0.5, 0.25, 0.125, 0.0625, 0.0625])
    q = torch.tensor([0.1, 0.2, 0.3, 0.2, 0.2])
    i32 = dict(dtype=torch.int32, device="cuda")
    for seed in range(4):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        drafts = torch.multinomial(q.cuda().expand(2 * n, V).contiguous(), 1, generator=g)[:, 0]
        got = cm.verify_drafts(p.cuda().expand(2 * n, V).contiguous(), drafts,
                               torch.tensor([-1, 0] * n, **i32), torch.arange(0, 2 * n + 1, 2, **i32),
                               torch.rand(2 * n, generator=g, device="cuda"),
                               torch.rand(n, generator=g, device="cuda"),
                               draft_probs=q.cuda().expand(2 * n, V).contiguous())
        first = torch.where(got.counts == 2, drafts[1::2], got.tokens)
        total += torch.bincount(first.cpu(), minlength=V)
    share = total / (4 * n)
    assert bool(((share - p).abs() <= 5 * (p * (1 - p) / (4 * n)).sqrt()).all())


def test_another_stream_and_a_graph():
    c = case([5, 9, 3], 3001, 2, BF16, True, seed=14)
    i32 = dict(dtype=torch.int32, device="cuda")
    tensors = [c["probs"], c["drafts"], torch.tensor(c["parents"], **i32), torch.tensor(c["rows"], **i32),
               torch.tensor(c["accept"], device="cuda"), torch.tensor(c["sample"], device="cuda")]
    want = cm.verify_drafts(*tensors, draft_probs=c["draft_probs"])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = cm.verify_drafts(*tensors, draft_probs=c["draft_probs"], stream=side)
    torch.cuda.current_stream().wait_stream(side)
    for a, b in ((got.path, want.path), (got.counts, want.counts), (got.tokens, want.tokens)):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        got = cm.verify_drafts(*tensors, draft_probs=c["draft_probs"])
    for n in range(3):
        tensors[4].copy_(torch.rand(17, device="cuda"))
        tensors[5].copy_(torch.rand(3, device="cuda"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = cm.verify_drafts(*tensors, draft_probs=c["draft_probs"])
        for a, b in ((got.path, want.path), (got.counts, want.counts), (got.tokens, want.tokens)):
            assert torch.equal(a, b)


@pytest.mark.parametrize("sampled", [True, False])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,V", [(1, 200_003), (3, 100_001), (40, 33_000), (1, 600_000)])
def test_shared_and_alone(n, V, dtype, sampled):
    """Requests that several workgroups share have the results that one workgroup gives them, call after
    call, and leave the workspace zero."""
    c = case([int(x) for x in np.random.default_rng(V).integers(4, 12, size=n)], V, 3, dtype, sampled, seed=V)
    if not sampled:                                      # (drafts that are likely: some are accepted)
        c["probs"][:, :4] *= V / 8
    check(c)
    i32 = dict(dtype=torch.int32, device="cuda")
    parents, rows = torch.tensor(c["parents"], **i32), torch.tensor(c["rows"], **i32)
    u, s = torch.tensor(c["accept"], device="cuda"), torch.tensor(c["sample"], device="cuda")
    many = [cm.verify_drafts(c["probs"], c["drafts"], parents, rows, u, s, draft_probs=c["draft_probs"])
            for _ in range(8)]
    T, q = len(c["parents"]), c["draft_probs"]
    path, counts, tokens = torch.empty(T, **i32), torch.empty(n, **i32), torch.empty(n, dtype=torch.int64, device="cuda")
    step = C.CmDrafts(n, C.CM_BF16 if dtype is BF16 else C.CM_F32, T, V, c["probs"].data_ptr(), V,
                      None if q is None else q.data_ptr(), V, c["drafts"].data_ptr(), parents.data_ptr(),
                      rows.data_ptr(), u.data_ptr(), s.data_ptr(), path.data_ptr(), counts.data_ptr(),
                      tokens.data_ptr())
    stream = torch.cuda.current_stream().cuda_stream
    assert C.lib().cm_verify_drafts(ctypes.byref(step), stream) == C.CM_OK
    for got in many:
        assert torch.equal(got.path, path) and torch.equal(got.counts, counts) and torch.equal(got.tokens, tokens)
    need = ctypes.c_size_t(0)
    assert C.lib().cm_verify_drafts_size(ctypes.byref(step), ctypes.byref(need)) == C.CM_OK and need.value > 0
    ws = torch.zeros(need.value, dtype=torch.uint8, device="cuda")
    step.workspace, step.workspace_bytes = ws.data_ptr(), need.value - 1
    assert C.lib().cm_verify_drafts(ctypes.byref(step), stream) == C.CM_EWORKSPACE
    step.workspace_bytes = need.value
    for x in (path, counts, tokens):
        x.fill_(-7)
    assert C.lib().cm_verify_drafts(ctypes.byref(step), stream) == C.CM_OK
    assert torch.equal(tokens, many[0].tokens) and torch.equal(path, many[0].path)
    assert not bool(ws.any())


def test_shared_on_two_streams_and_in_a_graph():
    """Calls on two streams at once, and a graph replayed beside them, have workspaces of their own."""
    cases = [case([9, 5], 150_001, 3, BF16, True, seed=s) for s in (21, 22)]
    i32 = dict(dtype=torch.int32, device="cuda")
    args = [(c["probs"], c["drafts"], torch.tensor(c["parents"], **i32), torch.tensor(c["rows"], **i32),
             torch.tensor(c["accept"], device="cuda"), torch.tensor(c["sample"], device="cuda"), c["draft_probs"])
            for c in cases]
    want = [cm.verify_drafts(*a) for a in args]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        inside = cm.verify_drafts(*args[0])
    streams = [torch.cuda.Stream() for _ in args]
    for _ in range(6):
        inside.tokens.fill_(-5)
        graph.replay()
        got = [cm.verify_drafts(*a, stream=s) for a, s in zip(args, streams)]
        torch.cuda.synchronize()
        for g, w in zip(got + [inside], want + [want[0]]):
            assert torch.equal(g.tokens, w.tokens) and torch.equal(g.path, w.path) and torch.equal(g.counts, w.counts)
