"""The 8-bit paged cache on the GPU against 64-bit results (tests/qcache_ref.py):
tables and slots exactly, codes and scales exactly, attention within the bounds that
its roundings allow."""

import numpy as np
import pytest
import torch

import paper_2607_01308_amd as cm
import qcache_ref as ref
from paper_2607_01308_amd import _cabi as C

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def filled(P, H, B, d, seed, spread=1.0, layers=1):
    """Random pages as the cache holds them: codes, with scales that are powers of two."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.randn((layers, 2, P, H, B, d), generator=g, device="cuda") * spread
    amax = x.abs().amax((-2, -1))
    s = torch.exp2(torch.ceil(torch.log2(amax / 448)))
    codes = (x / s[..., None, None]).to(torch.float8_e4m3fn)
    return codes, s


def deal(lens, B, spare=3, seed=0, width=None):
    """A block table over shuffled pages: (table, pages of the pool)."""
    rng = np.random.default_rng(seed)
    need = [-(-max(t, 0) // B) for t in lens]
    P = sum(need) + spare
    order = rng.permutation(P)
    width = width or max(need) + 2
    table = np.full((len(lens), width), -1, dtype=np.int32)
    at = 0
    for r, k in enumerate(need):
        table[r, :k] = order[at:at + k]
        at += k
    return table, P


def queries(R, Hq, d, dtype, seed, spread=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + 1)
    return (torch.randn((R, Hq, d), generator=g, device="cuda") * spread).to(dtype)


def check_attention(q, codes, scales, layer, table, lens, counts, window=0, scale=None, got=None,
                    device="cpu"):
    rows = [0] + [int(x) for x in np.cumsum(counts)]
    if got is None:
        cache = cm.QCache(codes, scales)
        got = cm.qcache_attention(cache, layer, q, ints(table), ints(lens), rows=ints(rows),
                                  max_rows=max(max(counts), 1), window=window, scale=scale)
    out, lse, A, X = ref.attend(q.double().to(device), codes[layer].view(torch.uint8).to(device),
                                scales[layer].to(device), table, lens, rows, window, scale, device)
    bo, bl = ref.attend_bounds(q.dtype, q.shape[2], max(max(lens), 1), out, A, X)
    go, gl = got[0].double().to(device), got[1].double().to(device)
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


EDGES = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 65, 127, 128, 129, 200, 511, 513, 1025]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d,B,H,G", [(64, 16, 2, 1), (128, 16, 2, 4), (128, 32, 1, 7), (256, 64, 1, 2),
                                     (64, 128, 1, 16), (256, 128, 1, 3), (128, 64, 3, 5)])
def test_one_row_a_request(dtype, d, B, H, G):
    lens = EDGES
    table, P = deal(lens, B)
    codes, scales = filled(P, H, B, d, seed=d + B + G, layers=2)
    q = queries(len(lens), H * G, d, dtype, seed=G)
    got = check_attention(q, codes, scales, 1, table, lens, [1] * len(lens))
    # rows left out: one row a request
    again = cm.qcache_attention(cm.QCache(codes, scales), 1, q, ints(table), ints(lens))
    assert torch.equal(again[0], got[0]) and torch.equal(again[1], got[1])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d,B,H,G,window", [(128, 16, 2, 4, 0), (64, 32, 1, 3, 0), (256, 16, 1, 2, 40),
                                            (128, 128, 1, 8, 1), (64, 16, 2, 1, 17),
                                            (256, 32, 2, 5, 0), (128, 32, 1, 16, 300)])
def test_ragged_rows(dtype, d, B, H, G, window):
    """Several rows a request: none, one, more than the context holds (rows that stand
    before its first token see nothing), prompts over nothing and over a context."""
    lens = [0, 0, 1, 5, 33, 64, 100, 257, 300, 130, 700]
    counts = [0, 2, 1, 9, 33, 3, 0, 40, 1, 130, 77]
    table, P = deal(lens, B, seed=3)
    codes, scales = filled(P, H, B, d, seed=d + window, spread=1.5)
    q = queries(sum(counts), H * G, d, dtype, seed=window)
    check_attention(q, codes, scales, 0, table, lens, counts, window)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,d,B,G,window", [(20011, 128, 16, 4, 0), (70000, 64, 32, 2, 0),
                                            (33333, 256, 16, 8, 9000), (40001, 128, 128, 16, 0)])
def test_long_axis(dtype, T, d, B, G, window):
    """One long context: split into many ranges, joined."""
    table, P = deal([T], B, seed=T)
    codes, scales = filled(P, 1, B, d, seed=T)
    q = queries(2, G, d, dtype, seed=T)
    check_attention(q, codes, scales, 0, table, [T], [2], window, device="cuda")


@pytest.mark.parametrize("n", [2, 63, 64, 65, 200, 1024])
def test_many_requests(n):
    rng = np.random.default_rng(n)
    lens = [int(x) for x in rng.integers(0, 90, size=n)]
    counts = [int(x) for x in rng.integers(0, 3, size=n)]
    table, P = deal(lens, 16, seed=n)
    codes, scales = filled(P, 1, 16, 64, seed=n)
    q = queries(sum(counts), 2, 64, BF16, seed=n)
    check_attention(q, codes, scales, 0, table, lens, counts)


def test_prompt_of_many_rows():
    lens, counts = [900, 1300], [700, 513]
    table, P = deal(lens, 16, seed=9)
    for dtype, H, G, d in ((BF16, 1, 4, 128), (F32, 1, 2, 128), (BF16, 2, 1, 64), (F32, 1, 1, 256)):
        codes, scales = filled(P, H, 16, d, seed=9)
        q = queries(sum(counts), H * G, d, dtype, seed=9)
        check_attention(q, codes, scales, 0, table, lens, counts, device="cuda")


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("counts", [[1, 1, 1], [6, 20, 37]])
def test_what_is_not_seen_has_no_effect(dtype, counts):
    """NaN codes and scales in every place that a row does not see: rows of the last
    page past the length, later tokens, tokens before the window, pages of nobody."""
    lens, B, H, G, d = [50, 77, 333], 32, 2, 3, 128
    table, P = deal(lens, B, seed=4)
    codes, scales = filled(P, H, B, d, seed=4)
    q = queries(sum(counts), H * G, d, dtype, seed=4)
    clean = check_attention(q, codes, scales, 0, table, lens, counts)
    raw = codes.view(torch.uint8)
    used = set()
    for r, T in enumerate(lens):
        for t in range(T, -(-T // B) * B):
            raw[0, :, int(table[r, t // B]), :, t % B] = 0x7F + 0x80 * (t & 1)
        used |= {int(p) for p in table[r, :-(-T // B)]}
    for p in set(range(P)) - used:
        raw[0, :, p] = 0xFF
        scales[0, :, p] = float("nan")
    got = check_attention(q, codes, scales, 0, table, lens, counts)
    assert torch.equal(got[0], clean[0]) and torch.equal(got[1], clean[1])
    # the last token of each request turns to NaN: only rows that stand on it see it
    for r, T in enumerate(lens):
        raw[0, :, int(table[r, (T - 1) // B]), :, (T - 1) % B, 5] = 0x7F
    got = check_attention(q, codes, scales, 0, table, lens, counts)
    rows = np.cumsum([0] + counts)
    for r, c in enumerate(counts):
        assert torch.equal(got[0][rows[r]:rows[r + 1] - 1], clean[0][rows[r]:rows[r + 1] - 1])
        assert bool(torch.isnan(got[0][rows[r + 1] - 1]).all())
    # V alone: only its column
    raw[0, 0] = codes.view(torch.uint8)[0, 0] & 0x77
    got = check_attention(q, codes, scales, 0, table, lens, counts)
    last = got[0][rows[1] - 1].float()
    assert bool(torch.isnan(last[:, 5]).all()) and not bool(torch.isnan(last[:, 6:]).any())
    # a window hides the early tokens, NaN among them
    codes, scales = filled(P, H, B, d, seed=4)
    raw = codes.view(torch.uint8)
    clean = check_attention(q, codes, scales, 0, table, lens, counts, window=11)
    for r, T in enumerate(lens):
        for t in range(max(0, T - counts[r] - 10)):
            raw[0, :, int(table[r, t // B]), :, t % B] = 0x7F
    got = check_attention(q, codes, scales, 0, table, lens, counts, window=11)
    assert torch.equal(got[0], clean[0])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("counts", [[1, 1, 1, 1], [3, 50, 1, 20]])
def test_absent_pages_hide_their_tokens(dtype, counts):
    lens, B, H, G, d = [100, 200, 64, 90], 16, 1, 2, 64
    table, P = deal(lens, B, seed=6)
    codes, scales = filled(P, H, B, d, seed=6)
    codes.view(torch.uint8)[0, :, 0, :, 3] = 0x7F      # page 0 stands in for absent pages' loads
    for r in range(4):
        table[r][table[r] == 0] = P - 1
    table[0, 2] = -1
    table[1, :5] = -1
    table[1, 7] = P                                    # beyond the pool
    table[2, :] = -1                                   # everything evicted
    q = queries(sum(counts), H * G, d, dtype, seed=6)
    out, lse = check_attention(q, codes, scales, 0, table, lens, counts)
    assert bool((lse[sum(counts[:2]):sum(counts[:3])] == -np.inf).all())


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_any_scales_and_large_scores(dtype):
    """Scales that are no powers of two and lie far apart; scores of hundreds."""
    lens, counts, B, H, G, d = [300, 77], [1, 19], 16, 2, 4, 128
    table, P = deal(lens, B, seed=8)
    codes, scales = filled(P, H, B, d, seed=8)
    rng = np.random.default_rng(8)
    scales *= torch.tensor(np.exp(rng.uniform(-3, 3, size=tuple(scales.shape))), device="cuda").float()
    q = queries(sum(counts), H * G, d, dtype, seed=8, spread=3.0)
    check_attention(q, codes, scales, 0, table, lens, counts)
    check_attention(q, codes, scales, 0, table, lens, counts, scale=-0.7)
    scales[0, 1] *= 2.0 ** -100                        # tiny V
    check_attention(q, codes, scales, 0, table, lens, counts)
    q[0, 0, 3] = float("nan")                          # a query of NaN spoils its own row alone
    out, _ = check_attention(q, codes, scales, 0, table, lens, counts)
    assert bool(torch.isnan(out[0, 0]).all()) and not bool(torch.isnan(out[0, 1:]).any())


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_strides_streams_and_buffers(dtype):
    lens, counts, B, H, G, d = [90, 0, 260], [4, 1, 9], 16, 2, 2, 128
    R, Hq = sum(counts), H * G
    table, P = deal(lens, B, seed=2)
    codes, scales = filled(P, H, B, d, seed=2)
    qkv = queries(R, Hq + 2 * H, d, dtype, seed=2)      # a fused projection
    q = qkv[:, :Hq]
    rows, cache = [0] + [int(x) for x in np.cumsum(counts)], cm.QCache(codes, scales)
    dense = check_attention(q.contiguous(), codes, scales, 0, table, lens, counts)
    wide = torch.full((Hq, R, d + 8), 7.0, dtype=dtype, device="cuda")
    out = wide.transpose(0, 1)[:, :, :d]                # head-major, padded rows
    lse = torch.full((R, Hq), 7.0, device="cuda")
    t, ln, rw = ints(table), ints(lens), ints(rows)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = cm.qcache_attention(cache, 0, q, t, ln, rows=rw, max_rows=9, out=out, lse=lse, stream=side)
    side.synchronize()
    assert got[0] is out and got[1] is lse
    assert torch.equal(out, dense[0]) and torch.equal(lse, dense[1])
    assert bool((wide[:, :, d:] == 7).all())            # nothing past the rows' ends
    with torch.cuda.stream(side):
        again = cm.qcache_attention(cache, 0, q, t, ln, rows=rw)
    side.synchronize()
    assert torch.equal(again[0], dense[0])


def test_lengths_beyond_the_table_and_rows_beyond_the_tensor():
    """Device values that do not fit are cut to what does: no access leaves the buffers."""
    B, H, G, d = 16, 1, 2, 64
    table, P = deal([64, 64], B, spare=0, width=4)
    codes, scales = filled(P, H, B, d, seed=1)
    q = queries(5, G, d, BF16, seed=1)
    cache = cm.QCache(codes, scales)
    got = cm.qcache_attention(cache, 0, q, ints(table), ints([10 ** 9, -5]), rows=ints([0, 2, 5]),
                              max_rows=3)
    check_attention(q, codes, scales, 0, table, [64, 0], [2, 3], got=got)
    out = torch.full((5, G, d), 7.0, dtype=BF16, device="cuda")
    cm.qcache_attention(cache, 0, q, ints(table), ints([64, 64]), rows=ints([3, 9, 2 ** 30]),
                        max_rows=100, out=out)
    cm.qcache_attention(cache, 0, q, ints(table), ints([64, 64]), rows=ints([-4, 1, -7]),
                        max_rows=100, out=out)
    torch.cuda.synchronize()
    assert bool((out[1:3] == 7).all())


def test_offsets_past_32_bits():
    """A pool whose layers lie past 4 GiB and whose K and V slices are longer than that."""
    B, H, G, d = 16, 8, 2, 128
    P = 2 ** 32 // (H * B * d) + 40
    codes = torch.zeros((1, 2, P, H, B, d), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    scales = torch.ones((1, 2, P, H), device="cuda")
    lens, counts = [300, 37], [1, 8]
    need = [-(-t // B) for t in lens]
    table = np.full((2, max(need)), -1, dtype=np.int32)
    table[0, :need[0]] = P - 1 - np.arange(need[0])
    table[1, :need[1]] = P - 1 - need[0] - 7 * np.arange(need[1]) % 20
    rng = np.random.default_rng(0)
    # written there by the operator: K and V of both requests
    tokens = sum(lens)
    k, v = (torch.tensor(rng.standard_normal((tokens, H, d)), dtype=BF16, device="cuda") for _ in "kv")
    slots = [int(table[r, t // B]) * B + t % B for r in range(2) for t in range(lens[r])]
    cache = cm.QCache(codes, scales)
    cm.qcache_write(cache, 0, k, v, torch.tensor(slots, device="cuda"))
    used = np.unique(table[table >= 0])
    part = codes.view(torch.uint8)[0, :, torch.tensor(used.astype(np.int64), device="cuda")].cpu().numpy()
    sub = scales[0, :, torch.tensor(used.astype(np.int64), device="cuda")].cpu().numpy()
    place = {int(p): i for i, p in enumerate(used)}
    small = [place[s // B] * B + s % B for s in slots]
    for w, x in enumerate((k, v)):
        c = np.zeros_like(part[w])
        s = np.ones_like(sub[w])
        ref.write(c, s, x.double().cpu().numpy(), small)
        assert np.array_equal(s, sub[w]) and np.array_equal(c, part[w])
    q = queries(sum(counts), H * G, d, BF16, seed=0)
    got = cm.qcache_attention(cache, 0, q, ints(table), ints(lens), rows=ints([0, 1, 9]), max_rows=8)
    tab = np.array([[place.get(int(p), -1) for p in row] for row in table], dtype=np.int32)
    check_attention(q, torch.tensor(part, device="cuda").view(torch.float8_e4m3fn)[None],
                    torch.tensor(sub, device="cuda")[None], 0, tab, lens, counts, got=got)


def test_same_bits_every_time():
    lens, counts = [5000, 40, 1777], [1, 30, 2]
    table, P = deal(lens, 16, seed=5)
    codes, scales = filled(P, 2, 16, 128, seed=5)
    q = queries(sum(counts), 8, 128, BF16, seed=5)
    first = check_attention(q, codes, scales, 0, table, lens, counts)
    for _ in range(5):
        again = check_attention(q, codes, scales, 0, table, lens, counts, device="cuda")
        assert torch.equal(again[0], first[0]) and torch.equal(again[1], first[1])


# ------------------------------------------------------------------ tables

def run_tables(pages, block, held, new, free, table, tokens=None):
    t = ints(table)
    step = cm.qcache_tables(pages, block, ints(held), ints(new), ints(free), t,
                            sum(new) if tokens is None else tokens)
    return t, step


@pytest.mark.parametrize("block", [16, 32, 64, 128])
@pytest.mark.parametrize("n", [1, 2, 5, 255, 256, 257, 1024])
def test_tables(block, n):
    rng = np.random.default_rng(n + block)
    held = [int(x) for x in rng.integers(0, 200, size=n)]
    new = [int(x) for x in rng.choice([0, 1, 1, 5, 40, 300], size=n)]
    held[0] = 0 if n > 1 else block
    table, P = deal(held, block, spare=0, seed=n, width=64)
    free = [int(x) for x in rng.permutation(sum(-(-w // block) + 1 for w in new) + 3) + P]
    want = ref.tables(P + len(free), block, held, new, free, table)
    t, step = run_tables(P + len(free), block, held, new, free, table)
    step.check()
    assert np.array_equal(t.cpu().numpy(), want[0])
    assert step.slots.tolist() == want[1] and step.rows.tolist() == want[2]
    assert step.lens.tolist() == want[3]
    assert step.info.tolist() == [0, sum(new), want[4], max(want[3])]


def test_tables_nothing_new_and_long_prompts():
    table, P = deal([5, 16], 16, width=4)
    t, step = run_tables(P, 16, [5, 16], [0, 0], [], table)
    assert step.check().slots.numel() == 0 and step.rows.tolist() == [0, 0, 0]
    assert np.array_equal(t.cpu().numpy(), table)
    held, new = [3, 0, 77], [30000, 1, 12345]
    table, P = deal(held, 32, seed=1, width=2000)
    free = list(range(P, P + 1400))
    want = ref.tables(P + 1400, 32, held, new, free, table)
    t, step = run_tables(P + 1400, 32, held, new, free, table)
    assert np.array_equal(t.cpu().numpy(), want[0]) and step.slots.tolist() == want[1]


def test_tables_pages_outside_the_pool_get_no_slot():
    table = np.array([[-1, 7, 7, 7]], dtype=np.int32)
    t, step = run_tables(6, 16, [10], [30], [5, 99], table)
    step.check()
    want = ref.tables(6, 16, [10], [30], [5, 99], table)
    assert step.slots.tolist() == want[1] and step.slots.tolist()[:6] == [-1] * 6
    assert t.tolist() == want[0].tolist() == [[-1, 5, 99, 7]]


@pytest.mark.parametrize("held,new,free,tokens", [
    ([3, -1], [1, 1], [4, 5], 2),              # a negative length
    ([3, 1], [1, -1], [4, 5], 2),
    ([16, 16], [1, 1], [4], 2),                # the free list is short
    ([3, 1], [1, 1], [4, 5], 3),               # other than the tokens given
    ([3, 60], [1, 5], [4, 5], 6),              # a table row is short
    ([2 ** 31 - 1, 1], [2 ** 31 - 1, 1], [4], 2),
])
def test_tables_refused_steps(held, new, free, tokens):
    table = np.array([[0, -1, -1, -1], [1, -1, -1, -1]], dtype=np.int32)
    t, step = run_tables(9, 16, held, new, free, table, tokens)
    with pytest.raises(cm.CmError) as e:
        step.check()
    assert e.value.status == C.CM_EINVAL
    assert np.array_equal(t.cpu().numpy(), table)
    assert step.slots.tolist() == [-1] * tokens and step.rows.tolist() == [0, 0, 0]
    assert step.lens.tolist() == [max(h, 0) for h in held]


# ------------------------------------------------------------------ write

@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d,B,H,L", [(64, 16, 2, 1), (128, 16, 3, 2), (64, 32, 1, 1), (128, 32, 2, 1),
                                     (64, 128, 1, 1), (256, 32, 1, 1), (128, 128, 1, 2),
                                     (256, 128, 2, 1), (256, 16, 1, 3)])
def test_write(dtype, d, B, H, L):
    """Rows that begin pages, continue them (with and without a greater scale), skip
    tokens, end inside pages; two writes one after another."""
    held = [0, 5, B, B + 1, 3, 2 * B - 1, 0, 7]
    new = [1, 3, 2 * B + 1, B, 1, 2, 0, 1]
    spread = [1.0, 30.0, 1.0, 0.01, 1.0, 1.0, 1.0, 1e4]
    rng = np.random.default_rng(d + B + H)
    total = [h + w for h, w in zip(held, new)]
    table, P = deal(total, B, seed=d)
    codes, scales = filled(P, H, B, d, seed=B, layers=L + 1)
    cache = cm.QCache(codes, scales)
    slots, amp = [], []
    for r in range(len(held)):
        for p in range(held[r], total[r]):
            slots.append(int(table[r, p // B]) * B + p % B)
            amp.append(spread[r])
    slots[len(slots) // 2] = -1
    slots.append(P * B)                       # past the pool
    amp.append(1.0)
    T = len(slots)
    x = rng.standard_normal((2, L, T, H, d)) * np.array(amp)[None, None, :, None, None]
    x[:, :, 0] = 0.0                          # a page that begins with zeros
    x[0, 0, 2, 0, 1] = np.inf
    x[1, 0, 3, 0, 2] = np.nan
    x[0, 0, 4, 0, :] = [np.inf, -np.inf] * (d // 2)
    kv = torch.tensor(x, dtype=dtype, device="cuda")
    want_c, want_s = codes.view(torch.uint8).cpu().numpy().copy(), scales.cpu().numpy().copy()
    for _ in range(2):
        for w in range(2):
            for l in range(L):
                ref.write(want_c[l + 1, w], want_s[l + 1, w], kv[w, l].double().cpu().numpy(), slots)
        cm.qcache_write(cache, 1, kv[0], kv[1], torch.tensor(slots, device="cuda"))
        got_c, got_s = codes.view(torch.uint8).cpu().numpy(), scales.cpu().numpy()
        assert np.array_equal(got_s, want_s)
        # the sign of a NaN does not matter
        same = (got_c == want_c) | (((got_c & 0x7F) == 0x7F) & ((want_c & 0x7F) == 0x7F))
        assert same.all(), np.argwhere(~same)[:5]


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_write_scales_at_their_edges(dtype):
    """Greatest values around 448 * 2^e, the least and the greatest of the type, subnormals."""
    tops = [448.0, 449.0, 450.0, 447.0, 0.0, 2.0 ** -126, 2.0 ** -130, 3.0e38, 2.0 ** -112,
            448 * 2.0 ** -120, 450 * 2.0 ** -120, 1.0, 1.75, 1.7578125, 256.0]
    d, B, H = 64, 16, 1
    codes, scales = filled(len(tops), H, B, d, seed=0)
    x = np.zeros((len(tops), H, d))
    for i, t in enumerate(tops):
        x[i, 0] = t * np.linspace(-1, 1, d)
    k = torch.tensor(x, dtype=dtype, device="cuda")
    slots = [B * i for i in range(len(tops))]
    want_c, want_s = codes.view(torch.uint8).cpu().numpy().copy(), scales.cpu().numpy().copy()
    for w in range(2):
        ref.write(want_c[0, w], want_s[0, w], k.double().cpu().numpy(), slots)
    cm.qcache_write(cm.QCache(codes, scales), 0, k, k, torch.tensor(slots, device="cuda"))
    assert np.array_equal(scales.cpu().numpy(), want_s)
    assert np.array_equal(codes.view(torch.uint8).cpu().numpy(), want_c)


def test_write_strides_streams_and_many_tokens():
    """Head-major rows of a merged cache, token-major rows of a fused projection, on a
    stream of their own, enough tokens for each way of dealing out the work."""
    L, H, d, B, T = 2, 4, 128, 16, 3001
    P = -(-T // B)
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    merged = torch.randn((L, 2, 1, H, T, d), generator=g, device="cuda").to(BF16)
    slots = torch.arange(T, device="cuda")
    want_c = np.zeros((L, 2, P, H, B, d), dtype=np.uint8)
    want_s = np.zeros((L, 2, P, H), dtype=np.float32)
    for l in range(L):
        for w in range(2):
            ref.write(want_c[l, w], want_s[l, w],
                      merged[l, w, 0].transpose(0, 1).double().cpu().numpy(), slots.tolist())
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for stream in (None, side):
        cache = cm.QCache.empty(L, H, d, P, B)
        torch.cuda.synchronize()
        cm.qcache_write(cache, 0, merged[:, 0, 0].transpose(1, 2), merged[:, 1, 0].transpose(1, 2),
                        slots, stream=stream)
        torch.cuda.synchronize()
        assert np.array_equal(cache.codes.view(torch.uint8).cpu().numpy(), want_c)
        assert np.array_equal(cache.scales.cpu().numpy(), want_s)
    qkv = torch.empty((T, 3 * H, d), dtype=BF16, device="cuda")
    qkv[:, H:2 * H], qkv[:, 2 * H:] = merged[1, 0, 0].transpose(0, 1), merged[1, 1, 0].transpose(0, 1)
    cache = cm.QCache.empty(1, H, d, P, B)
    for a, b in ((0, 1), (1, 700), (700, T)):           # in parts: the same pages in the end
        cm.qcache_write(cache, 0, qkv[a:b, H:2 * H], qkv[a:b, 2 * H:], slots[a:b])
    c2, s2 = np.zeros((2, P, H, B, d), np.uint8), np.zeros((2, P, H), np.float32)
    for w in range(2):
        x = merged[1, w, 0].transpose(0, 1).double().cpu().numpy()
        for a, b in ((0, 1), (1, 700), (700, T)):
            ref.write(c2[w], s2[w], x[a:b], slots[a:b].tolist())
    assert np.array_equal(cache.codes.view(torch.uint8).cpu().numpy()[0], c2)
    assert np.array_equal(cache.scales.cpu().numpy()[0], s2)


def test_step_by_step_equals_its_parts_and_a_graph():
    """A decoding loop (tables, write, attention, the lengths kept on the device) captured
    once and replayed, with eager work between the replays, against the same loop run
    eagerly."""
    n, H, G, d, B, L = 3, 2, 2, 64, 16, 1
    steps = 20
    P, width = 24, 8
    rng = np.random.default_rng(0)
    xs = torch.tensor(rng.standard_normal((steps, 3, n, H, d)), dtype=BF16, device="cuda")
    qs = torch.tensor(rng.standard_normal((steps, n, H * G, d)), dtype=BF16, device="cuda")
    free0 = ints(rng.permutation(P))
    one = ints([1] * n)

    def state():
        s = dict(cache=cm.QCache.empty(L, H, d, P, B), held=ints([0, 5, 15]),
                 free=free0.clone(), table=ints(np.full((n, width), -1)),
                 k=torch.zeros((n, H, d), dtype=BF16, device="cuda"),
                 q=torch.zeros((n, H * G, d), dtype=BF16, device="cuda"))
        s["table"][1, 0], s["table"][2, 0] = P - 1, P - 2
        s["free"] = ints([p for p in free0.tolist() if p < P - 2])
        s["out"] = torch.zeros((n, H * G, d), dtype=BF16, device="cuda")
        s["lse"] = torch.zeros((n, H * G), device="cuda")
        s["info"] = torch.zeros(4, dtype=torch.int64, device="cuda")
        return s

    def body(s):
        step = cm.qcache_tables(P, B, s["held"], one, s["free"], s["table"], n)
        cm.qcache_write(s["cache"], 0, s["k"], s["k"], step.slots)
        cm.qcache_attention(s["cache"], 0, s["q"], s["table"], step.lens, rows=step.rows,
                            max_rows=1, out=s["out"], lse=s["lse"])
        s["info"].copy_(step.info)
        s["held"].copy_(step.lens)
        # the taken pages leave the front of the list
        place = (torch.arange(s["free"].numel(), device="cuda") + step.info[2]).clamp(
            max=s["free"].numel() - 1)
        s["free"].copy_(s["free"][place])

    eager, results = state(), []
    for t in range(steps):
        eager["k"].copy_(xs[t, 0])
        eager["q"].copy_(qs[t])
        body(eager)
        assert int(eager["info"][0]) == 0
        results.append((eager["out"].clone(), eager["lse"].clone()))
    side = torch.cuda.Stream()
    warm = state()
    with torch.cuda.stream(side):
        body(warm)
    side.synchronize()
    s = state()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        body(s)
    for t in range(steps):
        s["k"].copy_(xs[t, 0])
        s["q"].copy_(qs[t])
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(s["out"], results[t][0]), f"replay {t}"
        assert torch.equal(s["lse"], results[t][1]), f"replay {t}"
    assert torch.equal(s["cache"].codes.view(torch.uint8), eager["cache"].codes.view(torch.uint8))
