"""The operators that serve a merged cache from 8-bit pages, as cases that can be
prepared, run in plain torch operations or through the library, computed in 64 bits
and timed.

The cache is paged, for each layer and K/V: codes [L, 2, P, H, B, d] in float8_e4m3fn
and scales [L, 2, P, H] in float32, one scale for the B tokens of a page and a head; a
stored value is code * scale. Three operators work on it:

  tables  block tables and slot maps from the requests' lengths: request r holds
          held[r] tokens and brings new[r]; its table row keeps the pages it has and
          takes the next ones of the free list (in the order of the requests); token i
          of the step, the requests' new tokens one after another, goes to slot
          page * B + row; rows = exclusive prefix sums of new, lens = held + new.
  write   the step's K and V rows [layers, tokens, H, d] into their slots. Of a page's
          head the scale is the least power of two 2^e, e >= -120, with
          amax <= 448 * 2^e over the finite new values; a page whose first new token
          is not its row 0 keeps the greater of that and its old scale, and its old
          codes are rounded again where the scale grew. Codes are value / scale
          rounded to nearest even.
  attend  softmax attention of the step's queries [tokens, H * G, d] over one layer: the
          i-th of request r's queries lies at position p = lens[r] - new[r] + i and sees
          the positions max(0, p - window + 1) .. p (window 0: all up to p); a query
          that sees nothing gives zeros and a log-sum-exp of -inf. Outputs: the
          attention in the queries' type and the log-sum-exp in float32.

A case is a dict of plain values:
  op         "tables" | "write" | "attend"
  L, H, d    layers (of the cache for write; the cache of attend has one more than
             the layer that is read), KV heads, head dimension
  G          query heads for each KV head (attend)
  dtype      of the rows and the queries, "bfloat16" | "float32"
  block      B, tokens a page
  n          requests
  held, new  ranges "a,b" of the requests' tokens, spread evenly over a..b and dealt
             out by the seed
  idle       requests of the batch that hold nothing and bring a query that sees
             nothing: the padding of a batch of fixed size (attend)
  window     (attend)
"""

import math

import numpy as np
import torch

own = False

_DT = {"bfloat16": torch.bfloat16, "float32": torch.float32}
_MAX_CODE = 448.0


def listed():
    qwen = dict(H=8, d=128, dtype="bfloat16", block=16)

    def case(name, op, n, held, new, L=1, G=0, idle=0, window=0, **shape):
        return dict(name=name, op=op, n=n, held=held, new=new, L=L, G=G, idle=idle,
                    window=window, **shape)

    return [
        # one decoding step of a batch: 32 requests, one token each; latency
        case("tables-step", "tables", 32, "100,4000", "1,1", **qwen),
        # many prompts admitted in one step: 262 thousand new tokens
        case("tables-prompts", "tables", 256, "0,8191", "1,2047", **qwen),
        # the K and V of one layer appended for that step: one token in a part-filled page each
        case("write-append", "write", 32, "100,4000", "1,1", **qwen),
        # a merged cache of four thoughts of 4096 tokens (4B shape) laid into pages, every layer
        case("write-merged-4b-n4", "write", 1, "0,0", "16384,16384", L=36, **qwen),
        # float32 rows of ragged prompts that continue part-filled pages of 32 tokens
        case("write-fp32-ragged", "write", 12, "0,500", "1,333", L=12, H=4, d=128,
             dtype="float32", block=32),
        # one agent reads the smallest ordinary merge (512 + 768 tokens, 1.7B shape): latency
        case("attend-1.7b-n2", "attend", 1, "1279,1279", "1,1", G=2, **qwen),
        # a decoding batch of ragged contexts: bandwidth
        case("attend-batch", "attend", 64, "127,16383", "1,1", G=4, **qwen),
        # one agent reads the largest merge, 264 thousand tokens: one long axis to split
        case("attend-4b-large", "attend", 1, "264180,264180", "1,1", G=4, **qwen),
        # float32 queries, an odd group, a sliding window, three idle places of the batch
        case("attend-fp32-window", "attend", 24, "0,5000", "1,1", G=7, idle=3, window=1000, H=4,
             d=64, dtype="float32", block=32),
        # short questions after long contexts: a few rows more than one for each request
        case("attend-questions", "attend", 16, "1000,9000", "13,29", G=4, H=2, d=256,
             dtype="bfloat16", block=64),
        # a long question over a merged cache: arithmetic
        case("attend-prompt-4b-n4", "attend", 1, "16384,16384", "4096,4096", G=4, **qwen),
        # float32 prompts of uneven lengths, some over nothing held before
        case("attend-prompts-fp32", "attend", 6, "0,2000", "101,1501", G=2, H=4, d=128,
             dtype="float32", block=32),
    ]


def _log(rng, a, b):
    return int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))


def draw(rng):
    """One more case of any operator: one to 512 requests of one token to 260 thousand, decoding
    steps, short questions and prompts, each type, head dimension and page size, groups of one to
    sixteen."""
    op = rng.choice(["tables", "write", "attend", "attend", "attend"])
    H, d = rng.choice([1, 2, 4, 8]), rng.choice([64, 128, 128, 256])
    dtype = rng.choice(["bfloat16", "bfloat16", "float32"])
    block = rng.choice([16, 16, 32, 64, 128])
    kind = rng.choice(["step", "step", "question", "prompt"])
    n = _log(rng, 1, 512)
    # tokens held in all requests together
    total = _log(rng, max(64, n), 400_000 if op != "attend" else 2 ** 29 // (H * d))
    hi = max(1, min(260_000, total // n))
    lo = rng.randint(0, hi)
    new_hi = {"step": 1, "question": rng.randint(2, 40), "prompt": _log(rng, 41, 4096)}[kind]
    new_lo = 1 if kind == "step" else rng.randint(1, new_hi)
    L = _log(rng, 1, 36) if op == "write" else 1
    G = rng.choice([1, 2, 4, 4, 5, 8, 16]) if op == "attend" else 0
    if op == "attend":
        # scores of the plain form: at most 2 GB in 32 bits
        while n * H * G * new_hi * (hi + new_hi) > 2 ** 29:
            if n > 1:
                n = max(1, n // 2)
            elif new_hi > 1:
                new_hi = max(1, new_hi // 2)
            else:
                hi = hi // 2
            new_lo, lo = min(new_lo, new_hi), min(lo, hi)
    else:
        most = 262_144 if op == "tables" else int(1.2e9) // (L * H * d * 4)
        n = max(1, min(n, most // new_hi))
        new_hi = min(new_hi, most)
        new_lo = min(new_lo, new_hi)
    idle = rng.randint(1, n - 1) if op == "attend" and kind == "step" and n > 2 and rng.random() < 0.3 else 0
    window = _log(rng, 1, hi + 1) if op == "attend" and rng.random() < 0.3 else 0
    return dict(op=op, n=n, held="%d,%d" % (lo, hi), new="%d,%d" % (new_lo, new_hi), L=L, G=G,
                idle=idle, window=window, H=H, d=d, dtype=dtype, block=block)


# ------------------------------------------------------------------ lengths

def _spread(text, n):
    a, b = (int(x) for x in text.split(","))
    return b - (b - a) * np.arange(n, dtype=np.int64) // max(1, n - 1)


def _lengths(case):
    """(held, new) of the requests before the seed deals them out, int64 arrays: the sums and so
    the shapes of the outputs are the same for every seed."""
    n = case["n"]
    held, new = _spread(case["held"], n), _spread(case["new"], n)
    new = new[np.random.default_rng(n).permutation(n)]      # long prompts on long and short contexts
    if case["idle"]:
        held[-case["idle"]:] = -1                           # one query, nothing held: lens 0
    return held, new


def _seen(case):
    """(keys read, (query, key) pairs) over all requests."""
    held, new = _lengths(case)
    lens, w = held + new, case["window"]
    first = np.maximum(0, held - w + 1) if w else np.zeros_like(held)
    first = np.minimum(first, lens)
    keys = int((lens - first).sum())
    if not w:
        return keys, int((new * (held + 1) + new * (new - 1) // 2)[lens > 0].sum())
    # sum over i of min(held + i + 1, w)
    short = np.clip(w - held - 1, 0, new)                   # queries that see less than the window
    pairs = short * (held + 1) + short * (short - 1) // 2 + (new - short) * w
    return keys, int(pairs[lens > 0].sum())


# ------------------------------------------------------------------ inputs

def _codes(x):
    """Rows x [.., P, H, B, d] (float32) as 8-bit pages: (codes, scales)."""
    scales = _power(x.abs().amax((-2, -1)))
    return (x / scales[..., None, None]).to(torch.float8_e4m3fn), scales


def _power(amax):
    """The least 2^e, e >= -120, with amax <= 448 * 2^e (448 = 0.875 * 2^9), exactly."""
    m, x = torch.frexp(amax)
    e = torch.where(m > 0.875, x - 8, x - 9)
    e = torch.where(amax > 0, e, torch.full_like(e, -120)).clamp(min=-120)
    return ((e + 127) << 23).to(torch.int32).view(torch.float32)


def prepare(case, seed):
    op, n, B, H, d = case["op"], case["n"], case["block"], case["H"], case["d"]
    rng = np.random.default_rng([int(seed), n, 7])
    g = torch.Generator(device="cuda")
    g.manual_seed(1_000_003 * int(seed) + 29)
    deal = rng.permutation(n)
    held, new = (x[deal] for x in _lengths(case))
    lens = held + new
    have = -(-(held if op == "tables" else lens) // B)
    have = np.maximum(have, 0)
    width = int(-(-lens.max() // B)) + 3                    # a table is made for more than is used
    P = int((-(-lens // B)).sum()) + 5
    order = torch.randperm(P, generator=g, device="cuda").int()
    filled = torch.as_tensor(np.arange(width) < have[:, None], device="cuda")
    table = torch.full((n, width), -1, dtype=torch.int32, device="cuda")
    table[filled] = order[:int(have.sum())]

    def ints(x):
        return torch.as_tensor(x, dtype=torch.int32, device="cuda")

    s = dict(case=case, table=table, lens=ints(lens), tokens=int(new.sum()), longest=int(new.max()))
    if op == "tables":
        s.update(held=ints(held), new=ints(new), free=order[int(have.sum()):].contiguous(), pages=P)
        return s
    at = np.concatenate([[0], np.cumsum(new)])
    s["rows"] = ints(at)
    layers = case["L"] if op == "write" else case["L"] + 1
    codes = torch.empty((layers, 2, P, H, B, d), dtype=torch.float8_e4m3fn, device="cuda")
    scales = torch.empty((layers, 2, P, H), device="cuda")
    spread = float(np.exp(0.3 * rng.standard_normal()))     # K of one context: log-normal scale
    for l in range(layers):
        for kv in (0, 1):
            x = torch.randn((P, H, B, d), generator=g, device="cuda")
            x.mul_(spread if kv == 0 else 1.0)
            codes[l, kv], scales[l, kv] = _codes(x)
            del x
    s.update(codes=codes, scales=scales)
    dt = _DT[case["dtype"]]
    if op == "write":
        # K and V as a merged cache holds them, [layers, 2, H, tokens, d], here seen token by token
        kv = torch.empty((layers, 2, H, s["tokens"], d), dtype=dt, device="cuda")
        for l in range(layers):
            x = torch.randn((2, H, s["tokens"], d), generator=g, device="cuda")
            x[0].mul_(1.2 * spread)                         # now and then greater than what is there
            kv[l] = x
        s["k"], s["v"] = kv[:, 0].transpose(1, 2), kv[:, 1].transpose(1, 2)
        r = np.repeat(np.arange(n), new)
        pos = held[r] + np.arange(s["tokens"]) - at[r]
        where = torch.as_tensor(r, device="cuda"), torch.as_tensor(pos // B, device="cuda")
        s["slots"] = table[where].long() * B + torch.as_tensor(pos % B, device="cuda")
        return s
    s["layer"] = layers - 1
    s["q"] = torch.randn((s["tokens"], H * case["G"], d), generator=g, device="cuda").to(dt)
    s["out"] = torch.empty_like(s["q"])
    s["lse"] = torch.empty((s["tokens"], H * case["G"]), device="cuda")
    return s


# ------------------------------------------------------------------ one pass

def run(s):
    op = s["case"]["op"]
    if own:
        return {"tables": _own_tables, "write": _own_write, "attend": _own_attend}[op](s)
    return {"tables": _tables, "write": _write, "attend": _attend}[op](s)


def _own_tables(s):
    import paper_2607_01308_amd as cm
    r = cm.qcache_tables(s["pages"], s["case"]["block"], s["held"], s["new"], s["free"], s["table"],
                         s["tokens"])
    return dict(table=s["table"], slots=r.slots, rows=r.rows, lens=r.lens)


def _own_write(s):
    import paper_2607_01308_amd as cm
    cm.qcache_write(cm.QCache(s["codes"], s["scales"]), 0, s["k"], s["v"], s["slots"])
    return dict(codes=s["codes"], scales=s["scales"])


def _own_attend(s):
    import paper_2607_01308_amd as cm
    cm.qcache_attention(cm.QCache(s["codes"], s["scales"]), s["layer"], s["q"], s["table"],
                        s["lens"], rows=s["rows"], max_rows=s["longest"],
                        window=s["case"]["window"], out=s["out"], lse=s["lse"])
    return dict(out=s["out"], lse=s["lse"])


def _tables(s):
    B, table = s["case"]["block"], s["table"]
    held, new = s["held"].long(), s["new"].long()
    lens = held + new
    have, want = (held + B - 1) // B, (lens + B - 1) // B
    first = torch.cumsum(want - have, 0) - (want - have)
    ends = torch.cumsum(new, 0)
    rows = torch.cat([ends.new_zeros(1), ends])
    j = torch.arange(table.shape[1], device=table.device)[None]
    fresh = (j >= have[:, None]) & (j < want[:, None])
    take = torch.where(fresh, first[:, None] + j - have[:, None], 0)
    table.copy_(torch.where(fresh, s["free"][take], table))
    i = torch.arange(s["tokens"], device=table.device)
    r = torch.searchsorted(ends, i, right=True)
    pos = held[r] + i - rows[r]
    slots = table[r, pos // B].long() * B + pos % B
    return dict(table=table, slots=slots, rows=rows.int(), lens=lens.int())


def _write(s):
    """Pages that a request's first new token enters in the middle are given as the first slots of
    the requests, which the step's rows tell."""
    slots = s["slots"]
    B = s["case"]["block"]
    page, row = slots // B, slots % B
    first = slots[s["rows"][:-1].long()]
    part = torch.where(first % B > 0, 1.0, 0.0)
    held, begin = first // B, first % B
    _write_rows(s["k"], s["codes"][:, 0], s["scales"][:, 0], page, row, held, begin, part)
    _write_rows(s["v"], s["codes"][:, 1], s["scales"][:, 1], page, row, held, begin, part)
    return dict(codes=s["codes"], scales=s["scales"])


def _at(codes, pages):
    """The codes of pages [.., n, H, B, d] as 32-bit numbers."""
    return codes.view(torch.uint8)[:, pages].view(torch.float8_e4m3fn).float()


def _write_rows(x, codes, scales, page, row, held, begin, part):
    x = x.float()
    high = torch.where(x.isfinite(), x.abs(), 0.0).amax(-1)                     # [layers, tokens, H]
    amax = torch.zeros_like(scales).index_reduce_(1, page, high, "amax")
    touched = torch.zeros_like(scales[:1, :, :1]).index_fill_(1, page, 1.0)
    old = scales[:, held]                                                       # [layers, n, H]
    was = _at(codes, held)                                                      # [layers, n, H, B, d]
    fresh = torch.where(touched > 0, _power(amax), scales)
    kept = torch.zeros_like(scales).index_copy_(1, held, old * part[None, :, None])
    now = torch.maximum(fresh, kept)
    # the old rows of the pages entered in the middle
    again = was * (old / now[:, held])[..., None, None]
    stays = torch.arange(codes.shape[3], device=x.device)[None, :, None] < begin[:, None, None]
    again = torch.where(stays[:, None], again, was).to(codes.dtype)
    codes.view(torch.uint8)[:, held] = again.view(torch.uint8)
    scales.copy_(now)
    put = (x / now[:, page][..., None]).to(codes.dtype)
    codes.view(torch.uint8)[:, page, :, row] = put.view(torch.uint8).transpose(0, 1)


def _attend(s):
    case = s["case"]
    B, H, G, d, n = case["block"], case["H"], case["G"], case["d"], case["n"]
    Q = s["longest"]
    rows, lens = s["rows"].long(), s["lens"].long()
    new = rows[1:] - rows[:-1]
    table = s["table"].long().clamp(min=0)
    T = table.shape[1] * B
    k = _pages(s, 0, table)                                                     # [n, H, T, d]
    i = torch.arange(Q, device=table.device)[None]
    place = (rows[:-1, None] + i).clamp(max=s["tokens"] - 1)                    # [n, Q]
    q = s["q"].float()[place].view(n, Q, H, G, d).permute(0, 2, 3, 1, 4).reshape(n, H, G * Q, d)
    x = torch.matmul(q, k.transpose(2, 3).contiguous()).view(n, H, G, Q, T)
    del k
    x *= d ** -0.5
    p = (lens - new)[:, None] + i                                               # [n, Q]
    t = torch.arange(T, device=table.device)
    sees = t[None, None] <= p[..., None]
    if case["window"]:
        sees &= t[None, None] > p[..., None] - case["window"]
    x.masked_fill_(~sees[:, None, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    low = torch.where(top == -math.inf, 0.0, top)
    x = x.sub_(low).exp_()
    total = x.sum(-1, keepdim=True)
    y = torch.matmul(x.view(n, H, G * Q, T), _pages(s, 1, table)).view(n, H, G, Q, d)
    y = y / torch.where(total == 0, 1.0, total)
    lse = (total.log() + low)[..., 0]
    # back to the step's rows
    r = torch.searchsorted(rows[1:], torch.arange(s["tokens"], device=table.device), right=True)
    at = torch.arange(s["tokens"], device=table.device) - rows[r]
    s["out"].copy_(y[r, :, :, at].reshape(s["tokens"], H * G, d))
    s["lse"].copy_(lse[r, :, :, at].reshape(s["tokens"], H * G))
    return dict(out=s["out"], lse=s["lse"])


def _pages(s, kv, table):
    """The values of every request's pages in order, [n, H, T, d] in 32 bits."""
    case, l = s["case"], s["layer"]
    x = _at(s["codes"][l:l + 1, kv], table)[0]
    x *= s["scales"][l, kv][table][..., None, None]
    return x.permute(0, 2, 1, 3, 4).reshape(case["n"], case["H"], -1, case["d"])


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    """tables: lengths, the free pages taken, the new table entries, the slots. write: the rows
    read, the pages' codes of the new rows written (and the old rows of part-filled pages read and
    written). attend: the visible codes and their scales, queries, outputs; two products of 2 d
    operations for each visible (query, key) pair and query head."""
    held, new = _lengths(case)
    lens, B, H, d, n = held + new, case["block"], case["H"], case["d"], case["n"]
    tokens = int(new.sum())
    e = 2 if case["dtype"] == "bfloat16" else 4
    pages = int((-(-lens // B)).sum())
    if case["op"] == "tables":
        taken = pages - int((-(-held // B)).sum())
        return {"bytes": 8 * n + 8 * taken + 8 * tokens + 4 * (n + 1) + 4 * n, "flops": 0}
    if case["op"] == "write":
        part = int((held % B)[new > 0].sum())
        touched = pages - int((held // B).sum())
        values = 2 * case["L"] * H * d
        return {"bytes": values * (tokens * (e + 1) + 2 * part) + 8 * tokens
                + 4 * 2 * case["L"] * H * touched,
                "flops": 2 * values * tokens}
    keys, pairs = _seen(case)
    Hq = H * case["G"]
    return {"bytes": 2 * H * d * keys + 8 * H * -(-keys // B) + 4 * -(-keys // B)
            + tokens * Hq * (2 * e * d + 4) + 8 * n,
            "flops": 4 * d * Hq * pairs}


# ------------------------------------------------------------------ the same in 64 bits

def exact(case, seed):
    if case["op"] == "tables":
        return None                                         # whole numbers only
    s = prepare(case, seed)
    if case["op"] == "write":
        return _write_exact(s)
    rows, lens = s["rows"].tolist(), s["lens"].tolist()
    B, H, G, d, w, l = (case[k] for k in ("block", "H", "G", "d", "window", "L"))
    out = torch.zeros((s["tokens"], H * G, d), dtype=torch.float64, device="cuda")
    lse = torch.full((s["tokens"], H * G), -math.inf, dtype=torch.float64, device="cuda")
    for r, T in enumerate(lens):
        count = rows[r + 1] - rows[r]
        if T < 1 or count < 1:
            continue
        pages = s["table"][r, :-(-T // B)].long()
        pos = T - count + torch.arange(count, device="cuda")
        t = torch.arange(T, device="cuda")
        hidden = t[None] > pos[:, None]
        if w:
            hidden |= t[None] <= pos[:, None] - w
        hidden |= (pos < 0)[:, None]
        for h in range(H):
            k, v = ((s["codes"][l, kv, :, h].view(torch.uint8)[pages].view(torch.float8_e4m3fn)
                     .double() * s["scales"][l, kv, pages, h].double()[:, None, None])
                    .reshape(-1, d)[:T] for kv in (0, 1))
            kt = k.t().contiguous()
            for j in range(h * G, (h + 1) * G):
                z = s["q"][rows[r]:rows[r + 1], j].double() @ kt / math.sqrt(d)
                z.masked_fill_(hidden, -math.inf)
                one = torch.logsumexp(z, -1)
                lse[rows[r]:rows[r + 1], j] = one
                z = (z - one[:, None]).exp_()
                out[rows[r]:rows[r + 1], j] = z @ v
    return dict(out=out, lse=lse)


def _e4m3(y):
    """y (64 bits, within +-448) rounded to the nearest of float8_e4m3fn, ties to even: three bits
    after the leading one down to 2^-6, steps of 2^-9 below."""
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step


def _write_exact(s):
    B = s["case"]["block"]
    codes, scales = s["codes"].double(), s["scales"].double()
    slots, first = s["slots"], s["slots"][s["rows"][:-1].long()]
    for kv, x in ((0, s["k"]), (1, s["v"])):
        high = torch.zeros_like(scales[:, kv])
        a = x.double().abs().amax(-1)
        high.index_reduce_(1, slots // B, a, "amax")
        new = torch.exp2(torch.ceil(torch.log2(high / _MAX_CODE))).clamp(min=2.0 ** -120)
        used = torch.zeros(scales.shape[2], dtype=torch.bool, device="cuda")
        used[slots // B] = True
        for page, row in zip((first // B).tolist(), (first % B).tolist()):
            if row == 0:
                continue
            old = scales[:, kv, page]
            grown = torch.maximum(old, new[:, page])
            codes[:, kv, page, :, :row] = _e4m3(codes[:, kv, page, :, :row]
                                                * (old / grown)[..., None, None])
            new[:, page] = grown
        scales[:, kv] = torch.where(used[None, :, None], new, scales[:, kv])
        y = _e4m3(x.double() / scales[:, kv][:, slots // B][..., None])
        codes[:, kv, slots // B, :, slots % B] = y.transpose(0, 1)
    return dict(codes=codes, scales=scales)
