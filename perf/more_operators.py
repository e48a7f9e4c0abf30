"""The operators that decode with drafted tokens over an 8-bit paged cache, as cases that can be
prepared, run in plain torch operations or through the library, computed in 64 bits and timed.

A step brings each request a tree of drafted nodes: node 0 is the token that was sampled last, node i
hangs on parents[i] < i (parents[0] = -1). A request of c nodes has lens tokens in its pages, the
nodes last: the first held = lens - c are its context, node i lies at place held + i, and its position
is held + the number of its ancestors. The cache is paged, for each layer and K/V: codes
[L, 2, P, H, B, d] in float8_e4m3fn and scales [L, 2, P, H] in float32; a stored value is code * scale.

  rotate  norms of queries and keys for each head and the rotation for their positions:
          y = x / sqrt(mean(x^2) + eps) * w over the d elements of a head; pair i of y is turned by
          the angle position * base^(-2i/d), pairs (i, i + d/2) ("half") or (2i, 2i + 1).
  attend  softmax attention of the nodes' queries [tokens, H * G, d] over one layer: a node sees the
          context (with a window: its last window positions, itself included) and the nodes whose
          bits are set in its mask, its ancestors and itself. Outputs: the attention in the
          queries' type and the log-sum-exp in float32.
  verify  drafted nodes against the target's probabilities p [tokens, V] (row i: of the token after
          node i), from given random numbers. From node 0 on, the node's children x in order are
          tried: with r = p's row, m = 1 at first, x is accepted if u_x q(t_x) m < r(t_x), t_x its
          token and q the row of draft probabilities that the node's children were sampled from;
          otherwise r = max(r - m q, 0), m = sum r. Without q a drafted token counts as certain
          (q is 1 there): u_x m < r(t_x), otherwise m -= r(t_x), r(t_x) = 0. The first accepted child is
          the next node; where there is none, the token sampled is the first v with
          r_0 + .. + r_v > s sum r. Outputs: the accepted nodes in order (path, -1 behind
          them), how many, and the token sampled.
  keep    the accepted nodes' K and V in every layer, moved to the front of the nodes' places: place
          held + i takes what lies at held + path[i]. The scale of a page that takes rows is the
          greatest among the pages they come from and, where it holds rows before them, its own;
          codes are rounded again where the scale grows. Outputs: the cache, the lengths held +
          counts, and the pages that the other nodes leave, in order.
  copy    whole pages of every layer, codes and scales, to other pages.

A case is a dict of plain values:
  op         "rotate" | "attend" | "verify" | "keep" | "copy"
  H, d, G    KV heads, head dimension, query heads for each KV head (rotate, attend)
  dtype      of the rows, the queries or the probabilities, "bfloat16" | "float32"
  block, L   B, tokens a page; layers of the cache (attend: one less than it has)
  n          requests (copy: pages)
  held, new  ranges "a,b" of the requests' context and nodes, spread evenly over a..b and dealt out
             by the seed (rotate: tokens, from positions held on)
  branch     the most children that a node has (attend, verify)
  window     (attend)
  style, base  of the rotation
  V, sampled the vocabulary; whether the drafts were sampled from probabilities (verify)
  kept       range "a,b" of the nodes accepted (keep)
"""

import math

import numpy as np
import torch

own = False

_DT = {"bfloat16": torch.bfloat16, "float32": torch.float32}
_EPS = 1e-6


def listed():
    qwen = dict(H=8, d=128, dtype="bfloat16", block=16)

    def attend(name, n, held, new, branch, G, window=0, **shape):
        return dict(name=name, op="attend", n=n, held=held, new=new, branch=branch, G=G, window=window,
                    L=1, **shape)

    return [
        # queries and keys of one decoding step of 32 requests, a token each; latency
        dict(name="rotate-step", op="rotate", n=32, held="100,4000", new="1,1", G=4, style="half",
             base=1e6, **qwen),
        # a prompt of 16384 tokens over nothing held (4B shape): bandwidth
        dict(name="rotate-prompt", op="rotate", n=1, held="0,0", new="16384,16384", G=4, style="half",
             base=1e6, **qwen),
        # one agent's eight drafted nodes over the smallest ordinary merge (512 + 768 tokens): latency
        attend("tree-1.7b-n2", 1, "1280,1280", "8,8", 2, 2, **qwen),
        # a decoding batch, sixteen nodes each over ragged contexts
        attend("tree-batch", 32, "127,8191", "16,16", 3, 4, **qwen),
        # one agent's wide tree over the largest merge, 264 thousand tokens: one long axis to split
        attend("tree-4b-large", 1, "264180,264180", "32,32", 4, 4, **qwen),
        # float32 queries, an odd group, ragged trees, a sliding window
        attend("tree-fp32-window", 24, "0,5000", "1,23", 4, 3, window=1000, H=4, d=64,
               dtype="float32", block=32),
        # chains of five for a few requests, a small vocabulary: latency
        dict(name="verify-chains", op="verify", n=4, held="0,0", new="5,5", branch=1, V=32768,
             sampled=True, dtype="float32"),
        # trees for a batch over a large odd vocabulary, drafts sampled from their probabilities
        dict(name="verify-trees", op="verify", n=32, held="0,0", new="9,25", branch=3, V=100003,
             sampled=True, dtype="bfloat16"),
        # the accepted nodes of a batch's trees of sixteen, every layer: latency
        dict(name="keep-batch", op="keep", n=32, L=36, held="16,400", new="16,16", kept="1,6", **qwen),
        # long trees of a full batch over pages of 64 tokens, many nodes accepted
        dict(name="keep-wide", op="keep", n=256, L=12, held="1,200", new="17,64", kept="0,40", H=4, d=256,
             dtype="bfloat16", block=64),
        # eight places begin as copies of one: its part-filled page for each
        dict(name="copy-fork", op="copy", n=8, L=36, **qwen),
        # a context of 16384 tokens copied whole (4B shape): bandwidth
        dict(name="copy-context", op="copy", n=1024, L=36, **qwen),
    ]


def _log(rng, a, b):
    return int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))


def draw(rng):
    """One more case of any operator: one to 512 requests, one to 128 nodes, contexts of none to 260
    thousand tokens, each type, head dimension, page size and style, groups of one to sixteen,
    vocabularies of 100 to 200 thousand."""
    op = rng.choice(["rotate", "attend", "attend", "attend", "verify", "verify", "keep", "copy"])
    H, d = rng.choice([1, 2, 4, 8]), rng.choice([64, 128, 128, 256])
    dtype = rng.choice(["bfloat16", "bfloat16", "float32"])
    block = rng.choice([16, 16, 32, 64, 128])
    shape = dict(H=H, d=d, dtype=dtype, block=block)
    n = _log(rng, 1, 512)
    nodes = _log(rng, 1, 128)
    least = rng.randint(1, nodes)
    if op == "rotate":
        G = rng.choice([1, 2, 4, 5, 8])
        most = 2 ** 27 // (H * (G + 1) * d * (2 if dtype == "float32" else 1))
        n = min(n, most)
        tokens = _log(rng, 1, most // n)
        first = rng.randint(0, 260_000)
        return dict(op=op, n=n, held="%d,%d" % (0, first), new="%d,%d" % (max(1, tokens // 2), tokens), G=G,
                    style=rng.choice(["half", "half", "interleaved"]), base=rng.choice([1e4, 5e5, 1e6]),
                    **shape)
    if op == "attend":
        G = rng.choice([1, 2, 4, 4, 5, 8, 16])
        hi = max(1, min(260_000, _log(rng, 64, 2 ** 29 // (H * d)) // n))
        # scores of the plain form: at most 2 GB in 32 bits
        while n * H * G * nodes * (hi + nodes) > 2 ** 29:
            if n > 1:
                n = max(1, n // 2)
            else:
                hi, nodes = max(1, hi // 2), max(1, nodes // 2)
        least = min(least, nodes)
        window = _log(rng, 1, hi + 1) if rng.random() < 0.3 else 0
        return dict(op=op, n=n, held="%d,%d" % (rng.randint(0, hi), hi), new="%d,%d" % (least, nodes),
                    branch=rng.randint(1, 5), G=G, window=window, L=1, **shape)
    if op == "verify":
        V = _log(rng, 100, 200_000)
        n = max(1, min(n, int(5e7) // (V * nodes)))
        return dict(op=op, n=n, held="0,0", new="%d,%d" % (least, nodes), branch=rng.randint(1, 4), V=V,
                    sampled=rng.random() < 0.6, dtype=dtype)
    L = _log(rng, 1, 36)
    if op == "keep":
        kept = rng.randint(0, least)
        hi = _log(rng, 1, 400)
        pages = max(1, 2 ** 29 // (L * 2 * H * block * d))
        n = max(1, min(n, pages // (2 + (hi + nodes) // block)))
        return dict(op=op, n=n, L=L, held="%d,%d" % (rng.randint(0, hi), hi), new="%d,%d" % (least, nodes),
                    kept="%d,%d" % (min(1, kept), kept), **shape)
    most = int(1.2e9) // (L * 2 * H * block * d)
    return dict(op=op, n=max(1, min(_log(rng, 1, 4096), most)), L=L, **shape)


# ------------------------------------------------------------------ lengths

def _spread(text, n):
    a, b = (int(x) for x in text.split(","))
    return b - (b - a) * np.arange(n, dtype=np.int64) // max(1, n - 1)


def _lengths(case):
    """(held, new) of the requests before the seed deals them out, int64 arrays: the sums and so
    the shapes of the outputs are the same for every seed."""
    n = case["n"]
    new = _spread(case["new"], n)
    return _spread(case["held"], n), new[np.random.default_rng(n).permutation(n)]


# ------------------------------------------------------------------ inputs

def _power(amax):
    """The least 2^e, e >= -120, with amax <= 448 * 2^e (448 = 0.875 * 2^9), exactly."""
    m, x = torch.frexp(amax)
    e = torch.where(m > 0.875, x - 8, x - 9)
    e = torch.where(amax > 0, e, torch.full_like(e, -120)).clamp(min=-120)
    return ((e + 127) << 23).to(torch.int32).view(torch.float32)


def _cache(case, layers, P, g, spread):
    """Pages as writes leave them: K of log-normal spread from page to page, V of one."""
    H, B, d = case["H"], case["block"], case["d"]
    codes = torch.empty((layers, 2, P, H, B, d), dtype=torch.float8_e4m3fn, device="cuda")
    scales = torch.empty((layers, 2, P, H), device="cuda")
    for l in range(layers):
        for kv in (0, 1):
            x = torch.randn((P, H, B, d), generator=g, device="cuda")
            if kv == 0:
                x *= spread
                if case["op"] == "keep":
                    x *= torch.exp(0.5 * torch.randn((P, H, 1, 1), generator=g, device="cuda"))
            s = _power(x.abs().amax((-2, -1)))
            codes[l, kv] = (x / s[..., None, None]).to(codes.dtype)
            scales[l, kv] = s
    return dict(codes=codes, scales=scales)


def _trees(rng, new, branch):
    """parents of all nodes, request after request, -1 for node 0: a node hangs on one of the last few
    nodes that have fewer than `branch` children."""
    out = []
    for c in new:
        children = np.zeros(c, dtype=np.int64)
        for i in range(c):
            room = np.nonzero(children[:i] < branch)[0]
            p = int(room[max(0, len(room) - 1 - int(rng.integers(0, 2 * branch)))]) if i else -1
            if i:
                children[p] += 1
            out.append(p)
    return np.array(out, dtype=np.int64)


def _ancestors(parents, at, window):
    """Masks [tokens, words] and depths [tokens]: bit j of node i's row is set for j = i and i's
    ancestors, with a window only those less than that many steps up."""
    tokens = len(parents)
    words = -(-int((at[1:] - at[:-1]).max()) // 64)
    bits = np.zeros((tokens, words * 64), dtype=np.uint8)
    depth = np.zeros(tokens, dtype=np.int64)
    for a, b in zip(at[:-1], at[1:]):
        for i in range(a, b):
            j, up = i - a, 0
            while j >= 0:
                if not window or up < window:
                    bits[i, j] = 1
                j, up = parents[a + j], up + 1
            depth[i] = up - 1
    masks = np.packbits(bits, axis=1, bitorder="little").view(np.int64)
    return np.ascontiguousarray(masks), depth


def prepare(case, seed):
    op, n = case["op"], case["n"]
    rng = np.random.default_rng([int(seed), n, 11])
    g = torch.Generator(device="cuda")
    g.manual_seed(1_000_003 * int(seed) + 31)

    def ints(x):
        return torch.as_tensor(x, dtype=torch.int32, device="cuda")

    if op == "copy":
        s = dict(case=case, **_cache(case, case["L"], 2 * n + 3, g, 1.0))
        order = torch.randperm(2 * n + 3, generator=g, device="cuda").int()
        s.update(src=order[:n].contiguous(), dst=order[n:2 * n].contiguous())
        return s
    deal = rng.permutation(n)
    held, new = (x[deal] for x in _lengths(case))
    tokens = int(new.sum())
    at = np.concatenate([[0], np.cumsum(new)])
    s = dict(case=case, tokens=tokens, longest=int(new.max()), rows=ints(at))
    if op == "rotate":
        H, G, d, dt = case["H"], case["G"], case["d"], _DT[case["dtype"]]
        # one projection's output, queries then keys (then values, which stay as they are)
        x = torch.randn((tokens, (G + 2) * H, d), generator=g, device="cuda")
        x *= torch.exp(0.5 * torch.randn((1, 1, d), generator=g, device="cuda"))
        s["x"] = x.to(dt)
        for name in ("q_weight", "k_weight"):
            s[name] = (1 + 0.3 * torch.randn(d, generator=g, device="cuda")).to(dt)
        s["positions"] = ints(np.concatenate([np.arange(h, h + c) for h, c in zip(held, new)]))
        return s
    if op == "verify":
        V, dt = case["V"], _DT[case["dtype"]]
        parents = _trees(rng, new, case["branch"])
        s["parents"] = ints(parents)
        x = 3 * torch.randn((tokens, V), generator=g, device="cuda")
        s["probs"] = torch.softmax(x, 1).to(dt)
        # the draft model's view of the same
        x += 1.5 * torch.randn((tokens, V), generator=g, device="cuda")
        q = torch.softmax(x, 1).to(dt)
        first = np.repeat(at[:-1], new)
        of = torch.as_tensor(np.where(parents < 0, first, first + parents), device="cuda")
        s["drafts"] = torch.multinomial(q.float(), 4, replacement=True, generator=g)[of].gather(
            1, torch.randint(0, 4, (tokens, 1), generator=g, device="cuda"))[:, 0]
        s["draft_probs"] = q if case["sampled"] else None
        s["accept"] = torch.rand(tokens, generator=g, device="cuda")
        s["sample"] = torch.rand(n, generator=g, device="cuda")
        return s
    B = case["block"]
    lens = held + new
    have = -(-lens // B)
    width = int(have.max()) + 3                             # a table is made for more than is used
    P = int(have.sum()) + 5
    order = torch.randperm(P, generator=g, device="cuda").int()
    table = torch.full((n, width), -1, dtype=torch.int32, device="cuda")
    table[torch.as_tensor(np.arange(width) < have[:, None], device="cuda")] = order[:int(have.sum())]
    spread = float(np.exp(0.3 * rng.standard_normal()))     # K of one context: log-normal scale
    s.update(_cache(case, case["L"] + (op == "attend"), P, g, spread), table=table, lens=ints(lens))
    if op == "keep":
        counts = np.minimum(_spread(case["kept"], n)[deal], new)
        path = np.full(tokens, -1, dtype=np.int64)
        for r in range(n):
            if counts[r]:
                some = 1 + rng.permutation(new[r] - 1)[:counts[r] - 1]
                path[at[r]:at[r] + counts[r]] = np.concatenate([[0], np.sort(some)])
        s.update(path=ints(path), counts=ints(counts), kept=int(counts.sum()), most=int((have - held // B).max()))
        s["freed"] = torch.full((int((have - held // B).sum()) + 1,), -1, dtype=torch.int32, device="cuda")
        return s
    masks, depth = _ancestors(_trees(rng, new, case["branch"]), at, case["window"])
    Hq, dt = case["H"] * case["G"], _DT[case["dtype"]]
    s.update(masks=torch.as_tensor(masks, device="cuda"), positions=ints(np.repeat(held, new) + depth),
             layer=case["L"], q=torch.randn((tokens, Hq, case["d"]), generator=g, device="cuda").to(dt))
    s["out"] = torch.empty_like(s["q"])
    s["lse"] = torch.empty((tokens, Hq), device="cuda")
    return s


# ------------------------------------------------------------------ one pass

def run(s):
    op = s["case"]["op"]
    if own:
        return {"rotate": _own_rotate, "attend": _own_attend, "verify": _own_verify, "keep": _own_keep,
                "copy": _own_copy}[op](s)
    return {"rotate": _rotate, "attend": _attend, "verify": _verify, "keep": _keep, "copy": _copy}[op](s)


def _own_rotate(s):
    import paper_2607_01308_amd as cm
    case = s["case"]
    q, k, _ = s["x"].split((case["H"] * case["G"], case["H"], case["H"]), 1)
    q, k = cm.norm_rotate(q, k, s["positions"], case["base"], style=case["style"],
                          q_weight=s["q_weight"], k_weight=s["k_weight"], eps=_EPS)
    return dict(q=q, k=k)


def _own_attend(s):
    import paper_2607_01308_amd as cm
    tree = cm.QCacheTree(s["masks"], s["positions"], s["case"]["window"])
    cm.qcache_tree_attention(cm.QCache(s["codes"], s["scales"]), s["layer"], s["q"], s["table"],
                             s["lens"], s["rows"], tree, max_rows=s["longest"], out=s["out"],
                             lse=s["lse"])
    return dict(out=s["out"], lse=s["lse"])


def _own_verify(s):
    import paper_2607_01308_amd as cm
    v = cm.verify_drafts(s["probs"], s["drafts"], s["parents"], s["rows"], s["accept"], s["sample"],
                         draft_probs=s["draft_probs"])
    return dict(path=v.path, counts=v.counts, tokens=v.tokens)


def _own_keep(s):
    import paper_2607_01308_amd as cm
    k = cm.qcache_keep(cm.QCache(s["codes"], s["scales"]), s["table"], s["lens"], s["rows"], s["path"],
                       s["counts"], freed=s["freed"])
    return dict(codes=s["codes"], scales=s["scales"], lens=k.lens, freed=s["freed"])


def _own_copy(s):
    import paper_2607_01308_amd as cm
    cm.qcache_copy(cm.QCache(s["codes"], s["scales"]), s["src"], s["dst"])
    return dict(codes=s["codes"], scales=s["scales"])


def _request(s):
    """(request, number within it) of every row of the step."""
    rows = s["rows"].long()
    i = torch.arange(s["tokens"], device=rows.device)
    r = torch.searchsorted(rows[1:], i, right=True)
    return r, i - rows[r]


def _rotate(s):
    case = s["case"]
    H, G, d = case["H"], case["G"], case["d"]
    q, k, _ = s["x"].split((H * G, H, H), 1)
    freq = case["base"] ** (-2 * torch.arange(d // 2, device=q.device, dtype=torch.float64) / d)
    angle = s["positions"].double()[:, None] * freq         # far positions: in 64 bits
    c, t = angle.cos().float()[:, None], angle.sin().float()[:, None]

    def one(x, w):
        y = x.float()
        y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + _EPS) * w.float()
        if case["style"] == "half":
            a, b = y[..., :d // 2], y[..., d // 2:]
            return torch.cat((a * c - b * t, b * c + a * t), -1).to(x.dtype)
        a, b = y[..., ::2], y[..., 1::2]
        return torch.stack((a * c - b * t, b * c + a * t), -1).flatten(-2).to(x.dtype)

    return dict(q=one(q, s["q_weight"]), k=one(k, s["k_weight"]))


def _at(codes, pages):
    """The codes of pages [.., n, H, B, d] as 32-bit numbers."""
    return codes.view(torch.uint8)[:, pages].view(torch.float8_e4m3fn).float()


def _pages(s, kv, table):
    """The values of every request's pages in order, [n, H, T, d] in 32 bits."""
    case, l = s["case"], s["layer"]
    x = _at(s["codes"][l:l + 1, kv], table)[0]
    x *= s["scales"][l, kv][table][..., None, None]
    return x.permute(0, 2, 1, 3, 4).reshape(case["n"], case["H"], -1, case["d"])


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
    t = torch.arange(T, device=table.device)[None]
    held = (lens - new)[:, None]
    # the nodes' bits where they lie, the context as its window says
    j = t - held                                                                # [n, T]
    word = (j // 64).clamp(0, s["masks"].shape[1] - 1)
    bit = s["masks"][place].gather(2, word[:, None].expand(n, Q, T)) >> (j % 64)[:, None] & 1
    context = (t < held)[:, None].expand(n, Q, T)
    if case["window"]:
        context = context & (t[:, None] > s["positions"].long()[place][..., None] - case["window"])
    sees = context | (bit == 1) & ((j >= 0) & (t < lens[:, None]))[:, None]
    x.masked_fill_(~sees[:, None, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    low = torch.where(top == -math.inf, 0.0, top)
    x = x.sub_(low).exp_()
    total = x.sum(-1, keepdim=True)
    y = torch.matmul(x.view(n, H, G * Q, T), _pages(s, 1, table)).view(n, H, G, Q, d)
    y = y / torch.where(total == 0, 1.0, total)
    lse = (total.log() + low)[..., 0]
    r, at = _request(s)                                     # back to the step's rows
    s["out"].copy_(y[r, :, :, at].reshape(s["tokens"], H * G, d))
    s["lse"].copy_(lse[r, :, :, at].reshape(s["tokens"], H * G))
    return dict(out=s["out"], lse=s["lse"])


def _verify(s):
    """Every node's own test, as if its parent had been reached, one child of each node after another;
    then the nodes whose ancestors and selves were chosen. In 64 bits: numbers next to a border."""
    rows, parents, drafts = s["rows"].long(), s["parents"].long(), s["drafts"]
    T = s["tokens"]
    request, at = _request(s)
    base = rows[request]
    i = torch.arange(T, device=rows.device)
    over = torch.where(parents >= 0, parents + base, -1)    # the parent's row, -1 for node 0
    family = over[:, None] == over[None]                    # siblings
    rank = (family & (i[None] < i[:, None])).sum(1)
    p = s["probs"].double()
    q = s["draft_probs"]
    r, m = p, torch.ones(T, dtype=torch.float64, device=rows.device)
    chosen = torch.zeros(T, dtype=torch.bool, device=rows.device)
    row = over.clamp(min=0)
    for k in range(s["case"]["branch"]):
        mine = (over >= 0) & (rank == k)
        open_to = torch.zeros(T + 1, device=rows.device).index_put_((torch.where(chosen, over, T),),
                                                                    torch.ones(T, device=rows.device))
        left = r[row, drafts]
        certain = 1.0 if q is None else q[row, drafts].double()
        ok = mine & (open_to[row] == 0) & (s["accept"].double() * certain * m[row] < left)
        chosen = chosen | ok
        # the rows whose k-th child was not accepted lose what it stood for
        lost = torch.zeros(T + 1, dtype=torch.long, device=rows.device).index_put_(
            (torch.where(mine & ~ok, over, T),), i)[:T]
        has = torch.zeros(T + 1, dtype=torch.bool, device=rows.device).index_put_(
            (torch.where(mine & ~ok, over, T),), torch.ones(T, dtype=torch.bool, device=rows.device))[:T]
        if q is None:
            gone = drafts[lost][:, None]
            had = r.gather(1, gone)
            r = torch.where(has[:, None], r.scatter(1, gone, 0.0), r)
            m = torch.where(has, m - had[:, 0], m)
        else:
            then = torch.clamp(r - m[:, None] * q.double(), min=0.0)
            m = torch.where(has, then.sum(1), m)
            r = torch.where(has[:, None], then, r)
    # reached: every node from the root on chosen (matrix of "is a descendant of or is")
    root = at == 0
    up = torch.zeros((T, T), device=rows.device).index_put_((i, row), (over >= 0).float())
    step = up + torch.eye(T, device=rows.device)
    for _ in range(max(1, math.ceil(math.log2(max(2, s["longest"]))))):
        step = (torch.matmul(step, step) > 0).float()
    reached = torch.matmul(step, (~(chosen | root)).float()) == 0
    counts = torch.zeros(s["case"]["n"], dtype=torch.long, device=rows.device).index_add_(0, request, reached.long())
    before = torch.cumsum(reached.long(), 0) - reached.long()
    place = torch.where(reached, base + before - before[base], T)
    path = torch.full((T + 1,), -1, dtype=torch.long, device=rows.device).index_put_((place,), at)[:T]
    # the token after the last of them
    last = rows[:-1] + path[rows[:-1] + counts - 1]
    sums = torch.cumsum(r[last], 1)
    want = s["sample"].double()[:, None] * sums[:, -1:]
    tokens = torch.searchsorted(sums, want, right=True)[:, 0].clamp(max=sums.shape[1] - 1)
    return dict(path=path.int(), counts=counts.int(), tokens=tokens)


def _moves(s):
    """Of every kept row: request, and slots (page, row) that it comes from and goes to."""
    B, rows, lens = s["case"]["block"], s["rows"].long(), s["lens"].long()
    counts, table = s["counts"].long(), s["table"].long()
    held = lens - (rows[1:] - rows[:-1])
    ends = torch.cumsum(counts, 0)
    i = torch.arange(s["kept"], device=rows.device)
    r = torch.searchsorted(ends, i, right=True)
    i = i - (ends - counts)[r]
    to = held[r] + i
    come = held[r] + s["path"].long()[rows[r] + i]
    return held, (table[r, come // B], come % B), (table[r, to // B], to % B)


def _keep(s):
    B, table = s["case"]["block"], s["table"].long()
    held, (sp, sr), (dp, dr) = _moves(s)
    counts = s["counts"].long()
    codes, scales = s["codes"].flatten(0, 1), s["scales"].flatten(0, 1)         # [2 L, P, ..]
    # rows that lie before the first kept one in its page
    first = table[torch.arange(len(held), device=held.device), held // B]
    begin = torch.where(counts > 0, held % B, 0)
    old = scales[:, first]
    grown = torch.zeros_like(scales).index_reduce_(1, dp, scales[:, sp], "amax")
    part = torch.zeros_like(scales).index_reduce_(1, first, old * (begin > 0)[:, None], "amax")
    touched = torch.zeros_like(scales[:1, :, :1]).index_fill_(1, dp, 1.0)
    now = torch.where(touched > 0, torch.maximum(grown, part), scales)
    was = _at(codes, first)                                                     # [2 L, n, H, B, d]
    stays = torch.arange(B, device=held.device)[None, :, None] < begin[:, None, None]
    again = torch.where(stays[:, None], was * (old / now[:, first])[..., None, None], was).to(codes.dtype)
    raw = codes.view(torch.uint8)
    moved = raw[:, sp, :, sr].view(codes.dtype).float()                         # [kept, 2 L, H, d]
    moved = moved * (scales[:, sp] / now[:, dp]).transpose(0, 1)[..., None]
    raw[:, first] = again.view(torch.uint8)
    raw[:, dp, :, dr] = moved.to(codes.dtype).view(torch.uint8)
    scales.copy_(now)
    # pages behind the kept tokens
    lens = held + counts
    have, end = (lens + B - 1) // B, (s["lens"].long() + B - 1) // B
    j = have[:, None] + torch.arange(s["most"] + 1, device=held.device)[None]
    out = j < end[:, None]
    place = torch.where(out, torch.cumsum(out.flatten().long(), 0).view_as(out) - 1, len(s["freed"]))
    pages = table.gather(1, j.clamp(max=table.shape[1] - 1)).int()
    freed = torch.cat((s["freed"], s["freed"][:1])).scatter_(0, place.flatten(), pages.flatten())
    s["freed"].copy_(freed[:-1])
    return dict(codes=s["codes"], scales=s["scales"], lens=lens.int(), freed=s["freed"])


def _copy(s):
    src, dst, raw = s["src"].long(), s["dst"].long(), s["codes"].view(torch.uint8)
    raw[:, :, dst] = raw[:, :, src]
    s["scales"][:, :, dst] = s["scales"][:, :, src]
    return dict(codes=s["codes"], scales=s["scales"])


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    """rotate: every row read and written. attend: the visible codes and their scales, queries, outputs;
    two products of 2 d operations for each query head and (node, token of the context or itself).
    verify: the row of the last node of each request. keep: the codes of the nodes moved (the first
    stays). copy: pages read and written."""
    op, n = case["op"], case["n"]
    if op == "copy":
        return {"bytes": 4 * n * case["L"] * case["H"] * (case["block"] * case["d"] + 4), "flops": 0}
    held, new = _lengths(case)
    tokens = int(new.sum())
    e = 2 if case["dtype"] == "bfloat16" else 4
    if op == "verify":
        return {"bytes": n * case["V"] * e * (2 if case["sampled"] else 1) + 24 * tokens,
                "flops": n * case["V"] * (4 if case["sampled"] else 1)}
    H, d = case["H"], case["d"]
    if op == "rotate":
        rows = tokens * H * (case["G"] + 1)
        return {"bytes": 2 * rows * d * e + 4 * tokens, "flops": 8 * rows * d}
    if op == "keep":
        moved = int(np.maximum(np.minimum(_spread(case["kept"], n), int(new.max())) - 1, 0).sum())
        return {"bytes": 2 * max(moved, 1) * 2 * case["L"] * H * d + 12 * tokens, "flops": 0}
    w, B, Hq = case["window"], case["block"], H * case["G"]
    seen = np.minimum(held, w) if w else held               # of the context, by the request's first node
    keys = int((seen + new).sum())
    pairs = int((new * (seen + 1)).sum())
    return {"bytes": 2 * H * d * keys + 8 * H * -(-keys // B) + 4 * -(-keys // B)
            + tokens * (Hq * (2 * e * d + 4) + 12),
            "flops": 4 * d * Hq * pairs}


# ------------------------------------------------------------------ the same in 64 bits

def exact(case, seed):
    op = case["op"]
    if op == "verify":
        return None                                         # whole numbers only
    s = prepare(case, seed)
    return {"rotate": _rotate_exact, "attend": _attend_exact, "keep": _keep_exact,
            "copy": _copy_exact}[op](s)


def _rotate_exact(s):
    case = s["case"]
    d = case["d"]
    half = torch.exp(torch.arange(d // 2, device="cuda").double() * (-2.0 / d * math.log(case["base"])))
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"),
                       s["positions"].double()[:, None, None] * half)
    out, begin = {}, 0
    for name, heads in (("q", case["H"] * case["G"]), ("k", case["H"])):
        x = s["x"][:, begin:begin + heads].double()
        begin += heads
        x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / d + _EPS) * s[name + "_weight"].double()
        if case["style"] == "half":
            z = torch.complex(x[..., :d // 2], x[..., d // 2:]) * turn
            out[name] = torch.cat((z.real, z.imag), -1)
        else:
            z = torch.complex(x[..., 0::2], x[..., 1::2]) * turn
            out[name] = torch.view_as_real(z).reshape(x.shape)
    return out


def _attend_exact(s):
    case = s["case"]
    rows, lens = s["rows"].tolist(), s["lens"].tolist()
    B, H, G, d, w, l = (case[k] for k in ("block", "H", "G", "d", "window", "L"))
    out = torch.zeros((s["tokens"], H * G, d), dtype=torch.float64, device="cuda")
    lse = torch.full((s["tokens"], H * G), -math.inf, dtype=torch.float64, device="cuda")
    for r, T in enumerate(lens):
        a, b = rows[r], rows[r + 1]
        held = T - (b - a)
        pages = s["table"][r, :-(-T // B)].long()
        hidden = torch.zeros((b - a, T), dtype=torch.bool, device="cuda")
        if w:
            t = torch.arange(held, device="cuda")
            hidden[:, :held] = t[None] + w <= s["positions"][a:b, None]
        for j in range(b - a):
            hidden[:, held + j] = (s["masks"][a:b, j // 64] >> (j % 64)) & 1 == 0
        for h in range(H):
            k, v = ((s["codes"][l, kv, :, h].view(torch.uint8)[pages].view(torch.float8_e4m3fn)
                     .double() * s["scales"][l, kv, pages, h].double()[:, None, None])
                    .reshape(-1, d)[:T] for kv in (0, 1))
            kt = k.t().contiguous()
            for j in range(h * G, (h + 1) * G):
                z = s["q"][a:b, j].double() @ kt / math.sqrt(d)
                z.masked_fill_(hidden, -math.inf)
                one = torch.logsumexp(z, -1)
                lse[a:b, j] = one
                out[a:b, j] = (z - one[:, None]).exp_() @ v
    return dict(out=out, lse=lse)


def _e4m3(y):
    """y (64 bits, within +-448) rounded to the nearest of float8_e4m3fn, ties to even: three bits
    after the leading one down to 2^-6, steps of 2^-9 below."""
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step


def _keep_exact(s):
    B = s["case"]["block"]
    codes, scales = s["codes"].flatten(0, 1).double(), s["scales"].flatten(0, 1).double()
    rows, lens, counts = (s[k].tolist() for k in ("rows", "lens", "counts"))
    table, path = s["table"].tolist(), s["path"].tolist()
    for r, T in enumerate(lens):
        held = T - (rows[r + 1] - rows[r])
        come = [held + path[rows[r] + i] for i in range(counts[r])]
        for j in range(held // B, -(-(held + counts[r]) // B) if counts[r] else 0):
            page = table[r][j]
            here = [i for i in range(counts[r]) if (held + i) // B == j]
            begin = (held + here[0]) % B
            from_pages = [table[r][come[i] // B] for i in here]
            new = scales[:, from_pages].amax(1)                                 # [2 L, H]
            if begin:
                new = torch.maximum(new, scales[:, page])
                codes[:, page, :, :begin] = _e4m3(codes[:, page, :, :begin]
                                                  * (scales[:, page] / new)[..., None, None])
            moved = [_e4m3(codes[:, p, :, come[i] % B] * (scales[:, p] / new)[..., None])
                     for i, p in zip(here, from_pages)]
            for i, x in zip(here, moved):
                codes[:, page, :, (held + i) % B] = x
            scales[:, page] = new
    return dict(codes=codes.view(s["codes"].shape), scales=scales.view(s["scales"].shape), lens=None,
                freed=None)


def _copy_exact(s):
    codes, scales = s["codes"].double(), s["scales"].double()
    for a, b in zip(s["src"].tolist(), s["dst"].tolist()):
        codes[:, :, b], scales[:, :, b] = codes[:, :, a], scales[:, :, a]
    return dict(codes=codes, scales=scales)
