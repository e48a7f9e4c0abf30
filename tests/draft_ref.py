"""The operators of drafted decoding in 64 bits, written from their definitions with loops over
requests, nodes and pages; nothing here comes from the library."""

import math

import numpy as np
import torch

import qcache_ref as ref


def ancestors(parents):
    """Of each node of one request the nodes above it and itself."""
    out = []
    for i, p in enumerate(parents):
        out.append((out[p] if p >= 0 else set()) | {i})
    return out


def tree(parents, held, window=0):
    """(sets of the nodes that each node sees, positions)."""
    up = ancestors(parents)
    depth = [len(a) - 1 for a in up]
    sees = [{j for j in a if not window or depth[i] - depth[j] < window} for i, a in enumerate(up)]
    return sees, [held + e for e in depth]


def random_tree(rng, c, branch):
    children, parents = [0] * c, []
    for i in range(c):
        if i == 0:
            parents.append(-1)
            continue
        room = [j for j in range(i) if children[j] < branch]
        p = int(room[rng.integers(max(0, len(room) - 2 * branch), len(room))])
        children[p] += 1
        parents.append(p)
    return parents


def norm_rotate(x, positions, base, style, weight=None, eps=1e-6):
    """y of x [T, heads, d] (double, CPU) and, for the bounds, |y_a| + |y_b| of each element's pair."""
    T, _, d = x.shape
    if weight is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * weight
    out, size = torch.empty_like(x), torch.empty_like(x)
    for i in range(d // 2):
        a, b = (i, i + d // 2) if style == "half" else (2 * i, 2 * i + 1)
        angle = [math.fmod(int(p) * base ** (-2.0 * i / d), 2 * math.pi) for p in positions]
        c = torch.tensor([math.cos(t) for t in angle], dtype=torch.float64)[:, None]
        s = torch.tensor([math.sin(t) for t in angle], dtype=torch.float64)[:, None]
        out[..., a] = x[..., a] * c - x[..., b] * s
        out[..., b] = x[..., b] * c + x[..., a] * s
        size[..., a] = size[..., b] = x[..., a].abs() + x[..., b].abs()
    return out, size


def norm_rotate_bound(dtype, out, size, positions, normed):
    """How far the kernel's arithmetic may be off. In units of 2^-24 of a value: the sum of squares is
    of at most 256 products of fp32, added by at most 16 in a lane and 5 across lanes, so off by 21,
    its root's part 10.5; root, division, product with the mean's factor and eps 3; two products 2:
    16 in all. Sine and cosine are of an angle in half turns of at most 1, rounded once (2^-25 of it,
    so pi 2^-25), by a function within 4 units, with two products and a sum: 9. The angle in fp64 is off by
    at most four roundings of the position times at most 1, in turns: 2 pi 2^-51 |p|, here twice that.
    bf16 rounds once more, by 2^-8."""
    p = torch.tensor([abs(int(x)) for x in positions], dtype=torch.float64)[:, None, None]
    off = size * ((16 if normed else 0) * 2.0 ** -24 + 9 * 2.0 ** -24 + p * 2.0 ** -47)
    if dtype == torch.bfloat16:
        off = off + 2.0 ** -8 * (out.abs() + off)
    return off * 1.001 + 1e-37


def clean(x):
    x = np.asarray(x, dtype=np.float64)
    return np.where(np.isfinite(x) & (x > 0), x, 0.0)


def verify(probs, drafts, parents, rows, accept, sample, draft_probs=None):
    """(path, counts, tokens), lists: a walk through each request's tree with r as a whole row."""
    path, counts, tokens = [], [], []
    V = probs.shape[1]
    for a, b, s in zip(rows[:-1], rows[1:], sample):
        if b == a:
            counts.append(0)
            tokens.append(-1)
            continue
        node, kept = 0, []
        while True:
            kept.append(node)
            p = clean(probs[a + node])
            q = None if draft_probs is None else clean(draft_probs[a + node])
            r, m, taken = p.copy(), 1.0, None
            for x in range(node + 1, b - a):
                if parents[a + x] != node:
                    continue
                t, u = int(drafts[a + x]), float(accept[a + x])
                here = 0 <= t < V
                rt = r[t] if here else 0.0
                if q is None:
                    if u * m < rt:
                        taken = x
                        break
                    m -= rt
                    if here:
                        r[t] = 0.0
                else:
                    if u * (q[t] if here else 0.0) * m < rt:
                        taken = x
                        break
                    r = np.maximum(r - m * q, 0.0)
                    m = math.fsum(r)
            if taken is None:
                break
            node = taken
        if not r.any():
            r = p
        sums = np.cumsum(r)
        over = np.nonzero((sums > float(s) * sums[-1]) & (r > 0))[0]
        some = np.nonzero(r)[0]
        tokens.append(int(over[0]) if len(over) else int(some[-1]) if len(some) else -1)
        counts.append(len(kept))
        path += kept + [-1] * (b - a - len(kept))
    return path, counts, tokens


def keep(codes, scales, table, lens, rows, path, counts):
    """codes [L, 2, P, H, B, d] uint8 and scales [L, 2, P, H] float32 in place; (lengths, pages
    freed)."""
    L, _, P, H, B, d = codes.shape
    out, freed = [], []
    for r, T in enumerate(lens):
        a, c = rows[r], rows[r + 1] - rows[r]
        held = T - c
        come = [held + path[a + i] for i in range(counts[r])]
        for l in range(L):
            for w in range(2):
                for h in range(H):
                    code, scale = codes[l, w, :, h], scales[l, w, :, h]
                    old = {p: (code[p].copy(), np.float32(scale[p])) for p in set(int(x) for x in table[r] if 0 <= x < P)}
                    i = 0
                    while i < counts[r]:
                        j = (held + i) // B
                        n = min(counts[r], (j + 1) * B - held) - i
                        page, begin = int(table[r][j]), (held + i) % B
                        if 0 <= page < P:
                            src = [int(table[r][come[i + k] // B]) for k in range(n)]
                            good = [k for k in range(n) if 0 <= src[k] < P]
                            new = max([old[src[k]][1] for k in good] + ([old[page][1]] if begin or len(good) < n else []))
                            if begin and new != old[page][1]:
                                code[page, :begin] = scaled(old[page][0][:begin], old[page][1], new)
                            for k in good:
                                was, s = old[src[k]]
                                code[page, begin + k] = scaled(was[come[i + k] % B], s, new)
                            scale[page] = new
                        i += n
        out.append(held + counts[r])
        freed += [int(table[r][j]) for j in range(-(-out[-1] // B), min(-(-T // B), len(table[r])))]
    return out, freed


def scaled(codes, old, new):
    """Codes times old / new, the ratio and the products in fp32, rounded again."""
    if old == new:
        return codes
    return ref.encode((ref.E4M3[codes].astype(np.float32) * np.float32(old / new)).astype(np.float64))


def attend(q, codes, scales, table, lens, rows, sees, positions, window=0, scale=None, device="cpu"):
    """out, lse and, for the bounds, A and X as qcache_ref.attend: row i of a request of c nodes sees its
    context (the places before lens - c) and the nodes in sees[i]."""
    lut = torch.tensor(ref.E4M3, device=device)
    q = torch.as_tensor(q, dtype=torch.float64, device=device)
    codes = torch.as_tensor(codes, device=device)
    scales = torch.as_tensor(scales, device=device).double()
    R, Hq, d = q.shape
    _, P, H, B, _ = codes.shape
    G = Hq // H
    scale = d ** -0.5 if scale is None else scale
    out = torch.zeros((R, Hq, d), dtype=torch.float64, device=device)
    lse = torch.full((R, Hq), -math.inf, dtype=torch.float64, device=device)
    A, X = torch.zeros_like(out), torch.zeros_like(lse)
    for r, T in enumerate(lens):
        T = min(max(T, 0), table.shape[1] * B)
        a, c = rows[r], rows[r + 1] - rows[r]
        ids = [int(p) for p in table[r][:-(-T // B)]]
        there = torch.tensor([0 <= p < P for p in ids for _ in range(B)], dtype=torch.bool,
                             device=device)[:T]
        idx = torch.tensor([p if 0 <= p < P else 0 for p in ids], dtype=torch.long, device=device)
        t = torch.arange(T, device=device)
        see = torch.zeros((c, T), dtype=torch.bool, device=device)
        for i in range(c):
            see[i] = t < T - c
            if window:
                see[i] &= t > positions[a + i] - window
            for j in sees[a + i]:
                if 0 <= T - c + j < T:
                    see[i, T - c + j] = True
        see &= there
        for h in range(H):
            k, v = (((lut[codes[w, idx, h].long()] * scales[w, idx, h][:, None, None]).reshape(-1, d)[:T])
                    for w in (0, 1))
            for i in range(c):
                if not bool(see[i].any()):
                    continue
                kk, vv = k[see[i]], v[see[i]]
                for j in range(h * G, (h + 1) * G):
                    qq = q[a + i, j]
                    x = (kk @ qq) * scale
                    one = torch.logsumexp(x, 0)
                    e = torch.exp(x - one)
                    out[a + i, j], lse[a + i, j] = e @ vv, one
                    A[a + i, j] = e @ vv.abs()
                    X[a + i, j] = (kk.abs() @ qq.abs()).max() * abs(scale)
    return out, lse, A, X


def attend_bounds(dtype, d, T, out, A, X):
    """(largest |error| of out, of lse) that the kernel's arithmetic allows, from its roundings.

    A score is a sum of d products in fp32 (exact products, d additions, a factor and the running
    exponent's subtraction): off by at most e = (d + 8) 2^-24 X. Weights and their sum then by
    2 e + 2^-21 (an exp2 within two units, twice) + T 2^-24 for T additions, scaled by the joins of at most
    some hundred parts (2^-17 in all). Weights enter as two bf16 terms for bf16 queries, the
    rest after which is at most 2^-8 of 2^-8, as three for fp32 ones (2^-24); the output is
    rounded once (2^-8, 2^-24)."""
    e = (d + 8) * 2.0 ** -24 * X
    p = (2 * e + 2.0 ** -21 + T * 2.0 ** -24 + 2.0 ** -17)[..., None]
    w, r = (2.0 ** -16, 2.0 ** -8) if dtype == torch.bfloat16 else (2.0 ** -24, 2.0 ** -24)
    off = (p + w) * A * 1.01
    return off + r * (out.abs() + off) + 1e-30, e + 2.0 ** -17 + 2.0 ** -22 * X
