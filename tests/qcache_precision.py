"""How many bits the 8-bit cache's attention holds: tolerances that follow the roundings of its
arithmetic where the errors of different tokens are independent, inputs that make them add up, and
the same attention in 64 bits with an arithmetic of the caller's for the weights, queries and values.

A row's output is sum_j w_j v_j with weights w_j that are off by factors 1 + e_j, |e_j| <= eps, which
for values of either sign adds up to at most about eps * S, S = (sum_j w_j^2 v_j^2)^(1/2), in the
mean square over a head's columns. eps is made of
  2^-21                 exp2, the sums of the waves and the final quotient, two units each
  2^-23 Y               the score: products are exact, their sum, the scale's factor and the
                        maximum's subtraction are rounded in fp32;
                        Y = max_j |x_j| + |scale| (sum_i q_i^2 k_ij^2)^(1/2)
  2^-24 (3 T / 16)^(1/2) the sums over T tokens, 16 and one of three terms at a time, at most 2048 in
                        a row (longer contexts are cut)
  2^-18                 for bf16 queries, whose weights are two bf16 terms (2^-9 of 2^-9)
and rounding the output to its type then changes the error by at most twice as much, on top of
what rounding the exact output costs: |round(o + e) - o| <= |round(o) - o| + 2 |e|."""

import math

import torch

from qcache_ref import E4M3


def terms(x, n):
    """x as n bf16 terms, each the rounding of what the ones before have left."""
    total, rest = torch.zeros_like(x), x
    for _ in range(n):
        t = rest.to(torch.bfloat16).to(x.dtype)
        total, rest = total + t, rest - t
    return total


def attend(q, codes, scales, table, lens, counts, window=0, scale=None, weights=None,
           values=None):
    """(out, lse, S, Y), each row's attention in 64 bits: q [R, Hq, d], codes [2, P, H, B, d] uint8,
    scales [2, P, H], table [n, width] of pages that are all there. weights, values: what becomes
    of exp(x - max), [rows, heads, T], in the products with the values, and of these, [H, T, d]."""
    dev = q.device
    lut = torch.tensor(E4M3, device=dev)
    q = q.double()
    R, Hq, d = q.shape
    H, B = codes.shape[2:4]
    G = Hq // H
    scale = d ** -0.5 if scale is None else scale
    out = torch.zeros((R, Hq, d), dtype=torch.float64, device=dev)
    lse = torch.full((R, Hq), -math.inf, dtype=torch.float64, device=dev)
    S, Y = torch.zeros_like(lse), torch.zeros_like(lse)
    at = 0
    for r, (T, count) in enumerate(zip(lens, counts)):
        if T < 1 or count < 1:
            at += count
            continue
        pages = torch.as_tensor(table[r][:-(-T // B)], dtype=torch.long, device=dev)
        k, v = ((lut[codes[w, pages].long()] * scales[w, pages].double()[:, :, None, None])
                .transpose(0, 1).reshape(H, -1, d)[:, :T] for w in (0, 1))
        if values is not None:
            v = values(v)
        p = T - count + torch.arange(count, device=dev)
        t = torch.arange(T, device=dev)
        hidden = t[None] > p[:, None]
        if window:
            hidden |= t[None] <= p[:, None] - window
        for h in range(H):
            qq = q[at:at + count, h * G:(h + 1) * G].reshape(count * G, d)
            gone = hidden.repeat_interleave(G, 0)
            kt = k[h].t().contiguous()
            x = (qq @ kt * scale).masked_fill(gone, -math.inf)
            top = x.amax(1, keepdim=True)
            low = torch.where(top == -math.inf, 0.0, top)
            e = torch.exp(x - low)
            l = e.sum(1, keepdim=True)
            here = slice(at, at + count), slice(h * G, (h + 1) * G)
            norm = ((qq ** 2) @ (kt ** 2)).sqrt() * abs(scale)
            whole = torch.where(l == 0, 1.0, l)
            w = (e if weights is None else weights(e)) / whole
            out[here] = (w @ v[h]).view(count, G, d)
            lse[here] = (l.log() + low).view(count, G)
            S[here] = ((w ** 2) @ (v[h] ** 2).mean(1, keepdim=True)).sqrt().view(count, G)
            Y[here] = (x.abs() + norm).masked_fill(gone, 0.0).amax(1).view(count, G)
        at += count
    return out, lse, S, Y


def allowed(dtype, T, out, lse, S, Y):
    """(root mean square over a head's columns of the output's error, largest error of lse)."""
    eps = 2.0 ** -21 + 2.0 ** -23 * Y + 2.0 ** -24 * min(3 * T / 16, 2048) ** 0.5
    if dtype is torch.bfloat16:
        eps = eps + 2.0 ** -18
    own = (out.to(dtype).double() - out).pow(2).mean(-1).sqrt()
    return (own + 2 * eps * S,
            2.0 ** -21 + 2.0 ** -23 * (Y + lse.abs() + math.log2(T)))


def check(got, dtype, T, out, lse, S, Y):
    """The worst of the errors relative to what is allowed: (of the output, of lse)."""
    bo, bl = allowed(dtype, T, out, lse, S, Y)
    none = lse == -math.inf
    far = (got[0].double() - out).pow(2).mean(-1).sqrt()
    assert torch.equal(got[1] == -math.inf, none) and bool((got[0][none] == 0).all())
    if bool(none.all()):
        return 0.0, 0.0
    return (float((far / bo)[~none].max()),
            float(((got[1].double() - lse).abs() / bl)[~none].max()))


# ------------------------------------------------------------------ errors that add up
#
# Rows of equal elements a over keys of equal codes: every score is the same multiple of a, and the
# logarithm of the sum is that score, so what is lost of a is lost of it: a third term dropped
# is up to 2^-18 of it, about 2^-18.3 at the worst of 64 rows. And values that are all
# equal: the output is that value if the weights in the products are those in their sum; a third
# term dropped of the weights costs it as much. Three terms hold 2^-27, the sums of fp32 of such
# numbers some 2^-22.
LINED_UP = 2.0 ** -20


def lined_up(d, rows, seed):
    """(rows [rows] of fp32 in 1 .. 2, their multiples of a score)."""
    g = torch.Generator().manual_seed(seed)
    return 1 + torch.rand(rows, generator=g)
