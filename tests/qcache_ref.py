"""The 8-bit paged cache's operators in 64 bits, written from their definitions with
loops over requests, pages and heads (numpy for codes, torch double for products);
nothing here comes from the library."""

import math

import numpy as np
import torch


def e4m3_table():
    """Value of each of the 256 codes: 1 sign, 4 exponent (bias 7), 3 mantissa bits;
    S.1111.111 is NaN, there is no infinity."""
    out = np.empty(256)
    for c in range(256):
        s, e, m = c >> 7, (c >> 3) & 15, c & 7
        if e == 15 and m == 7:
            v = math.nan
        elif e == 0:
            v = m * 2.0 ** -9
        else:
            v = (1 + m / 8) * 2.0 ** (e - 7)
        out[c] = -v if s else v
    return out


E4M3 = e4m3_table()
_POS = E4M3[:127]                     # 0 .. 448, ascending


def encode(y):
    """Codes of values |y| <= 448 or NaN (numpy float64), nearest, ties to the even code."""
    y = np.asarray(y, dtype=np.float64)
    a = np.abs(y)
    nan = ~np.isfinite(y)
    a = np.where(nan, 0, a)
    hi = np.clip(np.searchsorted(_POS, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - _POS[lo], _POS[hi] - a
    code = np.where(dl < dh, lo, np.where(dh < dl, hi, np.where(lo % 2 == 0, lo, hi)))
    code = np.where(nan, 127, code)
    return (code + np.where(np.signbit(y), 128, 0)).astype(np.uint8)


def power_scale(amax):
    """The least 2^e, e >= -120, with amax <= 448 * 2^e."""
    e = -120
    while amax > 448 * 2.0 ** e:
        e += 1
    return 2.0 ** e


def tables(pages, block, held, new, free, table):
    """(table, slots, rows, lens, taken) of a step, or None where it has to be refused."""
    table = np.array(table)
    slots, rows, taken = [], [0], 0
    if min(held) < 0 or min(new) < 0:
        return None
    for r, (h, w) in enumerate(zip(held, new)):
        if -(-(h + w) // block) > table.shape[1]:
            return None
        for p in range(h, h + w):
            if p % block == 0:
                if taken >= len(free):
                    return None
                table[r, p // block] = free[taken]
                taken += 1
            page = int(table[r, p // block])
            slots.append(page * block + p % block if 0 <= page < pages else -1)
        rows.append(rows[-1] + w)
    return table, slots, rows, [h + w for h, w in zip(held, new)], taken


def write(codes, scales, x, slots):
    """codes [P, H, B, d] uint8, scales [P, H], rows x [T, H, d] (float64), in place."""
    P, H, B, d = codes.shape
    i = 0
    while i < len(slots):
        if not 0 <= slots[i] < P * B:
            i += 1
            continue
        j = i
        while j < len(slots) and 0 <= slots[j] < P * B and slots[j] // B == slots[i] // B:
            j += 1
        page, rows = slots[i] // B, [s % B for s in slots[i:j]]
        for h in range(H):
            y = x[i:j, h]
            fin = np.abs(y[np.isfinite(y)])
            s = power_scale(float(fin.max()) if fin.size else 0.0)
            if rows[0] > 0:
                old = float(scales[page, h])
                if s > old:
                    was = E4M3[codes[page, h, :rows[0]]]
                    codes[page, h, :rows[0]] = encode(was * (old / s))
                else:
                    s = old
            scales[page, h] = s
            codes[page, h, rows] = encode(y / s)
        i = j


def attend(q, codes, scales, table, lens, rows, window=0, scale=None, device="cpu"):
    """out, lse and, for the bounds, A = sum p |v| and X = the largest sum |q| |k| * scale of a row:
    q [R, Hq, d] float64, codes [2, P, H, B, d] uint8, scales [2, P, H]."""
    lut = torch.tensor(E4M3, device=device)
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
        count = rows[r + 1] - rows[r]
        nb = -(-T // B)
        ids = [int(p) for p in table[r][:nb]]
        there = torch.tensor([0 <= p < P for p in ids for _ in range(B)], dtype=torch.bool,
                             device=device)[:T]
        idx = torch.tensor([p if 0 <= p < P else 0 for p in ids], dtype=torch.long, device=device)
        t = torch.arange(T, device=device)
        for h in range(H):
            kv = []
            for w in (0, 1):
                x = lut[codes[w, idx, h].long()] * scales[w, idx, h][:, None, None]
                kv.append(x.reshape(-1, d)[:T])
            for i in range(count):
                p = T - count + i
                see = (t <= p) & there
                if window:
                    see &= t > p - window
                if not bool(see.any()):
                    continue
                k, v = kv[0][see], kv[1][see]
                for j in range(h * G, (h + 1) * G):
                    qq = q[rows[r] + i, j]
                    x = (k @ qq) * scale
                    one = torch.logsumexp(x, 0)
                    e = torch.exp(x - one)
                    out[rows[r] + i, j] = e @ v
                    lse[rows[r] + i, j] = one
                    A[rows[r] + i, j] = e @ v.abs()
                    X[rows[r] + i, j] = (k.abs() @ qq.abs()).max() * abs(scale)
    return out, lse, A, X


def attend_bounds(dtype, d, T, out, A, X):
    """(largest |error| of out, of lse) that the kernel's arithmetic allows, from its roundings.

    A score is a sum of d products of 24-bit and 4-bit numbers in fp32 (exact products, d
    additions, a factor and the running maximum's subtraction): off by at most
    e = (d + 8) 2^-24 X. Probabilities and their sum then by 2 e + 2^-21 (an exp2 within two
    units, twice) + T 2^-24 for T additions, scaled by the joins of at most some hundred parts
    (2^-17 in all). In bf16 a probability is rounded once to 8 bits (2^-9), and so is the output."""
    e = (d + 8) * 2.0 ** -24 * X
    p = 2 * e + 2.0 ** -21 + T * 2.0 ** -24 + 2.0 ** -17
    if dtype == torch.bfloat16:
        bound = (p[..., None] + 2.0 ** -9) * A * 1.01 + 2.0 ** -9 * (out.abs() + (p[..., None] + 2.0 ** -9) * A)
    else:
        bound = p[..., None] * A + 2.0 ** -24 * out.abs()
    return bound + 1e-30, e + 2.0 ** -17 + 2.0 ** -22 * X
