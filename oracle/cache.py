"""Rotary positions, the 8-bit paged cache of keys and values and attention over it, in plain numpy.  TEST INFRASTRUCTURE ONLY
(see ops.py).  Pages hold the numbers that codes stand for, before their scale; keys [pages, heads, page, dh], values [pages, heads, dh, page]."""
from __future__ import annotations

import numpy as np


# ----------------------------------------------------------------------------- rotary positions
def rotary(x, pos, freq, rot, interleaved, scale=1.0, backward=False):
    """x [rows, heads, dh]; the first `rot` columns of every head are turned."""
    y = x.copy()
    angle = np.asarray(pos, np.float64)[:, None] * freq * (-1 if backward else 1)
    cos, sin = scale * np.cos(angle)[:, None], scale * np.sin(angle)[:, None]
    one, two = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    y[..., one], y[..., two] = x[..., one] * cos - x[..., two] * sin, x[..., one] * sin + x[..., two] * cos
    return y


def rotary_frequencies(rot, base, factor, low, high, context):
    out = []
    for i in range(rot // 2):
        f = base ** (-2.0 * i / rot)
        turns = context * f / (2 * np.pi)
        kept = 1.0 if turns >= high else 0.0 if turns <= low else (turns - low) / (high - low)
        out.append(kept * f + (1 - kept) * f / factor)
    return np.array(out)


# ----------------------------------------------------------------------------- the cache
def e4m3(x):
    """The nearest of the numbers +-m 2^e, m of 4 bits, that e4m3 holds (|x| up to 448; 2^-9 the smallest), ties to even."""
    x = np.asarray(x, np.float64)
    with np.errstate(divide="ignore", invalid="ignore"):
        step = np.exp2(np.maximum(np.floor(np.log2(np.abs(x))), -6.0) - 3.0)
        return np.where(x == 0, x, np.rint(x / step) * step)


def scale_for(most):
    """The least power of two s, 2^-126 or more, with most / s <= 448."""
    if most == 0:
        return 2.0 ** -126
    s = 2.0 ** np.floor(np.log2(most / 448.0))
    return max(s if most / s <= 448 else 2 * s, 2.0 ** -126)


def sequences(starts, lens, B, T, rows, most):
    """(first row, new rows, length) of every sequence."""
    out = []
    for b in range(B):
        lo, hi = (b * T, b * T + T) if starts is None else (int(starts[b]), int(starts[b + 1]))
        if not (0 <= lo <= hi <= rows and hi - lo <= T):
            lo = hi = 0
        out.append((lo, hi - lo, min(max(int(lens[b]), 0), most)))
    return out


def _page(table, pages, b, pos, P):
    p = table[b, pos // P] if pos >= 0 else -1
    return int(p) if 0 <= p < pages else -1


def append(x, pool, scale, values, seqs, table):
    """Rows x [rows, heads, dh] of one side into its pages, in place."""
    heads, P = pool.shape[1], pool.shape[3 if values else 2]
    side = pool.transpose(0, 1, 3, 2) if values else pool               # a view: [pages, heads, page, dh]
    for b, (first, n, length) in enumerate(seqs):
        for slot in range((length - n) // P, -(-length // P)):
            lo, hi = max(0, length - n - slot * P), min(P, length - slot * P)
            p = _page(table, pool.shape[0], b, slot * P, P)
            if p < 0:
                continue
            new = x[first + slot * P + lo - (length - n):][:hi - lo].astype(np.float64)
            new = np.where(np.isfinite(new), new, np.nan)
            for h in range(heads):
                part = new[:, h]
                need = scale_for(np.nanmax(np.abs(part)) if np.isfinite(part).any() else 0.0)
                s = max(scale[p, h], need) if lo > 0 else need
                if lo > 0 and s > scale[p, h]:
                    side[p, h, :lo] = e4m3(side[p, h, :lo] * (scale[p, h] / s))
                side[p, h, lo:hi] = e4m3(part / s)
                scale[p, h] = s


def token(pool, scale, values, p, at):
    """[heads, dh] of one token of a page."""
    t = pool[p, :, :, at] if values else pool[p, :, at]
    return t * scale[p][:, None]


def read(pool, scale, values, seqs, table, rows):
    """Rows [rows, heads, dh] of the sequences' last positions (zeros in all others)."""
    heads, P, dh = pool.shape[1], pool.shape[3 if values else 2], pool.shape[2 if values else 3]
    out = np.zeros((rows, heads, dh))
    for b, (first, n, length) in enumerate(seqs):
        for t in range(n):
            pos = length - n + t
            p = _page(table, pool.shape[0], b, pos, P)
            if p >= 0:
                out[first + t] = token(pool, scale, values, p, pos % P)
    return out


def attention(q, kpool, vpool, kscale, vscale, seqs, table, causal):
    """q [rows, heads, dh].  Returns o, lse [rows, heads], and for error bounds the largest sum of |q_i k_i| dh^-1/2 of a row and the weighted sum of |v|;
    rows of no sequence are NaN."""
    rows, H, dh = q.shape
    Hkv, P = kpool.shape[1], kpool.shape[2]
    G = H // Hkv
    o, lse = np.full((rows, H, dh), np.nan), np.full((rows, H), np.nan)
    size, mass = np.zeros((rows, H)), np.zeros((rows, H, dh))
    for b, (first, n, length) in enumerate(seqs):
        where = [(pos, _page(table, kpool.shape[0], b, pos, P)) for pos in range(length)]
        where = [(pos, p) for pos, p in where if p >= 0]
        pos = np.array([w[0] for w in where], int)
        k = np.array([token(kpool, kscale, False, p, at % P) for at, p in where]).reshape(-1, Hkv, dh)
        v = np.array([token(vpool, vscale, True, p, at % P) for at, p in where]).reshape(-1, Hkv, dh)
        for t in range(n):
            seen = pos <= length - n + t if causal else pos < length
            for h in range(H):
                r, kk, vv = first + t, k[seen, h // G], v[seen, h // G]
                if not seen.any():
                    o[r, h], lse[r, h] = 0.0, -np.inf
                    continue
                s = kk @ q[r, h] / np.sqrt(dh)
                top = s.max()
                w = np.exp(s - top)
                o[r, h] = w @ vv / w.sum()
                lse[r, h] = top + np.log(w.sum())
                size[r, h] = (np.abs(kk) @ np.abs(q[r, h])).max() / np.sqrt(dh)
                mass[r, h] = w @ np.abs(vv) / w.sum()
    return o, lse, size, mass
