"""fp64 oracle of the paged key / value cache (test infrastructure only): the plain definitions, position by position, with numpy.

quantise: scale = max |x| / L (L = 448 for e4m3, 127 for int8) rounded up to twelve significant bits, at least 2^-100; the code is the representable
value nearest to the real quotient x / scale, the even one of two.  A row with an infinity or NaN: scale NaN, codes 0.

attend: O[t, h] = sum_j softmax_j(scale <q[t, h], K_j>) V_j over the positions that the token sees; zeros where it sees none.
"""
from __future__ import annotations

import numpy as np

LARGEST = {"e4m3": 448.0, "i8": 127.0}
# the non-negative values of e4m3: 2^-9 steps below 2^-6, then eight to an octave; the largest is 448
E4M3 = np.array([m * 2.0 ** -9 for m in range(8)] + [(8 + m) * 2.0 ** (e - 10) for e in range(1, 16) for m in range(8)][:-1])


def up12(x):
    """x > 0 rounded up to twelve significant bits."""
    m, e = np.frexp(x)
    return np.ldexp(np.ceil(m * 4096.0), e - 12)


def quantise(x, kind, dtype=None):
    """(values of the codes, scales) of the rows along the last axis; dtype "f16": the scale keeps L * scale, rounded to fp16, finite."""
    x = np.asarray(x, np.float64)
    top = np.abs(x).max(axis=-1)
    good = np.isfinite(top)
    s = np.maximum(up12(np.where(good, top, 1.0) / LARGEST[kind]), 2.0 ** -100)
    if dtype == "f16":
        grid = np.arange(2048, 4096) * {"e4m3": 2.0 ** -4, "i8": 2.0 ** -2}[kind]          # twelve bits, around the scale of the largest numbers
        s = np.minimum(s, grid[grid * LARGEST[kind] < 65520.0].max())
    y = np.where(good[..., None], x, 0.0) / s[..., None]
    if kind == "i8":
        return np.rint(y), np.where(good, s, np.nan)
    a = np.abs(y)
    above = np.clip(np.searchsorted(E4M3, a, side="left"), 1, len(E4M3) - 1)      # E4M3[above - 1] < a <= E4M3[above]
    lo, hi = E4M3[above - 1], E4M3[above]
    up = (a - lo > hi - a) | ((a - lo == hi - a) & (above % 2 == 0))              # (index = code: even codes win ties)
    return np.copysign(np.where(up, hi, lo), y), np.where(good, s, np.nan)


def attend(q, k, v, table, starts, lengths, scale=None, causal=True, window=0):
    """q [tokens, query heads, size]; k, v [pages, page_size, heads, size] in fp64.  Returns the output, for each output the sum of p |v| (what an
    error of the weights is relative to), and for each row its largest |score|; rows of no sequence are zeros."""
    q = np.asarray(q, np.float64)
    T, Hq, D = q.shape
    P, ps, H, _ = k.shape
    G = Hq // H
    scale = 1.0 / np.sqrt(D) if scale is None else scale
    out, size, peak = np.zeros((T, Hq, D)), np.zeros((T, Hq, D)), np.zeros((T, Hq, 1))
    for b in range(len(lengths)):
        s0, n, length = int(starts[b]), int(starts[b + 1] - starts[b]), max(0, int(lengths[b]))
        for i in range(n):
            pos = length - n + i
            hi = min(pos + 1, length) if causal else length
            lo = max(0, pos - window + 1) if window else 0
            if hi <= lo:
                continue
            at = np.arange(lo, hi)
            entry = at // ps
            page = np.array([table[b, e] if e < table.shape[1] else -1 for e in entry])
            if ((page < 0) | (page >= P)).any():
                out[s0 + i] = np.nan
                continue
            kk, vv = k[page, at % ps], v[page, at % ps]                           # [keys, heads, size]
            for h in range(Hq):
                z = (kk[:, h // G] @ q[s0 + i, h]) * scale
                top = z.max()
                if top == -np.inf:
                    continue
                p = np.exp(z - top)
                p /= p.sum()
                out[s0 + i, h] = p @ vv[:, h // G]
                size[s0 + i, h] = p @ np.abs(vv[:, h // G])
                peak[s0 + i, h] = np.abs(z[np.isfinite(z)]).max(initial=0.0)
    return out, size, peak
