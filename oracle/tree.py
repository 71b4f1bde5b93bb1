"""Oracle of drafted tokens over a paged cache (test infrastructure only): the plain definitions, one sequence, token and page after the other, with numpy and fp64."""
from __future__ import annotations

import numpy as np


def fit(lengths, counts, page, table, held, free, free_count, tokens):
    """table (array), held and free (lists) are changed in place; returns (starts, new lengths, slots, positions, free_count)."""
    width, B = table.shape[1], len(lengths)
    lengths, counts = [max(0, int(n)) for n in lengths], [max(0, int(n)) for n in counts]
    new = [n + m for n, m in zip(lengths, counts)]
    want = [min(-(-n // page), width) for n in new]
    top = max(0, free_count)
    for b in reversed(range(B)):
        for e in reversed(range(want[b], held[b])):
            free[top] = int(table[b, e])
            top += 1
    for b in range(B):
        have = min(held[b], want[b])
        for e in range(held[b], want[b]):
            top -= 1
            table[b, e] = free[top] if top >= 0 else -1
            have += top >= 0
        held[b] = have
    starts, slots, positions = [0], [], []
    for b in range(B):
        for p in range(lengths[b], new[b]):
            e = p // page
            slots.append(int(table[b, e]) * page + p % page if e < held[b] and table[b, e] >= 0 else -1)
            positions.append(p)
        starts.append(len(slots))
    pad = max(0, tokens - len(slots))
    return starts, new, (slots + [-1] * pad)[:tokens], (positions + [0] * pad)[:tokens], top


def ancestors(parents, window=0):
    """Of each token of one tree: the numbers that its mask has (itself and its ancestors, `window` of them at most), and its depth."""
    seen, depths = [], []
    for i in range(len(parents)):
        chain, j = [], i
        while True:
            chain.append(j)
            p = int(parents[j])
            if not 0 <= p < j:
                break
            j = p
        seen.append(chain[:window] if window else chain)
        depths.append(len(chain) - 1)
    return seen, depths


def masks(seen, words):
    out = np.zeros((len(seen), words), np.uint64)
    for row, s in zip(out, seen):
        for j in s:
            if j < 64 * words:
                row[j // 64] |= np.uint64(1) << np.uint64(j % 64)
    return out.view(np.int64)


def attend(q, k, v, table, starts, lengths, mask, depths=None, window=0, scale=None):
    """q [tokens, query heads, size]; k, v [pages, page_size, heads, size] in fp64; mask int64 [tokens, words].  Returns the output, sum p |v| of each output, and for each row the
    largest sum of |scale q k| of a key that it sees."""
    q = np.asarray(q, np.float64)
    T, Hq, D = q.shape
    P, ps, H, _ = k.shape
    G = Hq // H
    scale = 1.0 / np.sqrt(D) if scale is None else scale
    bits = np.asarray(mask).view(np.uint64)
    out, size, peak = np.zeros((T, Hq, D)), np.zeros((T, Hq, D)), np.zeros((T, Hq, 1))
    for b in range(len(lengths)):
        s0, n, length = int(starts[b]), int(starts[b + 1] - starts[b]), max(0, int(lengths[b]))
        past = length - n
        for i in range(n):
            t = s0 + i
            lo = max(0, past + min(max(0, int(depths[t])), n - 1) - window + 1) if window else 0
            at = list(range(lo, max(lo, past)))
            at += [past + j for j in range(min(n, 64 * bits.shape[1])) if past + j >= 0 and (int(bits[t, j // 64]) >> (j % 64)) & 1]
            if not at:
                continue
            at = np.array(at)
            entry = at // ps
            page = np.where(entry < table.shape[1], table[b, np.minimum(entry, table.shape[1] - 1)] if table.shape[1] else -1, -1)
            if ((page < 0) | (page >= P)).any():
                out[t] = np.nan
                continue
            kk, vv = k[page, at % ps], v[page, at % ps]                           # [keys, heads, size]
            for h in range(Hq):
                z = (kk[:, h // G] @ q[t, h]) * scale
                peak[t, h] = (np.abs(kk[:, h // G][np.isfinite(z)]) @ np.abs(q[t, h])).max(initial=0.0) * abs(scale)
                top = z.max()
                if top == -np.inf:
                    continue
                p = np.exp(z - top)
                p /= p.sum()
                with np.errstate(invalid="ignore"):
                    out[t, h] = p @ vv[:, h // G]
                    size[t, h] = p @ np.abs(vv[:, h // G])
    return out, size, peak


def _weights(row):
    row = np.asarray(row, np.float64)
    return np.where(np.isfinite(row) & (row > 0), row, 0.0)


def verify(target, draft, ids, parents, starts, uniform, last, room):
    """target, draft [tokens, vocabulary] (fp64 arrays, draft or None).  Returns (paths, accepted, next)."""
    paths, accepted, following = [], [], []
    V = target.shape[1]
    for b in range(len(last)):
        s, n = int(starts[b]), int(starts[b + 1] - starts[b])
        if n == 0:
            paths.append([-1] * room)
            accepted.append(0)
            following.append(-1)
            continue
        path, w, m, walking = [0], _weights(target[s]), 1.0, True
        while walking and len(path) < room:
            walking, tried = False, 0
            node = path[-1]
            q = None if draft is None else _weights(draft[s + node])
            for i in range(node + 1, n):
                x = int(ids[s + i])
                if parents[s + i] != node or not 0 <= x < V:
                    continue
                if tried == 64:
                    break
                if float(uniform[s + i]) * (1.0 if q is None else q[x]) * m < w[x]:
                    path.append(i)
                    w, m, walking = _weights(target[s + i]), 1.0, True
                    break
                tried += 1
                if q is None:
                    m = max(0.0, m - w[x])
                    w[x] = 0.0
                else:
                    w = np.maximum(w / m - q, 0.0) if m > 0 else np.zeros(V)
                    m = w.sum()
        if not w.sum() > 0:
            w = _weights(target[s + path[-1]])
        total = w.sum()
        if total > 0:
            above = np.nonzero(np.cumsum(w) > float(last[b]) * total)[0]
            following.append(int(above[0]) if len(above) else int(np.nonzero(w)[0][-1]))
        else:
            following.append(-1)
        accepted.append(len(path))
        paths.append(path + [-1] * (room - len(path)))
    return paths, accepted, following


def compact(cache, table, lengths, path, accepted):
    """cache: an array [pages, page_size, ...], changed in place."""
    P, ps = cache.shape[:2]

    def place(b, p):
        e = p // ps
        page = int(table[b, e]) if p >= 0 and e < table.shape[1] else -1
        return (page, p % ps) if 0 <= page < P else None
    for b in range(len(lengths)):
        past = int(lengths[b]) - int(accepted[b])
        moves = [(place(b, past + int(path[b, i])), place(b, past + i)) for i in range(min(int(accepted[b]), path.shape[1])) if path[b, i] > i]
        held = [(cache[f].copy(), t) for f, t in moves if f is not None and t is not None]
        for x, t in held:
            cache[t] = x
