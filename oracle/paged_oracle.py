"""Plain 64-bit definition of the paged cache's operators (include/kvx.h: kv_paged_append, kv_paged_attend, kv_paged_evict),
one sequence, one head and one row at a time, on numpy arrays.  Test infrastructure: the product never calls it.

A pool is a dict: k, v [pages, slots, heads, d] (values as they are stored), table [sequences, entries], and where they are
kept weights and ids [pages, heads, slots].  Page numbers outside the pool hold no tokens.
"""
from __future__ import annotations

import numpy as np


def rope_frequencies(rotary, scaling="plain", base=10000.0, factor=1.0, original=0, low=1.0, high=4.0):
    """Radians per position of each pair."""
    w = []
    for i in range(rotary // 2):
        b = base * factor ** (rotary / (rotary - 2)) if scaling == "base" else base
        x = b ** (-2.0 * i / rotary)
        if scaling == "linear":
            x /= factor
        elif scaling == "parts":
            turns = original * x / (2 * np.pi)
            if turns <= low:
                x /= factor
            elif turns < high:
                t = (turns - low) / (high - low)
                x = (1 - t) * x / factor + t * x
        w.append(x)
    return np.array(w, np.float64)


def rotate(x, positions, freqs, interleaved, magnitude=1.0):
    """x [n, heads, d] with its first 2 len(freqs) channels turned by positions [n]."""
    x = np.asarray(x, np.float64)
    y, r = x.copy(), len(freqs)
    for i in range(r):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + r)
        angle = np.asarray(positions, np.float64) * freqs[i]
        c, s = (magnitude * np.cos(angle))[:, None], (magnitude * np.sin(angle))[:, None]
        y[:, :, a] = x[:, :, a] * c - x[:, :, b] * s
        y[:, :, b] = x[:, :, b] * c + x[:, :, a] * s
    return y


def place(pool, seq, j):
    """(page, slot) of cached token j of a sequence; None where its page is outside the pool."""
    size = pool["k"].shape[1]
    page = int(pool["table"][seq, j // size])
    return (page, j % size) if 0 <= page < pool["k"].shape[0] else None


def attend(pool, q, start, lens, scale, causal=True, window=0, k_scale=None, v_scale=None):
    """out, lse, weights gained [pages, heads, slots], and the sums of |p v| and |q||k| that error bounds go by."""
    q = np.asarray(q, np.float64)
    n_rows, hq, d = q.shape
    n_pages, size, hkv, _ = pool["k"].shape
    group = hq // hkv
    ks = np.ones(hkv) if k_scale is None else np.asarray(k_scale, np.float64)
    vs = np.ones(hkv) if v_scale is None else np.asarray(v_scale, np.float64)
    out, absolute = np.zeros((n_rows, hq, d)), np.zeros((n_rows, hq, d))
    lse, reach = np.full((n_rows, hq), -np.inf), np.zeros((n_rows, hq))
    gained = np.zeros((n_pages, hkv, size))
    for b in range(len(lens)):
        new, length = int(start[b + 1] - start[b]), int(lens[b])
        places = [place(pool, b, j) for j in range(length)]
        there = np.array([p is not None for p in places], bool)
        pg = np.array([p[0] if p else 0 for p in places], np.int64)
        sl = np.array([p[1] if p else 0 for p in places], np.int64)
        for h in range(hkv):
            k, v = pool["k"][pg, sl, h].astype(np.float64) * ks[h], pool["v"][pg, sl, h].astype(np.float64) * vs[h]
            for i in range(new):
                at = length - new + i
                j = np.arange(length)
                see = there & ((j <= at) if causal else True) & ((j > at - window) if window else True)
                if not see.any():
                    continue
                for g in range(h * group, (h + 1) * group):
                    row = start[b] + i
                    z = scale * (k[see] @ q[row, g])
                    with np.errstate(invalid="ignore"):
                        top = z.max()
                        e = np.exp(z - top)
                        total = e.sum()
                        p = e / total
                    out[row, g], absolute[row, g] = p @ v[see], p @ np.abs(v[see])
                    lse[row, g] = top + np.log(total)
                    reach[row, g] = scale * (np.abs(k[see]) @ np.abs(q[row, g])).max()
                    np.add.at(gained, (pg[see], h, sl[see]), p)
    return out, lse, gained, absolute, reach


def evict(pool, lens, seen, budget, sinks, recent):
    """Moves made on copies: k, v, weights, ids and the new lengths; also which slots of weights and ids the call writes."""
    k, v, w, ids = (pool[n].copy() for n in ("k", "v", "weights", "ids"))
    hkv = k.shape[2]
    written = np.zeros(w.shape, bool)
    for b in range(len(lens)):
        length = int(lens[b])
        for h in range(hkv):
            where = [place(pool, b, j) for j in range(length)]
            rank = []
            for j, p in enumerate(where):
                if p is None:
                    rank.append((3, 0.0))
                    continue
                token, weight = int(ids[p[0], h, p[1]]), float(w[p[0], h, p[1]])
                if token < sinks or token >= int(seen[b]) - recent:
                    rank.append((0, 0.0))
                elif np.isnan(weight):
                    rank.append((2, 0.0))
                else:
                    rank.append((1, -weight))
            order = sorted(range(length), key=lambda j: (rank[j], j))
            stay = set(order[:budget])
            holes = [j for j in range(min(budget, length)) if j not in stay]
            movers = [j for j in range(budget, length) if j in stay]
            for src, dst in zip(movers, holes):
                a, c = where[src], where[dst]
                if a is None or c is None:
                    continue
                for x in (k, v):
                    x[c[0], c[1], h] = x[a[0], a[1], h]
                for x in (w, ids):
                    x[c[0], h, c[1]] = x[a[0], h, a[1]]
            for j in range(min(budget, length)):
                if where[j] is not None:
                    written[where[j][0], h, where[j][1]] = True
    return k, v, w, ids, np.minimum(np.asarray(lens), budget), written
