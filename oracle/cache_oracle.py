"""Plain NumPy fp64 oracle of the paged K/V cache (append, attention of new
tokens, accumulated weights, eviction), slot by slot from the definitions in
include/gmc.h.  Test infrastructure; shares no code with the HIP path.

A cache is a dict: k, v [n_pages][hkv][page][dh] float64, table [B][max_pages],
lens [B], and for caches that evict seen [B], slot_pos and weights
[B][hkv][slots].  The functions change it in place.
"""
import numpy as np


def row_of(cache, b, h, s):
    """(page, row) of a slot, None where its page id is none."""
    page = cache["k"].shape[2]
    p = int(cache["table"][b][s // page])
    return (p, s % page) if 0 <= p < cache["k"].shape[0] else None


def capacity(cache):
    return cache["table"].shape[1] * cache["k"].shape[2]


def held(cache, b):
    return int(min(max(int(cache["lens"][b]), 0), capacity(cache)))


def append(cache, k, v, counts, rows):
    """rows[b][i]: row of k and v that becomes new row i < counts[b] of b."""
    for b, n in enumerate(counts):
        first = held(cache, b)
        n = min(n, capacity(cache) - first)
        for i in range(n):
            for h in range(cache["k"].shape[1]):
                at = row_of(cache, b, h, first + i)
                if cache.get("slot_pos") is not None:
                    cache["slot_pos"][b, h, first + i] = cache["seen"][b] + i
                if cache.get("weights") is not None:
                    cache["weights"][b, h, first + i] = 0
                if at is not None:
                    cache["k"][at[0], h, at[1]] = k[rows[b][i], h]
                    cache["v"][at[0], h, at[1]] = v[rows[b][i], h]
        cache["lens"][b] = first + n
        if cache.get("seen") is not None:
            cache["seen"][b] += n


def _keys(cache, b, h, n):
    """K and V of the first n slots; rows that are not held are zero and flagged."""
    dh = cache["k"].shape[3]
    k, v, ok = np.zeros((n, dh)), np.zeros((n, dh)), np.zeros(n, bool)
    for s in range(n):
        at = row_of(cache, b, h, s)
        if at is not None:
            k[s], v[s], ok[s] = cache["k"][at[0], h, at[1]], cache["v"][at[0], h, at[1]], True
    return k, v, ok


def attend(cache, q, first, counts, scale, window=0, sinks=0):
    """q [rows][hq][dh]; the queries of sequence b are rows first[b] + i, i <
    counts[b].  Returns a dict of arrays over the rows (rows of no sequence NaN):
    out, lse; probs[b][h][s], the weights a sequence's queries put on each slot;
    and what error bounds need: mass = sum_s a_s |v_s|, size = the largest
    |scale| sum_d |q_d k_d| and most = keys seen."""
    rows, hq, dh = q.shape
    hkv = cache["k"].shape[1]
    hg = hq // hkv
    out, mass = np.full((rows, hq, dh), np.nan), np.full((rows, hq, dh), np.nan)
    lse, size, most = (np.full((rows, hq), np.nan) for _ in range(3))
    probs = np.zeros((len(counts), hkv, capacity(cache)))
    for b, n in enumerate(counts):
        length = held(cache, b)
        for h in range(hkv):
            k, v, ok = _keys(cache, b, h, length)
            pos = np.arange(length) if cache.get("slot_pos") is None else cache["slot_pos"][b, h, :length].astype(np.int64)
            for i in range(n):
                t = length - n + i
                see = ok & (np.arange(length) <= t)
                if window > 0 and t >= 0:
                    see &= (pos[t] - pos < window) | (pos < sinks)
                idx = np.nonzero(see)[0]
                for j in range(h * hg, (h + 1) * hg):
                    r = first[b] + i
                    if len(idx) == 0:
                        out[r, j], lse[r, j], mass[r, j], size[r, j], most[r, j] = 0, -np.inf, 0, 0, 0
                        continue
                    x = scale * (k[idx] @ q[r, j])
                    m = x.max()
                    e = np.exp(x - m)
                    a = e / e.sum()
                    out[r, j], lse[r, j] = a @ v[idx], m + np.log(e.sum())
                    mass[r, j] = a @ np.abs(v[idx])
                    size[r, j] = abs(scale) * (np.abs(k[idx]) @ np.abs(q[r, j])).max()
                    most[r, j] = len(idx)
                    probs[b, h, idx] += a
    return dict(out=out, lse=lse, mass=mass, size=size, most=most, probs=probs)


def evict(cache, budget, sinks=0, recent=0):
    for b in range(len(cache["lens"])):
        n = held(cache, b)
        if n <= budget:
            continue
        for h in range(cache["k"].shape[1]):
            w = cache["weights"][b, h, :n].astype(np.float64)
            pos = cache["slot_pos"][b, h, :n]
            safe = (pos < sinks) | (pos >= cache["seen"][b] - recent)
            rank = lambda s: (1, 0, 0, s) if safe[s] else (2, 1, 0, s) if np.isnan(w[s]) else (2, 0, -w[s], s)  # noqa: E731
            order = sorted(range(n), key=rank)
            kept = set(order[:budget])
            to = [s for s in range(budget) if s not in kept]
            at = [s for s in range(budget, n) if s in kept]
            assert len(to) == len(at)
            for x, y in zip(to, at):
                cache["weights"][b, h, x] = cache["weights"][b, h, y]
                cache["slot_pos"][b, h, x] = cache["slot_pos"][b, h, y]
                p, r = row_of(cache, b, h, x), row_of(cache, b, h, y)
                if p is not None and r is not None:
                    cache["k"][p[0], h, p[1]] = cache["k"][r[0], h, r[1]]
                    cache["v"][p[0], h, p[1]] = cache["v"][r[0], h, r[1]]
        cache["lens"][b] = budget
