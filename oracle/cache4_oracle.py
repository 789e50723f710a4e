"""Plain NumPy oracle of the rotation on the way into the paged cache and of
caches in 4 bits, element by element from the definitions in include/gmc.h.
Test infrastructure; shares no code with the HIP path.

A cache of 4 bits is a dict as in cache_oracle with the values in k and v, so
that its attention is that module's, and beside them k_codes, v_codes
[n_pages][hkv][page][dh] (0 to 15, one an element) and k_scales, v_scales
[n_pages][hkv][page][dh / 32].
"""
import math

import numpy as np

from . import cache_oracle

MAGNITUDES = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def value(code, e):
    if e == 255:
        return math.nan
    return (-1.0 if code & 8 else 1.0) * MAGNITUDES[code & 7] * 2.0 ** (int(e) - 127)


def quantise(block):
    """(codes, e) of 32 numbers."""
    block = [float(x) for x in block]
    if not all(math.isfinite(x) for x in block):
        return None, 255            # the codes of such a block are anything
    top = max(abs(x) for x in block)
    e = 1
    while e < 252 and top > 7 * 2.0 ** (e - 127):
        e += 1
    codes = []
    for x in block:
        size = abs(x) / 2.0 ** (e - 127)
        off = [abs(size - m) for m in MAGNITUDES]
        near = [i for i in range(8) if off[i] == min(off)]
        code = near[0] if len(near) == 1 else [i for i in near if i % 2 == 0][0]
        codes.append(code + (8 if math.copysign(1.0, x) < 0 else 0))
    return codes, e


def rotate(x, cos, sin, rot, interleaved):
    """One head's row in float32: products rounded, then their sum; cos and sin
    of each pair."""
    x = np.array(x, np.float32)
    for j in range(rot // 2):
        a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + rot // 2)
        c, s, u, v = np.float32(cos[j]), np.float32(sin[j]), x[a], x[b]
        x[a], x[b] = np.float32(u * c) - np.float32(v * s), np.float32(v * c) + np.float32(u * s)
    return x


def turn(rows, rotary, pos):
    """rows [n][heads][dh] by positions [n] or [n][3] -> float32."""
    cos, sin, rot = rotary["cos"], rotary["sin"], 2 * rotary["cos"].shape[1]
    axis = np.zeros(rot // 2, int)
    if rotary.get("sections"):
        axis = np.repeat(np.arange(3), rotary["sections"])
    out = np.zeros(rows.shape, np.float32)
    for i in range(len(rows)):
        p = np.asarray(pos[i]).reshape(-1)
        p = np.broadcast_to(p, (3,)) if len(p) == 1 else p
        at = np.clip(p[axis], 0, len(cos) - 1), np.arange(rot // 2)
        for h in range(rows.shape[1]):
            out[i, h] = rotate(rows[i, h], cos[at], sin[at], rot, rotary["interleaved"])
    return out


def append4(cache, k, v, counts, rows):
    """cache_oracle.append into a cache of 4 bits; k, v float32."""
    for b, n in enumerate(counts):
        first = cache_oracle.held(cache, b)
        n = min(n, cache_oracle.capacity(cache) - first)
        for i in range(n):
            at = cache_oracle.row_of(cache, b, 0, first + i)
            if at is None:
                continue
            for name, x in (("k", k), ("v", v)):
                for h in range(cache["k"].shape[1]):
                    for blk in range(cache["k"].shape[3] // 32):
                        to = slice(32 * blk, 32 * blk + 32)
                        codes, e = quantise(x[rows[b][i], h, to])
                        where = (at[0], h, at[1])
                        cache[name + "_scales"][where + (blk,)] = e
                        if codes is None:
                            cache[name][where + (to,)] = math.nan
                        else:
                            cache[name + "_codes"][where + (to,)] = codes
                            cache[name][where + (to,)] = [value(c, e) for c in codes]
        cache["lens"][b] = first + n
