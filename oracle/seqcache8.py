"""Ring caches of e4m3 codes with a power-of-two scale for every 16 slots, in
float64: fill, append and the attention of a single event.  A cache is a dict
of k, v (codes, uint8 [caches, heads, slots, ld]) and ks, vs (scales [caches,
heads, blocks]).
"""
import numpy as np

from .fp8 import e4m3_code, e4m3_value
from .seqattn import slot_of

BLOCK = 16


def block_scale(top):
    """The smallest power of two s >= 2^-117 with top <= 448 s; 1 for 0."""
    if not top > 0:
        return 1.0
    s = 2.0 ** -117
    while top > 448 * s:
        s *= 2
    return s


def encode(x, reached):
    """(scale, codes) of a block [16, D]; rows that are not reached count for
    nothing.  Values that are not finite become NaN (0x7f)."""
    live = np.where(reached[:, None], x, 0)
    fin = np.isfinite(live)
    s = block_scale(np.abs(np.where(fin, live, 0)).max(initial=0))
    top = 240.0 if s >= 2.0 ** 120 else 448.0
    c = e4m3_code(np.clip(np.where(fin, live, 0) / s, -top, top))
    return s, np.where(fin, c, 0x7F).astype(np.uint8)


def value(codes, scales, D):
    """Values [heads, slots, D] of one cache."""
    s = np.repeat(scales.astype(np.float64), BLOCK, axis=-1)[:, :codes.shape[1]]
    return e4m3_value(codes[..., :D]) * s[..., None]


def put(cache, at, rows, end):
    """Rows {slot: (k, v)} of [heads, D] into cache `at`, whose slots below `end`
    are reached afterwards.  Blocks that take rows are encoded anew."""
    J, cap = cache["k"].shape[1:3]
    for b in sorted({s // BLOCK for s in rows}):
        lo, hi = b * BLOCK, min((b + 1) * BLOCK, cap)
        reached = np.arange(lo, lo + BLOCK) < min(end, cap)
        for side in (0, 1):
            c, s = (cache["k"], cache["ks"]) if side == 0 else (cache["v"], cache["vs"])
            for j in range(J):
                D = next(iter(rows.values()))[side].shape[-1]
                x = np.zeros((BLOCK, D))
                fresh = np.zeros(BLOCK, bool)
                for i in range(lo, hi):
                    if i in rows:
                        x[i - lo], fresh[i - lo] = rows[i][side][j], True
                    elif reached[i - lo]:
                        x[i - lo] = e4m3_value(c[at, j, i, :D]) * float(s[at, j, b])
                sc, codes = encode(x, reached)
                same = (reached & ~fresh).any() and sc == s[at, j, b]
                for i in range(lo, hi):
                    if fresh[i - lo] or (reached[i - lo] and not same):
                        c[at, j, i, :D] = codes[i - lo]
                        c[at, j, i, D:] = 0
                s[at, j, b] = sc


def fill(cache, k, v, offsets, window, sinks, index, first):
    for s, (a, e) in enumerate(zip(offsets[:-1], offsets[1:])):
        if not 0 <= index[s] < cache["k"].shape[0] or e <= a:
            continue
        rows = {}
        for t in range(a, e):
            rows[slot_of(int(first[s]) + t - a, window, sinks)] = (k[t], v[t])
        put(cache, index[s], rows, int(first[s]) + e - a)


def attend(K, V, q, n, scale):
    """(out, P, sum |P v|, largest sum |q k| scale) of one head over slots 0 .. n - 1."""
    s = K[:n] @ q * scale
    p = np.exp(s - s.max())
    P = p / p.sum()
    return P @ V[:n], P @ np.abs(V[:n]), (np.abs(K[:n]) @ np.abs(q)).max() * scale
