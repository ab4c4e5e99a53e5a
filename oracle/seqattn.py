"""Event-sequence operators in float64 (Sections 3.3.1, 3.3.2, 3.3.4): per-head
RMSNorm with rotary positions, windowed attention with sinks over jagged
sequences, the ring cache and the single-event step.  Plain loops over
sequences and heads; masks are built pair by pair from the definition.

The `*_bound` results say how far a correct evaluation in `storage` precision
may lie from the exact value, element by element, from the roundings it makes:
u = half a step of the storage type for each rounding to it, 2^-24 for each
fp32 operation of a sum.
"""
import numpy as np

U32 = 2.0 ** -24
HALF_STEP = {"f32": U32, "bf16": 2.0 ** -8}


def positions_of(offsets, rows):
    p = np.zeros(rows, np.int64)
    for a, e in zip(offsets[:-1], offsets[1:]):
        p[a:e] = np.arange(e - a)
    return p


def angles(pos, rotary, theta):
    """Angle of every (position, pair), reduced to [0, 2 pi) in extended precision."""
    m = np.arange(rotary // 2, dtype=np.longdouble)
    turns = np.asarray(pos, np.longdouble)[:, None] * np.longdouble(theta) ** (-2 * m / max(rotary, 1)) / (
        2 * np.longdouble("3.14159265358979323846264338327950288"))
    return ((turns - np.floor(turns)) * 2 * np.longdouble("3.14159265358979323846264338327950288")).astype(np.float64)


def pair_index(rotary, interleaved):
    m = np.arange(rotary // 2)
    return (2 * m, 2 * m + 1) if interleaved else (m, m + rotary // 2)


def qk_rope(x, gain, pos, rotary, theta, eps, interleaved):
    """x [rows, heads, D] -> (y, z): rotated and unrotated normalised vectors."""
    r = 1 / np.sqrt((x ** 2).mean(-1, keepdims=True) + eps)
    z = x * r * gain
    y = z.copy()
    u, v = pair_index(rotary, interleaved)
    a = angles(pos, rotary, theta)[:, None, :]
    y[..., u] = z[..., u] * np.cos(a) - z[..., v] * np.sin(a)
    y[..., v] = z[..., u] * np.sin(a) + z[..., v] * np.cos(a)
    return y, z


def qk_rope_bwd(x, gain, pos, rotary, theta, eps, interleaved, dy):
    """(dx, dgain, terms): terms = sum of |dz n| behind dgain."""
    D = x.shape[-1]
    r = 1 / np.sqrt((x ** 2).mean(-1, keepdims=True) + eps)
    n = x * r
    dz = dy.copy()
    u, v = pair_index(rotary, interleaved)
    a = angles(pos, rotary, theta)[:, None, :]
    dz[..., u] = dy[..., u] * np.cos(a) + dy[..., v] * np.sin(a)
    dz[..., v] = -dy[..., u] * np.sin(a) + dy[..., v] * np.cos(a)
    h = dz * gain
    dx = r * (h - n * (h * n).sum(-1, keepdims=True) / D)
    return dx, (dz * n).sum((0, 1)), np.abs(dz * n).sum((0, 1))


def visible(n, window, sinks, shown):
    """[n, n] truth of (row, key) pairs of one sequence."""
    i, j = np.arange(n)[:, None], np.arange(n)[None, :]
    return (j <= i) & ((i - j < window) | (j < sinks)) & shown[None, :]


def attn(q, k, v, offsets, window, sinks, scale, shown, storage="f32"):
    """Returns dict(o, lse, o_bound, o_wide): o_wide bounds the output before
    its rounding to the storage type, with 2^-16 for the pair (out, out_lo)."""
    rows, H, D = q.shape
    J = k.shape[1]
    u = HALF_STEP[storage]
    o, ob, ow = np.zeros(q.shape), np.zeros(q.shape), np.zeros(q.shape)
    lse = np.full((H, rows), -np.inf)
    for a, e in zip(offsets[:-1], offsets[1:]):
        n = e - a
        see = visible(n, window, sinks, shown[a:e])
        kk, vv = np.where(shown[a:e, None, None], k[a:e], 0), np.where(shown[a:e, None, None], v[a:e], 0)
        for h in range(H):
            j = h // (H // J)
            P, L, es = _probabilities(q[a:e, h], kk[:, j], see, scale)
            lse[h, a:e] = L
            o[a:e, h] = P @ vv[:, j]
            ow[a:e, h] = ((u if storage != "f32" else 0) + 2 * es[:, None] + (n + 4) * U32) * (P @ np.abs(vv[:, j]))
            ob[a:e, h] = ow[a:e, h] * (1 + u) + u * np.abs(o[a:e, h])
            ow[a:e, h] += min(u, 2.0 ** -16) * np.abs(o[a:e, h]) * (1 + u)
    return dict(o=o, lse=lse, o_bound=ob, o_wide=ow)


def _probabilities(q, k, see, scale):
    """P, lse and the relative error bound of fp32 probabilities, per row."""
    n, D = q.shape
    s = np.where(see, q @ k.T * scale, -np.inf)
    top = np.where(see.any(1), s.max(1, initial=-np.inf), 0.0)
    p = np.exp(s - top[:, None])
    t = p.sum(1)
    with np.errstate(divide="ignore", invalid="ignore"):
        P = np.where(t[:, None] > 0, p / t[:, None], 0.0)
        L = np.where(t > 0, top + np.log(t), -np.inf)
    size = np.where(see, np.abs(q) @ np.abs(k).T * scale, 0).max(1, initial=0)
    # the product's sum, its scaling, the exponent's argument, exp2, the row sum and lse
    return P, L, (D + 8) * U32 * size + 4 * U32 * (1 + size) + (n + 8) * U32


def attn_bwd(q, k, v, offsets, window, sinks, scale, shown, do, storage="f32"):
    """Returns dict of dq, dk, dv and their bounds."""
    rows, H, D = q.shape
    J = k.shape[1]
    u = HALF_STEP[storage]
    r = u if storage != "f32" else 0.0            # rounding of a product's operand
    g = {m: np.zeros(x.shape) for m, x in (("dq", q), ("dk", k), ("dv", v))}
    b = {m: np.zeros(x.shape) for m, x in g.items()}
    f = attn(q, k, v, offsets, window, sinks, scale, shown, storage)
    for a, e in zip(offsets[:-1], offsets[1:]):
        n = e - a
        see = visible(n, window, sinks, shown[a:e])
        kk, vv = np.where(shown[a:e, None, None], k[a:e], 0), np.where(shown[a:e, None, None], v[a:e], 0)
        for h in range(H):
            j = h // (H // J)
            Q, K, V, G = q[a:e, h], kk[:, j], vv[:, j], do[a:e, h]
            P, _, es = _probabilities(Q, K, see, scale)
            dP = G @ V.T
            delta = (G * f["o"][a:e, h]).sum(1, keepdims=True)
            dS = P * (dP - delta)
            # errors of dP, of delta (from out and out_lo) and of P
            e_delta = (np.abs(G) * f["o_wide"][a:e, h]).sum(1, keepdims=True) + (D + 2) * U32 * (
                np.abs(G) * np.abs(f["o"][a:e, h])).sum(1, keepdims=True)
            e_dP = (D + 2) * U32 * (np.abs(G) @ np.abs(V).T)
            e_dS = P * (e_dP + e_delta) + 2 * es[:, None] * np.abs(dS) + r * np.abs(dS) + 4 * U32 * np.abs(P) * (
                np.abs(dP) + np.abs(delta))
            N = n * (H // J) + 8
            g["dq"][a:e, h] = scale * dS @ K
            b["dq"][a:e, h] = scale * (e_dS @ np.abs(K) + (n + 4) * U32 * np.abs(dS) @ np.abs(K))
            g["dk"][a:e, j] += scale * dS.T @ Q
            b["dk"][a:e, j] += scale * (e_dS.T @ np.abs(Q) + N * U32 * np.abs(dS).T @ np.abs(Q))
            g["dv"][a:e, j] += P.T @ G
            b["dv"][a:e, j] += ((r + 2 * es[None, :] + N * U32) * P.T) @ np.abs(G)
    for m in g:
        b[m] = b[m] * (1 + u) + u * np.abs(g[m])
    return g, b


def slot_of(p, window, sinks):
    return p if p < sinks else sinks + (p - sinks) % window


def cache_fill(kc, vc, k, v, offsets, window, sinks, index, first):
    """Caches [C, J, slots, D] after the sequences' rows went in one by one."""
    kc, vc = kc.copy(), vc.copy()
    for s, (a, e) in enumerate(zip(offsets[:-1], offsets[1:])):
        if not 0 <= index[s] < kc.shape[0]:
            continue
        for t in range(a, e):
            x = slot_of(int(first[s]) + t - a, window, sinks)
            kc[index[s], :, x], vc[index[s], :, x] = k[t], v[t]
    return kc, vc
