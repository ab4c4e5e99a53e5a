"""Dropout from a counter-based generator, and the root-mean-square norm of a
residual sum with its 8-bit output (Sections 3.3.4, 3.5.2), in float64.

The bounds count the roundings of a correct evaluation: U32 = 2^-24 for an
fp32 operation, half a step of the storage type for each rounding to it.
"""
import numpy as np

from .fp8 import E4M3_MAX

U32 = 2.0 ** -24
HALF_STEP = {"f32": U32, "bf16": 2.0 ** -8}


def philox4x32(counter, key, rounds=10):
    """Philox4x32 (Salmon et al., 2011) of 32-bit words as Python integers."""
    c, k = list(counter), list(key)
    for _ in range(rounds):
        a, b = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(b >> 32) ^ c[1] ^ k[0], b & 0xFFFFFFFF, (a >> 32) ^ c[3] ^ k[1], a & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def threshold(p):
    return int(np.floor(p * 65536 + 0.5))


def numbers(rows, cols, seed, step, site):
    """The 16-bit numbers of elements [rows, cols] (rows: their indices)."""
    groups = -(-cols // 8)
    rows = np.asarray(rows, np.uint64)
    m = np.uint64(0xFFFFFFFF)
    c = [np.broadcast_to(x, (rows.size, groups)).astype(np.uint64) for x in
         (np.arange(groups, dtype=np.uint64), rows[:, None], np.uint64(site), np.uint64(step & 0xFFFFFFFF))]
    k = [seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF]
    s = np.uint64(32)
    for _ in range(10):
        a, b = np.uint64(0xD2511F53) * c[0], np.uint64(0xCD9E8D57) * c[2]
        c = [(b >> s) ^ c[1] ^ np.uint64(k[0]), b & m, (a >> s) ^ c[3] ^ np.uint64(k[1]), a & m]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    w = np.stack(c, -1)                                      # [rows, groups, 4]
    n = np.stack([w & np.uint64(0xFFFF), w >> np.uint64(16)], -1)
    return n.reshape(rows.size, groups * 8)[:, :cols].astype(np.int64)


def factor(rows, cols, p, seed, step, site):
    """What dropout multiplies each element by: 0 or 65536 / (65536 - t)."""
    t = threshold(p)
    if t == 0:
        return np.ones((len(rows), cols))
    return (numbers(rows, cols, seed, step, site) >= t) * (65536.0 / (65536 - t))


def rmsnorm(h, gain, eps):
    """(y, rho)."""
    rho = 1 / np.sqrt((h ** 2).mean(-1, keepdims=True) + eps)
    return h * rho * gain, rho


def rmsnorm_bwd(h, gain, eps, dy, dh=None):
    """(dr, dgain) of the norm's input and gain; dh: what reaches h besides."""
    n, rho = h * (r := 1 / np.sqrt((h ** 2).mean(-1, keepdims=True) + eps)), r
    dn = dy * gain
    dr = rho * (dn - n * (dn * n).mean(-1, keepdims=True)) + (0 if dh is None else dh)
    return dr, (dy * n).sum(0)


# Relative error of rho: a lane adds up at most 16 squares or 32, its wave's lanes are joined in
# 6 sums, and a row's waves one after another, at most 16 where lanes have 16 squares and 8
# where they have 32: 16 + 6 + 15 or 32 + 6 + 7 = 45 sums and the squares' own
# rounding; half of that, and the mean's two products, eps, the root and the division.
RHO = (32 + 13 + 2) / 2 * U32 + 5 * U32


def y_bound(y, dtype):
    """Of the norm's result in the storage type: rho, two products, the rounding."""
    u = HALF_STEP[dtype]
    return np.abs(y) * (RHO + 2 * U32 + u * (dtype != "f32")) * (1 + 1e-3)


def dr_bound(h, gain, eps, dy, dh, dtype):
    rho = 1 / np.sqrt((h ** 2).mean(-1, keepdims=True) + eps)
    n, dn = h * rho, dy * gain
    mean = np.abs((dn * n).mean(-1, keepdims=True))
    # sum(dn h): two products a term, 32 + 13 sums; then rho twice, the mean, two products
    e_mean = (45 + 2 + 3) * U32 * np.abs(dn * n).mean(-1, keepdims=True) + 2 * RHO * mean
    e = np.abs(rho * dn) * (RHO + 3 * U32) + np.abs(n) * e_mean + np.abs(n) * mean * (RHO + 4 * U32)
    total = np.abs(rho * dn) + np.abs(n) * mean + (0 if dh is None else np.abs(dh))
    dr, _ = rmsnorm_bwd(h, gain, eps, dy, dh)
    u = HALF_STEP[dtype]
    return e + 3 * U32 * total + u * np.abs(dr) * (1 + 1e-3) + (e + 3 * U32 * total) * u


def dgain_bound(h, eps, dy):
    """Any order of the sum over rows."""
    rho = 1 / np.sqrt((h ** 2).mean(-1, keepdims=True) + eps)
    return (RHO + (3 + h.shape[0]) * U32) * np.abs(dy * h * rho).sum(0)


def scale_of(y):
    top = np.abs(y).max(-1)
    return np.where(top > 0, np.maximum(top / E4M3_MAX, 2.0 ** -126), 1.0)


def code_bound(y, scale):
    """Of a code's value: half a step of e4m3, and what rho, the products and the
    scale bring before it."""
    return (np.maximum(2.0 ** -4 * np.abs(y), 2.0 ** -10 * scale[:, None]) + 3 * (RHO + 4 * U32) * np.abs(y)) * (1 + 1e-5)
