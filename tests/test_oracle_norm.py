"""Pins of the oracle of dropout, the residual norm and the 8-bit ring caches."""
import numpy as np
import pytest

from oracle import fp8
from oracle import norm as o
from oracle import seqcache8 as c8


@pytest.mark.parametrize("counter,key,want", [
    # the published known-answer vectors of Philox4x32-10
    ([0] * 4, [0] * 2, [0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]),
    ([0xffffffff] * 4, [0xffffffff] * 2, [0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd]),
    ([0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344], [0xa4093822, 0x299f31d0],
     [0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1])])
def test_philox_known_answers(counter, key, want):
    assert o.philox4x32(counter, key) == want


def test_numbers_are_the_generators_halves():
    seed, step, site, rows, cols = 0x123456789abcdef0, 0x1_0000_0005, 7, [0, 3, 2 ** 30 - 1], 21
    got = o.numbers(rows, cols, seed, step, site)
    for i, r in enumerate(rows):
        for c in range(cols):
            w = o.philox4x32([c // 8, r, site, step & 0xffffffff], [seed & 0xffffffff, seed >> 32])[c % 8 // 2]
            assert got[i, c] == (w >> 16 if c % 2 else w & 0xffff)


@pytest.mark.parametrize("p", [0.0, 2.0 ** -18, 0.1, 0.5, 0.9, 65535 / 65536])
def test_dropout_keeps_its_share_and_its_mean(p):
    f = o.factor(np.arange(2000), 333, p, 11, 5, 1)
    t = o.threshold(p) / 65536
    n = f.size
    assert abs((f == 0).mean() - t) <= 5 * np.sqrt(max(t * (1 - t), 1e-12) / n)
    if t < 0.99:
        assert abs(f.mean() - 1) <= 5 * np.sqrt(t / (1 - t) / n) + 1e-12
    # another step, site or seed drops others
    if 0.05 < t < 0.95:
        for other in (o.factor(np.arange(2000), 333, p, 11, 6, 1), o.factor(np.arange(2000), 333, p, 11, 5, 2),
                      o.factor(np.arange(2000), 333, p, 12, 5, 1), o.factor(np.arange(1, 2001), 333, p, 11, 5, 1)):
            same = ((f == 0) == (other == 0)).mean()
            assert abs(same - (t * t + (1 - t) ** 2)) <= 5 / np.sqrt(n)


def test_norm_gradient_against_differences():
    rng = np.random.default_rng(0)
    h, dy, dh, gain = rng.standard_normal((3, 7)), rng.standard_normal((3, 7)), rng.standard_normal((3, 7)), rng.standard_normal(7)
    dr, dg = o.rmsnorm_bwd(h, gain, 1e-3, dy, dh)
    f = lambda h, g: (o.rmsnorm(h, g, 1e-3)[0] * dy).sum() + (h * dh).sum()  # noqa: E731
    e = 1e-6
    for i in np.ndindex(*h.shape):
        d = np.zeros_like(h)
        d[i] = e
        assert abs((f(h + d, gain) - f(h - d, gain)) / (2 * e) - dr[i]) < 1e-7
    for i in range(7):
        d = np.zeros(7)
        d[i] = e
        assert abs((f(h, gain + d) - f(h, gain - d)) / (2 * e) - dg[i]) < 1e-7


def test_block_scale_is_the_smallest_power_that_holds():
    for top in (448.0, np.nextafter(448.0, 1e9), 447.0, 1.0, 3e-5, 3.4e38, 0.4375, 2.0 ** -120, 7 * 2.0 ** 40):
        s = c8.block_scale(top)
        assert np.log2(s) % 1 == 0 and top <= 448 * s and (s == 2.0 ** -117 or top > 224 * s)
    assert c8.block_scale(0.0) == 1.0


def test_encoding_an_encoded_block_again_changes_nothing():
    rng = np.random.default_rng(3)
    x = rng.standard_normal((16, 24)) * 10.0 ** rng.integers(-3, 4, (16, 1))
    s, c = c8.encode(x, np.ones(16, bool))
    s2, c2 = c8.encode(fp8.e4m3_value(c) * s, np.ones(16, bool))
    # the largest value may have been rounded down over the border of a smaller scale, not up
    assert s2 == s and np.array_equal(c, c2)


def test_a_fill_is_the_rows_one_by_one_where_scales_stay():
    rng = np.random.default_rng(4)
    J, D, W, N = 2, 8, 21, 3
    cap, n = W + N, 60
    k, v = (np.float64(np.sign(rng.standard_normal((n, J, D))) * 448) for _ in "kv")    # every row sets the same scale
    mk = lambda: dict(k=np.zeros((1, J, cap, 16), np.uint8), v=np.zeros((1, J, cap, 16), np.uint8),  # noqa: E731
                      ks=np.ones((1, J, 2), np.float32), vs=np.ones((1, J, 2), np.float32))
    a, b = mk(), mk()
    c8.fill(a, k, v, [0, n], W, N, [0], [0])
    for t in range(n):
        c8.fill(b, k[t:t + 1], v[t:t + 1], [0, 1], W, N, [0], [t])
    for x in a:
        assert np.array_equal(a[x], b[x])
