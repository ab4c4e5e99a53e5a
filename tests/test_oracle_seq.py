"""Pins of the event-sequence oracle: masks against hand-written lists, the
rotation against complex numbers and its known invariances, attention and its
gradients against direct sums and central differences, the ring cache against
the visible set's definition."""
import numpy as np
import pytest

from oracle import seqattn as o

rng = np.random.default_rng(7)


def test_visible_pairs_by_hand():
    see = o.visible(6, 2, 1, np.ones(6, bool))
    want = [[0], [0, 1], [0, 1, 2], [0, 2, 3], [0, 3, 4], [0, 4, 5]]
    assert [list(np.flatnonzero(r)) for r in see] == want
    shown = np.array([0, 1, 1, 0, 1, 1], bool)
    assert [list(np.flatnonzero(r)) for r in o.visible(6, 2, 1, shown)] == [[], [1], [1, 2], [2], [4], [4, 5]]
    assert (o.visible(5, 99, 0, np.ones(5, bool)) == np.tril(np.ones((5, 5), bool))).all()


@pytest.mark.parametrize("inter", [False, True])
def test_rotation_is_a_complex_product_and_keeps_relative_positions(inter):
    x = rng.standard_normal((2, 1, 16))
    gain = 1 + 0.1 * rng.standard_normal(16)
    y, z = o.qk_rope(x, gain, [5, 9], 8, 100.0, 0.0, inter)
    u, v = o.pair_index(8, inter)
    for t, p in enumerate((5, 9)):
        w = (z[t, 0, u] + 1j * z[t, 0, v]) * np.exp(1j * p * 100.0 ** (-2 * np.arange(4) / 8))
        assert np.allclose(y[t, 0, u] + 1j * y[t, 0, v], w)
    assert np.array_equal(y[..., 8:], z[..., 8:])
    y2, _ = o.qk_rope(x, gain, [1005, 1009], 8, 100.0, 0.0, inter)
    assert np.isclose((y[0] * y[1]).sum(), (y2[0] * y2[1]).sum())
    assert np.allclose((x[0, 0] * 1.0 / np.sqrt((x[0, 0] ** 2).mean())) * gain, z[0, 0])


@pytest.mark.parametrize("inter", [False, True])
def test_rope_gradient_by_differences(inter):
    x, dy = rng.standard_normal((3, 2, 8)), rng.standard_normal((3, 2, 8))
    gain, pos = 1 + 0.1 * rng.standard_normal(8), np.array([0, 3, 77])
    f = lambda x_, g_: (o.qk_rope(x_, g_, pos, 8, 50.0, 1e-3, inter)[0] * dy).sum()  # noqa: E731
    dx, dg, _ = o.qk_rope_bwd(x, gain, pos, 8, 50.0, 1e-3, inter, dy)
    for _ in range(5):
        d, h = rng.standard_normal(x.shape), 1e-5
        assert np.isclose((f(x + h * d, gain) - f(x - h * d, gain)) / (2 * h), (dx * d).sum(), rtol=1e-6)
        e = rng.standard_normal(8)
        assert np.isclose((f(x, gain + h * e) - f(x, gain - h * e)) / (2 * h), (dg * e).sum(), rtol=1e-6)


def _problem(shown=None):
    off = np.array([0, 1, 8, 8, 13])
    q, k, v = rng.standard_normal((13, 4, 8)), rng.standard_normal((13, 2, 8)), rng.standard_normal((13, 2, 8))
    return q, k, v, off, np.ones(13, bool) if shown is None else shown


def test_attention_by_direct_sums():
    shown = rng.random(13) > 0.3
    shown[8] = False
    q, k, v, off, shown = _problem(shown)
    f = o.attn(q, k, v, off, 3, 1, 0.4, shown)
    for a, e in zip(off[:-1], off[1:]):
        for i in range(a, e):
            js = [j for j in range(a, i + 1) if shown[j] and (i - j < 3 or j - a < 1)]
            for h in range(4):
                w = np.exp([0.4 * q[i, h] @ k[j, h // 2] for j in js])
                want = sum((x * v[j, h // 2] for x, j in zip(w, js)), np.zeros(8)) / (w.sum() if js else 1)
                assert np.allclose(f["o"][i, h], want)
                assert (np.isclose(f["lse"][h, i], np.log(w.sum())) if js else f["lse"][h, i] == -np.inf)
    assert (f["o"][8] == 0).all()                      # its only key is hidden


def test_attention_gradient_by_differences():
    q, k, v, off, shown = _problem()
    do = rng.standard_normal(q.shape)
    f = lambda a, b, c: (o.attn(a, b, c, off, 3, 2, 0.3, shown)["o"] * do).sum()  # noqa: E731
    g, _ = o.attn_bwd(q, k, v, off, 3, 2, 0.3, shown, do)
    h = 1e-5
    for m, i in (("dq", 0), ("dk", 1), ("dv", 2)):
        for _ in range(3):
            x = [q, k, v]
            d = rng.standard_normal(x[i].shape)
            up, dn = list(x), list(x)
            up[i], dn[i] = x[i] + h * d, x[i] - h * d
            assert np.isclose((f(*up) - f(*dn)) / (2 * h), (g[m] * d).sum(), rtol=1e-6), m


@pytest.mark.parametrize("window,sinks", [(1, 0), (3, 0), (3, 2), (5, 4), (40, 1)])
def test_ring_holds_exactly_the_visible_rows(window, sinks):
    n = 23
    k = np.arange(n, dtype=float).reshape(n, 1, 1) + 1
    see = o.visible(n, window, sinks, np.ones(n, bool))
    for p in range(n):
        kc, _ = o.cache_fill(np.zeros((1, 1, window + sinks, 1)), np.zeros((1, 1, window + sinks, 1)), k[:p + 1],
                             k[:p + 1], [0, p + 1], window, sinks, [0], [0])
        slots = min(p + 1, window + sinks)
        assert sorted(kc[0, 0, :slots, 0] - 1) == list(np.flatnonzero(see[p])), p


def test_bounds_cover_an_evaluation_in_fp32_and_are_not_vacuous():
    q, k, v, off, shown = _problem()
    do = rng.standard_normal(q.shape)
    q, k, v, do = (x.astype(np.float32).astype(np.float64) for x in (q, k, v, do))
    f = o.attn(q, k, v, off, 4, 1, 0.35, shown)
    g, b = o.attn_bwd(q, k, v, off, 4, 1, 0.35, shown, do)
    h = o.attn(*(x.astype(np.float32) for x in (q, k, v)), off, 4, 1, np.float32(0.35), shown)
    assert (np.abs(h["o"].astype(np.float32) - f["o"]) <= f["o_bound"] + 1e-30).all()
    assert f["o_bound"].max() < 1e-4 and max(x.max() for x in b.values()) < 1e-3
    assert max(np.abs(x).max() for x in g.values()) > 0.1
