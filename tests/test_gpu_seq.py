"""Event-sequence operators on the GPU against the float64 oracle: every row,
head and gradient element within the bound that follows from the roundings a
correct evaluation makes (oracle/seqattn.py)."""
import numpy as np
import pytest
import torch

from oracle import seqattn as o

DEV = "cuda"
TT = {"bf16": torch.bfloat16, "f32": torch.float32}
pytestmark = pytest.mark.gpu


def randn(rng, *shape):
    return torch.from_numpy(rng.standard_normal(shape).astype(np.float32))


def f64(t):
    return t.detach().float().cpu().double().numpy()


def offs(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)


def within(got, want, bound, what):
    g = f64(got)
    assert np.isfinite(g).all(), f"{what}: not finite"
    over = np.abs(g - want) - bound
    i = np.unravel_index(np.argmax(over), over.shape)
    assert over[i] <= 1e-30, f"{what} at {i}: {g[i]} against {want[i]}, bound {bound[i]}"


# ---------------------------------------------------------------------------
LENS = {"one": [1], "two": [2], "empty": [0, 5, 0, 0, 3, 0], "edges": [63, 64, 65, 1, 127, 128, 129],
        "ones": [1] * 70, "short": [20, 3, 31, 8, 1, 60, 17] * 9, "long": [700], "mixed": [300, 1, 0, 129, 400]}


def plan(lens, pad=0, max_len=0):
    from paper_2512_09200_amd import api
    off = offs(lens)
    rows = int(off[-1]) + pad
    return off, rows, api.lattice_seq_plan(torch.from_numpy(off.astype(np.int32)).to(DEV), rows, max_len=max_len,
                                           padded=pad > 0)


@pytest.mark.parametrize("lens", list(LENS))
@pytest.mark.parametrize("pad", [0, 37])
def test_plan(lens, pad):
    off, rows, s = plan(LENS[lens], pad)
    want = np.full((rows, 2), 0)
    want[:, 0] = 2 ** 31 - 1
    for a, e in zip(off[:-1], off[1:]):
        want[a:e] = a, e
    assert np.array_equal(s.span.cpu().numpy(), want)


# ---------------------------------------------------------------------------
ROPE = [("bf16", 4, 2, 64, 64, False), ("f32", 2, 1, 32, 32, True), ("bf16", 3, 3, 96, 64, True),
        ("f32", 5, 1, 40, 24, False), ("bf16", 1, 1, 8, 8, False), ("f32", 2, 2, 128, 0, False),
        ("bf16", 8, 1, 128, 128, False), ("bf16", 2, 1, 24, 8, True), ("f32", 4, 4, 16, 16, False)]


@pytest.mark.parametrize("dt,H,J,D,R,inter", ROPE)
@pytest.mark.parametrize("far", [False, True])
def test_qk_rope(dt, H, J, D, R, inter, far):
    from paper_2512_09200_amd import api
    rng = np.random.default_rng(D * 100 + H)
    lens = [37, 1, 90, 0, 5]
    off, rows, s = plan(lens, pad=3)
    n = int(off[-1])
    # q and k side by side in one projection's rows
    qk = randn(rng, rows, H + J, D).to(TT[dt]).to(DEV)
    q, k = qk[:, :H], qk[:, H:]
    gq, gk = (1 + 0.2 * randn(rng, D)).to(DEV), (1 + 0.2 * randn(rng, D)).to(DEV)
    pos = rng.integers(-2 ** 31, 2 ** 31, rows) if far else o.positions_of(off, rows)
    kw = dict(gain_q=gq, gain_k=gk, theta=10000.0, rotary=R, interleaved=inter, eps=1e-5,
              positions=torch.from_numpy(pos.astype(np.int32)).to(DEV) if far else None)
    buf = torch.full((rows, H + J, D), 7.0, dtype=TT[dt], device=DEV)
    yq, yk = api.lattice_qk_rope_fwd(s, q, k, q_out=buf[:, :H], k_out=buf[:, H:], **kw)
    dq_, dk_ = randn(rng, rows, H, D).to(TT[dt]).to(DEV), randn(rng, rows, J, D).to(TT[dt]).to(DEV)
    gbuf = torch.full((rows, H + J, D), 7.0, dtype=TT[dt], device=DEV)
    dq, dk, dgq, dgk = api.lattice_qk_rope_bwd(s, q, k, dq_, dk_, dq=gbuf[:, :H], dk=gbuf[:, H:], **kw)
    u = o.HALF_STEP[dt]
    for x, g, y, dy, dx, dg, name in ((q, gq, yq, dq_, dq, dgq, "q"), (k, gk, yk, dk_, dk, dgk, "k")):
        X, G, DY = f64(x)[:n], f64(g), f64(dy)[:n]
        want, z = o.qk_rope(X, G, pos[:n], R, 10000.0, 1e-5, inter)
        # norm (D squares summed, square root, division, two products), angle
        # (reduced to 2^-24 turns or better) and its sine, two products and a sum
        size = np.abs(z).copy()
        a, b = o.pair_index(R, inter)
        both = np.hypot(z[..., a], z[..., b])
        size[..., a], size[..., b] = both, both
        within(y[:n], want, u * np.abs(want) + (D + 40) * o.U32 * size, "y" + name)
        wdx, wdg, terms = o.qk_rope_bwd(X, G, pos[:n], R, 10000.0, 1e-5, inter, DY)
        r = 1 / np.sqrt((X ** 2).mean(-1, keepdims=True) + 1e-5)
        h = np.abs(G) * (np.abs(DY).max(-1, keepdims=True) * 1.5)
        bound = u * np.abs(wdx) + (2 * D + 64) * o.U32 * r * (h + np.abs(X * r) * (h * np.abs(X * r)).mean(-1, keepdims=True))
        within(dx[:n], wdx, bound, "d" + name)
        # (terms' size before the rotation mixes pairs: at most sqrt(2) times)
        big = (np.abs(X * r) * np.abs(DY).max(-1, keepdims=True) * 1.5).sum((0, 1))
        within(dg, wdg, o.U32 * ((D + 64) * big + 300 * terms), "dgain_" + name)
    assert (buf[n:] == 7).all() and (gbuf[n:] == 7).all()          # rows behind the last sequence


def test_qk_rope_in_place_without_plan_or_gains():
    from paper_2512_09200_amd import api
    rng = np.random.default_rng(3)
    x = randn(rng, 50, 3, 32).to(DEV)
    pos = torch.arange(50, dtype=torch.int32, device=DEV)
    ref = api.lattice_qk_rope_fwd(None, x[:, :2], x[:, 2:], positions=pos)
    dref = api.lattice_qk_rope_bwd(None, x[:, :2], x[:, 2:], *ref, positions=pos)
    assert dref[2] is None and dref[3] is None
    want, _ = o.qk_rope(f64(x[:, :2]), 1.0, np.arange(50), 32, 1e4, 1e-6, False)
    assert np.abs(f64(ref[0]) - want).max() < 1e-5
    d = [t.clone() for t in ref]
    api.lattice_qk_rope_bwd(None, x[:, :2], x[:, 2:], *d, positions=pos, dq=d[0], dk=d[1])
    y = x.clone()
    api.lattice_qk_rope_fwd(None, y[:, :2], y[:, 2:], positions=pos, q_out=y[:, :2], k_out=y[:, 2:])
    assert torch.equal(y, torch.cat(ref, 1)) and torch.equal(d[0], dref[0]) and torch.equal(d[1], dref[1])


# ---------------------------------------------------------------------------
def attn_case(dt, H, J, D, lens, W, N, hidden=0.0, pad=0, max_len=0, seed=0, all_hidden=False):
    from paper_2512_09200_amd import api
    rng = np.random.default_rng(seed + D + H)
    off, rows, s = plan(lens, pad, max_len)
    qkv = randn(rng, rows, H + 2 * J, D).to(TT[dt]).to(DEV)
    q, k, v = qkv[:, :H], qkv[:, H:H + J], qkv[:, H + J:]
    do = randn(rng, rows, H, D).to(TT[dt]).to(DEV)
    shown = rng.random(rows) >= hidden
    if all_hidden:
        shown[:] = False
    mask = torch.from_numpy(shown.astype(np.uint8)).to(DEV) if hidden or all_hidden else None
    kw = dict(window=W, sinks=N, key_mask=mask)
    out, lse = api.lattice_seq_attn_fwd(s, q, k, v, **kw)
    dq, dk, dv = api.lattice_seq_attn_bwd(s, q, k, v, out, lse, do, **kw)
    return dict(off=off, rows=rows, s=s, q=q, k=k, v=v, do=do, shown=shown, kw=kw, out=out, lse=lse, dq=dq, dk=dk, dv=dv)


def check_attn(c, dt, W, N):
    n, D = int(c["off"][-1]), c["q"].shape[2]
    a = [f64(c[m])[:n] for m in ("q", "k", "v")]
    W = min(W, n + 1)
    f = o.attn(*a, c["off"], W, N, D ** -0.5, c["shown"][:n], dt)
    within(c["out"][:n], f["o"], f["o_bound"], "out")
    L = f64(c["lse"].lse)[:, :n]
    empty = np.isneginf(f["lse"])
    assert np.array_equal(np.isneginf(L), empty)
    assert np.abs(np.where(empty, 0, L - np.where(empty, 0, f["lse"]))).max(initial=0) < 1e-4
    g, b = o.attn_bwd(*a, c["off"], W, N, D ** -0.5, c["shown"][:n], f64(c["do"])[:n], dt)
    for m in ("dq", "dk", "dv"):
        within(c[m][:n], g[m], b[m], m)


SHAPES = [("bf16", 4, 2, 64), ("bf16", 1, 1, 32), ("f32", 2, 2, 32), ("bf16", 8, 2, 128), ("f32", 3, 1, 128),
          ("bf16", 6, 2, 96), ("f32", 4, 1, 40), ("bf16", 3, 3, 8), ("f32", 8, 1, 64), ("bf16", 16, 1, 16)]


@pytest.mark.parametrize("lens", list(LENS))
@pytest.mark.parametrize("dt,H,J,D", SHAPES[:5])
def test_attention_lengths(dt, H, J, D, lens):
    check_attn(attn_case(dt, H, J, D, LENS[lens], 48, 3, pad=5), dt, 48, 3)


@pytest.mark.parametrize("W,N", [(1, 0), (1, 1), (2, 7), (16, 5), (16, 40), (31, 64), (64, 0), (100, 33), (129, 1),
                                 (300, 4), (701, 4), (2 ** 31 - 1, 0), (2 ** 31 - 1, 64)])
@pytest.mark.parametrize("dt,H,J,D", [SHAPES[0], SHAPES[4]])
def test_attention_windows(dt, H, J, D, W, N):
    check_attn(attn_case(dt, H, J, D, [700, 90, 1], W, N, max_len=700), dt, W, N)


@pytest.mark.parametrize("dt,H,J,D", SHAPES)
def test_attention_shapes_with_hidden_events(dt, H, J, D):
    check_attn(attn_case(dt, H, J, D, LENS["mixed"], 37, 6, hidden=0.4, pad=3), dt, 37, 6)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_attention_rows_that_see_nothing(dt):
    c = attn_case(dt, 4, 2, 64, [90, 40], 20, 2, all_hidden=True)
    for m in ("out", "dq", "dk", "dv"):
        assert (c[m] == 0).all(), m
    assert torch.isneginf(c["lse"].lse).all()
    check_attn(attn_case(dt, 4, 2, 64, [90, 40], 3, 1, hidden=0.8), dt, 3, 1)


def test_sinks_of_very_long_sequences_in_many_splits():
    # 64 splits of late rows; the oracle's own work bounds the length
    check_attn(attn_case("bf16", 2, 1, 32, [3, 2600, 10], 8, 35), "bf16", 8, 35)


@pytest.mark.parametrize("dt,H,J,D", [("bf16", 4, 2, 32), ("f32", 2, 1, 40), ("bf16", 2, 2, 128)])
@pytest.mark.parametrize("W,N", [(30, 5), (1, 1), (6, 64), (200, 3)])
@pytest.mark.parametrize("known", [False, True])
def test_a_long_history_among_many_short_ones(dt, H, J, D, W, N, known):
    """Far more sequences than rows / (sinks + window), some of which just have
    rows behind every sink's window or just do not."""
    edge = [W + N - 1, W + N, W + N + 1]
    lens = [3, 20, 1, 0, 9] * 20 + edge + [900] + edge[::-1] + [7, 2, 2] * 30
    check_attn(attn_case(dt, H, J, D, lens, W, N, pad=3, max_len=900 if known else 0), dt, W, N)


def banded(q, k, v, do, start, W, N, dt, longest):
    """One head over rows of sequences that begin at `start`, in float64 by each
    row's W + N keys: values and bounds of out, dq, dk, dv as oracle.seqattn has
    them."""
    T, D = q.shape
    u, U, scale = o.HALF_STEP[dt], o.U32, D ** -0.5
    r = u if dt == "bf16" else 0.0
    row = torch.arange(T, device=DEV)[:, None]
    win, sink = row - torch.arange(W, device=DEV), start[:, None] + torch.arange(N, device=DEV)
    ok = torch.cat([win >= start[:, None], sink <= row - W], 1)
    at = torch.cat([win, sink], 1).clamp(0, T - 1)
    K, V, Q, G = k[at], v[at], q[:, None], do[:, None]
    score = (Q * K).sum(-1) * scale
    P = torch.softmax(torch.where(ok, score, -torch.inf), 1)
    size = torch.where(ok, (Q.abs() * K.abs()).sum(-1) * scale, 0.0).amax(1, keepdim=True)
    es = (D + 8) * U * size + 4 * U * (1 + size) + (W + N + 8) * U
    out, mag = (P[..., None] * V).sum(1), (P[..., None] * V.abs()).sum(1)
    wide = (r + 2 * es + (W + N + 4) * U) * mag
    e_out, wide = wide * (1 + u) + u * out.abs(), wide + min(u, 2.0 ** -16) * out.abs() * (1 + u)
    dP, absdP = (G * V).sum(-1), (G.abs() * V.abs()).sum(-1)
    delta = (do * out).sum(1, keepdim=True)
    e_delta = (do.abs() * wide).sum(1, keepdim=True) + (D + 2) * U * (do.abs() * out.abs()).sum(1, keepdim=True)
    dS = P * (dP - delta)
    e_dS = P * ((D + 2) * U * absdP + e_delta) + (2 * es + r) * dS.abs() + 4 * U * P * (dP.abs() + delta.abs())
    n = longest + 8

    def per_key(w, x):                                       # sum over the rows of w x
        y = torch.zeros_like(x)
        return y.index_add_(0, at[ok], (w[..., None] * x[:, None])[ok])
    dq = scale * (dS[..., None] * K).sum(1)
    b = scale * ((e_dS + (W + N + 4) * U * dS.abs())[..., None] * K.abs()).sum(1)
    dk, bk = scale * per_key(dS, q), scale * per_key(e_dS + n * U * dS.abs(), q.abs())
    dv, bv = per_key(P, do), per_key((r + 2 * es + n * U) * P, do.abs())
    return [(out, e_out)] + [(x, y * (1 + u) + u * x.abs()) for x, y in ((dq, b), (dk, bk), (dv, bv))]


@pytest.mark.parametrize("dt,D,lens,W,N", [
    # more than 8192 late rows: pieces longer than a tile, up to 64 of them
    ("bf16", 32, [7, 12000, 300], 8, 5), ("f32", 40, [9000], 3, 40), ("bf16", 128, [20, 8300, 40, 9500], 40, 16),
    # more than 524288 rows: tiles above 128 rows
    ("bf16", 8, [3, 1, 11, 2] * 30000 + [20000] + [9, 4] * 4000, 4, 3)])
@pytest.mark.parametrize("known", [False, True])
def test_late_rows_in_long_pieces(dt, D, lens, W, N, known):
    off, T, s = plan(lens, max_len=max(lens) if known else 0)
    from paper_2512_09200_amd import api
    g = torch.Generator(device=DEV)
    g.manual_seed(D)
    q, k, v, do = (torch.randn(T, 1, D, generator=g, device=DEV).to(TT[dt]) for _ in range(4))
    out, saved = api.lattice_seq_attn_fwd(s, q, k, v, W, N)
    got = (out,) + tuple(api.lattice_seq_attn_bwd(s, q, k, v, out, saved, do, W, N))
    start = torch.from_numpy(np.repeat(off[:-1], np.diff(off))).to(DEV)
    want = banded(*(x[:, 0].double() for x in (q, k, v, do)), start, W, N, dt, max(lens))
    for x, (w, b), name in zip(got, want, ("out", "dq", "dk", "dv")):
        over = (x[:, 0].double() - w).abs() - b
        assert over.max() <= 1e-30, (name, int(over.amax(1).argmax()), float(over.max()))


@pytest.mark.parametrize("n,D", [(20, 64), (20, 32), (37, 128), (20, 8)])
def test_what_rounding_took_from_out_reaches_the_gradients(n, D):
    """Scores of 0 (q or k all zeros), so that probabilities are 1 / row count
    without rounding, and values between 1 and 1 + 3 / 128, whose differences are
    no larger than the rounding of out: a backward whose delta is from out
    alone is 5 to 80 times over these bounds."""
    from paper_2512_09200_amd import api
    rng = np.random.default_rng(n + D)
    U, u, sc = o.U32, o.HALF_STEP["bf16"], D ** -0.5
    off, rows, s = plan([n])
    bf = lambda x: torch.from_numpy(x.astype(np.float32)).to(torch.bfloat16)[:, None].to(DEV)  # noqa: E731
    V, DO = 1 + rng.integers(0, 4, (n, D)) * 2.0 ** -7, rng.choice([-1.0, 1.0], (n, D))
    x, zero = bf(1 + 0.5 * rng.random((n, D))), bf(np.zeros((n, D)))
    v, do, X = bf(V), bf(DO), f64(x)[:, 0]
    count = np.arange(1, n + 1)[:, None]
    P = np.tril(np.ones((n, n))) / count
    out = P @ V
    dP, delta = DO @ V.T, (DO * out).sum(1, keepdims=True)
    dS = P * (dP - delta)
    # out and out_lo: 2^-8 of 2^-8 of out, and the sum of `count` values
    e_out = (2.0 ** -16 + (count + 4) * U) * out
    e_dS = P * (D * U * np.abs(DO) @ V.T + (e_out + D * U * out).sum(1, keepdims=True)) + (u + 24 * U) * np.abs(dS)
    for q, k, which in ((zero, x, 1), (x, zero, 2)):
        y, saved = api.lattice_seq_attn_fwd(s, q, k, v, n)
        within(y.float() + saved.out_lo.float(), out[:, None], e_out[:, None], "out + out_lo")
        g = api.lattice_seq_attn_bwd(s, q, k, v, y, saved, do, n)[which - 1]
        w, e = (dS, e_dS) if which == 1 else (dS.T, e_dS.T)
        want = sc * w @ X
        bound = sc * (e @ X + (n + 4) * U * np.abs(w) @ X)
        within(g, want[:, None], (bound * (1 + u) + u * np.abs(want))[:, None], ("dq", "dk")[which - 1])


@pytest.mark.parametrize("dt,H,J,D", [("bf16", 4, 2, 64), ("f32", 2, 1, 40), ("bf16", 2, 1, 128)])
def test_attention_without_statistics_and_without_out_lo(dt, H, J, D):
    """lse=False gives the same out; without out_lo the rounding of out (u of it)
    enters delta."""
    from paper_2512_09200_amd import api
    W, N, n = 30, 3, 170
    c = attn_case(dt, H, J, D, [90, 80], W, N, hidden=0.1)
    out, none = api.lattice_seq_attn_fwd(c["s"], c["q"], c["k"], c["v"], lse=False, **c["kw"])
    assert none is None and torch.equal(out, c["out"])
    saved = api.SeqAttnSaved(c["lse"].lse, None)
    got = api.lattice_seq_attn_bwd(c["s"], c["q"], c["k"], c["v"], out, saved, c["do"], **c["kw"])
    if dt == "f32":
        assert all(torch.equal(a, c[m]) for a, m in zip(got, ("dq", "dk", "dv")))
        return
    q, k, v, do = (f64(c[m]) for m in ("q", "k", "v", "do"))
    sc, u = D ** -0.5, o.HALF_STEP[dt]
    f = o.attn(q, k, v, c["off"], W, N, sc, c["shown"], dt)
    g, b = o.attn_bwd(q, k, v, c["off"], W, N, sc, c["shown"], do, dt)
    assert torch.equal(got[2], c["dv"])
    e = u * (np.abs(do) * np.abs(f["o"])).sum(-1)                    # [rows, heads]
    for a, z in ((0, 90), (90, 170)):
        see = o.visible(z - a, W, N, c["shown"][a:z])
        for h in range(H):
            j = h // (H // J)
            P, _, _ = o._probabilities(q[a:z, h], np.where(c["shown"][a:z, None], k[a:z, j], 0), see, sc)
            w = P * e[a:z, h][:, None] * sc * (1 + u)
            b["dq"][a:z, h] += w @ np.where(c["shown"][a:z, None], np.abs(k[a:z, j]), 0)
            b["dk"][a:z, j] += w.T @ np.abs(q[a:z, h])
    assert n == c["rows"]
    within(got[0], g["dq"], b["dq"], "dq")
    within(got[1], g["dk"], b["dk"], "dk")


@pytest.mark.parametrize("dt,D", [("bf16", 64), ("f32", 128)])
def test_rows_behind_the_last_sequence_stay(dt, D):
    from paper_2512_09200_amd import api
    c = attn_case(dt, 4, 2, D, [70, 60], 40, 2, pad=130)
    n = 130
    qn, kn, vn, don = (c[m].clone() for m in ("q", "k", "v", "do"))
    for t in (qn, kn, vn, don):
        t[n:] = float("nan")
    mk = lambda t: torch.full_like(t, 3.0)  # noqa: E731
    out, lse = api.lattice_seq_attn_fwd(c["s"], qn, kn, vn, out=mk(c["out"]), **c["kw"])
    g = api.lattice_seq_attn_bwd(c["s"], qn, kn, vn, out, lse, don, dq=mk(c["dq"]), dk=mk(c["dk"]), dv=mk(c["dv"]),
                                 **c["kw"])
    for got, m in zip((out,) + tuple(g), ("out", "dq", "dk", "dv")):
        assert torch.equal(got[:n], c[m][:n]), m
        assert (got[n:] == 3).all(), m
        assert (c[m][n:] == 0).all(), m                # allocated by the call: zeros


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("dt,D", [("bf16", 64), ("f32", 32), ("bf16", 128)])
def test_nonfinite_values_reach_only_rows_that_see_them(dt, D, bad):
    from paper_2512_09200_amd import api
    lens, W, N = [90, 70, 140], 24, 2
    c = attn_case(dt, 4, 2, D, lens, W, N, hidden=0.2)
    n = sum(lens)
    see = np.zeros((n, n), bool)
    for a, e in zip(c["off"][:-1], c["off"][1:]):
        see[a:e, a:e] = o.visible(e - a, W, N, c["shown"][a:e])
    hidden = int(np.flatnonzero(~c["shown"])[3])
    shown = int(np.flatnonzero(c["shown"][100:])[5]) + 100
    # (which, row): rows of out / dq that may change, keys of dk / dv that may
    for which, at in (("k", hidden), ("v", hidden), ("k", shown), ("v", shown), ("q", 33), ("do", 200)):
        x = {m: c[m].clone() for m in ("q", "k", "v", "do")}
        x[which][at, :, 3] = bad
        out, lse = api.lattice_seq_attn_fwd(c["s"], x["q"], x["k"], x["v"], **c["kw"])
        dq, dk, dv = api.lattice_seq_attn_bwd(c["s"], x["q"], x["k"], x["v"], out, lse, x["do"], **c["kw"])
        if which in "kv":
            rows = see[:, at].copy()                   # rows that see it
            keys = see[rows].any(0)
            if which == "v":
                assert not np.isfinite(f64(out)[rows, :, 3]).any(), which
                rest = np.delete(f64(out), 3, axis=2)
                assert np.isfinite(rest).all()         # other dimensions of v are as they were
        else:
            rows = np.zeros(n, bool)
            rows[at] = True
            keys = see[at]
            if which == "do":
                assert torch.equal(out, c["out"])
        for m, touched in (("out", rows), ("dq", rows), ("dk", keys), ("dv", keys)):
            g = f64({"out": out, "dq": dq, "dk": dk, "dv": dv}[m])
            w = f64(c[m])
            assert np.isfinite(g[~touched]).all(), (which, at, m)
            assert np.allclose(g[~touched], w[~touched], rtol=2e-2, atol=1e-2 if dt == "bf16" else 1e-5), (which, at, m)


@pytest.mark.parametrize("dt,D,W,N", [("bf16", 64, 64, 2), ("f32", 32, 64, 0), ("bf16", 128, 64, 2), ("f32", 128, 12, 3),
                                      ("bf16", 32, 12, 3), ("bf16", 128, 12, 3)])
def test_nonfinite_values_stay_in_their_sequence_and_dimension(dt, D, W, N):
    """Bad values in different dimensions of two sequences that share tiles: an
    element is what the rows it is made of give, +-inf or NaN included."""
    from paper_2512_09200_amd import api
    inf, nan = float("inf"), float("nan")
    c = attn_case(dt, 2, 1, D, [40, 50], W, N)
    kw, n = c["kw"], 90
    see = np.zeros((n, n), bool)
    for a, e in ((0, 40), (40, 90)):
        see[a:e, a:e] = o.visible(e - a, W, N, np.ones(e - a, bool))

    def terms(bad, pairs):
        """What the bad elements (row, dimension, value) make of the elements
        [rows, dimensions] that have a positive weight for the row by pairs."""
        w = np.zeros((n, D))
        with np.errstate(invalid="ignore"):
            for at, d, x in bad:
                w[:, d] += np.where(pairs[:, at], x, 0.0)
        return w

    def check(got, want, bound, add, what):
        g = f64(got)
        add = np.broadcast_to(add[:, None, :], g.shape)
        ok = np.isfinite(add)
        assert np.array_equal(g[~ok], add[~ok], equal_nan=True), what
        over = np.where(ok, np.abs(g - want) - bound, -1.0)
        assert (over <= 1e-30).all(), (what, np.argwhere(~(over <= 1e-30))[:3])

    A3 = [f64(c[m]) for m in ("q", "k", "v")]
    all_shown, sc = np.ones(n, bool), D ** -0.5
    # v: +inf, -inf and both in one dimension, -inf and NaN of the other sequence in two others
    bad = [(5, 3, inf), (9, 3, -inf), (60, 5, nan), (45, 4, -inf)]
    v = c["v"].clone()
    for at, d, x in bad:
        v[at, :, d] = x
    out, sv = api.lattice_seq_attn_fwd(c["s"], c["q"], c["k"], v, **kw)
    f = o.attn(*A3, c["off"], W, N, sc, all_shown, dt)
    add = terms(bad, see)
    check(out, f["o"], f["o_bound"], add, "out")
    if sv.out_lo is not None:
        fine = torch.from_numpy(np.isfinite(add)).to(DEV)[:, None, :].expand_as(out)
        assert (sv.out_lo[fine].float().abs() <= 2.0 ** -8 * out[fine].float().abs()).all()
    # d_out: dv is its sum with positive weights
    bad = [(30, 3, inf), (33, 3, inf), (35, 2, -inf), (70, 5, nan), (66, 4, inf)]
    do = c["do"].clone()
    for at, d, x in bad:
        do[at, :, d] = x
    dq, dk, dv = api.lattice_seq_attn_bwd(c["s"], c["q"], c["k"], c["v"], c["out"], c["lse"], do, **kw)
    g, b = o.attn_bwd(*A3, c["off"], W, N, sc, all_shown, f64(c["do"]), dt)
    check(dv, g["dv"], b["dv"], terms(bad, see.T), "dv")
    touched = see[[at for at, _, _ in bad]].any(0)
    assert np.isfinite(f64(dk)[~touched]).all()
    # k: a key whose score is -inf has no weight, but 0 * inf in one dimension of
    # dq, and the other sequence's NaN is in another
    q, k = c["q"].clone(), c["k"].clone()
    q[:40, :, 3] = -q[:40, :, 3].abs() - 0.5
    k[7, :, 3], k[60, :, 5] = inf, nan
    out, sv = api.lattice_seq_attn_fwd(c["s"], q, k, c["v"], **kw)
    dq, dk, dv = api.lattice_seq_attn_bwd(c["s"], q, k, c["v"], out, sv, c["do"], **kw)
    k0 = c["k"].clone()
    shown = all_shown.copy()
    shown[7] = False
    B3 = f64(q), f64(k0), f64(c["v"])
    f = o.attn(*B3, c["off"], W, N, sc, shown, dt)
    g, b = o.attn_bwd(*B3, c["off"], W, N, sc, shown, f64(c["do"]), dt)
    rows = see[:, 60]                                            # all of their scores are NaN
    keys = see[rows].any(0)
    mine = see[:, 7].copy()
    for got, want, bound, hit, dims in ((out, f["o"], f["o_bound"], rows, []), (dk, g["dk"], b["dk"], keys, []),
                                        (dv, g["dv"], b["dv"], keys, []), (dq, g["dq"], b["dq"], rows, [3])):
        add = np.zeros((n, D))
        add[np.ix_(mine, dims)] = nan
        add[hit] = nan
        check(got, want, bound, add, "k")


@pytest.mark.parametrize("dt,D,W,N", [("bf16", 64, 24, 2), ("f32", 32, 24, 2), ("bf16", 128, 24, 0), ("bf16", 32, 200, 0),
                                      ("f32", 128, 1, 0)])
def test_rows_whose_scores_are_all_minus_infinity(dt, D, W, N):
    """Such a row is not one that sees nothing: its softmax is 0 / 0, in the
    batch and in the step alike; rows that see nothing keep their zeros."""
    from paper_2512_09200_amd import api
    c = attn_case(dt, 4, 2, D, [90, 1, 140], W, N, hidden=0.2)
    see = np.zeros((231, 231), bool)
    for a, e in zip(c["off"][:-1], c["off"][1:]):
        see[a:e, a:e] = o.visible(e - a, W, N, c["shown"][a:e])
    q, k = c["q"].clone(), c["k"].clone()
    k[:, :, 3] = k[:, :, 3].abs() + 1
    at = [0, 33, 90, 91, 130, 230] + list(np.flatnonzero(~see.any(1))[:3])
    q[at, :, 3] = -float("inf")
    out, sv = api.lattice_seq_attn_fwd(c["s"], q, k, c["v"], **c["kw"])
    dq, dk, dv = api.lattice_seq_attn_bwd(c["s"], q, k, c["v"], out, sv, c["do"], **c["kw"])
    bad = np.zeros(231, bool)
    bad[at] = True
    none = ~see.any(1)
    want = bad & ~none
    assert want.sum() >= 4 and (W > 1 or none.any())
    for x in (out, dq):
        x = f64(x)
        assert np.isnan(x[want]).all() and np.isfinite(x[~want]).all() and (x[none] == 0).all()
    L = f64(sv.lse)
    assert np.isnan(L[:, want]).all() and np.isneginf(L[:, none]).all() and np.isfinite(L[:, ~want & ~none]).all()
    keys = see[want].any(0)
    for x in (dk, dv):
        assert np.isnan(f64(x)[keys]).all() and np.isfinite(f64(x)[~keys]).all()
    kc, vc = (torch.zeros(1, 2, N + W, D, dtype=TT[dt], device=DEV) for _ in range(2))
    step = api.lattice_seq_step(q[:1], k[:1], c["v"][:1], torch.zeros(1, dtype=torch.int32, device=DEV), kc, vc, W, N,
                                rope=False)
    assert torch.isnan(step).all()


def test_attention_twice_on_side_streams_and_in_a_graph_gives_the_same_bits():
    from paper_2512_09200_amd import api
    c = attn_case("bf16", 8, 2, 64, LENS["mixed"], 60, 4, hidden=0.1)
    names = ("out", "lse", "lo", "dq", "dk", "dv")
    c.update(lo=c["lse"].out_lo, lse=c["lse"].lse)

    def go():
        s = api.lattice_seq_plan(c["s"].offsets, c["rows"], max_len=400)
        out, lse = api.lattice_seq_attn_fwd(s, c["q"], c["k"], c["v"], **c["kw"])
        return (out, lse.lse, lse.out_lo) + tuple(api.lattice_seq_attn_bwd(s, c["q"], c["k"], c["v"], out, lse, c["do"],
                                                                           **c["kw"]))

    def same(r):
        for x, m in zip(r, names):
            assert torch.equal(x, c[m]), m

    same(go())
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s1):
        r1 = go()
    with torch.cuda.stream(s2):
        r2 = go()
    torch.cuda.synchronize()
    same(r1)
    same(r2)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        rg = go()
    for _ in range(3):
        for x in rg:
            x.zero_()
        g.replay()
        same(go())                                     # eager work between the replays
        torch.cuda.synchronize()
        same(rg)


def test_hidden_sinks_get_no_gradient_from_late_rows_that_are_not_finite():
    from paper_2512_09200_amd import api
    rng = np.random.default_rng(11)
    off, rows, s = plan([200])
    q, do = (randn(rng, rows, 2, 32).to(DEV) for _ in "qo")
    k, v = (randn(rng, rows, 1, 32).to(DEV) for _ in "kv")
    mask = torch.ones(rows, dtype=torch.uint8, device=DEV)
    mask[1] = 0                                        # one of three sinks
    q[150] = float("nan")                              # behind every sink's window
    kw = dict(window=20, sinks=3, key_mask=mask)
    out, saved = api.lattice_seq_attn_fwd(s, q, k, v, **kw)
    dq, dk, dv = api.lattice_seq_attn_bwd(s, q, k, v, out, saved, do, **kw)
    seen = np.zeros(rows, bool)
    seen[[0, 2]] = True
    seen[131:151] = True
    for t in (dk, dv):
        assert np.array_equal(np.isfinite(f64(t)).all((1, 2)), ~seen)
    assert (dk[1] == 0).all() and (dv[1] == 0).all()


def test_rows_beyond_4_gib():
    """Row strides of 2^22 elements: byte offsets past 32 bits in every tensor."""
    from paper_2512_09200_amd import api
    rng = np.random.default_rng(2)
    T, H, J, D, ld = 600, 2, 1, 32, 1 << 22
    big = torch.empty(T * ld, dtype=torch.bfloat16, device=DEV).view(T, ld)
    q = randn(rng, T, H, D).to(torch.bfloat16).to(DEV)
    k, v = (randn(rng, T, J, D).to(torch.bfloat16).to(DEV) for _ in "kv")
    do = randn(rng, T, H, D).to(torch.bfloat16).to(DEV)
    wide = {}
    for i, (n, t) in enumerate((("q", q), ("k", k), ("v", v), ("do", do))):
        wide[n] = big[:, 256 * i:256 * i + t.shape[1] * D].view(T, t.shape[1], D)
        wide[n].copy_(t)
    off, rows, s = plan([T])
    kw = dict(window=70, sinks=4)
    out, sv = api.lattice_seq_attn_fwd(s, q, k, v, **kw)
    ref = api.lattice_seq_attn_bwd(s, q, k, v, out, sv, do, **kw)
    o2 = [big[:, 2048 + 256 * i:2048 + 256 * i + h * D].view(T, h, D) for i, h in enumerate((H, H, J, J, H, J))]
    out2, sv2 = api.lattice_seq_attn_fwd(s, wide["q"], wide["k"], wide["v"], out=o2[0], **kw)
    g2 = api.lattice_seq_attn_bwd(s, wide["q"], wide["k"], wide["v"], out2, sv2, wide["do"], dq=o2[1], dk=o2[2],
                                  dv=o2[3], **kw)
    assert torch.equal(out2, out) and all(torch.equal(a, b) for a, b in zip(g2, ref))
    r = api.lattice_qk_rope_fwd(s, q, k)
    r2 = api.lattice_qk_rope_fwd(s, wide["q"], wide["k"], q_out=o2[4], k_out=o2[5])
    assert all(torch.equal(a, b) for a, b in zip(r, r2))


def test_hundreds_of_thousands_of_sequences():
    """Sequences of one and two rows, far more than blocks or grid dimensions
    of 16 bits: values by hand (a row that sees only itself returns its v: the
    probability p and the sum l = p are the same number, so p v (1 / l) has three
    roundings, 2^-24 each)."""
    from paper_2512_09200_amd import api
    S, D = 300_000, 8
    lens = np.tile([1, 2, 1], S // 3)
    off = offs(lens)
    T = int(off[-1])
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    q, k, v, do = (torch.randn(T, 1, D, generator=g, device=DEV) for _ in range(4))
    s = api.lattice_seq_plan(torch.from_numpy(off.astype(np.int32)).to(DEV), T, max_len=3)
    out, sv = api.lattice_seq_attn_fwd(s, q, k, v, 1, 1)      # window 1: itself, and the first row
    dq, dk, dv = api.lattice_seq_attn_bwd(s, q, k, v, out, sv, do, 1, 1)
    second = torch.zeros(T, dtype=torch.bool, device=DEV)
    second[torch.from_numpy(off[:-1][lens == 2] + 1).to(DEV)] = True
    first = torch.roll(second, -1)
    assert ((out[~second] - v[~second]).abs() <= 4 * 2.0 ** -24 * v[~second].abs()).all()
    a, b = q[second].double(), torch.stack([k[first], k[second]]).double()
    P = torch.softmax((a * b).sum(-1, keepdim=True) * D ** -0.5, 0)
    w = (P * torch.stack([v[first], v[second]]).double()).sum(0)
    assert (out[second].double() - w).abs().max() < 1e-5
    # P = exp(s - lse): s and lse up to 8 with 2^-24 each for four roundings
    assert (dv[~second & ~first].double() - do[~second & ~first].double()).abs().max() < 1e-5
    assert (dv[second].double() - P[1] * do[second].double()).abs().max() < 1e-5
    assert (dv[first].double() - (do[first].double() + P[0] * do[second].double())).abs().max() < 1e-5


def test_caches_beyond_4_gib():
    from paper_2512_09200_amd import api
    rng = np.random.default_rng(4)
    J, D, W, N, C = 1, 128, 100_000, 4, 200              # 5 GB a cache tensor
    kc, vc = (torch.empty(C, J, W + N, D, dtype=torch.bfloat16, device=DEV) for _ in "kv")
    k1, v1 = (torch.zeros(1, J, W + N, D, dtype=torch.bfloat16, device=DEV) for _ in "kv")
    hist = 3000
    off, rows, s = plan([hist])
    kh, vh = (randn(rng, hist, J, D).to(torch.bfloat16).to(DEV) for _ in "kv")
    last = torch.tensor([C - 1], dtype=torch.int32, device=DEV)
    api.lattice_seq_cache_fill(s, kh, vh, kc, vc, W, N, cache_index=last)
    api.lattice_seq_cache_fill(s, kh, vh, k1, v1, W, N)
    assert torch.equal(kc[-1, :, :hist], k1[0, :, :hist]) and torch.equal(vc[-1, :, :hist], v1[0, :, :hist])
    q, k, v = (randn(rng, 1, h, D).to(torch.bfloat16).to(DEV) for h in (4, J, J))
    lens = torch.tensor([hist], dtype=torch.int32, device=DEV)
    a = api.lattice_seq_step(q, k, v, lens, kc, vc, W, N, cache_index=last)
    b = api.lattice_seq_step(q, k, v, lens, k1, v1, W, N)
    assert torch.equal(a, b) and torch.equal(kc[-1, :, hist], k1[0, :, hist])


def test_a_stream_of_its_own_keeps_its_memory():
    """Calls on a stream that is not the current one: their outputs and
    workspaces are not handed out again while that stream is behind."""
    from paper_2512_09200_amd import api
    c = attn_case("bf16", 4, 2, 64, [700, 300], 50, 4)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = []
    for _ in range(4):
        p = api.lattice_seq_plan(c["s"].offsets, c["rows"], stream=s)
        out, sv = api.lattice_seq_attn_fwd(p, c["q"], c["k"], c["v"], stream=s, **c["kw"])
        got.append(api.lattice_seq_attn_bwd(p, c["q"], c["k"], c["v"], out, sv, c["do"], stream=s, **c["kw"]))
        del p, out, sv
        torch.full((1 << 20,), -1.0, device=DEV)         # the current stream writes what it is given
    torch.cuda.synchronize()
    for g in got:
        assert all(torch.equal(x, c[m]) for x, m in zip(g, ("dq", "dk", "dv")))


def test_a_padded_batch_on_a_stream_of_its_own_while_the_current_one_is_behind():
    """Outputs of a padded plan are zero-filled on the call's own stream: a fill
    still queued on the current one would wipe them afterwards."""
    from paper_2512_09200_amd import api
    c = attn_case("bf16", 4, 2, 64, [700, 300], 50, 4, pad=40)
    s = torch.cuda.Stream()
    q0, k0 = api.lattice_qk_rope_fwd(c["s"], c["q"], c["k"])
    g0 = api.lattice_qk_rope_bwd(c["s"], c["q"], c["k"], c["do"], c["k"])[:2]
    want = [c["out"], c["dq"], c["dk"], c["dv"], q0, k0, *g0]
    busy = torch.zeros(8192, 8192, device=DEV)
    torch.mm(busy, busy)
    torch.cuda.synchronize()
    for _ in range(16):                                     # about a tenth of a second
        busy = torch.mm(busy, busy)
    out, sv = api.lattice_seq_attn_fwd(c["s"], c["q"], c["k"], c["v"], stream=s, **c["kw"])
    got = [out, *api.lattice_seq_attn_bwd(c["s"], c["q"], c["k"], c["v"], out, sv, c["do"], stream=s, **c["kw"])]
    got += api.lattice_qk_rope_fwd(c["s"], c["q"], c["k"], stream=s)
    got += api.lattice_qk_rope_bwd(c["s"], c["q"], c["k"], c["do"], c["k"], stream=s)[:2]
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert torch.equal(g, w)


def test_memory_of_a_call_on_its_own_stream_is_not_still_in_use_by_the_current_one():
    """Memory that was just freed while the current stream has yet to write it
    is not handed to a call on another stream."""
    from paper_2512_09200_amd import api
    c = attn_case("bf16", 4, 2, 64, [700, 300], 50, 4)
    s = torch.cuda.Stream()
    busy = torch.zeros(8192, 8192, device=DEV)
    torch.mm(busy, busy)
    torch.cuda.synchronize()
    for _ in range(16):
        busy = torch.mm(busy, busy)
    late = [torch.empty_like(c["q"]).fill_(-1.0) for _ in range(8)]
    del late
    out, sv = api.lattice_seq_attn_fwd(c["s"], c["q"], c["k"], c["v"], stream=s, **c["kw"])
    torch.cuda.synchronize()
    assert torch.equal(out, c["out"])


def test_a_step_and_a_fill_on_a_stream_of_its_own():
    from paper_2512_09200_amd import api
    rng = np.random.default_rng(11)
    s = torch.cuda.Stream()
    x = [randn(rng, 3, h, 64).to(DEV) for h in (4, 2, 2)]
    plan = api.lattice_seq_plan(torch.tensor([0, 3], dtype=torch.int32, device=DEV), 3)
    lens = torch.tensor([3, -1, 0], dtype=torch.int32, device=DEV)
    got = []
    for st in (None, s):
        kc, vc = (torch.zeros(3, 2, 12, 64, device=DEV) for _ in range(2))
        out = torch.full_like(x[0], 7.0)
        torch.cuda.synchronize()
        api.lattice_seq_cache_fill(plan, x[1], x[2], kc, vc, 8, 4, stream=st)
        assert api.lattice_seq_step(*x, lens, kc, vc, 8, 4, out=out, stream=st) is out
        torch.cuda.synchronize()
        got.append((out, kc, vc))
    for a, b in zip(*got):
        assert torch.equal(a, b)
    assert torch.all(got[0][0][1] == 7.0)


# ---------------------------------------------------------------------------
@pytest.mark.parametrize("dt,J,D,W,N", [("bf16", 2, 64, 30, 3), ("f32", 1, 8, 1, 0), ("bf16", 3, 40, 7, 64),
                                        ("f32", 2, 128, 200, 1), ("bf16", 40, 128, 20, 2)])
@pytest.mark.parametrize("first", [False, True])
def test_cache_fill(dt, J, D, W, N, first):
    from paper_2512_09200_amd import api
    rng = np.random.default_rng(W + D)
    lens = [3, 0, 300, 29, 1, 77]
    off, rows, s = plan(lens, pad=4)
    k, v = randn(rng, rows, J, D).to(TT[dt]).to(DEV), randn(rng, rows, J, D).to(TT[dt]).to(DEV)
    kc, vc = (randn(rng, 9, J, W + N, D).to(TT[dt]).to(DEV) for _ in "kv")
    index = np.array([4, 0, 8, 9, -1, 2])                  # the fourth and fifth are out of range
    f = np.array([0, 7, 5, 0, 3, 1000]) if first else np.zeros(6, int)
    want = o.cache_fill(f64(kc), f64(vc), f64(k), f64(v), off, W, N, index, f)
    i32 = lambda a: torch.from_numpy(a.astype(np.int32)).to(DEV)  # noqa: E731
    api.lattice_seq_cache_fill(s, k, v, kc, vc, W, N, cache_index=i32(index), first=i32(f) if first else None)
    assert np.array_equal(f64(kc), want[0]) and np.array_equal(f64(vc), want[1])


STEP = [("bf16", 4, 2, 64, 30, 3), ("f32", 2, 1, 32, 5, 0), ("bf16", 8, 1, 128, 700, 4), ("f32", 3, 3, 96, 129, 1),
        ("bf16", 20, 1, 40, 64, 64), ("f32", 17, 1, 128, 333, 7), ("bf16", 2, 2, 8, 1, 0), ("bf16", 32, 2, 128, 5000, 2)]


@pytest.mark.parametrize("dt,H,J,D,W,N", STEP)
@pytest.mark.parametrize("rope", [True, False])
def test_step_against_the_definition(dt, H, J, D, W, N, rope):
    from paper_2512_09200_amd import api
    rng = np.random.default_rng(H + D + W)
    cap = W + N
    lens = np.array([0, 1, N, cap - 1, cap, 3 * cap + 1, -1, min(cap, 200) // 2, 5])
    B = len(lens)
    index = rng.permutation(B + 2)[:B]
    index[8] = B + 2                                       # out of range
    q, k, v = (randn(rng, B, h, D).to(TT[dt]).to(DEV) for h in (H, J, J))
    kc, vc = (randn(rng, B + 2, J, cap, D).to(TT[dt]).to(DEV) for _ in "kv")
    for b in range(B):                                     # slots nothing was written to yet
        if 0 <= lens[b] < cap and index[b] < B + 2:
            kc[index[b], :, lens[b]:] = float("nan")
            vc[index[b], :, lens[b]:] = float("nan")
    pos = rng.integers(0, 2 ** 30, B)
    gq, gk = 1 + 0.1 * randn(rng, D), 1 + 0.1 * randn(rng, D)
    R = D // 16 * 8
    i32 = lambda a: torch.from_numpy(a.astype(np.int32)).to(DEV)  # noqa: E731
    kc0, vc0 = f64(kc), f64(vc)
    out = torch.full((B, H, D), 5.0, dtype=TT[dt], device=DEV)
    kw = dict(gain_q=gq.to(DEV), gain_k=gk.to(DEV), rotary=R, positions=i32(pos)) if rope else dict(rope=False)
    api.lattice_seq_step(q, k, v, i32(lens), kc, vc, W, N, cache_index=i32(index), out=out, **kw)
    Q, K, V = f64(q), f64(k), f64(v)
    u = o.HALF_STEP[dt]
    eq = np.zeros(B)
    if rope:
        Qr, _ = o.qk_rope(Q, f64(gq), pos, R, 1e4, 1e-6, False)
        Kr, _ = o.qk_rope(K, f64(gk), pos, R, 1e4, 1e-6, False)
    else:
        Qr, Kr = Q, K
    KC, VC = f64(kc), f64(vc)
    for b in range(B):
        at = index[b]
        if lens[b] < 0 or at >= B + 2:
            assert (out[b] == 5).all()
            if at < B + 2:
                assert np.array_equal(KC[at], kc0[at], equal_nan=True)
            continue
        slot, n = o.slot_of(int(lens[b]), W, N), min(lens[b] + 1, cap)
        kc0[at, :, slot], vc0[at, :, slot] = Kr[b], V[b]
        e = (u if rope else 0) * np.abs(Kr[b]) + (D + 40) * o.U32 * np.abs(Kr[b]).max() * 1.5
        assert (np.abs(KC[at, :, slot] - Kr[b]) <= e).all()
        assert np.array_equal(VC[at, :, slot], V[b])
        kc0[at, :, slot] = KC[at, :, slot]                 # the attention reads the stored key
        assert np.array_equal(KC[at], kc0[at], equal_nan=True) and np.array_equal(VC[at], vc0[at], equal_nan=True)
        for h in range(H):
            j = h // (H // J)
            kk, vv = KC[at, j, :n], VC[at, j, :n]
            s = kk @ Qr[b, h] / np.sqrt(D)
            size = (np.abs(kk) @ np.abs(Qr[b, h])).max() / np.sqrt(D)
            p = np.exp(s - s.max())
            P = p / p.sum()
            # the rotated query is rounded to the storage type (u per element of
            # each product), then as the batch's attention
            es = (u if rope else 0) * size + (2 * D + 48) * o.U32 * size * 1.5 + (n + 16) * o.U32
            r = u if dt == "bf16" else 0
            # P's error: exp(es) - 1 up, its normalisation the same
            bound = (r + 2 * np.expm1(es)) * (P @ np.abs(vv)) + u * np.abs(P @ vv) * (1 + r)
            within(out[b, h], P @ vv, bound, f"out {b} {h}")
    _ = eq


@pytest.mark.parametrize("H,J,D,W,N", [(8, 2, 64, 30, 3), (4, 4, 32, 5, 0), (20, 1, 40, 64, 36), (6, 3, 128, 20, 4)])
@pytest.mark.parametrize("rope", [True, False])
def test_step_rounds_the_query_and_the_probabilities_in_two_parts(H, J, D, W, N, rope):
    """Few slots, where one bf16 part of either would be 1.8 to 8 times over the
    bound: 2^-8 of 2^-8 for each, fp32 sums, one rounding of out."""
    from paper_2512_09200_amd import api
    rng = np.random.default_rng(D + W)
    B, cap, U, u = 6, W + N, o.U32, o.HALF_STEP["bf16"]
    q, k, v = (randn(rng, B, h, D).to(torch.bfloat16).to(DEV) for h in (H, J, J))
    kc, vc = (randn(rng, B, J, cap, D).to(torch.bfloat16).to(DEV) for _ in "kv")
    lens = torch.tensor([cap, cap + 1, 3 * cap, cap - 1, cap // 2, 5 * cap], dtype=torch.int32, device=DEV)
    gq, gk = (1 + 0.1 * randn(rng, D)).to(DEV), (1 + 0.1 * randn(rng, D)).to(DEV)
    kw = dict(gain_q=gq, gain_k=gk) if rope else dict(rope=False)
    out = api.lattice_seq_step(q, k, v, lens, kc, vc, W, N, **kw)
    Q, KC, VC = f64(q), f64(kc), f64(vc)
    if rope:
        Q, _ = o.qk_rope(Q, f64(gq), lens.cpu().numpy(), D, 1e4, 1e-6, False)
    for b in range(B):
        n = min(int(lens[b]) + 1, cap)
        for h in range(H):
            kk, vv = KC[b, h // (H // J), :n], VC[b, h // (H // J), :n]
            s = kk @ Q[b, h] / np.sqrt(D)
            P = np.exp(s - s.max())
            P /= P.sum()
            size = (np.abs(kk) @ np.abs(Q[b, h])).max() / np.sqrt(D)
            es = (2.0 ** -16 if rope else 0) * size + (2 * D + 48) * U * size * 1.5 + (n + 16) * U
            bound = (2.0 ** -16 + 2 * np.expm1(es)) * (P @ np.abs(vv)) + u * np.abs(P @ vv) * (1 + 2.0 ** -16)
            within(out[b, h], P @ vv, bound, f"out {b} {h}")


@pytest.mark.parametrize("dt,H,J,D,W,N", [("bf16", 4, 2, 64, 16, 2), ("f32", 4, 1, 32, 40, 0)])
def test_histories_trained_and_served_alike(dt, H, J, D, W, N):
    """Norm and rotation, attention, cache fill, then event by event: the
    served outputs are the batch's last rows, and the caches those that a
    fill with the whole history gives."""
    from paper_2512_09200_amd import api
    rng = np.random.default_rng(1)
    lens, more = np.array([5, 0, 33, 90]), 20
    full = lens + more
    off = offs(full)
    q, k, v = (randn(rng, int(off[-1]), h, D).to(TT[dt]).to(DEV) for h in (H, J, J))
    gq, gk = (1 + 0.1 * randn(rng, D)).to(DEV), (1 + 0.1 * randn(rng, D)).to(DEV)
    kw = dict(gain_q=gq, gain_k=gk, theta=500.0)
    i32 = lambda a: torch.from_numpy(np.asarray(a).astype(np.int32)).to(DEV)  # noqa: E731
    s = api.lattice_seq_plan(i32(off), int(off[-1]))
    qr, kr = api.lattice_qk_rope_fwd(s, q, k, **kw)
    ref, lse = api.lattice_seq_attn_fwd(s, qr, kr, v, W, N)
    # training: the chain's gradient against the oracle's chain
    do = randn(rng, *q.shape).to(TT[dt]).to(DEV)
    dqr, dkr, dv = api.lattice_seq_attn_bwd(s, qr, kr, v, ref, lse, do, W, N)
    dq, dk, dgq, dgk = api.lattice_qk_rope_bwd(s, q, k, dqr, dkr, **kw)
    pos = o.positions_of(off, int(off[-1]))
    Q, _ = o.qk_rope(f64(q), f64(gq), pos, D, 500.0, 1e-6, False)
    K, _ = o.qk_rope(f64(k), f64(gk), pos, D, 500.0, 1e-6, False)
    shown = np.ones(len(Q), bool)
    g, _ = o.attn_bwd(Q, K, f64(v), off, W, N, D ** -0.5, shown, f64(do))
    tol = 3e-2 if dt == "bf16" else 1e-5
    for x, gain, dy, dx, dg in ((q, gq, g["dq"], dq, dgq), (k, gk, g["dk"], dk, dgk)):
        wdx, wdg, _ = o.qk_rope_bwd(f64(x), f64(gain), pos, D, 500.0, 1e-6, False, dy)
        assert np.linalg.norm(f64(dx) - wdx) <= tol * np.linalg.norm(wdx)
        assert np.linalg.norm(f64(dg) - wdg) <= tol * np.linalg.norm(wdg)
    assert np.linalg.norm(f64(dv) - g["dv"]) <= tol * np.linalg.norm(g["dv"])
    # serving
    idx = i32([2, 0, 3, 1])
    kc = torch.zeros(4, J, W + N, D, dtype=TT[dt], device=DEV)
    vc = torch.zeros_like(kc)
    past = np.concatenate([np.arange(a, a + n) for a, n in zip(off[:-1], lens)])
    s0 = api.lattice_seq_plan(i32(offs(lens)), int(lens.sum()))
    api.lattice_seq_cache_fill(s0, kr[past], v[past], kc, vc, W, N, cache_index=idx)
    have = i32(lens)
    for t in range(more):
        rows = off[:-1] + lens + t
        out = api.lattice_seq_step(q[rows], k[rows], v[rows], have, kc, vc, W, N, cache_index=idx, **kw)
        # two correct evaluations of one row, each off by P's and its own rounding
        err = np.linalg.norm(f64(out) - f64(ref[rows]), axis=-1) / np.linalg.norm(f64(ref[rows]), axis=-1)
        assert err.max() <= (4 * 2.0 ** -8 * np.sqrt(W + N) if dt == "bf16" else 1e-5), t
        have += 1
    kc2, vc2 = torch.zeros_like(kc), torch.zeros_like(vc)
    api.lattice_seq_cache_fill(s, kr, v, kc2, vc2, W, N, cache_index=idx)
    assert torch.equal(vc, vc2)
    assert (kc.float() - kc2.float()).abs().max() <= (2 ** -5 if dt == "bf16" else 1e-5)


def test_step_in_a_graph_that_advances_by_itself():
    from paper_2512_09200_amd import api
    rng = np.random.default_rng(5)
    B, H, J, D, W, N = 3, 4, 2, 64, 900, 2
    q, k, v = (randn(rng, B, h, D).to(torch.bfloat16).to(DEV) for h in (H, J, J))
    kc, vc = (torch.zeros(B, J, W + N, D, dtype=torch.bfloat16, device=DEV) for _ in "kv")
    lens = torch.zeros(B, dtype=torch.int32, device=DEV)
    k2, v2, l2 = kc.clone(), vc.clone(), lens.clone()

    def go(kc, vc, lens):
        out = api.lattice_seq_step(q, k, v, lens, kc, vc, W, N)
        lens += 1
        return out
    go(k2, v2, l2)                                          # the library is loaded, kernels too
    k2.zero_(), v2.zero_(), l2.zero_()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        rg = go(kc, vc, lens)
    for t in range(5):
        q.copy_(randn(rng, B, H, D).to(DEV))
        k.copy_(randn(rng, B, J, D).to(DEV))
        g.replay()
        ref = go(k2, v2, l2)
        torch.cuda.synchronize()
        assert torch.equal(rg, ref), t
    assert torch.equal(kc, k2) and torch.equal(lens, l2)


def test_binding_refusals():
    from paper_2512_09200_amd import api
    from paper_2512_09200_amd._abi import LatticeError
    off, rows, s = plan([10, 6])
    q = torch.zeros(16, 4, 64, device=DEV)
    k = torch.zeros(16, 2, 64, device=DEV)
    with pytest.raises(ValueError):
        api.lattice_seq_attn_fwd(s, q[:15], k[:15], k[:15], 4)
    with pytest.raises(ValueError):
        api.lattice_seq_attn_fwd(s, q, k, k.bfloat16(), 4)
    with pytest.raises(ValueError):
        api.lattice_seq_attn_fwd(s, q, k, k.cpu(), 4)
    with pytest.raises(ValueError):
        api.lattice_qk_rope_fwd(None, q, k)
    with pytest.raises(LatticeError, match="INVALID_ARG"):
        api.lattice_seq_attn_fwd(s, q, k, k, 0)
    with pytest.raises(LatticeError, match="INVALID_ARG"):          # 4-byte aligned
        x = torch.zeros(16 * 256 + 1, device=DEV)[1:].view(16, 4, 64)
        api.lattice_seq_attn_fwd(s, x, k, k, 4)
    with pytest.raises(LatticeError, match="UNSUPPORTED"):
        api.lattice_seq_attn_fwd(s, torch.zeros(16, 1, 136, device=DEV), torch.zeros(16, 1, 136, device=DEV),
                                 torch.zeros(16, 1, 136, device=DEV), 4)
    with pytest.raises(TypeError):
        api.lattice_seq_attn_fwd(s, q.half(), k.half(), k.half(), 4)
    # no rows, no sequences
    none = api.lattice_seq_plan(torch.zeros(1, dtype=torch.int32, device=DEV), 0)
    out, lse = api.lattice_seq_attn_fwd(none, q[:0], k[:0], k[:0], 4)
    assert out.shape == (0, 4, 64) and lse.lse.shape == (4, 0)
    dq, dk, dgq, dgk = api.lattice_qk_rope_bwd(none, q[:0], k[:0], q[:0], k[:0], gain_q=torch.ones(64, device=DEV))
    assert (dgq == 0).all() and dgk is None
    api.lattice_seq_attn_bwd(none, q[:0], k[:0], k[:0], out, lse, q[:0], 4)
