"""Dropout and the residual norm on the GPU against the float64 oracle, element
by element within the bound that follows from the roundings (oracle/norm.py)."""
import numpy as np
import pytest
import torch

from oracle import fp8
from oracle import norm as o

DEV = "cuda"
TT = {"bf16": torch.bfloat16, "f32": torch.float32}
pytestmark = pytest.mark.gpu
SEED, STEP, SITE = 0x7edc_ba98_7654_3210, 0x1_2345_6789, 5


def f64(t):
    return t.detach().float().cpu().double().numpy()


def rng_state(seed=SEED, step=STEP):
    return torch.tensor([seed, step], dtype=torch.int64, device=DEV)


def randn(rng, dt, *shape):
    return torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(TT[dt]).to(DEV)


def within(got, want, bound, what):
    g = f64(got)
    assert np.isfinite(g).all(), f"{what}: not finite"
    over = np.abs(g - want) - bound
    i = np.unravel_index(np.argmax(over), over.shape)
    assert over[i] <= 1e-30, f"{what} at {i}: {g[i]} against {want[i]}, bound {np.broadcast_to(bound, over.shape)[i]}"


def rounded(x, dt):
    """x (float64) in the storage type, by way of fp32 as the kernel's sums are."""
    return torch.from_numpy(x.astype(np.float32)).to(TT[dt]).double().numpy()


# ---------------------------------------------------------------------------
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 8), (3, 7), (53, 33), (5, 1024), (700, 129), (2, 70001), (4099, 16),
                                       (1, 8192), (8193, 1)])
@pytest.mark.parametrize("p", [0.1, 0.5, 65535 / 65536])
def test_dropout(dt, rows, cols, p):
    from paper_2512_09200_amd import api
    r = np.random.default_rng(rows + cols)
    x = randn(r, dt, rows, cols)
    out = api.lattice_dropout(x, p, rng_state(), site=SITE)
    f = o.factor(np.arange(rows), cols, p, SEED, STEP, SITE)
    # the factor in fp32, the product, the rounding
    within(out, f64(x) * f, np.abs(f64(x) * f) * (2 * o.U32 + o.HALF_STEP[dt]) * 1.001, "out")
    assert torch.equal(out, api.lattice_dropout(x, p, rng_state(), site=SITE))


def test_dropout_strides_in_place_and_nothing_else_written():
    from paper_2512_09200_amd import api
    r = np.random.default_rng(1)
    buf = randn(r, "bf16", 77, 61)
    keep = buf.clone()
    x = buf[:, 3:54]                                          # 51 columns at an odd address
    want = api.lattice_dropout(x.contiguous(), 0.3, rng_state())
    got = api.lattice_dropout(x, 0.3, rng_state(), out=x)
    assert got.data_ptr() == x.data_ptr() and torch.equal(x, want)
    keep[:, 3:54] = want
    assert torch.equal(buf, keep)


def test_dropout_drops_nan_and_keeps_it():
    from paper_2512_09200_amd import api
    x = torch.full((40, 40), float("nan"), device=DEV)
    out = api.lattice_dropout(x, 0.5, rng_state())
    f = o.factor(np.arange(40), 40, 0.5, SEED, STEP, 0)
    assert np.array_equal(np.isnan(f64(out)), f > 0) and (f64(out)[f == 0] == 0).all()


def test_dropout_of_nothing_copies():
    from paper_2512_09200_amd import api
    x = torch.randn(9, 19, device=DEV)
    for p in (0.0, 2.0 ** -18):
        assert torch.equal(api.lattice_dropout(x, p, None), x)
    for shape in ((0, 5), (5, 0), (0, 0)):
        assert api.lattice_dropout(torch.empty(shape, device=DEV), 0.5, rng_state()).shape == shape


def test_dropout_of_more_elements_than_32_bits_count():
    from paper_2512_09200_amd import api
    rows, cols = 2_150_000, 2048                              # 4.4e9 elements
    x = torch.ones(rows, cols, dtype=torch.bfloat16, device=DEV)
    api.lattice_dropout(x, 0.5, rng_state(), site=1, out=x)
    for a in (0, 1_048_576, 2_097_151, rows - 3):
        f = o.factor(np.arange(a, a + 3), cols, 0.5, SEED, STEP, 1)
        assert np.array_equal(f64(x[a:a + 3]), f)


# ---------------------------------------------------------------------------
SIZES = [(1, 1), (3, 7), (5, 8), (7, 100), (130, 128), (9, 129), (33, 250), (64, 256), (41, 257), (40, 512), (21, 511),
         (50, 1000), (17, 1024), (5, 2048), (6, 1999), (3, 4096), (2, 4095), (5, 8192), (3, 8185), (2, 16384), (2, 16383)]


def run_case(dt, rows, cols, residual, p, out, gain=True, eps=1e-5, seed=0, make=None):
    from paper_2512_09200_amd import api
    r = np.random.default_rng(1000 * cols + rows + seed)
    make = make or (lambda *shape: randn(r, dt, *shape))
    c = dict(x=make(rows, cols), res=make(rows, cols) * 2 if residual else None, dy=make(rows, cols),
             dh=make(rows, cols) if residual else None,
             gain=torch.from_numpy(1 + 0.3 * r.standard_normal(cols)).float().to(DEV) if gain else None)
    drop = (p, rng_state(), SITE) if p else None
    kw = dict(gain=c["gain"], eps=eps, dropout=drop)
    c["h"], c["y"], c["codes"], c["scales"] = api.lattice_add_rmsnorm_fwd(c["x"], c["res"], out=out, **kw)
    c["dr"], c["dx"], c["dgain"] = api.lattice_add_rmsnorm_bwd(c["h"], c["dy"], c["dh"], **kw)
    return c


def check_case(c, dt, p, eps=1e-5):
    rows, cols = c["x"].shape
    u = o.HALF_STEP[dt]
    f = o.factor(np.arange(rows), cols, p, SEED, STEP, SITE)
    x, res = f64(c["x"]) * f, f64(c["res"]) if c["res"] is not None else 0.0
    # the factor, the product, the sum, the rounding
    within(c["h"], x + res, (2 * o.U32 * np.abs(x) + o.U32 * np.abs(x + res)) * 1.001 + u * np.abs(x + res) * 1.001
           if c["h"] is not c["x"] else 0 * x, "h")
    h, g = f64(c["h"]), f64(c["gain"]) if c["gain"] is not None else np.ones(cols)      # the norm is that of h as it is kept
    y, _ = o.rmsnorm(h, g, eps)
    if c["y"] is not None:
        within(c["y"], y, o.y_bound(y, dt), "y")
    if c["codes"] is not None:
        s = o.scale_of(y)
        got = f64(c["scales"])
        assert (np.abs(got - s) <= s * (o.RHO + 4 * o.U32)).all()
        codes = c["codes"].cpu().numpy()
        assert codes.shape == (rows, -(-cols // 16) * 16) and (codes[:, cols:] == 0).all()
        v = fp8.e4m3_value(codes[:, :cols]) * got[:, None]
        assert (np.abs(v - y) <= o.code_bound(y, s)).all()
        if dt == "f32" and c["y"] is not None:                # y is what was encoded
            q, sc = fp8.quantize(c["y"].cpu().numpy())
            assert np.array_equal(q, codes[:, :cols]) and np.array_equal(sc, c["scales"].cpu().numpy())
    dy, dh = f64(c["dy"]), f64(c["dh"]) if c["dh"] is not None else None
    dr, dg = o.rmsnorm_bwd(h, g, eps, dy, dh)
    b = o.dr_bound(h, g, eps, dy, dh, dt)
    within(c["dr"], dr, b, "d_residual")
    if p:
        # dx is made from the sum before its rounding
        within(c["dx"], dr * f, (b + 2 * (o.U32 + u * (dt == "bf16")) * np.abs(dr)) * f, "dx")
    else:
        assert c["dx"] is c["dr"]
    if c["gain"] is not None:
        within(c["dgain"], dg, o.dgain_bound(h, eps, dy), "dgain")
    else:
        assert c["dgain"] is None


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("residual,p,out", [(True, 0.0, "both"), (False, 0.0, "y"), (True, 0.2, "fp8"), (False, 0.6, "both")])
def test_norm(dt, rows, cols, residual, p, out):
    check_case(run_case(dt, rows, cols, residual, p, out), dt, p)


@pytest.mark.parametrize("dt,rows,cols", [("bf16", 70001, 24), ("f32", 50003, 9), ("bf16", 20003, 520), ("f32", 9001, 300),
                                          ("bf16", 3001, 4100), ("bf16", 1500, 16000)])
def test_norm_with_more_rows_than_a_launch_has_waves(dt, rows, cols):
    """Every wave takes several rows."""
    check_case(run_case(dt, rows, cols, True, 0.1, "both", seed=1), dt, 0.1)


def test_norm_without_gain():
    check_case(run_case("bf16", 19, 200, True, 0.0, "both", gain=False), "bf16", 0.0)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("cols", [51, 64, 1003])
def test_norm_of_strided_rows(dt, cols):
    r = np.random.default_rng(7)
    check_case(run_case(dt, 37, cols, True, 0.1, "both", make=lambda n, c: randn(r, dt, n, c + 13)[:, 5:5 + c]), dt, 0.1)


def test_norm_writes_in_place_and_only_its_rows():
    from paper_2512_09200_amd import api
    r = np.random.default_rng(8)
    for cols in (40, 43, 2500):
        x, res = randn(r, "bf16", 30, cols), randn(r, "bf16", 30, cols)
        gain = torch.rand(cols, device=DEV)
        h, y, _, _ = api.lattice_add_rmsnorm_fwd(x, res, gain)
        dy, dh = randn(r, "bf16", 30, cols), randn(r, "bf16", 30, cols)
        dr, _, dg = api.lattice_add_rmsnorm_bwd(h, dy, dh, gain)
        buf = torch.full((30, cols + 9), 3.0, dtype=torch.bfloat16, device=DEV)
        a, b = buf[:, 1:1 + cols], res.clone()
        a.copy_(x)
        h2, y2, _, _ = api.lattice_add_rmsnorm_fwd(a, b, gain, h=b, y=a)
        assert torch.equal(h2, h) and torch.equal(y2, y) and h2 is b and y2 is a
        assert (buf[:, :1] == 3).all() and (buf[:, 1 + cols:] == 3).all()
        d = dh.clone()
        dr2, _, dg2 = api.lattice_add_rmsnorm_bwd(h, dy, d, gain, d_residual=d)
        assert torch.equal(d, dr) and dr2 is d and torch.equal(dg, dg2)


def test_norm_of_no_rows():
    from paper_2512_09200_amd import api
    x, gain = torch.empty(0, 24, device=DEV), torch.ones(24, device=DEV)
    h, y, q, s = api.lattice_add_rmsnorm_fwd(x, x, gain, out="both")
    assert h.shape == y.shape == (0, 24) and q.shape == (0, 32) and s.shape == (0,)
    dr, dx, dg = api.lattice_add_rmsnorm_bwd(x, x, None, gain)
    assert dr.shape == (0, 24) and (dg == 0).all()


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("cols", [40, 700, 5003])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_rows_that_are_not_finite_say_so_and_stay_alone(dt, cols, bad):
    from paper_2512_09200_amd import api
    r = np.random.default_rng(2)
    x = randn(r, dt, 6, cols)
    clean = x.clone()
    x[2, cols - 1] = bad
    h, y, q, s = api.lattice_add_rmsnorm_fwd(x, None, out="both")
    _, y0, q0, s0 = api.lattice_add_rmsnorm_fwd(clean, None, out="both")
    others = [0, 1, 3, 4, 5]
    assert torch.equal(y[others], y0[others]) and torch.equal(q[others], q0[others]) and torch.equal(s[others], s0[others])
    assert torch.isnan(s[2]) and (q[2, :cols] == 0x7f).all() and (q[2, cols:] == 0).all()
    want, _ = o.rmsnorm(f64(x)[2:3], np.ones(cols), 1e-6) if np.isnan(bad) else (None, None)
    if want is not None:
        assert np.isnan(f64(y)[2]).all()
    else:
        assert np.isnan(f64(y)[2, -1])
    # the linear layer that takes the codes shows it too
    w, sw = api.lattice_fp8_quantize(torch.randn(16, cols, device=DEV))
    z = api.lattice_linear_fp8_fwd(q, s, w, sw, cols, out_dtype=torch.float32)
    assert torch.isnan(z[2]).all() and torch.isfinite(z[others]).all()


def test_rows_of_zeros():
    from paper_2512_09200_amd import api
    x = torch.zeros(5, 96, device=DEV)
    h, y, q, s = api.lattice_add_rmsnorm_fwd(x, None, eps=1e-6, out="both")
    assert (y == 0).all() and (q == 0).all() and (s == 1).all()
    _, y, q, s = api.lattice_add_rmsnorm_fwd(x, None, eps=0.0, out="both")      # 0 / 0
    assert torch.isnan(y).all() and torch.isnan(s).all()


def test_rows_of_the_smallest_and_the_largest_numbers():
    from paper_2512_09200_amd import api
    from oracle import fp8
    r = np.random.default_rng(11)
    x = randn(r, "f32", 6, 100)
    x *= torch.tensor([2.0 ** -149, 2.0 ** -140, 2.0 ** -130, 2.0 ** -122, 2.0 ** -117, 2.0 ** -110], device=DEV)[:, None]
    _, y, q, s = api.lattice_add_rmsnorm_fwd(x, None, eps=1.0, out="both")      # the square root is 1
    assert torch.equal(y, x) and (s >= 2.0 ** -126).all()
    got = fp8.e4m3_value(q.cpu().numpy()[:, :100]).astype(np.float64) * f64(s)[:, None]
    # half a step of a code, normal or not; the reciprocal, its product and the scale are off by 2^-24 each
    want, S = f64(x), f64(s)[:, None]
    step = np.maximum(2.0 ** -4 * np.abs(want), 2.0 ** -10 * S)
    assert (np.abs(got - want) <= step * (1 + 2.0 ** -20) + 2.0 ** -22 * np.abs(want)).all()
    big = torch.full((3, 70), 2.0 ** 70, device=DEV)                            # squares past fp32
    h, y, q, s = api.lattice_add_rmsnorm_fwd(big, None, out="both")
    assert torch.equal(h, big) and (y == 0).all() and torch.isnan(s).all() and (q[:, :70] == 0x7f).all()


@pytest.mark.parametrize("dt,cols", [("f32", 100), ("bf16", 24), ("bf16", 1500)])
def test_gradients_of_rows_whose_scale_has_an_infinite_square(dt, cols):
    """eps 0 and values around 2^-65: 1 / rms is 2^65, its square past fp32."""
    from paper_2512_09200_amd import api
    r = np.random.default_rng(13)
    h = torch.ldexp(randn(r, "f32", 9, cols).clamp(0.25, 4.0), torch.tensor(-65, device=DEV)).to(TT[dt])
    dy = randn(r, dt, 9, cols)
    gain = torch.from_numpy(1 + 0.3 * r.standard_normal(cols)).float().to(DEV)
    d, _, dg = api.lattice_add_rmsnorm_bwd(h, dy, None, gain, eps=0.0)
    H, Y, G = f64(h), f64(dy), f64(gain)
    want, wg = o.rmsnorm_bwd(H, G, 0.0, Y)
    # Besides the ordinary roundings: a square is at least 2^-134 and off by 2^-150, as is the
    # mean, which is above it, so 1 / rms is off by 2^-16 of itself
    n = H / np.sqrt((H ** 2).mean(-1, keepdims=True))
    rho, e = n / H, 2.0 ** -16
    terms = np.abs(rho * Y * G) + 3 * np.abs(n * rho) * np.abs(Y * G * n).mean(-1, keepdims=True)
    within(d, want, o.dr_bound(H, G, 0.0, Y, None, dt) + e * (1 + 2 * o.HALF_STEP[dt]) * terms, "d_residual")
    within(dg, wg, o.dgain_bound(H, 0.0, Y) + e * np.abs(Y * n).sum(0) * 1.001, "dgain")


def test_norm_beyond_4_gib():
    from paper_2512_09200_amd import api
    r = np.random.default_rng(5)
    stride, cols = 2_200_000_000, 300
    big = torch.empty(2 * stride + cols, dtype=torch.bfloat16, device=DEV)
    wide = big.as_strided((3, cols), (stride, 1))
    x = randn(r, "bf16", 3, cols)
    wide.copy_(x)
    h, y, _, _ = api.lattice_add_rmsnorm_fwd(x, x)
    h2, y2, _, _ = api.lattice_add_rmsnorm_fwd(wide, wide, h=wide)
    assert torch.equal(h, h2) and torch.equal(y, y2)
    dr, _, _ = api.lattice_add_rmsnorm_bwd(h, x, x)
    dr2, _, _ = api.lattice_add_rmsnorm_bwd(h2, x, x, d_residual=wide)
    assert torch.equal(dr, dr2)
    assert torch.equal(api.lattice_dropout(wide, 0.5, rng_state(), out=wide), api.lattice_dropout(dr, 0.5, rng_state()))


@pytest.mark.parametrize("dt,cols", [("bf16", c) for c in (16, 64, 200, 256, 512, 1001, 1024, 2048, 4096, 8192, 16384)]
                         + [("f32", 1024), ("f32", 1001)])
def test_backward_of_data_beyond_the_caches(dt, cols):
    """More than 256 MB in five tensors.  Every row's gradient is that of a call of fewer
    rows, bit for bit; some rows' and the gain's are the definition's."""
    from paper_2512_09200_amd import api
    rows = (1 << 28) // (5 * cols * (2 if dt == "bf16" else 4)) + 1 + 30
    rows += -rows % 2 + 1
    h, dy, dh = (torch.randn(rows, cols, device=DEV).to(TT[dt]) for _ in range(3))
    gain, drop = 1 + 0.3 * torch.randn(cols, device=DEV), (0.2, rng_state(), SITE)
    dr, dx, dg = api.lattice_add_rmsnorm_bwd(h, dy, dh, gain, dropout=drop)
    for a in range(0, rows, -(-rows // 4)):
        b = slice(a, a + -(-rows // 4))
        assert torch.equal(dr[b], api.lattice_add_rmsnorm_bwd(h[b], dy[b], dh[b], gain)[0]), a
    pick = [0, 1, rows // 3, rows - 2, rows - 1]
    H, Y, R, G, u = f64(h[pick]), f64(dy[pick]), f64(dh[pick]), f64(gain), o.HALF_STEP[dt]
    want, _ = o.rmsnorm_bwd(H, G, 1e-6, Y, R)
    f, b = o.factor(np.array(pick), cols, 0.2, SEED, STEP, SITE), o.dr_bound(H, G, 1e-6, Y, R, dt)
    within(dr[pick], want, b, "d_residual")
    within(dx[pick], want * f, (b + 2 * (o.U32 + u * (dt == "bf16")) * np.abs(want)) * f, "dx")
    n = h.double() / (h.double().square().mean(-1, keepdim=True) + 1e-6).sqrt()
    terms = dy.double() * n
    within(dg, f64(terms.sum(0)), (o.RHO + (3 + rows) * o.U32) * f64(terms.abs().sum(0)), "dgain")
    d = dh.clone()                                           # in an input's place
    dr2, dx2, dg2 = api.lattice_add_rmsnorm_bwd(h, dy, d, gain, dropout=drop, d_residual=d)
    assert dr2 is d and torch.equal(dr2, dr) and torch.equal(dx2, dx) and torch.equal(dg2, dg)


def test_backward_of_strided_rows_beyond_the_caches():
    """Rows that are not whole lines of memory: other kernels, the same bits."""
    from paper_2512_09200_amd import api
    rows, cols = 60000, 512
    h, dy, dh = (torch.randn(rows, cols, device=DEV).bfloat16() for _ in range(3))
    gain = torch.rand(cols, device=DEV)
    want = api.lattice_add_rmsnorm_bwd(h, dy, dh, gain)
    for ld, at in ((520, 0), (576, 0), (576, 3)):
        x, y, z, out = (torch.zeros(rows, ld, dtype=torch.bfloat16, device=DEV)[:, at:at + cols] for _ in range(4))
        for a, b in ((x, h), (y, dy), (z, dh)):
            a.copy_(b)
        got = api.lattice_add_rmsnorm_bwd(x, y, z, gain, d_residual=out)
        assert torch.equal(got[0], want[0]) and torch.equal(got[2], want[2]), (ld, at)
        base = out._base
        assert not base[:, :at].any() and not base[:, at + cols:].any()


@pytest.mark.parametrize("dt,cols", [("bf16", 1024), ("bf16", 1001), ("bf16", 24), ("f32", 1024), ("f32", 1001)])
def test_dropout_of_data_beyond_the_caches(dt, cols):
    from paper_2512_09200_amd import api
    rows = (1 << 28) // (2 * cols * (2 if dt == "bf16" else 4)) + 33
    x = torch.randn(rows, cols, device=DEV).to(TT[dt])
    out = api.lattice_dropout(x, 0.3, rng_state(), site=SITE)
    pick = [0, 1, rows // 3, rows - 2, rows - 1]
    f, X = o.factor(np.array(pick), cols, 0.3, SEED, STEP, SITE), f64(x[pick])
    within(out[pick], X * f, np.abs(X * f) * (2 * o.U32 + o.HALF_STEP[dt]) * 1.001, "out")
    # the first rows are those of a smaller call, and in its input's place nothing changes
    assert torch.equal(out[:rows // 3], api.lattice_dropout(x[:rows // 3], 0.3, rng_state(), site=SITE))
    api.lattice_dropout(x, 0.3, rng_state(), site=SITE, out=x)
    assert torch.equal(out, x)


# ---------------------------------------------------------------------------
def test_a_captured_step_draws_anew_and_repeats_the_eager_bits():
    """Two graphs that share a pool, replayed in turn with eager work between."""
    from paper_2512_09200_amd import api
    r = np.random.default_rng(3)
    x, res, dy, dh = (randn(r, "bf16", 300, 1000) for _ in range(4))
    gain, state = torch.rand(1000, device=DEV), rng_state(step=0)

    def step():
        h, y, q, s = api.lattice_add_rmsnorm_fwd(x, res, gain, dropout=(0.3, state, 2), out="both")
        dr, dx, dg = api.lattice_add_rmsnorm_bwd(h, dy, dh, gain, dropout=(0.3, state, 2))
        z = api.lattice_dropout(y, 0.5, state, site=9)
        state[1:] += 1
        return h, y, q, s, dr, dx, dg, z

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graphs, outs = [], []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, pool=graphs[0].pool() if graphs else None):
            outs.append(step())
        graphs.append(g)
    seen = []
    for n in range(6):
        state[1] = n
        want = [t.clone() for t in step()]
        state[1] = n
        graphs[n % 2].replay()
        assert int(state[1]) == n + 1
        for a, b in zip(outs[n % 2], want):
            assert torch.equal(a, b), n
        seen.append(want[0])
        _ = torch.randn(1000, 1000, device=DEV).sum().item()
    assert not torch.equal(seen[0], seen[1])


def test_a_stream_of_its_own():
    from paper_2512_09200_amd import api
    r = np.random.default_rng(4)
    x, res, dy = (randn(r, "f32", 500, 777) for _ in range(3))
    gain, side = torch.rand(777, device=DEV), torch.cuda.Stream()
    drop = (0.25, rng_state(), 1)
    want = api.lattice_add_rmsnorm_fwd(x, res, gain, dropout=drop, out="both")
    wantb = api.lattice_add_rmsnorm_bwd(want[0], dy, res, gain, dropout=drop)
    wantd = api.lattice_dropout(x, 0.5, drop[1])
    side.wait_stream(torch.cuda.current_stream())
    got = api.lattice_add_rmsnorm_fwd(x, res, gain, dropout=drop, out="both", stream=side)
    gotb = api.lattice_add_rmsnorm_bwd(got[0], dy, res, gain, dropout=drop, stream=side)
    gotd = api.lattice_dropout(x, 0.5, drop[1], stream=side)
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(want + wantb + (wantd,), got + gotb + (gotd,)):
        assert torch.equal(a, b)


def test_refusals_of_the_binding():
    from paper_2512_09200_amd import LatticeError
    from paper_2512_09200_amd import api
    x = torch.randn(8, 32, device=DEV)
    rs = rng_state()
    for call in (lambda: api.lattice_dropout(x[0], 0.5, rs), lambda: api.lattice_dropout(x.half(), 0.5, rs),
                 lambda: api.lattice_dropout(x.t(), 0.5, rs), lambda: api.lattice_dropout(x, 0.5, rs.float()),
                 lambda: api.lattice_dropout(x, 0.5, rs[:1]), lambda: api.lattice_dropout(x, 0.5, rs.cpu()),
                 lambda: api.lattice_dropout(x.cpu(), 0.5, rs), lambda: api.lattice_dropout(x, 1.0, rs),
                 lambda: api.lattice_dropout(x, -0.1, rs), lambda: api.lattice_dropout(x, 0.5, None),
                 lambda: api.lattice_dropout(x, 0.5, rs, out=x[:4]),
                 lambda: api.lattice_add_rmsnorm_fwd(x, x[:, :16]), lambda: api.lattice_add_rmsnorm_fwd(x, x.bfloat16()),
                 lambda: api.lattice_add_rmsnorm_fwd(x, out="int8"), lambda: api.lattice_add_rmsnorm_fwd(x, eps=-1.0),
                 lambda: api.lattice_add_rmsnorm_fwd(x, gain=torch.ones(16, device=DEV)),
                 lambda: api.lattice_add_rmsnorm_fwd(torch.zeros(2, 16385, device=DEV)),
                 lambda: api.lattice_add_rmsnorm_fwd(x, h=torch.empty_like(x), y=None, residual=x.cpu()),
                 lambda: api.lattice_add_rmsnorm_bwd(x, x[:4]), lambda: api.lattice_add_rmsnorm_bwd(x, x, x.bfloat16())):
        with pytest.raises((ValueError, TypeError, LatticeError)):
            call()
