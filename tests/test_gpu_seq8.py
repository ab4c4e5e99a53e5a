"""8-bit ring caches on the GPU: fill and single-event step against the float64
oracle (oracle/seqcache8.py).  Codes and scales of rows that are taken as they are
have to be the oracle's; outputs lie within the bound of their roundings."""
import numpy as np
import pytest
import torch

from oracle import fp8
from oracle import seqattn as o
from oracle import seqcache8 as c8

DEV = "cuda"
TT = {"bf16": torch.bfloat16, "f32": torch.float32}
pytestmark = pytest.mark.gpu


def randn(rng, *shape):
    return torch.from_numpy(rng.standard_normal(shape).astype(np.float32))


def f64(t):
    return t.detach().float().cpu().double().numpy()


def i32(a):
    return torch.from_numpy(np.asarray(a).astype(np.int32)).to(DEV)


def within(got, want, bound, what):
    g = f64(got)
    assert np.isfinite(g).all(), f"{what}: not finite"
    over = np.abs(g - want) - bound
    i = np.unravel_index(np.argmax(over), over.shape)
    assert over[i] <= 1e-30, f"{what} at {i}: {g[i]} against {want[i]}, bound {bound[i]}"


def ld(D):
    return -(-D // 16) * 16


def new_caches(C, J, cap, D, rng=None, garbage=True):
    """Caches on the GPU and their copy for the oracle.  Everything is garbage (NaN
    codes and scales among it) that the operators must not use."""
    nb = -(-cap // 16)
    k, v = (np.full((C, J, cap, ld(D)), 0x7F if garbage else 0, np.uint8) for _ in "kv")
    ks, vs = (np.full((C, J, nb), np.nan if garbage else 1, np.float32) for _ in "kv")
    host = dict(k=k, v=v, ks=ks, vs=vs)
    return host


def to_gpu(host):
    return tuple(torch.from_numpy(host[x].copy()).to(DEV) for x in ("k", "v", "ks", "vs"))


def same(gpu, host, what=""):
    for t, x in zip(gpu, ("k", "v", "ks", "vs")):
        g = t.cpu().numpy()
        bad = ~((g == host[x]) | ((g != g) & (host[x] != host[x])))
        assert not bad.any(), f"{what} {x} at {np.argwhere(bad)[0]}: {g[bad][0]} against {host[x][bad][0]}"


def plan(off, rows):
    from paper_2512_09200_amd import api
    return api.lattice_seq_plan(i32(off), rows)


def rows_of(rng, dt, n, J, D, scale):
    """Events whose sizes differ by powers of ten."""
    x = randn(rng, n, J, D) * torch.from_numpy(10.0 ** rng.integers(-scale, scale + 1, (n, J, 1))).float()
    return x.to(TT[dt]).to(DEV)


FILL = [("bf16", 2, 64, 30, 3), ("f32", 1, 8, 1, 0), ("bf16", 3, 40, 7, 64), ("f32", 2, 128, 100, 20), ("bf16", 1, 128, 16, 0),
        ("f32", 4, 32, 45, 5), ("bf16", 2, 24, 300, 1), ("f32", 1, 96, 13, 37), ("bf16", 2, 16, 64, 16)]


@pytest.mark.parametrize("dt,J,D,W,N", FILL)
@pytest.mark.parametrize("spread", [0, 4])
def test_fill(dt, J, D, W, N, spread):
    from paper_2512_09200_amd import api
    rng = np.random.default_rng(W + D)
    lens = np.array([1, 0, W + N, W + N + 1, 3 * (W + N) + 5, 2, max(W - 1, 1), 17, 5])
    S, cap, C = len(lens), W + N, len(lens) + 2
    off = np.concatenate([[0], np.cumsum(lens)])
    rows = int(off[-1]) + 3                                   # three rows behind the last sequence
    host = new_caches(C, J, cap, D)
    kc = to_gpu(host)
    index = rng.permutation(C)[:S]
    index[7], index[8] = -1, C                                # skipped
    qkv = torch.cat([rows_of(rng, dt, rows, J, D, spread) for _ in range(2)], 1)
    k, v = qkv[:, :J], qkv[:, J:]
    api.lattice_seq_cache8_fill(plan(off, rows), k, v, *kc, W, N, cache_index=i32(index))
    c8.fill(host, f64(k), f64(v), off, W, N, index, np.zeros(S, int))
    same(kc, host, "fill")
    # the histories go on: what is there already is scaled with the new rows
    more = np.array([1, 4, 0, 3, 2 * cap, cap, 7, 3, 2])
    off2 = np.concatenate([[0], np.cumsum(more)])
    k, v = (rows_of(rng, dt, int(off2[-1]), J, D, spread) for _ in "kv")
    first = lens.copy()
    first[6] = -1                                             # skipped
    api.lattice_seq_cache8_fill(plan(off2, int(off2[-1])), k, v, *kc, W, N, cache_index=i32(index), first=i32(first))
    idx = index.copy()
    idx[6] = -1
    c8.fill(host, f64(k), f64(v), off2, W, N, idx, first)
    same(kc, host, "second fill")


@pytest.mark.parametrize("dt,J,D,W,N", [("bf16", 2, 64, 500, 3), ("f32", 1, 40, 2000, 0), ("bf16", 3, 128, 90, 17)])
@pytest.mark.parametrize("max_len", [0, 900, 5])
def test_long_histories_among_many_short_ones(dt, J, D, W, N, max_len):
    """Long ones are spread over waves of their own (max_len 5: a wrong bound costs
    time, not results); empty ones, and rows behind the last, in between."""
    from paper_2512_09200_amd import api
    rng = np.random.default_rng(W)
    lens = np.array([3, 0, 1, 5] * 60)
    lens[[0, 101, 239]] = 900, 333, 128
    S, cap = len(lens), W + N
    off = np.concatenate([[0], np.cumsum(lens)])
    rows = int(off[-1]) + 70
    host = new_caches(S, J, cap, D)
    kc = to_gpu(host)
    k, v = (rows_of(rng, dt, rows, J, D, 1) for _ in "kv")
    index = rng.permutation(S)
    s = api.lattice_seq_plan(i32(off), rows, max_len=max_len)
    api.lattice_seq_cache8_fill(s, k, v, *kc, W, N, cache_index=i32(index))
    c8.fill(host, f64(k), f64(v), off, W, N, index, np.zeros(S, int))
    same(kc, host, "fill")
    api.lattice_seq_cache8_fill(s, v, k, *kc, W, N, cache_index=i32(index), first=i32(lens))
    c8.fill(host, f64(v), f64(k), off, W, N, index, lens)
    same(kc, host, "second fill")


@pytest.mark.parametrize("dt,J,D,W,N", [("bf16", 2, 64, 700, 3), ("bf16", 1, 128, 1200, 0), ("f32", 3, 24, 660, 20)])
def test_long_histories_among_middling_ones(dt, J, D, W, N):
    """The longest are 8 and more times as many blocks as a history of the mean length,
    which one just misses; another order of the sequences in the call that goes on."""
    from paper_2512_09200_amd import api
    rng = np.random.default_rng(W)
    lens = np.tile([40, 0, 61, 17, 70], 24)
    lens[[3, 50, 77, 100]] = 1300, 640, 639, 657
    S, cap = len(lens), W + N
    off = np.concatenate([[0], np.cumsum(lens)])
    rows = int(off[-1])
    assert -(-rows // S) // 16 + 1 == 5 and cap >= 8 * 5 * 16
    host = new_caches(S, J, cap, D)
    kc = to_gpu(host)
    k, v = (rows_of(rng, dt, rows, J, D, 1) for _ in "kv")
    index = rng.permutation(S)
    api.lattice_seq_cache8_fill(plan(off, rows), k, v, *kc, W, N, cache_index=i32(index))
    c8.fill(host, f64(k), f64(v), off, W, N, index, np.zeros(S, int))
    same(kc, host, "fill")
    order = np.concatenate([np.arange(78, S), np.arange(78)])
    off = np.concatenate([[0], np.cumsum(lens[order])])
    api.lattice_seq_cache8_fill(plan(off, rows), v, k, *kc, W, N, cache_index=i32(index[order]),
                                first=i32(lens[order]))
    c8.fill(host, f64(v), f64(k), off, W, N, index[order], lens[order])
    same(kc, host, "second fill")


def test_fill_of_positions_next_to_the_end_of_int32():
    from paper_2512_09200_amd import api
    rng = np.random.default_rng(0)
    J, D, W, N = 1, 16, 1000, 5
    first = np.array([2 ** 31 - 300, 2 ** 31 - 1])
    off = np.array([0, 299, 300])
    host = new_caches(2, J, W + N, D, garbage=False)
    host["k"][:] = 0x38
    kc = to_gpu(host)
    k, v = (randn(rng, 300, J, D).to(DEV) for _ in "kv")
    api.lattice_seq_cache8_fill(plan(off, 300), k, v, *kc, W, N, first=i32(first))
    c8.fill(host, f64(k), f64(v), off, W, N, [0, 1], first)
    same(kc, host)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_values_that_are_not_finite_become_nan_and_set_no_scale(bad):
    from paper_2512_09200_amd import api
    rng = np.random.default_rng(1)
    J, D, W = 1, 32, 40
    k, v = randn(rng, 20, J, D), randn(rng, 20, J, D)
    k[3, 0, 5], v[17, 0, 31] = bad, bad
    host = new_caches(1, J, W, D)
    kc = to_gpu(host)
    api.lattice_seq_cache8_fill(plan([0, 20], 20), k.to(DEV), v.to(DEV), *kc, W)
    c8.fill(host, k.double().numpy(), v.double().numpy(), [0, 20], W, 0, [0], [0])
    same(kc, host)
    assert (host["k"][0, 0, 3, 5] & 0x7F) == 0x7F
    # a step: what sees the key is NaN; of the value only its dimension
    q, kn, vn = (randn(rng, 1, 1, D).to(DEV) for _ in "qkv")
    out = api.lattice_seq_step8(q, kn, vn, i32([20]), *kc, W, rope=False)
    assert torch.isnan(out).all()
    kc[0][0, 0, 3, 5] = 0
    out = api.lattice_seq_step8(q, kn, vn, i32([20]), *kc, W, rope=False)
    assert torch.isnan(out[0, 0, 31]) and torch.isfinite(out[0, 0, :31]).all()


def test_values_next_to_the_ends_of_fp32():
    from paper_2512_09200_amd import api
    big = np.finfo(np.float32).max
    x = torch.zeros(48, 1, 8)
    x[0, 0] = torch.tensor([big, -big, 1.0, 2.0 ** 120, 2.0 ** 111, 0, 3e38, 1e38])
    x[16, 0] = torch.tensor([2.0 ** -149, 2.0 ** -126, 1e-40, 0, -2.0 ** -130, 2.0 ** -117, 2.0 ** -120, 0])
    host = new_caches(1, 1, 48, 8)
    kc = to_gpu(host)
    api.lattice_seq_cache8_fill(plan([0, 48], 48), x.to(DEV), x.to(DEV), *kc, 48)
    c8.fill(host, x.double().numpy(), x.double().numpy(), [0, 48], 48, 0, [0], [0])
    same(kc, host)
    assert np.isfinite(c8.value(host["k"][0], host["ks"][0], 8).astype(np.float32)).all()


# ---------------------------------------------------------------------------
def used_caches(rng, dt, C, J, cap, D, lens, index):
    """Caches as earlier events left them: reached slots hold codes under their
    block's scale, the others garbage."""
    host = new_caches(C, J, cap, D)
    for b, at in enumerate(index):
        n = min(max(int(lens[b]), 0), cap)
        if at >= C or n == 0:
            continue
        x = rng.standard_normal((2, n, J, D)) * 10.0 ** rng.integers(-2, 3, (2, n, J, 1))
        x = torch.from_numpy(x).to(TT[dt]).double().numpy()
        c8.put(host, at, {i: (x[0, i], x[1, i]) for i in range(n)}, n)
    return host


STEP = [("bf16", 4, 2, 64, 30, 3), ("f32", 2, 1, 32, 5, 0), ("bf16", 8, 1, 128, 700, 4), ("f32", 3, 3, 96, 129, 1),
        ("bf16", 20, 1, 40, 64, 64), ("f32", 17, 1, 128, 333, 7), ("bf16", 2, 2, 8, 1, 0), ("bf16", 40, 2, 128, 1500, 2),
        ("f32", 4, 4, 24, 50, 14), ("bf16", 6, 2, 32, 250, 6)]


@pytest.mark.parametrize("dt,H,J,D,W,N", STEP)
@pytest.mark.parametrize("rope", [True, False])
def test_step_against_the_definition(dt, H, J, D, W, N, rope):
    from paper_2512_09200_amd import api
    rng = np.random.default_rng(H + D + W)
    cap = W + N
    lens = np.array([0, 1, N, cap - 1, cap, 3 * cap + 1, -1, min(cap, 200) // 2, 5, cap + 15, 2 * cap + 7])
    B = len(lens)
    C = B + 2
    index = rng.permutation(C)[:B]
    index[8] = C                                              # out of range
    host = used_caches(rng, dt, C, J, cap, D, lens, index)
    kc = to_gpu(host)
    qkv = torch.cat([randn(rng, B, h, D) for h in (H, J, J)], 1).to(TT[dt]).to(DEV)
    q, k, v = qkv[:, :H], qkv[:, H:H + J], qkv[:, H + J:]
    pos = rng.integers(0, 2 ** 30, B)
    gq, gk = 1 + 0.1 * randn(rng, D), 1 + 0.1 * randn(rng, D)
    R = D // 16 * 8
    out = torch.full((B, H, D), 5.0, dtype=TT[dt], device=DEV)
    kw = dict(gain_q=gq.to(DEV), gain_k=gk.to(DEV), rotary=R, positions=i32(pos)) if rope else dict(rope=False)
    api.lattice_seq_step8(q, k, v, i32(lens), *kc, W, N, cache_index=i32(index), out=out, **kw)
    Q, K, V = f64(q), f64(k), f64(v)
    if rope:
        Q, _ = o.qk_rope(Q, f64(gq), pos, R, 1e4, 1e-6, False)
        K, _ = o.qk_rope(K, f64(gk), pos, R, 1e4, 1e-6, False)
        K = torch.from_numpy(K.astype(np.float32)).to(TT[dt]).double().numpy()
    got = {x: t.cpu().numpy() for x, t in zip(("k", "v", "ks", "vs"), kc)}
    u = o.HALF_STEP[dt]
    for b in range(B):
        at = index[b]
        if lens[b] < 0 or at >= C:
            assert (out[b] == 5).all()
            continue
        slot, n = o.slot_of(int(lens[b]), W, N), min(lens[b] + 1, cap)
        blk, lo = slot // 16, slot // 16 * 16
        before = {x: host[x][at].copy() for x in host}
        c8.put(host, at, {slot: (K[b], V[b])}, int(n))
        if rope:
            # the rotated key may lie next to a border: its code may be the neighbour's,
            # and where it sets the scale, the scale's and its block's with it
            for j in range(J):
                kv = c8.value(got["k"][at], got["ks"][at], D)[j, slot]
                e = np.maximum(2.0 ** -4 * np.abs(K[b, j]), 2.0 ** -10 * got["ks"][at, j, blk])
                assert (np.abs(kv - K[b, j]) <= e + (u + (D + 40) * o.U32 * 1.5) * np.abs(K[b, j]).max()).all()
                if got["ks"][at, j, blk] == host["ks"][at, j, blk]:
                    host["k"][at, j, slot] = got["k"][at, j, slot]
                else:
                    assert abs(np.log2(got["ks"][at, j, blk] / host["ks"][at, j, blk])) == 1
                    host["ks"][at, j, blk], host["k"][at, j, lo:lo + 16] = got["ks"][at, j, blk], got["k"][at, j, lo:lo + 16]
        del before
    same(kc, host, "caches")
    for b in range(B):
        at = index[b]
        if lens[b] < 0 or at >= C:
            continue
        n = int(min(lens[b] + 1, cap))
        KC, VC = c8.value(host["k"][at], host["ks"][at], D), c8.value(host["v"][at], host["vs"][at], D)
        for h in range(H):
            j = h // (H // J)
            want, mass, size = c8.attend(KC[j], VC[j], Q[b, h], n, D ** -0.5)
            # query and probabilities in two bf16 parts (three for fp32): 2^-16 (2^-24)
            # of each; rotation, products and sums in fp32
            r = 2.0 ** -16 if dt == "bf16" else 2.0 ** -23
            es = r * size + (2 * D + 48) * o.U32 * size * 1.5 + (n + 16) * o.U32
            within(out[b, h], want, (r + 2 * np.expm1(es)) * mass + u * np.abs(want) * (1 + r), f"out {b} {h}")


@pytest.mark.parametrize("dt,H,J,D,W,N,S", [("bf16", 4, 2, 64, 30, 3, 300), ("f32", 2, 2, 32, 60, 5, 700),
                                            ("bf16", 20, 1, 128, 17, 0, 300), ("f32", 3, 1, 40, 1, 1, 40),
                                            ("bf16", 6, 2, 104, 20, 64, 700), ("f32", 34, 2, 64, 9, 16, 200),
                                            ("f32", 8, 2, 128, 28, 4, 300), ("f32", 5, 1, 120, 40, 0, 700)])
@pytest.mark.parametrize("rope", [True, False])
def test_short_windows_of_many_users(dt, H, J, D, W, N, S, rope):
    """A wave each: the definition's outputs, and where a window is one tile those that
    each user gets in a batch of few, bit for bit; the same caches always."""
    from paper_2512_09200_amd import api
    rng = np.random.default_rng(S + D)
    cap = W + N
    assert cap <= S * J // 16
    lens = rng.integers(-1, 3 * cap, S)
    index = rng.permutation(S + 3)[:S]
    index[7] = S + 3
    host = used_caches(rng, dt, S + 3, J, cap, D, lens, index)
    kc, kf = to_gpu(host), to_gpu(host)
    q, k, v = (randn(rng, S, h, D).to(TT[dt]).to(DEV) for h in (H, J, J))
    kw = dict(gain_q=(1 + 0.1 * randn(rng, D)).to(DEV), gain_k=(1 + 0.1 * randn(rng, D)).to(DEV)) if rope else dict(rope=False)
    out = api.lattice_seq_step8(q, k, v, i32(lens), *kc, W, N, cache_index=i32(index), **kw)
    for a in range(0, S, 4):
        b = slice(a, min(a + 4, S))
        ref = api.lattice_seq_step8(q[b], k[b], v[b], i32(lens[b]), *kf, W, N, cache_index=i32(index[b]), **kw)
        live = [i for i in range(*b.indices(S)) if lens[i] >= 0 and index[i] < S + 3]
        if not live:
            continue
        got, want = out[live], ref[[i - a for i in live]]
        if cap <= 32:
            assert torch.equal(got, want)
    # Longer windows: two evaluations of one row, each as far from the definition as
    # test_step_against_the_definition allows.  (Events here differ by 10^4 in size, so scores
    # reach hundreds, and an exponent's fp32 argument is off by 2^-24 of that: no bound
    # relative to out alone holds.)
    Q = f64(q)
    if rope:
        Q, _ = o.qk_rope(Q, f64(kw["gain_q"]), np.maximum(lens, 0), D, 1e4, 1e-6, False)
    c = {x: t.cpu().numpy() for x, t in zip(("k", "v", "ks", "vs"), kc)}
    r, u = 2.0 ** -16 if dt == "bf16" else 2.0 ** -23, o.HALF_STEP[dt]
    for b in range(0, S, 9):
        at, n = index[b], int(min(lens[b] + 1, cap))
        if lens[b] < 0 or at >= S + 3:
            continue
        KC, VC = c8.value(c["k"][at], c["ks"][at], D), c8.value(c["v"][at], c["vs"][at], D)
        for h in range(H):
            j = h // (H // J)
            want, mass, size = c8.attend(KC[j], VC[j], Q[b, h], n, D ** -0.5)
            es = r * size + (2 * D + 48) * o.U32 * size * 1.5 + (n + 16) * o.U32
            within(out[b, h], want, (r + 2 * np.expm1(es)) * mass + u * np.abs(want) * (1 + r), f"out {b} {h}")
    for x, y in zip(kc, kf):
        assert ((x == y) | ((x != x) & (y != y))).all()


# (the last: more rounds of slots than a join has places for splits)
@pytest.mark.parametrize("dt,H,J,D,W,N,S", [("bf16", 16, 2, 128, 70000, 36, 2), ("f32", 2, 1, 64, 20000, 0, 1),
                                            ("bf16", 3, 1, 32, 150001, 7, 1)])
def test_step_of_long_windows_in_splits(dt, H, J, D, W, N, S):
    from paper_2512_09200_amd import api
    rng = np.random.default_rng(9)
    cap = W + N
    lens = np.array([3 * cap + 11, cap // 3])[:S]
    k, v = (torch.randint(0, 256, (S, J, cap, D), dtype=torch.uint8, device=DEV) for _ in "kv")
    for t in (k, v):
        t[(t & 0x7F) >= 0x78] = 0x30                          # no NaN, nothing above 240
    ks, vs = (torch.exp2(torch.randint(-9, -5, (S, J, -(-cap // 16)), device=DEV).float()) for _ in "kv")
    q, kn, vn = (randn(rng, S, h, D).to(TT[dt]).to(DEV) for h in (H, J, J))
    out = api.lattice_seq_step8(q, kn, vn, i32(lens), k, v, ks, vs, W, N, rope=False)
    u, r = o.HALF_STEP[dt], 2.0 ** -16 if dt == "bf16" else 2.0 ** -23
    for b in range(S):
        n = int(min(lens[b] + 1, cap))
        KC = c8.value(k[b].cpu().numpy(), ks[b].cpu().numpy(), D)
        VC = c8.value(v[b].cpu().numpy(), vs[b].cpu().numpy(), D)
        for h in range(H):
            j = h // (H // J)
            want, mass, size = c8.attend(KC[j], VC[j], f64(q)[b, h], n, D ** -0.5)
            es = r * size + (2 * D + 48) * o.U32 * size * 1.5 + (64 + 512) * o.U32
            within(out[b, h], want, (r + 2 * np.expm1(es) + 64 * o.U32) * mass + u * np.abs(want) * (1 + r), f"out {b} {h}")


@pytest.mark.parametrize("dt,H,J,D,W,N", [("bf16", 4, 2, 64, 16, 2), ("f32", 4, 1, 40, 40, 0), ("f32", 2, 2, 128, 9, 30)])
def test_events_one_by_one(dt, H, J, D, W, N):
    """A history from its first event on, wrapping several times: after every step
    codes and scales are the oracle's, so a block's many rewrites lose nothing
    but what the definition says."""
    from paper_2512_09200_amd import api
    rng = np.random.default_rng(2)
    cap, n = W + N, 4 * (W + N)
    host = new_caches(2, J, cap, D)
    kc = to_gpu(host)
    q = randn(rng, n, 2, H, D).to(TT[dt]).to(DEV)
    k, v = (rows_of(rng, dt, 2 * n, J, D, 2).view(n, 2, J, D) for _ in "kv")
    have = i32([0, 3])
    api.lattice_seq_cache8_fill(plan([0, 3], 3), k[:3, 1].contiguous(), v[:3, 1].contiguous(), *kc, W, N, cache_index=i32([1]))
    c8.fill(host, f64(k[:3, 1]), f64(v[:3, 1]), [0, 3], W, N, [1], [0])
    for t in range(n):
        api.lattice_seq_step8(q[t], k[t], v[t], have, *kc, W, N, rope=False)
        for b, p in ((0, t), (1, t + 3)):
            c8.put(host, b, {o.slot_of(p, W, N): (f64(k[t, b]), f64(v[t, b]))}, p + 1)
        have += 1
        if t % 7 == 0 or t > n - 3:
            same(kc, host, f"step {t}")


@pytest.mark.parametrize("dt,interleaved", [("bf16", False), ("bf16", True), ("f32", False), ("f32", True)])
def test_rotated_events_stepped_and_filled(dt, interleaved):
    """lattice_qk_rope_fwd and the fill against the step's own norm and rotation: a key's
    code is that of the definition's key rounded to the type, either way, but for keys that
    lie nearer to a border than the fp32 operator's roundings reach; values are the same."""
    from paper_2512_09200_amd import api
    rng = np.random.default_rng(21)
    B, H, J, D, W, N, n = 3, 4, 2, 64, 20, 3, 70
    q, k, v = (randn(rng, B * n, h, D).to(TT[dt]).to(DEV) for h in (H, J, J))
    gain = (1 + 0.1 * randn(rng, D)).to(DEV)
    kw = dict(gain_k=gain, rotary=48, interleaved=interleaved)
    s = plan(np.arange(B + 1) * n, B * n)
    filled, stepped = (to_gpu(new_caches(B, J, W + N, D)) for _ in "fs")
    _, kr = api.lattice_qk_rope_fwd(s, q, k, **kw)
    api.lattice_seq_cache8_fill(s, kr, v, *filled, W, N)
    rows = [x.view(B, n, -1, D) for x in (q, k, v)]
    for t in range(n):
        api.lattice_seq_step8(*(x[:, t] for x in rows), i32([t] * B), *stepped, W, N, **kw)
    pos = np.tile(np.arange(n), B)
    K, _ = o.qk_rope(f64(k), f64(gain), pos, 48, 1e4, 1e-6, interleaved)
    at = [t for t in range(n) if t < N or t >= n - W]
    slots = [o.slot_of(t, W, N) for t in at]
    u = o.HALF_STEP[dt]

    def typed(x):
        return torch.from_numpy(x.astype(np.float32)).to(TT[dt]).double().numpy()

    for side, x, e in (("k", K, (D + 40) * o.U32 * 1.5 * np.abs(K).max(-1, keepdims=True)), ("v", f64(v), 0.0)):
        S = c8.block_scale(np.abs(x).max())                  # no block had a larger one
        x, e = (np.broadcast_to(y, x.shape).reshape(B, n, J, D)[:, at].transpose(0, 2, 1, 3) for y in (x, e))
        # the code's value does not depend on the scale while it is normal
        lo, hi = (fp8.e4m3_value(fp8.e4m3_code(typed(y) / S)) * S for y in (x - e, x + e))
        normal = np.abs(x) - e >= 2.0 ** -6 * S
        assert normal.mean() > 0.9 and (lo == hi)[normal].mean() > 0.99
        for c in (filled, stepped):
            codes, scales = (c[0], c[2]) if side == "k" else (c[1], c[3])
            got = np.stack([c8.value(a, b, D) for a, b in zip(codes.cpu().numpy(), scales.cpu().numpy())])[:, :, slots]
            assert ((lo <= got) & (got <= hi))[normal].all(), side       # both roundings are monotonic
            # a subnormal one is off by half a step of each scale it was written under,
            # which double: twice the largest's at most
            assert (np.abs(got - x) <= (2.0 ** -4 + 2 * u) * np.abs(x) + 3 * 2.0 ** -10 * S + 2 * e).all(), side


def test_8_bit_caches_answer_nearly_as_bf16_ones():
    """The same histories served from both: the outputs differ by what the
    codes lose (at most 2^-4 of each key and value)."""
    from paper_2512_09200_amd import api
    rng = np.random.default_rng(6)
    H, J, D, W, N = 8, 2, 64, 100, 4
    lens = [250, 30, 104]
    off = np.concatenate([[0], np.cumsum(lens)])
    k, v = (randn(rng, int(off[-1]), J, D).bfloat16().to(DEV) for _ in "kv")
    s = plan(off, int(off[-1]))
    c16 = [torch.zeros(3, J, W + N, D, dtype=torch.bfloat16, device=DEV) for _ in "kv"]
    kc = to_gpu(new_caches(3, J, W + N, D, garbage=False))
    api.lattice_seq_cache_fill(s, k, v, *c16, W, N)
    api.lattice_seq_cache8_fill(s, k, v, *kc, W, N)
    q, kn, vn = (randn(rng, 3, h, D).bfloat16().to(DEV) for h in (H, J, J))
    a = api.lattice_seq_step(q, kn, vn, i32(lens), *c16, W, N)
    b = api.lattice_seq_step8(q, kn, vn, i32(lens), *kc, W, N)
    # scores off by scale sum |q k| 2^-4 at most; rounding errors of either sign make it far less
    assert (f64(a) - f64(b)).std() <= 0.1 * f64(a).std()


def test_skipped_users_and_unreached_slots_keep_their_memory():
    from paper_2512_09200_amd import api
    rng = np.random.default_rng(3)
    J, D, W, N = 2, 40, 37, 3
    host = new_caches(4, J, W + N, D)
    kc = to_gpu(host)
    q, k, v = (randn(rng, 3, h, D).to(DEV) for h in (4, J, J))
    api.lattice_seq_step8(q, k, v, i32([4, -1, 0]), *kc, W, N, cache_index=i32([7, 1, 2]), rope=False)
    c8.put(host, 2, {0: (f64(k[2]), f64(v[2]))}, 1)
    same(kc, host)
    assert (kc[0][2, :, 0, D:] == 0).all()                    # bytes past head_dim


def test_caches_beyond_4_gib():
    from paper_2512_09200_amd import api
    rng = np.random.default_rng(12)
    J, D, W = 1, 128, 600
    C = 2 ** 32 // (W * D) + 3
    k, v = (torch.zeros(C, J, W, D, dtype=torch.uint8, device=DEV) for _ in "kv")
    ks, vs = (torch.ones(C, J, -(-W // 16), device=DEV) for _ in "kv")
    x, y = randn(rng, 700, J, D).to(DEV), randn(rng, 700, J, D).to(DEV)
    api.lattice_seq_cache8_fill(plan([0, 700], 700), x, y, k, v, ks, vs, W, cache_index=i32([C - 1]))
    host = new_caches(1, J, W, D, garbage=False)
    c8.fill(host, f64(x), f64(y), [0, 700], W, 0, [0], [0])
    same((k[C - 1:], v[C - 1:], ks[C - 1:], vs[C - 1:]), host)
    q = randn(rng, 1, 2, D).to(DEV)
    out = api.lattice_seq_step8(q, x[:1], y[:1], i32([700]), k, v, ks, vs, W, cache_index=i32([C - 1]), rope=False)
    small = [t[C - 1:].clone() for t in (k, v, ks, vs)]
    assert torch.equal(out, api.lattice_seq_step8(q, x[:1], y[:1], i32([700]), *small, W, rope=False))
    assert not k[:C - 1].any()


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_millions_of_sequences(dt):
    """More sequences than a launch has waves for: the same as from calls of a few
    hundred thousand, and blocks that hold older events are made anew once."""
    from paper_2512_09200_amd import api
    S, J, D, W = 1_500_000, 3, 8, 5
    k, v = (torch.randn(2 * S, J, D, device=DEV, dtype=TT[dt]) for _ in "kv")
    k[1::2] *= 100
    whole = [torch.zeros(S, J, W, 16, dtype=torch.uint8, device=DEV) for _ in "kv"] + [
        torch.ones(S, J, 1, device=DEV) for _ in "kv"]
    parts = [t.clone() for t in whole]
    index = torch.randperm(S, device=DEV).int()

    def fill(caches, a, b, at, first):
        n = b - a
        s = api.lattice_seq_plan(torch.arange(n + 1, device=DEV, dtype=torch.int32), n)
        x, y = k[at::2][a:b], v[at::2][a:b]
        api.lattice_seq_cache8_fill(s, x.contiguous(), y.contiguous(), *caches, W, cache_index=index[a:b].contiguous(),
                                    first=torch.full((n,), first, dtype=torch.int32, device=DEV))

    for at in (0, 1):
        fill(whole, 0, S, at, at)
        for a in range(0, S, 250_000):
            fill(parts, a, a + 250_000, at, at)
    for a, b in zip(whole, parts):
        assert torch.equal(a, b)
    host = dict(k=np.zeros((3, J, W, 16), np.uint8), v=np.zeros((3, J, W, 16), np.uint8), ks=np.ones((3, J, 1), np.float32),
                vs=np.ones((3, J, 1), np.float32))
    for i, s in enumerate((0, 777_777, S - 1)):
        for at in (0, 1):
            c8.put(host, i, {at: (f64(k[2 * s + at]), f64(v[2 * s + at]))}, at + 1)
    pick = index[[0, 777_777, S - 1]].long()
    same([t[pick] for t in whole], host)


@pytest.mark.parametrize("long", [False, True])
def test_a_step_in_a_graph_that_advances_by_itself(long):
    from paper_2512_09200_amd import api
    rng = np.random.default_rng(5)
    B, H, J, D, W, N = (1, 4, 1, 64, 3000, 2) if long else (3, 4, 2, 64, 20, 2)
    kc = to_gpu(new_caches(B, J, W + N, D, garbage=False))
    q, k, v = (randn(rng, B, h, D).bfloat16().to(DEV) for h in (H, J, J))
    have, ref_have = torch.zeros(B, dtype=torch.int32, device=DEV), torch.zeros(B, dtype=torch.int32, device=DEV)
    ref = [t.clone() for t in kc]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        api.lattice_seq_step8(q, k, v, have, *[t.clone() for t in kc], W, N)
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = api.lattice_seq_step8(q, k, v, have, *kc, W, N)
        have += 1
    for t in range(40):
        x = randn(rng, B, J, D).bfloat16().to(DEV)
        k.copy_(x)
        g.replay()
        want = api.lattice_seq_step8(q, k, v, ref_have, *ref, W, N)
        ref_have += 1
        assert torch.equal(out, want), t
        for a, b in zip(kc, ref):
            assert torch.equal(a, b), t
        torch.cuda.synchronize()


def test_a_step_and_a_fill_on_a_stream_of_its_own():
    from paper_2512_09200_amd import api
    rng = np.random.default_rng(8)
    J, D, W, N = 2, 64, 5000, 4
    kc = to_gpu(new_caches(2, J, W + N, D, garbage=False))
    ref = [t.clone() for t in kc]
    k, v = (randn(rng, 700, J, D).bfloat16().to(DEV) for _ in "kv")
    s, q = plan([0, 300, 700], 700), randn(rng, 2, 4, D).bfloat16().to(DEV)
    api.lattice_seq_cache8_fill(s, k, v, *ref, W, N)
    want = api.lattice_seq_step8(q, k[:2], v[:2], i32([300, 400]), *ref, W, N)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    api.lattice_seq_cache8_fill(s, k, v, *kc, W, N, stream=side)
    got = api.lattice_seq_step8(q, k[:2], v[:2], i32([300, 400]), *kc, W, N, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want) and all(torch.equal(a, b) for a, b in zip(kc, ref))


# ---------------------------------------------------------------------------
def test_an_event_block_in_8_bits():
    """The operators as a served block uses them: residual norm to codes, FP8
    projection, step over the 8-bit cache, and the next residual norm; then the
    trained block's gradient through dropout and norm."""
    from oracle import norm as on
    from paper_2512_09200_amd import api
    rng = np.random.default_rng(7)
    B, cols, H, J, D, W = 5, 96, 4, 2, 32, 24
    x, res = randn(rng, B, cols).bfloat16().to(DEV), randn(rng, B, cols).bfloat16().to(DEV)
    gain = (1 + 0.1 * randn(rng, cols)).to(DEV)
    w = randn(rng, (H + 2 * J) * D, cols).bfloat16().to(DEV) / 8
    qw, sw = api.lattice_fp8_quantize(w)
    kc = to_gpu(new_caches(B, J, W, D, garbage=False))
    host = new_caches(B, J, W, D, garbage=False)
    lens = i32([0] * B)
    for t in range(30):
        h, _, q8, s8 = api.lattice_add_rmsnorm_fwd(x, res, gain, out="fp8")
        qkv = api.lattice_linear_fp8_fwd(q8, s8, qw, sw, cols).view(B, H + 2 * J, D)
        # the projection from the oracle's values of the codes
        A = fp8.e4m3_value(q8.cpu().numpy()[:, :cols]) * f64(s8)[:, None]
        Wt = fp8.e4m3_value(qw.cpu().numpy()[:, :cols]) * f64(sw)[:, None]
        assert np.abs(f64(qkv).reshape(B, -1) - A @ Wt.T).max() <= 2e-2 * np.abs(A @ Wt.T).max()
        q, k, v = qkv[:, :H], qkv[:, H:H + J], qkv[:, H + J:]
        out = api.lattice_seq_step8(q, k, v, lens, *kc, W, rope=False)
        for b in range(B):
            c8.put(host, b, {o.slot_of(t, W, 0): (f64(k)[b], f64(v)[b])}, t + 1)
            KC, VC = c8.value(host["k"][b], host["ks"][b], D), c8.value(host["v"][b], host["vs"][b], D)
            for hh in range(H):
                want, mass, _ = c8.attend(KC[hh // 2], VC[hh // 2], f64(q)[b, hh], min(t + 1, W), D ** -0.5)
                assert np.abs(f64(out)[b, hh] - want).max() <= (2.0 ** -8 + 2.0 ** -12) * mass.max()
        same(kc, host, f"event {t}")
        lens += 1
        x, res = out.reshape(B, H * D)[:, :cols].contiguous(), h
    # training: dropout, norm and a linear loss, gradients against the chain's
    state = torch.tensor([3, 4], device=DEV)
    h, y, _, _ = api.lattice_add_rmsnorm_fwd(x, res, gain, dropout=(0.3, state, 1))
    z = api.lattice_dropout(y, 0.2, state, site=2)
    dz, dh = randn(rng, B, cols).bfloat16().to(DEV), randn(rng, B, cols).bfloat16().to(DEV)
    dy = api.lattice_dropout(dz, 0.2, state, site=2)
    dr, dx, dg = api.lattice_add_rmsnorm_bwd(h, dy, dh, gain, dropout=(0.3, state, 1))
    f1, f2 = (on.factor(np.arange(B), cols, p, 3, 4, s) for p, s in ((0.3, 1), (0.2, 2)))
    assert np.abs(f64(h) - (f64(x) * f1 + f64(res))).max() <= 2.0 ** -8 * np.abs(f64(h)).max()
    yy, _ = on.rmsnorm(f64(h), f64(gain), 1e-6)
    assert np.abs(f64(z) - yy * f2).max() <= 2.0 ** -7 * np.abs(yy * f2).max()
    wr, wg = on.rmsnorm_bwd(f64(h), f64(gain), 1e-6, f64(dz) * f2, f64(dh))
    assert np.linalg.norm(f64(dr) - wr) <= 2.0 ** -7 * np.linalg.norm(wr)
    assert np.linalg.norm(f64(dx) - wr * f1) <= 2.0 ** -7 * np.linalg.norm(wr * f1)
    assert np.linalg.norm(f64(dg) - wg) <= 2.0 ** -7 * np.linalg.norm(wg)


def test_refusals_of_the_binding():
    from paper_2512_09200_amd import LatticeError, api
    J, D, W, N = 2, 40, 20, 2
    kc = to_gpu(new_caches(3, J, W + N, D, garbage=False))
    q, k, v = (torch.randn(2, h, D, device=DEV) for h in (4, J, J))
    lens = i32([0, 0])
    ok = (q, k, v, lens) + kc
    api.lattice_seq_step8(*ok, W, N)
    for i, bad in ((0, q[..., :32]), (1, k[:, :1]), (2, v.bfloat16()), (3, lens.long()), (3, lens[:1]), (4, kc[0][..., :D]),
                   (5, kc[1].view(torch.int8)), (6, kc[2][:, :, :1]), (7, kc[3].double()), (4, kc[0][:2]), (6, kc[2].cpu())):
        a = list(ok)
        a[i] = bad
        with pytest.raises((ValueError, TypeError, LatticeError)):
            api.lattice_seq_step8(*a, W, N)
    with pytest.raises(ValueError):
        api.lattice_seq_step8(*ok, W + 1, N)
    s = plan([0, 2], 2)
    for a in ((k, v[:1]), (k[:1], v[:1]), (k.cpu(), v.cpu())):
        with pytest.raises((ValueError, LatticeError)):
            api.lattice_seq_cache8_fill(s, *a, *kc, W, N)
