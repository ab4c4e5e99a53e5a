"""What an event block has between its products, and its cache in 8 bits
(`paper_2512_09200_amd.api`): root-mean-square norm of a residual sum with an
output in the storage type or in e4m3 codes, dropout from a counter-based
generator whose mask is never stored, and the single-event attention step with
its fill over ring caches of e4m3 codes with a scale for every 16 slots.

A case is a dict of plain values.  `listed()` names the fixed ones, `draw(rng)`
gives one more of the same ranges, `prepare(case, seed)` makes a call's inputs
on the GPU, `run(state)` is one pass (the plain torch form, or the framework's
kernels where `own` is true), `work(case)` its compulsory bytes and
operations, and `exact(case, seed)` the same outputs from the definition in
64 bits.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
EPS = 1e-6
THETA = 10000.0
BLOCK = 16                                  # slots that share a scale
F8 = torch.float8_e4m3fn
F8_MAX = 448.0
TORCH_TYPE = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------
def listed():
    return [
        # One user's event between two layers of a served model: the smallest
        # call, latency alone.
        dict(name="norm-event-bf16-fp8", kind="norm", dtype="bf16", rows=1, cols=512, train=False, residual=True,
             p=0.0, out="fp8"),
        # The same for a serving batch, in front of an FP8 projection.
        dict(name="norm-serve-bf16-fp8", kind="norm", dtype="bf16", rows=8192, cols=1024, train=False,
             residual=True, p=0.0, out="fp8"),
        # A large training batch of events: dropout of the layer's output,
        # residual, norm, and the gradients of all.
        dict(name="norm-train-large-bf16", kind="norm", dtype="bf16", rows=131072, cols=1024, train=True,
             residual=True, p=0.1, out="y"),
        # fp32 model, rows that no 16-byte load fits, no residual (the norm in
        # front of the first layer).
        dict(name="norm-train-odd-f32", kind="norm", dtype="f32", rows=5021, cols=1001, train=True, residual=False,
             p=0.0, out="y"),
        # Wide rows of mixed FP8 training: codes for the product and the
        # storage type for its weight gradient.
        dict(name="norm-train-wide-bf16-both", kind="norm", dtype="bf16", rows=2048, cols=8192, train=True,
             residual=True, p=0.0, out="both"),
        # Dropout of a small layer, forward and backward.
        dict(name="dropout-small-f32", kind="drop", dtype="f32", rows=53, cols=33, train=True, p=0.5),
        # Dropout of a large batch's activations.
        dict(name="dropout-large-bf16", kind="drop", dtype="bf16", rows=131072, cols=1024, train=False, p=0.1),
        # A few fp32 histories laid into their 8-bit caches.
        dict(name="fill8-small-f32", kind="fill8", dtype="f32", T=501, S=5, L=300, C=8, J=2, D=40, W=100, N=3),
        # The histories of a serving restart: only sinks and window are kept.
        dict(name="fill8-large-bf16", kind="fill8", dtype="bf16", T=262144, S=300, L=4096, C=400, J=2, D=128,
             W=508, N=4),
        # One user's next event: the smallest step.
        dict(name="step8-one-f32", kind="step8", dtype="f32", S=1, C=4, H=4, J=2, D=64, R=64, pairs="halves", W=252,
             N=4, far=False),
        # A serving batch, every user's window full or filling.
        dict(name="step8-batch-bf16", kind="step8", dtype="bf16", S=1024, C=1100, H=8, J=2, D=128, R=128,
             pairs="halves", W=1020, N=4, far=False),
        # Few users with very long windows: the cache's length is the only
        # axis to spread over the chip.
        dict(name="step8-long-bf16", kind="step8", dtype="bf16", S=3, C=3, H=16, J=2, D=128, R=64, pairs="halves",
             W=131013, N=36, far=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    biggest = {k: max(_cost(c) for c in listed() if c["kind"] == k) for k in ("norm", "drop", "fill8", "step8")}
    while True:
        kind = rng.choice(["norm", "norm", "norm", "drop", "fill8", "step8", "step8"])
        c = dict(kind=kind, dtype=rng.choice(["bf16", "bf16", "f32"]))
        if kind in ("norm", "drop"):
            c.update(rows=_log(rng, 1, 131072), cols=_log(rng, 8, 8192), train=rng.random() < 0.5)
            if rng.random() < 0.6:
                c["cols"] = -(-c["cols"] // 8) * 8
        if kind == "norm":
            c.update(residual=rng.random() < 0.7, p=rng.choice([0.0, 0.0, 0.1, round(rng.uniform(0.01, 0.7), 3)]),
                     out=rng.choice(["y", "y", "fp8", "both"]))
        elif kind == "drop":
            c.update(p=rng.choice([0.1, 0.5, round(rng.uniform(0.01, 0.9), 3)]))
        else:
            J = rng.choice([1, 1, 2, 3, 4])
            D = rng.choice([16, 32, 32, 40, 64, 64, 96, 128, 128])
            N = rng.choice([0, 1, 4, 16, 64])
            if kind == "step8":
                S = _log(rng, 1, 3000)
                c.update(S=S, C=S + rng.randint(0, 20), H=J * rng.choice([1, 2, 3, 4, 8]), J=J, D=D,
                         R=8 * rng.randint(1, D // 8), pairs=rng.choice(["halves", "neighbours"]),
                         W=_log(rng, 1, 60000), N=N, far=rng.random() < 0.5)
            else:
                S, L = _log(rng, 1, 4000), _log(rng, 1, 9000)
                mean = max(1, min(L, int(L * rng.uniform(0.3, 0.9))))
                c.update(T=max(S, min(S * mean, S * L)), S=S, L=L, C=S + rng.randint(0, 20), J=J, D=D,
                         W=_log(rng, 1, 4096), N=N)
        if _cost(c) <= biggest[kind]:
            return c


# ---------------------------------------------------------------------------
# compulsory work
# ---------------------------------------------------------------------------
def _lengths(T, S, L, seed):
    """S lengths in 1 .. L of sum T, spread like user activity (log-normal)."""
    rs = np.random.RandomState(seed % (1 << 31))
    w = rs.lognormal(0.0, 0.6, S)
    n = np.clip(np.floor(w / w.sum() * T).astype(np.int64), 1, L)
    while n.sum() != T:
        d = int(T - n.sum())
        can = np.flatnonzero(n < L) if d > 0 else np.flatnonzero(n > 1)
        room = (L - n[can]) if d > 0 else (n[can] - 1)
        take = np.minimum(room, max(1, abs(d) // can.size))
        order = rs.permutation(can.size)
        cut = np.minimum(np.cumsum(take[order]), abs(d))
        n[can[order]] += np.sign(d) * np.diff(cut, prepend=0)
    return n


def _history(c, seed):
    """Events each user of a step already has: full windows and filling ones."""
    rs = np.random.RandomState((seed + 7) % (1 << 31))
    full = c["N"] + c["W"]
    return np.floor(full * np.minimum(1.3, rs.uniform(0.3, 2.0, c["S"]))).astype(np.int64)


def _stores_h(c):
    return c["residual"] or c["p"] > 0


def work(case):
    c = case
    es = 2 if c["dtype"] == "bf16" else 4
    if c["kind"] == "drop":
        x = c["rows"] * c["cols"]
        passes = 2 if c["train"] else 1
        return {"bytes": passes * 2 * es * x, "flops": passes * x}
    if c["kind"] == "norm":
        x, n = c["rows"] * c["cols"], 4 * c["cols"]
        b = es * x * (1 + c["residual"] + _stores_h(c) + (c["out"] != "fp8")) + n
        b += (x + 4 * c["rows"]) if c["out"] != "y" else 0
        f = 6 * x
        if c["train"]:              # h, dy, the residual's gradient in; its, x's and the gain's out
            b += es * x * (2 + 2 * c["residual"] + (not c["residual"] or c["p"] > 0)) + 2 * n
            f += 12 * x
        return {"bytes": b, "flops": f}
    if c["kind"] == "step8":
        slots = float(_history(c, 1).clip(max=c["N"] + c["W"] - 1).sum() + c["S"])
        b = 2 * slots * c["J"] * (c["D"] + 4 / BLOCK) + c["S"] * (2 * c["H"] + 2 * c["J"]) * c["D"] * es
        return {"bytes": b, "flops": 4 * slots * c["H"] * c["D"]}
    kept = float(np.minimum(_lengths(c["T"], c["S"], c["L"], 1), c["W"] + c["N"]).sum())
    return {"bytes": 2 * kept * c["J"] * (c["D"] * (es + 1) + 4 / BLOCK), "flops": 4 * kept * c["J"] * c["D"]}


def _cost(c):
    w = work(c)
    extra = 0.0                     # what the plain form moves
    if c["kind"] == "norm" and c["p"] > 0:
        extra = 2.0 * w["bytes"]
    if c["kind"] == "fill8":
        extra = c["T"] * c["J"] * c["D"] * 4.0 + 0.5 * c["S"] * c["J"] * (c["N"] + c["W"]) * c["D"]
    if c["kind"] == "step8":
        extra = c["S"] * c["J"] * (c["N"] + c["W"]) * c["D"] * 2.0
    return max(w["bytes"], extra)


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


def _ld(D):
    """Bytes of a slot's codes: rows of whole 16 bytes."""
    return -(-D // 16) * 16


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    rs = np.random.RandomState((seed + 1) % (1 << 31))
    dt = TORCH_TYPE[c["dtype"]]

    def rand(*shape):
        return torch.randn(*shape, generator=g, device=DEV, dtype=dt)

    s = dict(case=c)
    if c["kind"] in ("norm", "drop"):
        shape = c["rows"], c["cols"]
        s["x"] = rand(*shape)
        # the generator's seed and the training step's number
        s["rng"] = torch.tensor([int(rs.randint(1 << 62)), int(rs.randint(1 << 20))], device=DEV)
        s["site"] = 3                       # which dropout of the model this is
        if c["train"]:
            s["dy"] = rand(*shape)
    if c["kind"] == "norm":
        s["residual"] = rand(*shape).mul_(2) if c["residual"] else None
        s["gain"] = 1 + 0.1 * _normal(g, c["cols"])
        s["dh"] = rand(*shape) if c["train"] and c["residual"] else None
    if c["kind"] in ("fill8", "step8"):
        J, D, cap = c["J"], c["D"], c["N"] + c["W"]
        nb, ld = -(-cap // BLOCK), _ld(c["D"])
        s["index"] = torch.from_numpy(rs.permutation(c["C"])[:c["S"]].astype(np.int32)).to(DEV)
        for x in ("k", "v"):
            s[x + "c"] = torch.zeros(c["C"], J, cap, ld, dtype=torch.uint8, device=DEV)
            s[x + "s"] = torch.ones(c["C"], J, nb, device=DEV)
    if c["kind"] == "fill8":
        n = _lengths(c["T"], c["S"], c["L"], seed)
        s["offsets"] = torch.from_numpy(np.concatenate([[0], np.cumsum(n)]).astype(np.int32)).to(DEV)
        s["k"], s["v"] = rand(c["T"], J, D), rand(c["T"], J, D)
    elif c["kind"] == "step8":
        S, H = c["S"], c["H"]
        s["q"], s["k"], s["v"] = rand(S, H, D), rand(S, J, D), rand(S, J, D)
        s["gq"], s["gk"] = 1 + 0.1 * _normal(g, D), 1 + 0.1 * _normal(g, D)
        n = _history(c, seed)
        s["lens"] = torch.from_numpy(n.astype(np.int32)).to(DEV)
        s["positions"] = torch.from_numpy((n + 25_000_000).astype(np.int32)).to(DEV) if c["far"] else None
        # what earlier events left: slots that none has reached hold zeros
        at = s["index"].long()
        for x in ("k", "v"):
            old = _normal(g, S, J, nb * BLOCK, D)
            old *= torch.arange(nb * BLOCK, device=DEV)[None, None, :, None] < s["lens"].clamp(max=cap)[:, None, None, None]
            scale, codes = _encode(old.view(S, J, nb, BLOCK, D))
            s[x + "s"][at] = scale
            s[x + "c"][at, :, :, :D] = codes.view(torch.uint8).view(S, J, nb * BLOCK, D)[:, :, :cap]
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    from paper_2512_09200_amd import api
    c = s["case"]
    if c["kind"] == "drop":
        o = {"out": api.lattice_dropout(s["x"], c["p"], s["rng"], site=s["site"])}
        if c["train"]:
            o["dx"] = api.lattice_dropout(s["dy"], c["p"], s["rng"], site=s["site"])
        return o
    if c["kind"] == "norm":
        drop = (c["p"], s["rng"], s["site"]) if c["p"] > 0 else None
        h, y, codes, scales = api.lattice_add_rmsnorm_fwd(s["x"], s["residual"], s["gain"], eps=EPS, dropout=drop,
                                                          out=c["out"])
        o = {}
        if _stores_h(c):
            o["h"] = h
        if c["out"] != "fp8":
            o["y"] = y
        if c["out"] != "y":
            o["codes"], o["scales"] = codes.view(F8)[:, :c["cols"]], scales
        if c["train"]:
            d_res, dx, dgain = api.lattice_add_rmsnorm_bwd(h, s["dy"], s["dh"], s["gain"], eps=EPS, dropout=drop)
            o["dgain"] = dgain
            if c["residual"]:
                o["d_residual"] = d_res
            if c["p"] > 0 or not c["residual"]:
                o["dx"] = dx
        return o
    caches = s["kc"], s["vc"], s["ks"], s["vs"]
    if c["kind"] == "fill8":
        seqs = api.lattice_seq_plan(s["offsets"], c["T"], max_len=c["L"])
        api.lattice_seq_cache8_fill(seqs, s["k"], s["v"], *caches, window=c["W"], sinks=c["N"], cache_index=s["index"])
        return _caches(s)
    out = api.lattice_seq_step8(s["q"], s["k"], s["v"], s["lens"], *caches, window=c["W"], sinks=c["N"],
                                cache_index=s["index"], gain_q=s["gq"], gain_k=s["gk"], theta=THETA, rotary=c["R"],
                                interleaved=c["pairs"] == "neighbours", eps=EPS, positions=s["positions"])
    return {"out": out, **_caches(s)}


def _run_plain(s):
    return {"norm": _plain_norm, "drop": _plain_drop, "fill8": _plain_fill, "step8": _plain_step}[s["case"]["kind"]](s)


def _caches(s):
    """The codes as the values they stand for, and their scales."""
    return {"kc": s["kc"].view(F8), "vc": s["vc"].view(F8), "ks": s["ks"], "vs": s["vs"]}


def _threshold(p):
    return int(math.floor(p * 65536 + 0.5))


LOW = 0xFFFFFFFF


def _philox_round(c, k):
    """One round of Philox4x32 on int64 tensors that hold 32-bit words.
    Products wrap at 64 bits, whose upper half the shift and mask give."""
    a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
    return (((b >> 32) & LOW) ^ c[1] ^ k[0], b & LOW, ((a >> 32) & LOW) ^ c[3] ^ k[1], a & LOW)


def _keep(s, p):
    """Which elements stay: [rows, cols], true or false.  Eight neighbouring
    columns take the eight 16-bit numbers of one block of the generator
    (counter: columns / 8, row, site, step; key: seed)."""
    c = s["case"]
    groups = -(-c["cols"] // 8)
    seed, step = s["rng"][0], s["rng"][1] & LOW
    like = torch.zeros(c["rows"], groups, dtype=torch.int64, device=DEV)
    w = (like + torch.arange(groups, device=DEV), like + torch.arange(c["rows"], device=DEV)[:, None], like + s["site"],
         like + step)
    for r in range(10):
        w = _philox_round(w, ((seed + r * 0x9E3779B9) & LOW, ((seed >> 32) + r * 0xBB67AE85) & LOW))
    w = torch.stack(w, -1)
    n = torch.stack([w & 0xFFFF, w >> 16], -1).view(c["rows"], groups * 8)
    return n[:, :c["cols"]] >= _threshold(p)


def _dropped(x, keep, p):
    return torch.where(keep, x.float() * (65536.0 / (65536 - _threshold(p))), 0.0)


def _plain_drop(s):
    p, dt, keep = s["case"]["p"], s["x"].dtype, _keep(s, s["case"]["p"])
    o = {"out": _dropped(s["x"], keep, p).to(dt)}
    if s["case"]["train"]:
        o["dx"] = _dropped(s["dy"], keep, p).to(dt)
    return o


def _plain_norm(s):
    c = s["case"]
    p, dt = c["p"], s["x"].dtype
    keep = _keep(s, p) if p > 0 else None
    h = _dropped(s["x"], keep, p) if p > 0 else s["x"].float()
    if c["residual"]:
        h = h + s["residual"].float()
    h = h.to(dt)                            # the residual stream is kept in the storage type
    o = {"h": h} if _stores_h(c) else {}
    h = h.float()
    rho = torch.rsqrt(h.square().mean(-1, keepdim=True) + EPS)
    n = h * rho
    y = n * s["gain"]
    if c["out"] != "fp8":
        o["y"] = y.to(dt)
    if c["out"] != "y":
        top = y.abs().amax(-1, keepdim=True)
        scale = torch.where(top > 0, top / F8_MAX, torch.ones_like(top))
        o["codes"] = (y * (1 / scale)).clamp(-F8_MAX, F8_MAX).to(F8)
        o["scales"] = scale[:, 0]
    if not c["train"]:
        return o
    dy = s["dy"].float()
    o["dgain"] = (dy * n).sum(0)
    dn = dy * s["gain"]
    d = rho * (dn - n * (dn * n).mean(-1, keepdim=True))
    if c["residual"]:
        d = d + s["dh"].float()
        o["d_residual"] = d.to(dt)
    if p > 0:
        o["dx"] = _dropped(d, keep, p).to(dt)
    elif not c["residual"]:
        o["dx"] = d.to(dt)
    return o


def _block_scale(top):
    """The smallest power of two s with top <= 448 s (1 for an empty block)."""
    m, e = torch.frexp(top)                 # top = m 2^e, m in [1/2, 1); 448 = 0.875 2^9
    s = torch.ldexp(torch.ones_like(top), (e - 9 + (m > 0.875).int()).clamp(min=-117))
    return torch.where(top > 0, s, torch.ones_like(top))


def _encode(x):
    """Scales [...] and codes of blocks [..., 16, D]."""
    s = _block_scale(x.abs().amax((-1, -2)))
    return s, (x / s[..., None, None]).to(F8)


def _slot(p, W, N):
    return torch.where(p < N, p, N + (p - N) % W)


def _plain_fill(s):
    """The kept rows in a float copy of their caches, whose blocks are then
    encoded (the caches are new: all that they hold comes from this call)."""
    c = s["case"]
    T, S, J, D, W, N = c["T"], c["S"], c["J"], c["D"], c["W"], c["N"]
    cap = N + W
    nb = -(-cap // BLOCK)
    row, off = torch.arange(T, device=DEV), s["offsets"].long()
    seq = torch.searchsorted(off, row, right=True) - 1
    p, n = row - off[seq], off[1:] - off[:-1]
    keep = (p < N) | (p >= n[seq] - W)
    seq, slot = seq[keep], _slot(p, W, N)[keep]
    at = s["index"].long()
    used = torch.arange(nb, device=DEV) * BLOCK < n.clamp(max=cap)[:, None]             # [S, nb]

    def lay(x, codes, scales):
        full = torch.zeros(S, J, nb * BLOCK, D, device=DEV)
        full[seq, :, slot] = x[keep].float()
        sc, q = _encode(full.view(S, J, nb, BLOCK, D))
        codes[at, :, :, :D] = q.view(torch.uint8).view(S, J, nb * BLOCK, D)[:, :, :cap]
        scales[at] = torch.where(used[:, None, :], sc, scales[at])

    lay(s["k"], s["kc"], s["ks"])
    lay(s["v"], s["vc"], s["vs"])
    return _caches(s)


def _turned(x, gain, pos, R, pairs):
    """Norm per head and rotation, in 64 bits: the result is rounded to eight
    bits, and a value next to a border must fall on its own side."""
    x = x.double()
    z = x / (x.square().mean(-1, keepdim=True) + EPS).sqrt() * gain.double()
    f = THETA ** (-2.0 * torch.arange(R // 2, device=DEV, dtype=torch.float64) / R)
    phi = (pos.double()[:, None] * f)[:, None, :]
    cos, sin = phi.cos(), phi.sin()
    if pairs == "halves":
        u, v = z[..., :R // 2], z[..., R // 2:R]
        return torch.cat([u * cos - v * sin, u * sin + v * cos, z[..., R:]], -1)
    u, v = z[..., 0:R:2], z[..., 1:R:2]
    return torch.cat([torch.stack([u * cos - v * sin, u * sin + v * cos], -1).flatten(-2), z[..., R:]], -1)


def _append(s, new, codes, scales):
    """Puts the events' rows [S, J, D] into their slots and encodes their
    blocks anew."""
    c = s["case"]
    D, W, N = c["D"], c["W"], c["N"]
    lens, at = s["lens"].long(), s["index"].long()
    slot = _slot(lens, W, N)
    b = slot // BLOCK
    places = b[:, None] * BLOCK + torch.arange(BLOCK, device=DEV)                       # [S, 16]
    live = (places < N + W) & ((places < lens[:, None]) | (places == slot[:, None]))
    got = torch.where(live, places, slot[:, None])          # in the place of the others: the new row once more
    mine = (got == slot[:, None])[:, :, None, None]
    x = codes[at[:, None], :, got][..., :D].view(F8).float() * scales[at, :, b][:, None, :, None]     # [S, 16, J, D]
    x = torch.where(mine, new[:, None].float(), x).transpose(1, 2)                      # [S, J, 16, D]
    sc, q = _encode(x)
    scales[at, :, b] = sc
    codes[at[:, None], :, got, :D] = q.view(torch.uint8).transpose(1, 2)


def _plain_step(s):
    c = s["case"]
    S, H, J, D, W, N = c["S"], c["H"], c["J"], c["D"], c["W"], c["N"]
    dt, lens, at = s["q"].dtype, s["lens"].long(), s["index"].long()
    pos = s["positions"] if s["positions"] is not None else lens
    q = _turned(s["q"], s["gq"], pos, c["R"], c["pairs"]).float()
    _append(s, _turned(s["k"], s["gk"], pos, c["R"], c["pairs"]).to(dt), s["kc"], s["ks"])
    _append(s, s["v"], s["vc"], s["vs"])

    def cache(codes, scales):
        return codes[at][..., :D].view(F8).float() * scales[at].repeat_interleave(BLOCK, -1)[..., :N + W, None]

    see = torch.arange(N + W, device=DEV)[None, :] <= lens[:, None]
    sc = q.view(S, J, H // J, D) @ cache(s["kc"], s["ks"]).transpose(-1, -2) * D ** -0.5
    sc = sc.masked_fill_(~see[:, None, None, :], -math.inf)
    p = torch.exp(sc - sc.amax(-1, keepdim=True))
    out = p @ cache(s["vc"], s["vs"]) / p.sum(-1, keepdim=True)
    return {"out": out.view(S, H, D).to(dt), **_caches(s)}


# ---------------------------------------------------------------------------
# the definition in 64 bits
# ---------------------------------------------------------------------------
def _exact_factor(s):
    """0 or 1 / (1 - t / 65536) of every element, on the host."""
    c = s["case"]
    rows, cols, groups = c["rows"], c["cols"], -(-c["cols"] // 8)
    seed, step = (int(v) for v in s["rng"].tolist())
    t = _threshold(c["p"])
    full = np.empty((rows, groups, 8), np.uint16)
    mask, at = np.uint64(LOW), max(1, (1 << 19) // groups)
    for r0 in range(0, rows, at):
        r1 = min(rows, r0 + at)
        x0, x1 = np.meshgrid(np.arange(groups, dtype=np.uint64), np.arange(r0, r1, dtype=np.uint64))
        x2, x3 = np.full_like(x0, s["site"]), np.full_like(x0, step & LOW)
        key = [seed & LOW, (seed >> 32) & LOW]
        for _ in range(10):
            lo, hi = np.uint64(0xD2511F53) * x0, np.uint64(0xCD9E8D57) * x2
            x0, x1, x2, x3 = ((hi >> np.uint64(32)) ^ x1 ^ np.uint64(key[0]), hi & mask,
                              (lo >> np.uint64(32)) ^ x3 ^ np.uint64(key[1]), lo & mask)
            key = [(key[0] + 0x9E3779B9) & LOW, (key[1] + 0xBB67AE85) & LOW]
        for i, x in enumerate((x0, x1, x2, x3)):
            full[r0:r1, :, 2 * i] = (x & np.uint64(0xFFFF)).astype(np.uint16)
            full[r0:r1, :, 2 * i + 1] = (x >> np.uint64(16)).astype(np.uint16)
    keep = torch.from_numpy(full.reshape(rows, groups * 8)[:, :cols] >= t).to(DEV)
    return keep.double() / (1 - t / 65536.0)


def _exact_norm(s):
    c = s["case"]
    factor = _exact_factor(s) if c["p"] > 0 else 1.0
    h = s["x"].double() * factor + (s["residual"].double() if c["residual"] else 0.0)
    o = {"h": h} if _stores_h(c) else {}
    h = h.to(s["x"].dtype).double()         # the norm is that of the sum as it is kept
    rms = (h.pow(2).sum(-1, keepdim=True) / c["cols"] + EPS).sqrt()
    gain = s["gain"].double()
    y = h / rms * gain
    if c["out"] != "fp8":
        o["y"] = y
    if c["out"] != "y":
        o["scales"] = y.abs().max(-1).values / F8_MAX
        o["codes"] = y / o["scales"][:, None]
    if c["train"]:
        dy = s["dy"].double()
        o["dgain"] = (dy * h / rms).sum(0)
        z = dy * gain
        d = z / rms - h * (z * h).sum(-1, keepdim=True) / (c["cols"] * rms.pow(3))
        if c["residual"]:
            d += s["dh"].double()
            o["d_residual"] = d
        if c["p"] > 0 or not c["residual"]:
            o["dx"] = d * factor
    return o


def _exact_drop(s):
    factor = _exact_factor(s)
    o = {"out": s["x"].double() * factor}
    if s["case"]["train"]:
        o["dx"] = s["dy"].double() * factor
    return o


def _power(top):
    """The block scale, from its definition."""
    if not top > 0:
        return 1.0
    s = 2.0 ** math.floor(math.log2(top / F8_MAX))
    while F8_MAX * s < top:
        s *= 2
    while F8_MAX * s / 2 >= top:
        s /= 2
    return s


def _exact_cache(s, x):
    """Codes and scales as numbers in 64 bits."""
    D = s["case"]["D"]
    codes = s[x + "c"].view(F8).double()
    codes[..., D:] = 0
    return codes, s[x + "s"].double()


def _exact_fill(s):
    c = s["case"]
    J, W, N, D = c["J"], c["W"], c["N"], c["D"]
    off, o = s["offsets"].tolist(), {}
    for x in ("k", "v"):
        codes, scales = _exact_cache(s, x)
        for b, at in enumerate(s["index"].tolist()):
            n = off[b + 1] - off[b]
            p = np.unique(np.concatenate([np.arange(min(n, N)), np.arange(max(0, n - W), n)]))
            slots = np.where(p < N, p, N + (p - N) % W)
            nb = int(slots.max()) // BLOCK + 1
            rows = torch.zeros(nb * BLOCK, J, D, dtype=torch.float64, device=DEV)
            rows[torch.from_numpy(slots).to(DEV)] = s[x][torch.from_numpy(p + off[b]).to(DEV)].double()
            top = rows.view(nb, BLOCK, J, D).abs().amax((1, 3)).T.cpu().numpy()
            sc = torch.tensor([[_power(float(t)) for t in r] for r in top], dtype=torch.float64, device=DEV)
            scales[at, :, :nb] = sc
            m = min(N + W, nb * BLOCK)
            codes[at, :, :m, :D] = rows.transpose(0, 1)[:, :m] / sc.repeat_interleave(BLOCK, 1)[:, :m, None]
        o[x + "c"], o[x + "s"] = codes, scales
    return o


def _exact_turn(x, pos, R, pairs):
    """Pairs as complex numbers, turned by position * frequency."""
    x = x.clone()
    u, v = (slice(0, R // 2), slice(R // 2, R)) if pairs == "halves" else (slice(0, R, 2), slice(1, R, 2))
    freq = torch.exp(-math.log(THETA) * 2.0 / R * torch.arange(R // 2, device=x.device, dtype=torch.float64))
    z = torch.complex(x[..., u], x[..., v]) * torch.exp(1j * pos.double()[:, None, None] * freq)
    x[..., u], x[..., v] = z.real, z.imag
    return x


def _exact_rms(x):
    x = x.double()
    return x / (x.pow(2).sum(-1, keepdim=True) / x.shape[-1] + EPS).sqrt()


def _exact_step(s):
    c = s["case"]
    W, N, G, D, J = c["W"], c["N"], c["H"] // c["J"], c["D"], c["J"]
    dt = s["q"].dtype
    pos = s["positions"] if s["positions"] is not None else s["lens"]
    q = _exact_turn(_exact_rms(s["q"]) * s["gq"].double(), pos, c["R"], c["pairs"])
    k = _exact_turn(_exact_rms(s["k"]) * s["gk"].double(), pos, c["R"], c["pairs"])
    new = {"k": k.to(dt).double(), "v": s["v"].double()}
    cache = {x: _exact_cache(s, x) for x in ("k", "v")}
    out = torch.zeros_like(q)
    for b, (n, at) in enumerate(zip(s["lens"].tolist(), s["index"].tolist())):
        slot = n if n < N else N + (n - N) % W
        m = min(n + 1, N + W)
        blk, lo = slot // BLOCK, slot // BLOCK * BLOCK
        hi = min(lo + BLOCK, m)
        seen = {}
        for x, (codes, scales) in cache.items():
            rows = codes[at, :, lo:hi, :D] * scales[at, :, blk, None, None]
            rows[:, slot - lo] = new[x][b]
            sc = torch.tensor([_power(float(t)) for t in rows.abs().amax((1, 2)).tolist()], dtype=torch.float64, device=DEV)
            codes[at, :, lo:hi, :D] = rows / sc[:, None, None]
            scales[at, :, blk] = sc
            # the attention reads the codes, which are rounded
            rounded = codes[at, :, :m, :D].clone()
            rounded[:, lo:hi] = rounded[:, lo:hi].float().to(F8).double()
            seen[x] = rounded * scales[at].repeat_interleave(BLOCK, 1)[:, :m, None]
        w = torch.softmax(torch.bmm(q[b].view(-1, G, D), seen["k"].mT.contiguous()) / math.sqrt(D), -1)
        out[b] = torch.bmm(w, seen["v"]).view(-1, D)
    o = {"out": out}
    for x, (codes, scales) in cache.items():
        o[x + "c"], o[x + "s"] = codes, scales
    return o


def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "drop": _exact_drop, "fill8": _exact_fill, "step8": _exact_step}[case["kind"]](s)
