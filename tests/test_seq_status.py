"""Refusals of the event-sequence entry points: statuses of the C ABI on a
machine without a GPU (raised before anything is enqueued; the pointers are
placeholders), the workspace queries, and the binding's own checks."""
import ctypes
from ctypes import byref
from types import SimpleNamespace

import pytest
import torch

from paper_2512_09200_amd import _abi as A
from paper_2512_09200_amd import api

OK, INVALID_ARG, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
P = 0x10000             # placeholder device pointer, never dereferenced here


def _gpu_visible():
    return torch.cuda.device_count() > 0


pytestmark = pytest.mark.skipif(_gpu_visible(), reason="placeholder pointers must never reach a GPU")


@pytest.fixture(scope="module")
def lib():
    return A.load()


def seqs(rows=100, num_seqs=3, offsets=P, span=P, max_len=0):
    return A.lattice_seqs(rows=rows, num_seqs=num_seqs, offsets=offsets, span=span, max_len=max_len)


def rope(dtype=A.BF16, heads=4, kv_heads=2, head_dim=64, rotary_dim=64, theta=1e4, eps=1e-6, positions=None):
    return A.lattice_qk_rope_desc(dtype=dtype, heads=heads, kv_heads=kv_heads, head_dim=head_dim,
                                  rotary_dim=rotary_dim, theta=theta, eps=eps, positions=positions)


def attn(dtype=A.BF16, heads=4, kv_heads=2, head_dim=64, window=8, sinks=2, scale=0.125, key_mask=None):
    return A.lattice_seq_attn_desc(dtype=dtype, heads=heads, kv_heads=kv_heads, head_dim=head_dim, window=window,
                                   sinks=sinks, scale=scale, key_mask=key_mask)


def cache(k=P, v=P, num_caches=4):
    return A.lattice_seq_cache(k=k, v=v, num_caches=num_caches)


QS, KS = 4 * 64, 2 * 64


def test_plan(lib):
    f = lib.lattice_seq_plan
    assert f(None, P, None) == INVALID_ARG
    assert f(byref(seqs(rows=-1)), P, None) == INVALID_ARG
    assert f(byref(seqs(num_seqs=-1)), P, None) == INVALID_ARG
    assert f(byref(seqs(max_len=-1)), P, None) == INVALID_ARG
    assert f(byref(seqs(rows=1 << 30)), P, None) == UNSUPPORTED
    assert f(byref(seqs()), None, None) == INVALID_ARG
    assert f(byref(seqs()), P + 4, None) == INVALID_ARG
    assert f(byref(seqs(offsets=None)), P, None) == INVALID_ARG
    assert f(byref(seqs(rows=0)), None, None) == OK


def _rope_fwd(lib, d, s, q=P, ldq=QS, k=P, ldk=KS, qo=P, ldqo=QS, ko=P, ldko=KS):
    return lib.lattice_qk_rope_fwd(byref(d) if d else None, byref(s) if s else None, q, ldq, k, ldk, qo, ldqo, ko,
                                   ldko, None)


BAD_HEADS = [(dict(dtype=7), INVALID_ARG), (dict(heads=0), INVALID_ARG), (dict(heads=2000), INVALID_ARG),
             (dict(kv_heads=0), INVALID_ARG), (dict(head_dim=0), UNSUPPORTED), (dict(head_dim=136), UNSUPPORTED),
             (dict(head_dim=60), UNSUPPORTED), (dict(head_dim=-8), UNSUPPORTED)]


@pytest.mark.parametrize("bad,status", BAD_HEADS + [
    (dict(rotary_dim=72), UNSUPPORTED), (dict(rotary_dim=4), UNSUPPORTED), (dict(rotary_dim=-8), UNSUPPORTED),
    (dict(theta=0.0), INVALID_ARG), (dict(theta=float("nan")), INVALID_ARG), (dict(eps=-1.0), INVALID_ARG)])
def test_rope_descriptor(lib, bad, status):
    assert _rope_fwd(lib, rope(**bad), seqs()) == status
    assert lib.lattice_qk_rope_bwd(byref(rope(**bad)), byref(seqs()), P, QS, P, KS, P, QS, P, KS, P, QS, P, KS, None,
                                   None, None, 0, None) == status
    assert lib.lattice_qk_rope_bwd_workspace(byref(rope(**bad)), 100) == 0


def test_rope_tensors(lib):
    assert _rope_fwd(lib, None, seqs()) == INVALID_ARG
    assert _rope_fwd(lib, rope(), None) == INVALID_ARG
    assert _rope_fwd(lib, rope(), seqs(span=None)) == INVALID_ARG
    for name in ("q", "k", "qo", "ko"):
        assert _rope_fwd(lib, rope(), seqs(), **{name: None}) == INVALID_ARG
        assert _rope_fwd(lib, rope(), seqs(), **{name: P + 8}) == INVALID_ARG
        ld = "ld" + name
        for v in ((QS if name[0] == "q" else KS) - 8, QS + 4, (1 << 22) + 8):
            assert _rope_fwd(lib, rope(), seqs(), **{ld: v}) == INVALID_ARG
    assert _rope_fwd(lib, rope(), seqs(rows=0)) == OK
    need = lib.lattice_qk_rope_bwd_workspace(byref(rope()), 100)
    assert need > 0
    for ws, n in ((None, need), (P, need - 1)):
        assert lib.lattice_qk_rope_bwd(byref(rope()), byref(seqs()), P, QS, P, KS, P, QS, P, KS, P, QS, P, KS, P, None,
                                       ws, n, None) == WORKSPACE


def _fwd(lib, d, s, q=P, ldq=QS, k=P, ldk=KS, v=P, ldv=KS, o=P, ldo=QS):
    return lib.lattice_seq_attn_fwd(byref(d), byref(s), q, ldq, k, ldk, v, ldv, o, ldo, None, None, None)


@pytest.mark.parametrize("bad,status", BAD_HEADS + [
    (dict(heads=3), INVALID_ARG), (dict(window=0), INVALID_ARG), (dict(window=-5), INVALID_ARG),
    (dict(sinks=-1), INVALID_ARG), (dict(sinks=65), INVALID_ARG), (dict(scale=0.0), INVALID_ARG),
    (dict(scale=-1.0), INVALID_ARG), (dict(scale=float("inf")), INVALID_ARG), (dict(scale=float("nan")), INVALID_ARG)])
def test_attn_descriptor(lib, bad, status):
    d, s, c = attn(**bad), seqs(), cache()
    assert _fwd(lib, d, s) == status
    assert lib.lattice_seq_attn_bwd(byref(d), byref(s), P, QS, P, KS, P, KS, P, QS, P, None, P, QS, P, QS, P, KS, P,
                                    KS, P, 1 << 40, None) == status
    assert lib.lattice_seq_cache_fill(byref(d), byref(s), P, KS, P, KS, None, None, byref(c), None) == status
    assert lib.lattice_seq_step(byref(d), None, 2, P, QS, P, KS, P, KS, P, None, byref(c), P, QS, P, 1 << 40,
                                None) == status
    assert lib.lattice_seq_attn_bwd_workspace(byref(d), byref(s)) == 0
    assert lib.lattice_seq_step_workspace(byref(d), 2) == 0


def test_attn_tensors(lib):
    assert _fwd(lib, attn(), seqs(span=None)) == INVALID_ARG
    for name in ("q", "k", "v", "o"):
        assert _fwd(lib, attn(), seqs(), **{name: None}) == INVALID_ARG
        assert _fwd(lib, attn(), seqs(), **{name: P + 2}) == INVALID_ARG
        assert _fwd(lib, attn(), seqs(), **{"ld" + name: 64}) == INVALID_ARG
    assert _fwd(lib, attn(), seqs(rows=0)) == OK
    assert _fwd(lib, attn(), seqs(num_seqs=0)) == OK
    assert _fwd(lib, attn(heads=1024, kv_heads=1024), seqs(rows=(1 << 30) - 1), ldq=65536, ldk=65536, ldv=65536,
                ldo=65536) == UNSUPPORTED
    d, s = attn(), seqs()
    need = lib.lattice_seq_attn_bwd_workspace(byref(d), byref(s))
    assert need > 0

    def bwd(lse=P, ws=P, n=need, s=s, go=P, lo=None):
        return lib.lattice_seq_attn_bwd(byref(d), byref(s), P, QS, P, KS, P, KS, P, QS, lse, lo, go, QS, P, QS, P, KS,
                                        P, KS, ws, n, None)
    assert bwd(lo=P + 8) == INVALID_ARG
    assert bwd(lse=None) == INVALID_ARG
    assert bwd(go=None) == INVALID_ARG
    assert bwd(s=seqs(offsets=None)) == INVALID_ARG
    assert bwd(ws=None) == WORKSPACE
    assert bwd(n=need - 1) == WORKSPACE
    assert bwd(ws=P + 4) == INVALID_ARG
    # only sequences that outgrow sinks + window need room for their sinks
    small = lib.lattice_seq_attn_bwd_workspace(byref(attn(window=90, sinks=2)), byref(seqs(max_len=91)))
    assert small < lib.lattice_seq_attn_bwd_workspace(byref(attn(window=80, sinks=2)), byref(seqs(max_len=91)))


@pytest.mark.parametrize("rows,S,kw", [
    (1_000_000, 500_000, dict(heads=2, kv_heads=2, head_dim=64, sinks=64, window=2048)),
    (10_000_000, 500_000, dict(heads=8, kv_heads=8, head_dim=128, sinks=4, window=256)),
    (1 << 20, 1, dict(heads=4, kv_heads=4, head_dim=128, sinks=64, window=1))])
@pytest.mark.parametrize("max_len", [0, 5000])
def test_backward_workspace_goes_by_rows_not_by_sequences(lib, rows, S, kw, max_len):
    """A sequence whose sinks need room of their own has sinks + window rows or
    more, so there are at most rows / (sinks + window) of them: their partial
    sums are at most 2 * 4 * rows * kv_heads * head_dim bytes for one split
    each, and another 4096 splits (of at most 64 sinks) for the whole call."""
    d, s = attn(dtype=A.BF16, **kw), seqs(rows=rows, num_seqs=S, max_len=max_len)
    need = lib.lattice_seq_attn_bwd_workspace(byref(d), byref(s))
    L, D, J = kw["sinks"] + kw["window"], kw["head_dim"], kw["kv_heads"]
    stats = 2 * (4 * rows * kw["heads"] + 256)
    part = 8 * kw["sinks"] * D
    assert 2 * 4 * rows * kw["heads"] < need <= stats + part * (J * (rows // L) + 4096 + 64 * J)


def test_late_rows_of_one_long_history_are_spread_whatever_else_is_in_the_batch(lib):
    """Room for its partial sums: as many as it has when it is alone."""
    d = attn(dtype=A.BF16, heads=8, kv_heads=2, head_dim=64, sinks=16, window=2048)
    alone, batch = seqs(rows=32000, num_seqs=1, max_len=32000), seqs(rows=92000, num_seqs=3001, max_len=32000)
    a, b = (lib.lattice_seq_attn_bwd_workspace(byref(d), byref(s)) - 2 * ((4 * s.rows * 8 + 255) // 256 * 256)
            for s in (alone, batch))
    assert b >= a >= 32 * 2 * 2 * 16 * 64 * 4                # 32 tiles of 1000 rows, 2 key heads


def test_cache_and_step(lib):
    d, c, r = attn(), cache(), rope()

    def step(d=d, r=None, B=2, q=P, k=P, v=P, lens=P, c=c, o=P, ws=P, n=1 << 40):
        return lib.lattice_seq_step(byref(d), byref(r) if r else None, B, q, QS, k, KS, v, KS, lens, None,
                                    byref(c) if c else None, o, QS, ws, n, None)
    for kw in (dict(B=-1), dict(q=None), dict(k=None), dict(v=None), dict(lens=None), dict(c=None), dict(o=None),
               dict(c=cache(k=None)), dict(c=cache(v=P + 4)), dict(c=cache(num_caches=-1)), dict(d=attn(key_mask=P)),
               dict(r=rope(head_dim=32, rotary_dim=32)), dict(r=rope(heads=2)), dict(r=rope(dtype=A.F32)),
               dict(r=rope(theta=-1.0))):
        assert step(**kw) == INVALID_ARG, kw
    assert step(d=attn(window=1 << 30, sinks=1)) == UNSUPPORTED
    assert step(B=1 << 30) == UNSUPPORTED
    assert step(B=0) == OK and step(c=cache(num_caches=0)) == OK
    wide = attn(window=60000)
    need = lib.lattice_seq_step_workspace(byref(wide), 2)
    assert need > 0 and lib.lattice_seq_step_workspace(byref(attn()), 2) == 0
    assert step(d=wide, n=need - 1) == WORKSPACE and step(d=wide, ws=None) == WORKSPACE
    _ = r

    def fill(s=seqs(), k=P, v=P, c=c):
        return lib.lattice_seq_cache_fill(byref(d), byref(s), k, KS, v, KS, None, None, byref(c) if c else None, None)
    assert fill(c=None) == INVALID_ARG and fill(k=None) == INVALID_ARG and fill(v=P + 4) == INVALID_ARG
    assert fill(s=seqs(offsets=None)) == INVALID_ARG
    assert fill(s=seqs(rows=0)) == OK and fill(c=cache(num_caches=0)) == OK


def test_a_cache_takes_no_hidden_events(lib):
    """Neither the fill nor the step: every slot of a ring is seen."""
    d, s, c = attn(key_mask=P), seqs(), cache()
    assert lib.lattice_seq_cache_fill(byref(d), byref(s), P, KS, P, KS, None, None, byref(c), None) == INVALID_ARG
    assert b"key_mask" in lib.lattice_last_error()
    assert lib.lattice_seq_step(byref(d), None, 2, P, QS, P, KS, P, KS, P, None, byref(c), P, QS, P, 1 << 40,
                                None) == INVALID_ARG


def test_binding_checks_before_it_calls():
    x = torch.zeros(4, 2, 64)
    like = 4, 64, torch.float32, -1
    with pytest.raises(ValueError, match="GPU"):
        api.lattice_qk_rope_fwd(None, x, x, positions=torch.zeros(4, dtype=torch.int32))
    with pytest.raises(ValueError, match="int32"):
        api.lattice_seq_plan(torch.zeros(3), 4)
    with pytest.raises(ValueError, match="contiguous"):
        api._heads(torch.zeros(4, 64, 2).transpose(1, 2), like, "q")
    with pytest.raises(ValueError, match="expected"):
        api._heads(x[:3], like, "q")
    with pytest.raises(ValueError, match="expected"):
        api._heads(x.bfloat16(), like, "q")
    with pytest.raises(ValueError, match="not on"):
        api._vec(torch.zeros(4, dtype=torch.int32), torch.int32, 4, "lens", 0)
    with pytest.raises(ValueError, match="heads, head_dim"):
        api.lattice_qk_rope_fwd(None, x[0], x[0])
    assert api._heads(torch.zeros(4, 6, 64)[:, 2:4], like, "k")[1] == 384
    with pytest.raises(ValueError, match="not on GPU"):
        api._heads(x, like[:3] + (0,), "q")
    with pytest.raises(ValueError, match="elements"):
        api._vec(torch.zeros(3, dtype=torch.int32), torch.int32, 4, "lens", 0)
    with pytest.raises(ValueError, match="caches"):
        api._cache(torch.zeros(2, 2, 9, 64), torch.zeros(2, 2, 9, 64), x, 2, 8, 2)


def test_a_stream_of_another_device_is_refused():
    other = SimpleNamespace(device=torch.device("cuda:1"))
    q = torch.zeros(2, 1, 8)
    with pytest.raises(ValueError, match="the stream is on cuda:1"):
        api.lattice_seq_plan(torch.zeros(2, dtype=torch.int32), 0, stream=other)
    with pytest.raises(ValueError, match="the stream is on cuda:1"):
        api.lattice_qk_rope_fwd(None, q, q, positions=torch.zeros(2, dtype=torch.int32), stream=other)
    with pytest.raises(ValueError, match="the stream is on cuda:1"):
        api.lattice_seq_step(q, q, q, torch.zeros(2, dtype=torch.int32), q, q, 1, stream=other)
