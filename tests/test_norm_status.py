"""Refusals of dropout, the residual norm and the 8-bit caches: statuses of the
C ABI on a machine without a GPU (raised before anything is enqueued; the
pointers are placeholders), and the workspace queries."""
import ctypes
import subprocess
from ctypes import byref

import pytest
import torch

from paper_2512_09200_amd import _abi as A
from paper_2512_09200_amd import api
from test_seq_status import attn, rope, seqs

OK, INVALID_ARG, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
P = 0x10000             # placeholder device pointer, never dereferenced here
BF16, F32 = A.BF16, A.F32

pytestmark = pytest.mark.skipif(torch.cuda.device_count() > 0, reason="placeholder pointers must never reach a GPU")


@pytest.fixture(scope="module")
def lib():
    return A.load()


def drop(p=0.5, rng=P, site=0):
    return A.lattice_dropout_desc(p, rng, site)


def norm(dtype=BF16, cols=64, eps=1e-6, gain=None, dropout=None):
    d = A.lattice_add_rmsnorm_desc(dtype, cols, eps, gain, ctypes.pointer(dropout) if dropout is not None else None)
    return d


def test_dropout(lib):
    def f(d=drop(), dt=BF16, rows=5, cols=8, x=P, xs=8, out=P, os=8):
        return lib.lattice_dropout(byref(d) if d is not None else None, dt, rows, cols, x, xs, out, os, None)
    assert f(None) == INVALID_ARG
    for p in (-0.1, 1.0, 1.5, float("nan"), float("inf"), 65535.5 / 65536):
        assert f(drop(p)) == INVALID_ARG, p
    assert f(drop(rng=None)) == INVALID_ARG
    assert f(drop(rng=P + 4)) == INVALID_ARG
    assert f(dt=7) == INVALID_ARG
    assert f(rows=-1) == INVALID_ARG and f(cols=-1) == INVALID_ARG
    assert f(rows=1 << 30) == UNSUPPORTED
    assert f(cols=1 << 30, xs=1 << 30, os=1 << 30) == UNSUPPORTED
    assert f(rows=1 << 29, cols=1024, xs=1024, os=1024) == UNSUPPORTED
    assert f(x=None) == INVALID_ARG and f(out=None) == INVALID_ARG
    assert f(x=P + 1) == INVALID_ARG and f(dt=F32, x=P + 2) == INVALID_ARG
    assert f(xs=7) == INVALID_ARG and f(os=7) == INVALID_ARG
    assert f(xs=16, os=24) == INVALID_ARG                                  # in place, other rows
    # nothing to do: no pointer is looked at
    assert f(rows=0, x=None, out=None) == OK and f(cols=0, x=None, out=None) == OK


def test_norm_forward(lib):
    def f(d, rows=5, x=P, xs=64, r=None, rs=0, h=None, hs=0, y=P + 4096, ys=64, q=None, ldq=0, sc=None):
        return lib.lattice_add_rmsnorm_fwd(byref(d) if d is not None else None, rows, x, xs, r, rs, h, hs, y, ys, q, ldq,
                                           sc, None)
    assert f(None) == INVALID_ARG
    for bad in (norm(dtype=9), norm(cols=0), norm(cols=-3), norm(eps=-1.0), norm(eps=float("nan")),
                norm(dropout=drop(1.0)), norm(dropout=drop(rng=None))):
        assert f(bad) == INVALID_ARG
    assert f(norm(cols=16385), xs=16385, ys=16385) == UNSUPPORTED
    assert f(norm(), rows=1 << 30) == UNSUPPORTED
    assert f(norm(), rows=-1) == INVALID_ARG
    assert f(norm(), x=None) == INVALID_ARG and f(norm(), xs=63) == INVALID_ARG and f(norm(), x=P + 1) == INVALID_ARG
    assert f(norm(), r=P, rs=63) == INVALID_ARG and f(norm(), h=P, hs=63) == INVALID_ARG and f(norm(), ys=63) == INVALID_ARG
    assert f(norm(dtype=F32), y=P + 2) == INVALID_ARG
    assert f(norm(), y=None) == INVALID_ARG
    assert f(norm(), h=P, hs=64, y=P) == INVALID_ARG
    assert f(norm(), h=P, hs=72) == INVALID_ARG and f(norm(), y=P, ys=72) == INVALID_ARG       # in place, other rows
    assert f(norm(), r=P + 8192, rs=64, h=P + 8192, hs=72) == INVALID_ARG
    assert f(norm(), r=P + 8192, rs=64, y=P + 8192, ys=72) == INVALID_ARG
    q = dict(y=None, q=P, ldq=64, sc=P)
    assert f(norm(), **{**q, "sc": None}) == INVALID_ARG
    assert f(norm(), **{**q, "ldq": 48}) == INVALID_ARG and f(norm(), **{**q, "ldq": 72}) == INVALID_ARG
    assert f(norm(), **{**q, "q": P + 8}) == INVALID_ARG
    assert f(norm(), rows=0, x=None, y=None) == OK


def test_norm_backward(lib):
    def f(d, rows=5, h=P, hs=64, dy=P, dys=64, dh=None, dhs=0, dr=P, drs=64, dx=None, dxs=0, dg=None, ws=None, wsb=0):
        return lib.lattice_add_rmsnorm_bwd(byref(d) if d is not None else None, rows, h, hs, dy, dys, dh, dhs, dr, drs,
                                           dx, dxs, dg, ws, wsb, None)
    assert f(None) == INVALID_ARG
    assert f(norm(), h=None) == INVALID_ARG and f(norm(), dy=None) == INVALID_ARG
    assert f(norm(), hs=63) == INVALID_ARG and f(norm(), dys=63) == INVALID_ARG and f(norm(), dh=P, dhs=63) == INVALID_ARG
    assert f(norm(), drs=63) == INVALID_ARG and f(norm(), dx=P + 4096, dxs=63) == INVALID_ARG
    assert f(norm(), dx=P, dxs=64) == INVALID_ARG                          # the same memory as d_residual
    for at in (dict(h=P + 64), dict(dy=P + 64), dict(dh=P + 64, dhs=64)):  # in place, other rows
        assert f(norm(), **at, dr=P + 64, drs=72) == INVALID_ARG and f(norm(), **at, dx=P + 64, dxs=72) == INVALID_ARG
    assert f(norm(cols=16385), hs=16385, dys=16385, drs=16385) == UNSUPPORTED
    w = lib.lattice_add_rmsnorm_bwd_workspace
    need = w(byref(norm()), 5)
    assert need > 0 and w(None, 5) == 0 and w(byref(norm()), -1) == 0 and w(byref(norm(cols=0)), 5) == 0
    assert w(byref(norm()), 0) == 0
    assert f(norm(), dg=P) == WORKSPACE and f(norm(), dg=P, ws=P, wsb=need - 1) == WORKSPACE
    assert f(norm(), dg=P, ws=P + 4, wsb=need) == INVALID_ARG
    # the workspace stops growing with the rows
    assert w(byref(norm()), 1 << 29) == w(byref(norm()), 1 << 28) <= 4 << 20


def cache8(k=P, v=P, ks=P, vs=P, n=4):
    return A.lattice_seq_cache8(k, v, ks, vs, n)


def test_cache8_fill(lib):
    def f(d=attn(), s=seqs(), k=P, kst=128, v=P, vst=128, c=cache8()):
        return lib.lattice_seq_cache8_fill(byref(d) if d is not None else None, byref(s) if s is not None else None, k, kst,
                                           v, vst, None, None, byref(c) if c is not None else None, None)
    assert f(None) == INVALID_ARG and f(s=None) == INVALID_ARG and f(c=None) == INVALID_ARG
    assert f(attn(key_mask=P)) == INVALID_ARG
    assert f(attn(head_dim=65)) == UNSUPPORTED and f(attn(head_dim=136)) == UNSUPPORTED
    assert f(attn(window=1 << 30, sinks=1)) == UNSUPPORTED
    for c in (cache8(k=None), cache8(v=None), cache8(ks=None), cache8(vs=None), cache8(k=P + 8), cache8(v=P + 8),
              cache8(ks=P + 2), cache8(vs=P + 2), cache8(n=-1)):
        assert f(c=c) == INVALID_ARG
    assert f(s=seqs(offsets=None)) == INVALID_ARG
    assert f(k=None) == INVALID_ARG and f(kst=120) == INVALID_ARG and f(v=P + 2) == INVALID_ARG and f(vst=132) == INVALID_ARG
    assert f(s=seqs(rows=0)) == OK and f(s=seqs(num_seqs=0)) == OK and f(c=cache8(k=None, v=None, ks=None, vs=None, n=0)) == OK


def test_step8(lib):
    def f(d=attn(), r=rope(), batch=2, q=P, qs=256, k=P, ks=128, v=P, vs=128, lens=P, c=cache8(), out=P, os=256, ws=P,
          wsb=1 << 30):
        return lib.lattice_seq_step8(byref(d) if d is not None else None, byref(r) if r is not None else None, batch, q, qs,
                                     k, ks, v, vs, lens, None, byref(c) if c is not None else None, out, os, ws, wsb, None)
    assert f(None) == INVALID_ARG and f(c=None) == INVALID_ARG and f(batch=-1) == INVALID_ARG
    assert f(attn(key_mask=P)) == INVALID_ARG
    assert f(r=rope(heads=8)) == INVALID_ARG and f(r=rope(dtype=F32)) == INVALID_ARG
    for c in (cache8(k=None), cache8(v=None), cache8(ks=None), cache8(vs=None), cache8(k=P + 8), cache8(vs=P + 1), cache8(n=-1)):
        assert f(c=c) == INVALID_ARG
    assert f(lens=None) == INVALID_ARG
    assert f(q=None) == INVALID_ARG and f(out=None) == INVALID_ARG and f(qs=248) == INVALID_ARG and f(k=P + 8) == INVALID_ARG
    assert f(batch=1 << 24) == UNSUPPORTED
    big = attn(window=100000)
    need = lib.lattice_seq_step8_workspace(byref(big), 2)
    assert need > 0 and f(big, wsb=need - 1) == WORKSPACE and f(big, ws=None, wsb=0) == WORKSPACE
    assert f(big, ws=P + 2) == INVALID_ARG
    assert lib.lattice_seq_step8_workspace(byref(attn()), 2) == 0
    assert lib.lattice_seq_step8_workspace(None, 2) == 0 and lib.lattice_seq_step8_workspace(byref(big), 0) == 0
    assert f(batch=0, lens=None) == OK and f(c=cache8(k=None, v=None, ks=None, vs=None, n=0)) == OK


def test_binding_refuses_cpu_tensors_and_wrong_caches():
    x = torch.randn(4, 16)
    with pytest.raises(ValueError):
        api.lattice_dropout(x, 0.5, torch.zeros(2, dtype=torch.int64))
    with pytest.raises(ValueError):
        api.lattice_add_rmsnorm_fwd(x)
    k = torch.zeros(4, 2, 24, dtype=torch.bfloat16)
    good = [torch.zeros(3, 2, 20, 32, dtype=torch.uint8), torch.zeros(3, 2, 20, 32, dtype=torch.uint8),
            torch.zeros(3, 2, 2), torch.zeros(3, 2, 2)]
    api._cache8(good, k, 2, 18, 2)
    for i, bad in ((0, good[0][..., :24]), (1, good[1].view(torch.int8)), (2, torch.zeros(3, 2, 3)),
                   (3, torch.zeros(3, 2, 2, dtype=torch.float64)), (0, good[0].transpose(0, 1))):
        with pytest.raises(ValueError):
            api._cache8([bad if j == i else t for j, t in enumerate(good)], k, 2, 18, 2)


def test_divisions_by_a_product(tmp_path):
    """FastDiv gives the quotient for every kind of divisor, at the edges of
    each multiple."""
    import os
    csrc = os.path.join(os.path.dirname(A.__file__), "csrc", "norm.h")
    text = open(csrc).read()
    cls = text[text.index("struct FastDiv {"):]
    cls = cls[:cls.index("};") + 2].replace("__host__ __device__", "")
    src = tmp_path / "div.cpp"
    src.write_text("""#include <cstdint>
#include <cstdio>
""" + cls + """
int main() {
  const uint32_t ds[] = {1, 2, 3, 5, 7, 8, 9, 125, 126, 127, 128, 129, 1000, 65535, 65536, 65537, 8750, 134217727,
                         134217728, 1073741823, 1073741825, 2147483647};
  for (uint32_t d : ds) {
    const FastDiv f(d);
    for (uint64_t q = 0; q * d < (1ull << 31); q += 1 + (2147483647ull / d) / 5000)
      for (int64_t e = -2; e <= 2; ++e) {
        const int64_t n = (int64_t)(q * d) + e;
        if (n >= 0 && n < (1ll << 31) && f((uint32_t)n) != (uint32_t)n / d) { printf("%u / %u\\n", (uint32_t)n, d); return 1; }
      }
  }
  return 0;
}
""")
    subprocess.run(["g++", "-O1", "-o", str(tmp_path / "div"), str(src)], check=True)
    r = subprocess.run([str(tmp_path / "div")], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout


def test_a_buffer_that_nothing_would_be_written_to():
    x = torch.zeros(2, 16)
    with pytest.raises(ValueError, match="out='fp8' writes none"):
        api.lattice_add_rmsnorm_fwd(x, out="fp8", y=torch.zeros(2, 16))


@pytest.mark.parametrize("site", [-1, 1 << 32, -(1 << 32)])
def test_sites_that_would_be_another_one(site):
    with pytest.raises(ValueError, match="site"):
        api._drop_desc((0.5, None, site), 0)
    assert api._drop_desc((0.5, None, (1 << 32) - 1), 0).site == (1 << 32) - 1


def test_the_memory_of_a_call_on_another_stream():
    """What a call on another stream keeps until that stream has passed it: the
    generator's state too, in a tuple or a list."""
    rng, x = torch.zeros(2, dtype=torch.int64), torch.zeros(2, 16)
    for drop in ((0.5, rng, 1), [0.5, rng, 1]):
        assert [t.data_ptr() for t in api._memory((x, None, drop, 0.1))] == [x.data_ptr(), rng.data_ptr()]
