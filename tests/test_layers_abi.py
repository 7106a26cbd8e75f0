"""CPU-only checks of the layer and optimizer entry points: workspace sizes,
and refusals with the documented status before the device is touched."""
import ctypes

import pytest

from paper_2205_14465_amd import binding as B

P = ctypes.c_void_p
X, Y, W, WS = P(0x10000), P(0x20000), P(0x30000), P(0x40000)


def test_layernorm_refusals():
    L = B.lib()

    def fwd(dtype=0, wdtype=0, rows=2, cols=8, x=X, ldx=8, w=W, b=W, eps=1e-5, y=Y, ldy=8, mean=None, rstd=None):
        return L.bytecomp_layernorm_forward(dtype, wdtype, rows, cols, x, ldx, w, b, eps, y, ldy, mean, rstd, None)

    assert fwd(dtype=3) == -3 and fwd(wdtype=1) == -3 and fwd(dtype=1, wdtype=2) == -3
    assert fwd(rows=1 << 31) == -5 and fwd(cols=1 << 24, ldx=1 << 24, ldy=1 << 24) == -5
    assert fwd(ldx=7) == -5 and fwd(ldy=7) == -5
    assert fwd(x=None) == -1 and fwd(y=None) == -1
    assert fwd(x=P(0x10002)) == -9 and fwd(dtype=1, y=P(0x20001)) == -9 and fwd(mean=P(0x11)) == -9
    for eps in (-1e-5, float("nan"), float("inf")):
        assert fwd(eps=eps) == -11
    assert fwd(rows=0) == 0 and fwd(cols=0) == 0

    def bwd(dtype=0, wdtype=0, rows=2, cols=8, dy=Y, x=X, mean=W, rstd=W, dx=Y, lddx=8, dw=W, db=W, ws=WS, n=1 << 20):
        return L.bytecomp_layernorm_backward(dtype, wdtype, rows, cols, dy, 8, x, 8, W, mean, rstd, dx, lddx, dw, db,
                                             ws, n, None)

    assert bwd(dtype=9) == -3 and bwd(dtype=2, wdtype=1) == -3
    assert bwd(dy=None) == -1 and bwd(mean=None) == -1 and bwd(rstd=None) == -1
    assert bwd(lddx=7) == -5
    assert bwd(ws=None) == -7 and bwd(n=16) == -7
    assert bwd(dw=P(0x30002)) == -9
    assert bwd(dx=None, dw=None, db=None) == 0
    need = B.bytecomp_layernorm_workspace_size(2, 8)
    assert 0 < need <= 4096 and bwd(n=need - 1) == -7
    assert B.bytecomp_layernorm_workspace_size(0, 8) == 0
    # the sums of the most workgroups, whatever the rows
    assert B.bytecomp_layernorm_workspace_size(1 << 20, 1600) <= 512 * 2 * 1600 * 4
    with pytest.raises(B.BytecompError) as e:
        B.bytecomp_layernorm_workspace_size(1 << 31, 8)
    assert e.value.code == -5


def test_status_text():
    assert B.lib().bytecomp_strerror(-11) not in (b"", b"unknown status")


def test_linear_refusals():
    L = B.lib()

    def fwd(dtype=1, rows=70, inner=64, cols=32, x=X, ldx=64, w=W, ldw=64, b=None, act=0, r=None, ldr=0, y=Y, ldy=32,
            z=None, ldz=0, ws=None, n=0):
        return L.bytecomp_linear_forward(dtype, rows, inner, cols, x, ldx, w, ldw, b, act, r, ldr, y, ldy, z, ldz, ws, n,
                                         None)

    assert fwd(dtype=3) == -3 and fwd(act=5) == -2 and fwd(act=-1) == -2
    assert fwd(rows=1 << 22) == -5 and fwd(inner=1 << 22) == -5 and fwd(cols=1 << 22) == -5
    assert fwd(ldx=63) == -5 and fwd(ldw=63) == -5 and fwd(ldy=31) == -5
    assert fwd(r=Y, ldr=31) == -5 and fwd(z=Y, ldz=31) == -5
    assert fwd(x=None) == -1 and fwd(w=None) == -1 and fwd(y=None) == -1
    assert fwd(x=P(0x10001)) == -9 and fwd(b=P(0x10001)) == -9 and fwd(ws=P(0x40008), n=1 << 30) == -9
    assert fwd(rows=0) == 0 and fwd(cols=0) == 0
    # fp32 and odd sizes are laid out first
    need = B.bytecomp_linear_workspace_size(0, 70, 64, 32)
    assert need > 0 and fwd(dtype=0) == -7 and fwd(dtype=0, ws=WS, n=need - 1) == -7
    assert fwd(inner=63) == -7
    assert B.bytecomp_linear_workspace_size(1, 64, 64, 32) == 0

    def bwd(dtype=1, gdtype=1, dy=Y, lddy=32, z=Y, ldz=32, act=1, x=X, ldx=64, w=W, ldw=64, dx=X, lddx=64, dw=W,
            lddw=64, db=W, ws=WS, n=1 << 30, rows=70):
        return L.bytecomp_linear_backward(dtype, gdtype, rows, 64, 32, dy, lddy, z, ldz, act, x, ldx, w, ldw, dx, lddx,
                                          dw, lddw, db, ws, n, None)

    assert bwd(gdtype=2) == -3 and bwd(dtype=0, gdtype=1) == -3 and bwd(act=9) == -2
    assert bwd(dy=None) == -1 and bwd(z=None) == -1 and bwd(x=None) == -1 and bwd(w=None) == -1
    assert bwd(lddx=63) == -5 and bwd(lddw=63) == -5 and bwd(ldz=31) == -5
    assert bwd(gdtype=0, dw=P(0x30002)) == -9
    need = B.bytecomp_linear_workspace_size(1, 70, 64, 32, True)
    assert bwd(n=need - 1) == -7 and bwd(ws=None) == -7
    assert bwd(dx=None, dw=None, db=None) == 0
    with pytest.raises(B.BytecompError) as e:
        B.bytecomp_linear_workspace_size(7, 1, 1, 1)
    assert e.value.code == -3


def test_orthogonalize_refusals():
    L = B.lib()
    abc = (ctypes.c_double * 3)(*B.MUON_COEFFICIENTS)

    def orth(dtype=0, T=1, steps=5, k=abc, eps=1e-7, ws=WS, n=1 << 30, update=0x10000, out=0x20000, ldu=8, ldo=8, rows=4,
             cols=8, null=False):
        t = (B.bc_update * 1)(B.bc_update(update, out, ldu, ldo, rows, cols))
        return L.bytecomp_orthogonalize(dtype, None if null else t, T, steps, k, eps, ws, n, None)

    assert orth(dtype=5) == -3 and orth(T=-1) == -6 and orth(T=(1 << 20) + 1) == -6
    assert orth(k=None) == -1 and orth(null=True) == -1 and orth(update=None) == -1 and orth(out=None) == -1
    assert orth(steps=0) == -11 and orth(steps=65) == -11 and orth(eps=-1.0) == -11 and orth(eps=float("nan")) == -11
    for bad in ((float("nan"), 0, 0), (1e300, 0, 0), (100.0, 0, 0), (3.0, 3.0, 3.0), (1.0, float("inf"), 0)):
        assert orth(k=(ctypes.c_double * 3)(*bad)) == -11
    assert orth(rows=1 << 22, cols=8) == -5 and orth(ldu=7) == -5 and orth(ldo=7) == -5
    assert orth(update=0x10002) == -9 and orth(ws=P(0x40010)) == -9
    assert orth(T=0) == 0 and orth(rows=0) == 0
    need = B.bytecomp_orthogonalize_workspace_size([(4, 8)])
    assert need > 0 and orth(n=need - 1) == -7 and orth(ws=None) == -7
    assert B.bytecomp_orthogonalize_workspace_size([]) == 0
    assert B.bytecomp_orthogonalize_workspace_size([(1600, 6400)]) <= 12 * 1600 * 6400 + 12 * 1600 * 1600 + (1 << 16)

    def muon(wd=0, gd=0, lr=0.1, mu=0.9, decay=0.0, momentum=0x30000, scale=1.0, ldm=8, n=1 << 30):
        t = (B.bc_param * 1)(B.bc_param(0x10000, 0x20000, momentum, 8, 8, ldm, 4, 8, scale))
        return L.bytecomp_muon_step(wd, gd, t, 1, lr, mu, 1, decay, 5, abc, 1e-7, WS, n, None)

    assert muon(wd=3) == -3 and muon(gd=-1) == -3
    for v in (float("nan"), float("inf")):
        assert muon(lr=v) == -11 and muon(mu=v) == -11 and muon(decay=v) == -11 and muon(scale=v) == -11
    assert muon(momentum=None) == -1 and muon(ldm=7) == -5 and muon(momentum=0x30002) == -9 and muon(n=0) == -7
