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
