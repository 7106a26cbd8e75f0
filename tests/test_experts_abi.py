"""CPU-only checks of the entry points of a block of experts and of the
gradients' norm and clipping: workspace sizes, and refusals with the documented
status before the device is touched."""
import ctypes

import pytest

from paper_2205_14465_amd import binding as B

P = ctypes.c_void_p
X, Y, W, WS, O, S = P(0x10000), P(0x20000), P(0x30000), P(0x40000), P(0x50000), P(0x60000)
ODD = P(0x10002)


def test_route_refusals():
    L = B.lib()

    def fwd(dtype=0, rows=4, experts=8, k=2, x=X, ld=8, w=W, e=Y, slot=S, src=S, off=O, ws=None, n=0):
        return L.bytecomp_route_forward(dtype, rows, experts, k, x, ld, 1, w, e, slot, src, off, ws, n, None)

    assert fwd(dtype=3) == -3
    for experts, k in ((0, 1), (1025, 1), (8, 0), (8, 9), (1024, 33)):
        assert fwd(experts=experts, k=k, ld=2000) == -6
    assert fwd(rows=1 << 29) == -5 and fwd(rows=1 << 28, k=8) == -5 and fwd(ld=7) == -5
    for name in ("x", "w", "e", "slot", "src", "off"):
        assert fwd(**{name: None}) == -1 and fwd(**{name: ODD}) == -9, name
    assert fwd(rows=0, off=None) == -1
    assert B.bytecomp_route_workspace_size(64, 8, 2) == 0
    need = B.bytecomp_route_workspace_size(65, 8, 2)
    assert need > 0 and fwd(rows=65) == -7 and fwd(rows=65, ws=WS, n=need - 1) == -7
    # at most 256 blocks of rows while the masks of the experts fit
    assert B.bytecomp_route_workspace_size(1 << 18, 64, 2) <= 257 * 64 * 4
    with pytest.raises(B.BytecompError) as e:
        B.bytecomp_route_workspace_size(1, 4, 5)
    assert e.value.code == -6

    def bwd(dtype=0, rows=4, experts=8, k=2, x=X, ld=8, norm=0, w=W, e=Y, dw=W, dx=Y, ldd=8):
        return L.bytecomp_route_backward(dtype, rows, experts, k, x, ld, norm, w, e, dw, dx, ldd, None)

    assert bwd(dtype=-1) == -3 and bwd(k=9) == -6 and bwd(rows=1 << 29) == -5
    assert bwd(ld=7) == -5 and bwd(ldd=7) == -5
    for name in ("x", "w", "e", "dw", "dx"):
        assert bwd(**{name: None}) == -1 and bwd(**{name: ODD}) == -9, name
    assert bwd(rows=0) == 0


def test_combine_refusals():
    L = B.lib()

    def fwd(dtype=1, rows=4, cols=8, k=2, slots=8, y=X, ldy=8, slot=S, w=W, r=None, ldr=0, out=Y, ldo=8):
        return L.bytecomp_combine_forward(dtype, rows, cols, k, slots, y, ldy, slot, w, r, ldr, out, ldo, None)

    assert fwd(dtype=7) == -3 and fwd(k=0) == -6 and fwd(k=33) == -6
    assert fwd(rows=1 << 29) == -5 and fwd(rows=1 << 27, k=16) == -5 and fwd(slots=1 << 31) == -5
    assert fwd(cols=1 << 24, ldy=1 << 24, ldo=1 << 24) == -5
    assert fwd(ldy=7) == -5 and fwd(ldo=7) == -5 and fwd(r=X, ldr=7) == -5
    for name in ("y", "slot", "out"):
        assert fwd(**{name: None}) == -1
    assert fwd(y=P(0x10001)) == -9 and fwd(slot=ODD) == -9 and fwd(w=ODD) == -9
    assert fwd(rows=0) == 0 and fwd(cols=0) == 0

    def bwd(dtype=1, rows=4, cols=8, k=2, slots=8, d=X, ldd=8, y=X, ldy=8, slot=S, w=W, dy=Y, lddy=8, dw=W):
        return L.bytecomp_combine_backward(dtype, rows, cols, k, slots, d, ldd, y, ldy, slot, w, dy, lddy, dw, None)

    assert bwd(dtype=7) == -3 and bwd(k=33) == -6 and bwd(slots=1 << 31) == -5
    for name in ("d", "y", "slot"):
        assert bwd(**{name: None}) == -1
    assert bwd(ldd=7) == -5 and bwd(ldy=7) == -5 and bwd(lddy=7) == -5 and bwd(dw=ODD) == -9
    assert bwd(dy=None, dw=None) == 0 and bwd(rows=0) == 0


def test_grouped_linear_refusals():
    L = B.lib()

    def fwd(dtype=1, rows=70, inner=64, cols=32, experts=3, off=O, x=X, ldx=64, src=None, x_rows=0, w=W, ldw=64,
            each=2048, b=None, ldb=32, act=0, y=Y, ldy=32, z=None, ldz=0, ws=None, n=0):
        return L.bytecomp_grouped_linear_forward(dtype, rows, inner, cols, experts, off, x, ldx, src, x_rows, w, ldw, each,
                                                 b, ldb, act, y, ldy, z, ldz, ws, n, None)

    assert fwd(dtype=3) == -3 and fwd(act=5) == -2 and fwd(experts=0) == -6 and fwd(experts=1025) == -6
    assert fwd(rows=1 << 22) == -5 and fwd(inner=1 << 20) == -5 and fwd(cols=1 << 20) == -5
    assert fwd(src=S, x_rows=1 << 31) == -5
    assert fwd(rows=1 << 20, cols=1 << 15) == -5 and fwd(inner=1 << 18, cols=1 << 18) == -5
    assert fwd(ldx=63) == -5 and fwd(ldw=63) == -5 and fwd(ldy=31) == -5 and fwd(each=2047) == -5
    assert fwd(b=X, ldb=31) == -5 and fwd(z=Y, ldz=31) == -5
    for name in ("off", "x", "w", "y"):
        assert fwd(**{name: None}) == -1
    assert fwd(x=P(0x10001)) == -9 and fwd(off=ODD) == -9 and fwd(src=ODD, x_rows=5) == -9
    assert fwd(ws=P(0x40008), n=1 << 30) == -9
    assert fwd(rows=0) == 0 and fwd(cols=0) == 0
    assert fwd(ldx=1 << 21) == -5 and fwd(ldw=1 << 21, each=1 << 30) == -5
    # many 16-bit rows of odd sizes are laid out first, fp32 ones that a gather's offsets do not reach
    need = B.bytecomp_grouped_linear_workspace_size(1, 700, 700, 63, 32, 3)
    assert need > 0 and fwd(rows=700, inner=63) == -7 and fwd(rows=700, inner=63, ws=WS, n=need - 257) == -7
    assert fwd(rows=700, inner=60) == -7
    assert fwd(dtype=0, rows=700, src=S, x_rows=1 << 30) == -7
    assert B.bytecomp_grouped_linear_workspace_size(0, 64, 64, 64, 32, 3) == 0
    assert B.bytecomp_grouped_linear_workspace_size(1, 64 + 8 * 3, 9, 63, 32, 3) == 0

    def bwd(dtype=1, gdtype=1, rows=70, off=O, dy=Y, lddy=32, z=Y, ldz=32, act=1, x=X, ldx=64, src=None, w=W, ldw=64,
            each=2048, dx=X, lddx=64, dw=W, lddw=64, each_d=2048, db=W, lddb=32, ws=WS, n=1 << 30):
        return L.bytecomp_grouped_linear_backward(dtype, gdtype, rows, 64, 32, 3, off, dy, lddy, z, ldz, act, x, ldx, src,
                                                  9, w, ldw, each, dx, lddx, dw, lddw, each_d, db, lddb, ws, n, None)

    assert bwd(gdtype=2) == -3 and bwd(dtype=0, gdtype=1) == -3 and bwd(act=9) == -2
    for name in ("off", "dy", "z", "x", "w"):
        assert bwd(**{name: None}) == -1, name
    for name in ("lddy", "ldz", "ldx", "ldw", "lddx", "lddw", "lddb"):
        assert bwd(**{name: 31}) == -5, name
    assert bwd(each=2047) == -5 and bwd(each_d=2047) == -5
    assert bwd(gdtype=0, dw=ODD) == -9
    need = B.bytecomp_grouped_linear_workspace_size(1, 70, 70, 64, 32, 3, True)
    assert bwd(n=need // 8) == -7 and bwd(ws=None) == -7
    assert bwd(dx=None, dw=None, db=None) == 0
    with pytest.raises(B.BytecompError) as e:
        B.bytecomp_grouped_linear_workspace_size(7, 1, 1, 1, 1, 1)
    assert e.value.code == -3


@pytest.mark.parametrize("dtype", [0, 1, 2])
@pytest.mark.parametrize("experts", [1, 3, 64, 1024])
@pytest.mark.parametrize("x_rows,ldx", [(1 << 25, 64), (1 << 10, 1 << 20), ((1 << 31) - 1, 65), (90, 64), (0, 64)])
def test_a_workspace_of_the_size_asked_for_is_enough(x_rows, ldx, experts, dtype):
    """Also where a source reads from more than 2 GB, on either side of the most rows that
    need none; the calls then get as far as the launch, which fails (-8) without a device."""
    import torch
    if torch.cuda.is_available():
        pytest.skip("would launch on addresses that are no memory")
    L = B.lib()
    few = 64 + 8 * experts
    for rows in (1, 64, 65, few - 1, few, few + 1, few + 700):
        for src, x, inner in ((S, X, 64), (S, X, 63), (None, X, 64), (S, ODD, 64), (S, X, 8)):
            if dtype == 0 and x is ODD:
                continue
            for backward in (False, True):
                need = B.bytecomp_grouped_linear_workspace_size(dtype, rows, x_rows if src else rows, inner, 32, experts, backward)
                ws = WS if need else None
                if backward:
                    rc = L.bytecomp_grouped_linear_backward(dtype, dtype, rows, inner, 32, experts, O, Y, 32, Y, 32, 1, x, ldx,
                                                            src, x_rows, W, 64, 2048, X, 64, W, 64, 2048, W, 32, ws, need, None)
                else:
                    rc = L.bytecomp_grouped_linear_forward(dtype, rows, inner, 32, experts, O, x, ldx, src, x_rows, W, 64, 2048,
                                                           None, 32, 0, Y, 32, None, 32, ws, need, None)
                assert rc == -8, (rows, inner, backward, need, rc)


def test_clip_refusals():
    L = B.lib()

    def grads(grad=0x10000, out=0x20000, ld=8, ldo=8, rows=4, cols=8, dtype=0):
        return (B.bc_grad * 1)(B.bc_grad(grad, out, ld, ldo, rows, cols, dtype, 0))

    need = B.bytecomp_grad_norm_workspace_size(1)

    def norm(t=None, T=1, kind=0, out=P(0x30000), ws=WS, n=need, **g):
        return L.bytecomp_grad_norm(grads(**g) if t is None else t, T, kind, out, ws, n, None)

    def clip(t=None, T=1, kind=0, most=1.0, given=None, out=None, factor=None, ws=WS, n=need, **g):
        return L.bytecomp_clip_grads(grads(**g) if t is None else t, T, kind, most, given, out, factor, ws, n, None)

    for call in (norm, clip):
        assert call(T=-1) == -6 and call(T=(1 << 20) + 1) == -6 and call(kind=2) == -2 and call(dtype=3) == -3
        assert call(ws=None) == -7 and call(n=need - 1) == -7 and call(ws=P(0x40008)) == -9
        assert call(ld=7) == -5 and call(rows=1 << 24, cols=1 << 24, ld=1 << 24, ldo=1 << 24) == -5
        assert call(grad=None) == -1 and call(grad=0x10002) == -9
        # a null table
        assert call(t=ctypes.cast(None, ctypes.POINTER(B.bc_grad))) == -1
    assert norm(out=None) == -1 and norm(out=P(0x30004)) == -9
    assert clip(out=P(0x30004)) == -9 and clip(given=P(0x30004)) == -9 and clip(factor=P(0x30002)) == -9
    g = B.bc_grad
    assert clip(ldo=7) == -5 and L.bytecomp_clip_grads((g * 1)(g(0x10000, None, 8, 8, 4, 8, 0, 0)), 1, 0, 1.0, None, None,
                                                       None, WS, need, None) == -1
    for most in (-1.0, float("nan")):
        assert clip(most=most) == -11
    with pytest.raises(B.BytecompError) as e:
        B.bytecomp_grad_norm_workspace_size(-1)
    assert e.value.code == -6


def test_grad_list_of_strided_and_contiguous():
    """Marshalling alone: a gradient and its out may lie differently."""
    import torch

    class Dev(torch.Tensor):
        is_cuda = True

    def dev(t):
        return t.as_subclass(Dev)
    g, wide = dev(torch.zeros(3, 5)), dev(torch.zeros(3, 8))
    a = B._grad_list([g, g, wide[:, :5], dev(torch.zeros(2, 3, 4))], [g, wide[:, :5], g, dev(torch.zeros(2, 3, 4))])
    assert [(x.rows, x.cols, x.ld_grad, x.ld_out) for x in a] == [(1, 15, 15, 15), (3, 5, 5, 8), (3, 5, 8, 5),
                                                                  (1, 24, 24, 24)]
    for bad in ([dev(torch.zeros(4, 5))], [dev(torch.zeros(3, 5, dtype=torch.float16))], [dev(torch.zeros(5, 3)).t()], []):
        with pytest.raises(ValueError):
            B._grad_list([g], bad)
    with pytest.raises(ValueError):
        B._grad_list([dev(torch.zeros(2, 3, 4)).transpose(0, 1)], None)
    with pytest.raises(ValueError):
        B._grad_list([torch.zeros(3)], None)


def test_combination_gradient_wants_what_it_reads():
    """Without y there is nothing to take dweight from, also where no dy tells the slots."""
    import torch

    class Dev(torch.Tensor):
        is_cuda = True

    def dev(*shape, dtype=torch.float32):
        return torch.zeros(*shape, dtype=dtype).as_subclass(Dev)
    class Stream:
        cuda_stream = 0
    dout, slot, weight, y = dev(4, 8), dev(4, 2, dtype=torch.int32), dev(4, 2), dev(8, 8)
    for dy in (None, dev(8, 8)):
        with pytest.raises(ValueError, match="y:"):
            B.CombineGradCall(dout, None, slot, weight, dy, dev(4, 2), Stream)
    for given, dy, dweight in ((None, dev(8, 8), None), (None, None, None), (y, None, dev(4, 2)), (dev(0, 8), None, dev(4, 2))):
        B.CombineGradCall(dout, given, slot, weight, dy, dweight, Stream)
