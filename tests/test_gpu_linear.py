"""The linear layer, forward and backward, against a plain implementation in
64 bits, over its paths: few rows, operands read where they lie, operands laid
out first (odd sizes, strides and starts, fp32), and the tile shapes.

Tolerances from the arithmetic: a product of k terms summed in fp32 is off by
at most k 2^-24 of the sum of magnitudes; fp32 operands in three bfloat16
parts add four units of 2^-24 of it; activations in fp32 add 2^-18 of their
argument (the hardware exponential at arguments of up to 30); dz in fp16 and
bfloat16 is rounded once more, half a unit of each term; a result is rounded
once to its type."""
import math

import numpy as np
import pytest

from tests.test_gpu_layernorm import F32, TINY, UNIT, close, f64, make, vec

pytestmark = pytest.mark.gpu
ACT = 2.0 ** -18


def erf(x):
    import torch
    return torch.erf(torch.from_numpy(x)).numpy()


def act_ref(name, z):
    if name == "relu":
        return np.maximum(z, 0)
    if name == "gelu":
        return 0.5 * z * (1 + erf(z / math.sqrt(2)))
    if name == "gelu_tanh":
        return 0.5 * z * (1 + np.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    if name == "silu":
        return z / (1 + np.exp(-z))
    return z


def slope_ref(name, z):
    if name == "relu":
        return (z > 0) * 1.0
    if name == "gelu":
        return 0.5 * (1 + erf(z / math.sqrt(2))) + z * np.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if name == "gelu_tanh":
        c = math.sqrt(2 / math.pi)
        t = np.tanh(c * (z + 0.044715 * z ** 3))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 3 * 0.044715 * z * z)
    if name == "silu":
        p = 1 / (1 + np.exp(-z))
        return p * (1 + z * (1 - p))
    return np.ones_like(z)


CASES = [  # rows, inner, cols, dtype, act, pad, shift, residual, save
    (1, 1, 1, "float32", "none", 0, 0, True, True),
    (1, 768, 1600, "float16", "gelu", 0, 0, False, False),
    (1, 6400, 130, "bfloat16", "none", 0, 0, True, False),
    (7, 33, 19, "bfloat16", "silu", 1, 1, True, True),
    (16, 250, 65, "float32", "gelu", 3, 1, True, True),
    (17, 257, 64, "float16", "relu", 0, 0, False, True),
    (33, 1001, 48, "float32", "silu", 0, 0, True, False),
    (64, 512, 515, "bfloat16", "gelu_tanh", 8, 0, True, True),
    (65, 64, 1, "float16", "none", 0, 0, True, True),
    (65, 1, 70, "float32", "relu", 0, 0, False, True),
    (128, 192, 128, "float16", "gelu_tanh", 0, 0, True, True),
    (129, 200, 257, "bfloat16", "gelu", 0, 0, True, True),
    (257, 64, 129, "float16", "silu", 64, 0, False, False),
    (300, 320, 333, "bfloat16", "relu", 8, 8, True, True),
    (301, 127, 255, "float16", "gelu", 5, 3, True, True),
    (777, 1001, 515, "float32", "relu", 0, 0, True, True),
    (513, 640, 129, "float32", "gelu_tanh", 1, 1, False, True),
    (4100, 256, 2600, "bfloat16", "gelu_tanh", 0, 0, True, True),
    (4100, 72, 2563, "float16", "none", 0, 0, True, False),
]


def setup(rows, inner, cols, dtype, pad, shift, seed):
    rng = np.random.default_rng(seed)
    x, _ = make((rows, inner), dtype, rng, pad, shift)
    w, _ = make((cols, inner), dtype, rng, pad, shift, scale=1 / math.sqrt(inner))
    return rng, x, w


@pytest.mark.parametrize("rows,inner,cols,dtype,act,pad,shift,residual,save", CASES)
def test_forward(rows, inner, cols, dtype, act, pad, shift, residual, save):
    import torch
    from paper_2205_14465_amd import binding as B
    rng, x, w = setup(rows, inner, cols, dtype, pad, shift, rows + inner)
    bias = vec(cols, dtype, rng)
    res, _ = make((rows, cols), dtype, rng, pad, shift) if residual else (None, None)
    y, ybuf = make((rows, cols), dtype, rng, pad, shift)
    z = make((rows, cols), dtype, rng, pad, shift)[0] if save else None
    ybuf.fill_(7.0)
    ws = B.alloc_linear_workspace(x, w)
    ws.fill_(255)
    B.bytecomp_linear_forward(x, w, bias, res, act, y, z, ws)
    X, W = f64(x), f64(w)
    wz = X @ W.T + f64(bias)
    ez = (inner + 6) * F32 * (np.abs(X) @ np.abs(W).T + np.abs(f64(bias)))
    if save:
        close(f64(z), wz, dtype, ez)
    R = f64(res) if residual else 0.0
    ey = 1.2 * ez + (ACT * np.abs(wz) if act not in ("none", "relu") else 0) + 2 * F32 * (np.abs(wz) + np.abs(R))
    close(f64(y), act_ref(act, wz) + R, dtype, ey)
    outside = ybuf.clone()
    outside[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols] = 7.0
    assert torch.equal(outside, torch.full_like(outside, 7.0))
    if residual:  # the residual's own place
        B.bytecomp_linear_forward(x, w, bias, res, act, res, None, ws)
        assert torch.equal(res, y)


@pytest.mark.parametrize("rows,inner,cols,dtype,act,pad,shift,residual,save", CASES)
def test_backward(rows, inner, cols, dtype, act, pad, shift, residual, save):
    import torch
    from paper_2205_14465_amd import binding as B
    rng, x, w = setup(rows, inner, cols, dtype, pad, shift, rows + cols)
    dy, _ = make((rows, cols), dtype, rng, pad, shift, scale=0.05)
    z = make((rows, cols), dtype, rng, pad, shift)[0] if act != "none" else None
    ws = B.alloc_linear_workspace(x, w, backward=True)
    ws.fill_(255)
    X, W, DY = f64(x), f64(w), f64(dy)
    dz = DY * (slope_ref(act, f64(z)) if z is not None else 1.0)
    half = UNIT[dtype] if dtype != "float32" else 0.0
    each = half + 6 * F32 + (ACT if act not in ("none", "relu") else 0)
    A = np.abs(dz) + (ACT + F32) * np.abs(DY)   # a slope near zero is off by units of one
    # gradients in the tensors' type, then dw and dbias in fp32
    for gd in {dtype, "float32"}:
        dx, dxbuf = make((rows, inner), dtype, rng, pad, shift)
        dw, dwbuf = make((cols, inner), gd, rng, pad, shift)
        db = torch.full((cols,), 9.0, dtype=getattr(torch, gd), device="cuda")
        dxbuf.fill_(7.0)
        dwbuf.fill_(7.0)
        B.bytecomp_linear_backward(dy, z, x, w, act, dx, dw, db, ws)
        tiny = TINY[dtype]
        close(f64(dx), dz @ W, dtype, (A * (each + cols * F32) + tiny) @ np.abs(W) + F32 * np.abs(DY) @ np.abs(W))
        close(f64(dw), dz.T @ X, gd, (A * (each + rows * F32) + tiny).T @ np.abs(X) + F32 * np.abs(DY).T @ np.abs(X))
        close(f64(db), dz.sum(0), gd, (A * (each - half + rows * F32) + F32 * np.abs(DY)).sum(0))
        for buf, r in ((dxbuf, rows), (dwbuf, cols)):
            outside = buf.clone()
            outside[shift:shift + r * (inner + pad)].view(r, inner + pad)[:, :inner] = 7.0
            assert torch.equal(outside, torch.full_like(outside, 7.0))
    one = torch.empty_like(dw), torch.empty_like(dx), torch.empty_like(db)
    B.bytecomp_linear_backward(dy, z, x, w, act, None, one[0], None, ws)
    B.bytecomp_linear_backward(dy, z, x, w, act, one[1], None, None, ws)
    B.bytecomp_linear_backward(dy, z, x, w, act, None, None, one[2], ws)
    assert torch.equal(one[0], dw) and torch.equal(one[1], dx) and torch.equal(one[2], db)


@pytest.mark.parametrize("act", ["none", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("rows", [12, 130])
def test_gradient_against_differences(rows, act):
    """dL along a direction for L = sum(g y), by central differences of the
    definition in 64 bits with a step of 1e-4 (their own error under 1e-6 of
    the derivative's scale), against the fp32 gradients."""
    import torch
    from paper_2205_14465_amd import binding as B
    rng = np.random.default_rng(rows)
    inner, cols = 70, 90
    X, g = rng.standard_normal((rows, inner)).astype(np.float32), rng.standard_normal((rows, cols)).astype(np.float32)
    W, b = (rng.standard_normal((cols, inner)) / 8).astype(np.float32), rng.standard_normal(cols).astype(np.float32)
    x, w, gy = (torch.from_numpy(v).cuda() for v in (X, W, g))
    y, z = torch.empty_like(gy), torch.empty_like(gy)
    dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty(cols, device="cuda")
    B.bytecomp_linear_forward(x, w, torch.from_numpy(b).cuda(), None, act, y, z, B.alloc_linear_workspace(x, w))
    B.bytecomp_linear_backward(gy, z, x, w, act, dx, dw, db, B.alloc_linear_workspace(x, w, backward=True))
    u, v, t = rng.standard_normal(X.shape), rng.standard_normal(W.shape), rng.standard_normal(cols)
    e = 1e-4

    def loss(s):
        return (g * act_ref(act, (X + s * u) @ (W + s * v).T + b + s * t)).sum()
    slope = (loss(e) - loss(-e)) / (2 * e)
    got = (f64(dx) * u).sum() + (f64(dw) * v).sum() + (f64(db) * t).sum()
    size = math.sqrt(sum((f64(d) ** 2).sum() for d in (dx, dw, db)))
    assert abs(got - slope) <= 1e-4 * size


def test_empty_special_and_other_stream():
    import torch
    from paper_2205_14465_amd import binding as B
    dev = "cuda"
    # no rows: dw and dbias are zero; no inner axis: the bias's activation
    x, w = torch.empty(0, 40, device=dev), torch.randn(30, 40, device=dev)
    dw, db = torch.ones_like(w), torch.ones(30, device=dev)
    e = torch.empty(0, 30, device=dev)
    B.bytecomp_linear_backward(e, None, x, w, "none", torch.empty_like(x), dw, db,
                               B.alloc_linear_workspace(x, w, backward=True))
    assert not dw.any() and not db.any()
    for rows in (5, 100):
        x, w, b = torch.empty(rows, 0, device=dev), torch.empty(30, 0, device=dev), torch.randn(30, device=dev)
        y = torch.empty(rows, 30, device=dev)
        B.bytecomp_linear_forward(x, w, b, None, "relu", y, None, B.alloc_linear_workspace(x, w))
        assert torch.equal(y, b.clamp(min=0).expand(rows, 30))
    # NaN stays in its row, also through relu
    for rows in (3, 200):
        x, w = torch.randn(rows, 64, device=dev, dtype=torch.float16), torch.randn(96, 64, device=dev).half()
        x[1, 5] = float("nan")
        y = torch.empty(rows, 96, device=dev, dtype=torch.float16)
        B.bytecomp_linear_forward(x, w, None, None, "relu", y, None, None)
        assert y[1].isnan().all() and y[0].isfinite().all() and y[2:].isfinite().all()
        s, y2 = torch.cuda.Stream(), torch.empty_like(y)
        s.wait_stream(torch.cuda.current_stream())
        B.bytecomp_linear_forward(x, w, None, None, "relu", y2, None, None, stream=s)
        torch.cuda.current_stream().wait_stream(s)
        assert torch.equal(torch.nan_to_num(y), torch.nan_to_num(y2))


def test_wrong_tensors_raise():
    import torch
    from paper_2205_14465_amd import binding as B
    x, w = torch.randn(70, 64, device="cuda"), torch.randn(32, 64, device="cuda")
    y = torch.empty(70, 32, device="cuda")
    ws = B.alloc_linear_workspace(x, w)
    for bad in (lambda: B.bytecomp_linear_forward(x, w.half(), None, None, "none", y, None, ws),
                lambda: B.bytecomp_linear_forward(x, w[:, :60], None, None, "none", y, None, ws),
                lambda: B.bytecomp_linear_forward(x.t().contiguous().t(), w, None, None, "none", y, None, ws),
                lambda: B.bytecomp_linear_forward(x, w, None, None, "swish", y, None, ws),
                lambda: B.bytecomp_linear_forward(x, w, torch.zeros(31, device="cuda"), None, "none", y, None, ws),
                lambda: B.bytecomp_linear_forward(x, w.cpu(), None, None, "none", y, None, ws)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(B.BytecompError) as err:
        B.bytecomp_linear_forward(x, w, None, None, "none", y, None, None)
    assert err.value.code == -7


@pytest.mark.parametrize("rows,inner,cols", [(1, 768, 1600), (300, 700, 90), (1024, 768, 768), (65, 1745, 3585)])
@pytest.mark.parametrize("dtype", ["float16", "float32"])
def test_gradients_do_not_depend_on_the_others(rows, inner, cols, dtype):
    """dx is the same bits with dw in either type, and without dw."""
    import torch
    from paper_2205_14465_amd import binding as B
    rng, x, w = setup(rows, inner, cols, dtype, 0, 0, 5)
    dy, _ = make((rows, cols), dtype, rng, 0, 0, scale=0.05)
    ws = B.alloc_linear_workspace(x, w, backward=True)
    got = []
    for gd in (None, dtype, "float32"):
        dx = torch.empty_like(x)
        dw = None if gd is None else torch.empty_like(w, dtype=getattr(torch, gd))
        B.bytecomp_linear_backward(dy, None, x, w, "none", dx, dw, None, ws)
        got.append(dx)
    assert torch.equal(got[0], got[1]) and torch.equal(got[0], got[2])


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("rows", [1, 2, 3, 4])
@pytest.mark.parametrize("inner", [1, 7, 8, 511, 512, 520, 1600, 2047, 2049, 8200])
def test_tokens(rows, inner, dtype):
    """A few tokens: rows of the weight that end anywhere in a wave's pieces."""
    import torch
    from paper_2205_14465_amd import binding as B
    rng, x, w = setup(rows, inner, 37, dtype, 0, 0, inner)
    y = torch.empty(rows, 37, dtype=x.dtype, device="cuda")
    B.bytecomp_linear_forward(x, w, None, None, "none", y, None, None)
    X, W = f64(x), f64(w)
    close(f64(y), X @ W.T, dtype, (inner + 6) * F32 * (np.abs(X) @ np.abs(W).T))
