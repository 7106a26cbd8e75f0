"""Layer norm, forward and backward, against a plain implementation in 64
bits, at the widths where the kernels change (a wave a row, a workgroup a row,
rows past the registers), with row strides, odd starts and special values.

Tolerances, all from the arithmetic: a result rounded to a type with p bits
of significand is off by at most 2^-p of itself (and half the smallest
subnormal); everything before is fp32 with the longest chain of additions at
most 64 + cols / 1024 + log2 terms long, each off by 2^-24 of the sum of
magnitudes."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

UNIT = {"float32": 2.0 ** -24, "float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}
TINY = {"float32": 2.0 ** -149, "float16": 2.0 ** -24, "bfloat16": 2.0 ** -133}
F32 = 2.0 ** -24


def chain(n):
    return 80 + n / 1024


def make(shape, dtype, rng, pad=0, shift=0, scale=1.0, offset=0.0):
    """A device matrix of `shape` whose rows are `pad` elements apart from each
    other and start `shift` elements into their storage."""
    import torch
    r, c = shape
    buf = torch.full((shift + r * (c + pad) + 8,), float("nan"), dtype=getattr(torch, dtype), device="cuda")
    t = buf[shift:shift + r * (c + pad)].view(r, c + pad)[:, :c]
    t.copy_(torch.from_numpy(rng.standard_normal(shape) * scale + offset).to(t.dtype))
    return t, buf


def vec(n, dtype, rng, scale=0.1, offset=0.0):
    import torch
    return torch.from_numpy(rng.standard_normal(n) * scale + offset).to(getattr(torch, dtype)).cuda()


def f64(t):
    return t.double().cpu().numpy()


def forward_ref(x, w, b, eps):
    mean = x.mean(1)
    var = ((x - mean[:, None]) ** 2).mean(1)
    rstd = 1 / np.sqrt(var + eps)
    return (x - mean[:, None]) * rstd[:, None] * w + b, mean, rstd


def backward_ref(dy, x, w, mean, rstd):
    xhat = (x - mean[:, None]) * rstd[:, None]
    h = dy * w
    dx = rstd[:, None] * (h - h.mean(1, keepdims=True) - xhat * (h * xhat).mean(1, keepdims=True))
    return dx, (dy * xhat).sum(0), dy.sum(0)


def close(got, want, dtype, slack):
    """|got - want| <= half a unit of the type + what fp32 arithmetic loses (slack)."""
    off = np.abs(got - want)
    most = UNIT[dtype] * (np.abs(want) + slack) + TINY[dtype] + slack
    assert np.all(off <= most), (float(np.max(off - most)), np.unravel_index(np.argmax(off - most), off.shape))


CASES = [  # rows, cols, dtype, wdtype, pad, shift
    (1, 1, "float32", "float32", 0, 0),
    (1, 768, "float16", "float16", 0, 0),
    (5, 7, "bfloat16", "float32", 1, 1),
    (3, 64, "float32", "float32", 0, 3),
    (9, 255, "float32", "float32", 5, 1),
    (4, 257, "float16", "float32", 0, 1),
    (1237, 1001, "float32", "float32", 0, 0),
    (70, 1025, "float32", "float32", 3, 0),
    (2100, 513, "float16", "float16", 8, 0),
    (65, 1600, "bfloat16", "bfloat16", 0, 0),
    (33, 2049, "float16", "float32", 0, 0),
    (700, 4095, "bfloat16", "float32", 1, 1),
    (17, 5000, "float32", "float32", 0, 2),
    (11, 8200, "float16", "float16", 0, 0),
    (6, 16390, "bfloat16", "bfloat16", 7, 1),
    (100, 9001, "float32", "float32", 0, 0),
    (2, 70001, "float32", "float32", 0, 0),
]


@pytest.mark.parametrize("rows,cols,dtype,wdtype,pad,shift", CASES)
def test_forward(rows, cols, dtype, wdtype, pad, shift):
    import torch
    from paper_2205_14465_amd import binding as B
    rng = np.random.default_rng(rows * 7 + cols)
    eps = 1e-5
    x, _ = make((rows, cols), dtype, rng, pad, shift, offset=0.3)
    y, ybuf = make((rows, cols), dtype, rng, pad + 2, shift)
    ybuf.fill_(7.0)
    w, b = vec(cols, wdtype, rng, offset=1.0), vec(cols, wdtype, rng)
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    B.bytecomp_layernorm_forward(x, w, b, eps, y, mean, rstd)
    X, W, Bv = f64(x), f64(w), f64(b)
    wy, wm, wr = forward_ref(X, W, Bv, eps)
    n = chain(cols)
    mag = np.abs(X).mean(1)
    em = n * F32 * mag                                   # of the mean
    close(f64(mean), wm, "float32", em)
    er = wr * (n * F32 + (em * wr))                      # of rstd: relative half of var's, generously
    close(f64(rstd), wr, "float32", er)
    xhat = np.abs((X - wm[:, None]) * wr[:, None])
    slack = np.abs(W) * (xhat * (er / wr)[:, None] + (em * wr)[:, None] + 4 * F32 * (xhat + (np.abs(X) * wr[:, None])))
    close(f64(y), wy, dtype, slack + 2 * F32 * np.abs(Bv))
    # nothing outside the rows was written
    outside = ybuf.clone()
    outside[shift:shift + rows * (cols + pad + 2)].view(rows, cols + pad + 2)[:, :cols] = 7.0
    assert torch.equal(outside, torch.full_like(outside, 7.0))


@pytest.mark.parametrize("rows,cols,dtype,wdtype,pad,shift", CASES)
def test_backward(rows, cols, dtype, wdtype, pad, shift):
    import torch
    from paper_2205_14465_amd import binding as B
    rng = np.random.default_rng(rows * 11 + cols)
    x, _ = make((rows, cols), dtype, rng, pad, shift, offset=0.3)
    dy, _ = make((rows, cols), dtype, rng, pad, shift, scale=0.05)
    dx, dxbuf = make((rows, cols), dtype, rng, pad, shift)
    w = vec(cols, wdtype, rng, offset=1.0)
    X, W, DY = f64(x), f64(w), f64(dy)
    _, m, r = forward_ref(X, W, 0.0, 1e-5)
    mean, rstd = torch.from_numpy(m).float().cuda(), torch.from_numpy(r).float().cuda()
    m, r = f64(mean), f64(rstd)
    dw, db = torch.full_like(w, 9.0), torch.full_like(w, 9.0)
    dxbuf.fill_(7.0)
    ws = B.alloc_layernorm_workspace(rows, cols)
    ws.fill_(255)
    B.bytecomp_layernorm_backward(dy, x, w, mean, rstd, dx, dw, db, ws)
    wdx, wdw, wdb = backward_ref(DY, X, W, m, r)
    n = chain(cols)
    xhat = np.abs((X - m[:, None]) * r[:, None])
    h = np.abs(DY * W)
    exh = 3 * F32 * (np.abs(X) + np.abs(m)[:, None]) * r[:, None]
    s2 = (h * xhat).mean(1, keepdims=True)
    es2 = n * F32 * s2 + (h * exh).mean(1, keepdims=True)
    slack = r[:, None] * (6 * F32 * h + n * F32 * h.mean(1, keepdims=True) + xhat * es2 + exh * s2 + 4 * F32 * xhat * s2)
    close(f64(dx), wdx, dtype, slack)
    k = chain(cols) + rows / 64
    close(f64(dw), wdw, wdtype, (np.abs(DY) * (k * F32 * xhat + exh)).sum(0))
    close(f64(db), wdb, wdtype, k * F32 * np.abs(DY).sum(0))
    outside = dxbuf.clone()
    outside[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols] = 7.0
    assert torch.equal(outside, torch.full_like(outside, 7.0))
    # each output alone, and again: the same bits
    again = [torch.empty_like(dx), torch.empty_like(dw), torch.empty_like(db)]
    B.bytecomp_layernorm_backward(dy, x, w, mean, rstd, again[0], None, None, None)
    B.bytecomp_layernorm_backward(dy, x, w, mean, rstd, None, again[1], None, ws)
    B.bytecomp_layernorm_backward(dy, x, w, mean, rstd, None, None, again[2], ws)
    assert torch.equal(again[0], dx) and torch.equal(again[1], dw) and torch.equal(again[2], db)


@pytest.mark.parametrize("cols", [40, 1500, 20000])
def test_gradient_against_differences(cols):
    """dL = <dx, u> + <dw, v> + <db, t> for L = sum(g y), by central differences
    of the forward definition in 64 bits (whose own error, with a step of 1e-4 of
    inputs of order one, is under 1e-6 of the derivative's scale)."""
    import torch
    from paper_2205_14465_amd import binding as B
    rng = np.random.default_rng(cols)
    rows, eps = 6, 1e-5
    X, g = (rng.standard_normal((rows, cols)).astype(np.float32) for _ in range(2))
    W, b = (1 + 0.1 * rng.standard_normal(cols)).astype(np.float32), np.zeros(cols, np.float32)
    x, w = torch.from_numpy(X).cuda(), torch.from_numpy(W).cuda()
    y, dx = torch.empty_like(x), torch.empty_like(x)
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    dw, db = torch.empty_like(w), torch.empty_like(w)
    B.bytecomp_layernorm_forward(x, w, torch.from_numpy(b).cuda(), eps, y, mean, rstd)
    B.bytecomp_layernorm_backward(torch.from_numpy(g).cuda(), x, w, mean, rstd, dx, dw, db,
                                  B.alloc_layernorm_workspace(rows, cols))
    u, v, t = rng.standard_normal((rows, cols)), rng.standard_normal(cols), rng.standard_normal(cols)
    e = 1e-4

    def loss(s):
        return (g * forward_ref(X + s * u, W + s * v, b + s * t, eps)[0]).sum()
    slope = (loss(e) - loss(-e)) / (2 * e)
    got = (f64(dx) * u).sum() + (f64(dw) * v).sum() + (f64(db) * t).sum()
    size = np.sqrt((f64(dx) ** 2).sum() + (f64(dw) ** 2).sum() + (f64(db) ** 2).sum())
    assert abs(got - slope) <= 1e-5 * size * 3


def test_special_rows():
    """A NaN or an infinity stays in its row; a constant row gives the bias."""
    import torch
    from paper_2205_14465_amd import binding as B
    for cols in (100, 3000, 20000):
        x = torch.randn(6, cols, device="cuda")
        x[1, 3], x[2, cols - 1], x[4] = float("nan"), float("inf"), 2.5
        w, b = torch.ones(cols, device="cuda"), torch.randn(cols, device="cuda")
        y, mean, rstd = torch.empty_like(x), torch.empty(6, device="cuda"), torch.empty(6, device="cuda")
        B.bytecomp_layernorm_forward(x, w, b, 1e-5, y, mean, rstd)
        assert y[1].isnan().all() and y[2].isnan().all()
        assert y[[0, 3, 5]].isfinite().all()
        assert torch.equal(y[4], b) and mean[4] == 2.5
        # no weights: 1 and 0; nothing kept; in place
        z = torch.empty_like(x)
        B.bytecomp_layernorm_forward(x, None, None, 1e-5, z)
        assert torch.equal(z[4], torch.zeros(cols, device="cuda"))
        c = x.clone()
        B.bytecomp_layernorm_forward(c, w, b, 1e-5, c)
        assert torch.equal(torch.nan_to_num(c), torch.nan_to_num(y))


def test_empty_and_other_stream():
    import torch
    from paper_2205_14465_amd import binding as B
    e = torch.empty(0, 48, device="cuda")
    w = torch.ones(48, device="cuda")
    none = torch.empty(0, device="cuda")
    B.bytecomp_layernorm_forward(e, w, w, 1e-5, e, none, none)
    dw, db = torch.ones(48, device="cuda"), torch.ones(48, device="cuda")
    B.bytecomp_layernorm_backward(e, e, w, none, none, e, dw, db, None)
    assert not dw.any() and not db.any()
    s = torch.cuda.Stream()
    x = torch.randn(300, 500, device="cuda")
    y, y2 = torch.empty_like(x), torch.empty_like(x)
    B.bytecomp_layernorm_forward(x, None, None, 1e-5, y)
    s.wait_stream(torch.cuda.current_stream())
    B.bytecomp_layernorm_forward(x, None, None, 1e-5, y2, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(y, y2)
