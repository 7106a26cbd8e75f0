"""fp32 linear layers with infinities, NaN and the largest finite numbers in
their operands, over the paths (few rows, tiles of each size, split products):
what the formulas give, whatever the number of rows.

Tolerance of finite results: tests/test_gpu_linear.py's for a product of k
terms, (k + 6) 2^-24 of the sum of magnitudes."""
import numpy as np
import pytest

from tests.test_gpu_layernorm import F32

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")
LARGEST = 3.4028234663852886e38
TIE = 3.3961775292304e38        # halfway from bfloat16's largest number to the next power of two
SHAPES = [(3, 40, 70), (8, 40, 70), (40, 100, 70), (65, 40, 70), (65, 1745, 400), (777, 1001, 515), (1500, 320, 1700),
          (4096, 800, 2048)]


def product(a, b):
    """a b^T in 64 bits, term by term, and the sums of the terms' magnitudes."""
    a, b = a.astype(np.float64), b.astype(np.float64)
    with np.errstate(invalid="ignore"):
        t = a[:, None, :] * b[None, :, :]
        return t.sum(2), np.abs(t).sum(2)


def same(got, want, size, k):
    got, want = got.astype(np.float64), want.copy()
    with np.errstate(over="ignore"):
        want = np.where(np.abs(want) > LARGEST, np.sign(want) * INF, want)
    odd = ~np.isfinite(want)
    assert np.array_equal(got[odd], want[odd], equal_nan=True)
    off = np.abs(got[~odd] - want[~odd])
    assert np.all(off <= (k + 6) * F32 * size[~odd]), float(np.max(off / size[~odd]))


def operand(rng, rows, cols, rare=()):
    v = np.clip(rng.standard_normal((rows, cols)) * 0.1, -0.4, 0.4)
    v = np.where(np.abs(v) < 1e-3, 1e-3, v).astype(np.float32)
    for (r, c), x in rare:
        if r < rows:
            v[r, c] = x
    return v


# rows of their own: an infinity; two that may cancel; NaN; numbers past
# bfloat16's largest, alone and among others
RARE = [((0, 3), LARGEST), ((1, 5), INF), ((2, 0), INF), ((2, 7), -INF), ((4, 2), -LARGEST), ((5, 9), NAN), ((6, 1), TIE),
        ((7, 8), -INF)]


def device(*arrays):
    import torch
    return [torch.from_numpy(a).cuda() for a in arrays]


@pytest.mark.parametrize("rows,inner,cols", SHAPES)
def test_forward(rows, inner, cols):
    import torch
    from paper_2205_14465_amd import binding as B
    rng = np.random.default_rng(rows + cols)
    X = operand(rng, rows, inner, RARE)
    W = operand(rng, cols, inner, [((4, 6), INF), ((9, 3), 1.5e38), ((11, 4), -LARGEST)])
    x, w = device(X, W)
    y, z = torch.empty(rows, cols, device="cuda"), torch.empty(rows, cols, device="cuda")
    B.bytecomp_linear_forward(x, w, None, None, "relu", y, z, B.alloc_linear_workspace(x, w))
    Z, Y = z.cpu().numpy(), y.cpu().numpy()
    few = min(rows, 8)
    same(Z[:few], *product(X[:few], W), inner)
    same(Z[:, :12], *product(X, W[:12]), inner)
    assert np.array_equal(Y, np.where(Z < 0, np.float32(0), Z), equal_nan=True)
    ordinary = np.ones_like(Z, dtype=bool)
    ordinary[[r for r in (1, 2, 5, 7) if r < rows]] = False
    ordinary[:, 4] = False
    ordinary[0, 9] = False  # LARGEST times 1.5e38
    assert np.isfinite(Z[ordinary]).all()


@pytest.mark.parametrize("rows,inner,cols", SHAPES)
def test_backward(rows, inner, cols):
    import torch
    from paper_2205_14465_amd import binding as B
    rng = np.random.default_rng(rows + cols)
    DY = operand(rng, rows, cols, RARE)
    X, W = operand(rng, rows, inner), operand(rng, cols, inner)
    dy, x, w = device(DY, X, W)
    dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty(cols, device="cuda")
    B.bytecomp_linear_backward(dy, None, x, w, "none", dx, dw, db, B.alloc_linear_workspace(x, w, backward=True))
    DX, DW, DB = dx.cpu().numpy(), dw.cpu().numpy(), db.cpu().numpy()
    few = min(rows, 8)
    same(DX[:few], *product(DY[:few], W.T), cols)
    assert np.isfinite(DX[few:]).all() and np.isfinite(DW[10:]).all()
    same(DW[:10], *product(DY[:, :10].T, X.T), rows)
    with np.errstate(invalid="ignore"):
        same(DB, DY.astype(np.float64).sum(0), np.abs(DY.astype(np.float64)).sum(0), rows)
