"""Layer norm of more rows than one launch takes: the same bits as calls on
parts of the rows, at both ends and where a launch ends, and the column sums
against 64 bits."""
import pytest

pytestmark = pytest.mark.gpu
ROWS, COLS = (1 << 26) + 5, 8


def test_layer_norm():
    import torch
    from paper_2205_14465_amd import binding as B
    g = torch.Generator(device="cuda").manual_seed(1)
    x, dy = (torch.randn(ROWS, COLS, generator=g, device="cuda", dtype=torch.float16) for _ in range(2))
    w, b = (torch.randn(COLS, generator=g, device="cuda") for _ in range(2))
    y, dx = torch.zeros_like(x), torch.zeros_like(x)
    mean, rstd = (torch.zeros(ROWS, device="cuda") for _ in range(2))
    dw, db = torch.zeros_like(w), torch.zeros_like(w)
    B.bytecomp_layernorm_forward(x, w, b, 1e-5, y, mean, rstd)
    B.bytecomp_layernorm_backward(dy, x, w, mean, rstd, dx, dw, db, B.alloc_layernorm_workspace(ROWS, COLS))
    for lo in (0, (1 << 24) - 3, (1 << 25) - 3, 3 * (1 << 24) - 3, (1 << 26) - 3, ROWS - 5):
        p = slice(lo, min(lo + 70, ROWS))
        y2, dx2, m2, r2 = torch.empty_like(y[p]), torch.empty_like(y[p]), torch.empty_like(mean[p]), torch.empty_like(mean[p])
        B.bytecomp_layernorm_forward(x[p], w, b, 1e-5, y2, m2, r2)
        B.bytecomp_layernorm_backward(dy[p], x[p], w, m2, r2, dx2, None, None, None)
        assert torch.equal(y[p], y2) and torch.equal(mean[p], m2) and torch.equal(rstd[p], r2) and torch.equal(dx[p], dx2)
    assert (rstd > 0).all() and y.isfinite().all()
    # Each of 512 x 4 waves adds rows / 2048 terms a column, then at most 80 sums
    # more: each off by 2^-24 of the sum of magnitudes.
    want_w, want_b, size_w, size_b = (torch.zeros(COLS, dtype=torch.float64, device="cuda") for _ in range(4))
    for lo in range(0, ROWS, 1 << 24):
        p = slice(lo, lo + (1 << 24))
        d = dy[p].double()
        xh = (x[p].double() - mean[p].double()[:, None]) * rstd[p].double()[:, None]
        want_w += (d * xh).sum(0)
        want_b += d.sum(0)
        size_w += (d * xh).abs().sum(0)
        size_b += d.abs().sum(0)
    k = (ROWS / 2048 + 80 + 4) * 2.0 ** -24
    assert ((dw - want_w).abs() <= k * size_w).all() and ((db - want_b).abs() <= k * size_b).all()
