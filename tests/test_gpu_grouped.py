"""The linear layer grouped by expert, forward and backward, against a plain
implementation in 64 bits over its paths: few rows, operands read where they lie
and laid out first, every tile shape, runs of any length (none, one row, ends
inside a tile), rows gathered from anywhere or nowhere, rows before the first and
behind the last run.  Everything beside the tensors' elements, and x and dy in
rows of no expert, is NaN.

Tolerances as for the linear layer (tests/test_gpu_linear.py): k 2^-24 of the sum
of magnitudes for a sum of k terms, the activations' 2^-18, a rounded dz's half a
unit, a result rounded once."""
import math

import numpy as np
import pytest

from tests.test_gpu_layernorm import F32, TINY, UNIT, close, f64, make
from tests.test_gpu_linear import ACT, act_ref, slope_ref

pytestmark = pytest.mark.gpu

CASES = [  # counts of the experts, rows before and behind, inner, cols, dtype, act, gather, pad, shift, bias, save
    ([1], 0, 0, 1, 1, "float32", "none", False, 0, 0, True, True),
    ([0, 1, 0, 1], 0, 0, 768, 130, "float16", "gelu", False, 0, 0, True, False),
    ([2, 0, 3, 1], 1, 2, 33, 19, "bfloat16", "silu", True, 1, 1, True, True),
    ([5, 9, 20], 0, 3, 257, 64, "float32", "relu", True, 0, 0, False, True),
    ([64], 0, 0, 512, 515, "bfloat16", "gelu_tanh", False, 8, 0, True, True),
    ([65], 0, 0, 64, 1, "float16", "none", False, 0, 0, True, True),
    ([30, 0, 64, 1], 0, 5, 1, 70, "float32", "relu", True, 0, 0, False, True),
    ([63, 64, 65], 0, 0, 192, 128, "float16", "gelu_tanh", False, 0, 0, True, True),
    ([0, 0, 0], 40, 60, 64, 64, "float16", "relu", False, 0, 0, True, True),
    ([129, 1, 0, 70], 3, 4, 200, 257, "bfloat16", "gelu", True, 0, 0, True, True),
    ([257, 0, 300], 0, 7, 72, 129, "float16", "silu", True, 8, 8, False, False),
    ([300, 17, 2], 5, 0, 320, 333, "bfloat16", "relu", False, 8, 8, True, True),
    ([127, 128, 129], 0, 1, 127, 255, "float16", "gelu", True, 5, 3, True, True),
    ([700, 70, 7], 0, 9, 1001, 515, "float32", "relu", True, 0, 0, True, True),
    ([200, 313], 1, 0, 640, 129, "float32", "gelu_tanh", False, 1, 1, False, True),
    ([3] * 70, 0, 0, 64, 64, "bfloat16", "none", True, 0, 0, True, True),
    ([2, 0] * 100, 0, 0, 96, 40, "float32", "none", True, 0, 0, True, False),
    ([4000, 100, 0, 2500], 0, 77, 256, 2600, "bfloat16", "gelu_tanh", True, 0, 0, True, True),
    ([1500, 2500], 0, 0, 72, 2568, "float16", "none", False, 0, 0, True, False),
]


def stack(experts, rows, cols, dtype, rng, pad, shift, scale=1.0):
    """[experts, rows, cols] with rows and matrices apart."""
    import torch
    m, buf = make((experts * rows + experts, cols), dtype, rng, pad, shift, scale)
    t = m.as_strided((experts, rows, cols), ((rows + 1) * (cols + pad), cols + pad, 1), m.storage_offset())
    return t, buf


class Case:
    def __init__(self, counts, before, behind, inner, cols, dtype, act, gather, pad, shift, seed):
        import torch
        self.rng = rng = np.random.default_rng(seed)
        self.counts, self.inner, self.cols, self.dtype, self.act = counts, inner, cols, dtype, act
        self.experts, self.pad, self.shift, self.gather = len(counts), pad, shift, gather
        self.first, self.total = before, sum(counts)
        self.rows = before + self.total + behind
        self.offsets = torch.from_numpy(np.cumsum([before] + counts).astype(np.int32)).cuda()
        self.own = np.arange(before, before + self.total)
        self.expert = np.repeat(np.arange(self.experts), counts)
        x_rows = max(1, self.rows * 2 // 3) if gather else self.rows
        self.x, _ = make((x_rows, inner), dtype, rng, pad, shift)
        if gather:
            # any row, some twice, some from nowhere; garbage where no expert's rows are
            src = rng.integers(0, x_rows, self.rows)
            src[rng.random(self.rows) < 0.1] = x_rows + 5
            src[rng.random(self.rows) < 0.05] = -1
            src[:before], src[before + self.total:] = 1 << 30, -(1 << 31)
            self.source = torch.from_numpy(src.astype(np.int32)).cuda()
            there = (src >= 0) & (src < x_rows)
            self.X = np.where(there[:, None], f64(self.x)[np.where(there, src, 0)], 0.0)[self.own]
        else:
            self.source = None
            self.x[:before] = float("nan")
            self.x[before + self.total:] = float("nan")
            self.X = f64(self.x)[self.own]
        self.w, _ = stack(self.experts, cols, inner, dtype, rng, pad, shift, 1 / math.sqrt(inner))
        self.W = f64(self.w)

    def each(self):
        """(expert, its rows among the experts' rows) of those that have some."""
        for e in range(self.experts):
            r = np.nonzero(self.expert == e)[0]
            if len(r):
                yield e, r

    def outputs(self, cols, dtype=None):
        t, buf = make((self.rows, cols), dtype or self.dtype, self.rng, self.pad, self.shift)
        buf.fill_(7.0)
        return t, buf

    def check_outside(self, buf, cols):
        """Nothing written but the experts' rows."""
        import torch
        rest = buf.clone()
        rest[self.shift:self.shift + self.rows * (cols + self.pad)].view(self.rows, cols + self.pad)[
            self.first:self.first + self.total, :cols] = 7.0
        assert torch.equal(rest, torch.full_like(rest, 7.0))


@pytest.mark.parametrize("counts,before,behind,inner,cols,dtype,act,gather,pad,shift,bias,save", CASES)
def test_forward(counts, before, behind, inner, cols, dtype, act, gather, pad, shift, bias, save):
    from paper_2205_14465_amd import binding as B
    c = Case(counts, before, behind, inner, cols, dtype, act, gather, pad, shift, sum(counts) + inner)
    b = make((c.experts, cols), dtype, c.rng, pad, shift)[0] if bias else None
    y, ybuf = c.outputs(cols)
    z, zbuf = c.outputs(cols) if save else (None, None)
    ws = B.alloc_grouped_linear_workspace(c.x, c.w, c.rows)
    ws.fill_(255)
    B.bytecomp_grouped_linear_forward(c.x, c.source, c.offsets, c.w, b, act, y, z, ws)
    bias_of = f64(b)[c.expert] if bias else np.zeros((c.total, cols))
    wz, mag = np.array(bias_of), np.abs(bias_of)
    for e, r in c.each():
        wz[r] += c.X[r] @ c.W[e].T
        mag[r] += np.abs(c.X[r]) @ np.abs(c.W[e]).T
    ez = (inner + 6) * F32 * mag
    if c.total:
        if save:
            close(f64(z)[c.own], wz, dtype, ez)
        ey = 1.2 * ez + (ACT * np.abs(wz) if act not in ("none", "relu") else 0) + 2 * F32 * np.abs(wz)
        close(f64(y)[c.own], act_ref(act, wz), dtype, ey)
    c.check_outside(ybuf, cols)
    if save:
        c.check_outside(zbuf, cols)


@pytest.mark.parametrize("counts,before,behind,inner,cols,dtype,act,gather,pad,shift,bias,save", CASES)
def test_backward(counts, before, behind, inner, cols, dtype, act, gather, pad, shift, bias, save):
    import torch
    from paper_2205_14465_amd import binding as B
    c = Case(counts, before, behind, inner, cols, dtype, act, gather, pad, shift, sum(counts) + cols)
    dy, _ = make((c.rows, cols), dtype, c.rng, pad, shift, scale=0.05)
    z = make((c.rows, cols), dtype, c.rng, pad, shift)[0] if act != "none" else None
    dy[:before] = float("nan")
    dy[before + c.total:] = float("nan")
    ws = B.alloc_grouped_linear_workspace(c.x, c.w, c.rows, backward=True)
    ws.fill_(255)
    DY = f64(dy)[c.own]
    dz = DY * (slope_ref(act, f64(z)[c.own]) if z is not None else 1.0)
    half = UNIT[dtype] if dtype != "float32" else 0.0
    each = half + 6 * F32 + (ACT if act not in ("none", "relu") else 0)
    A = np.abs(dz) + (ACT + F32) * np.abs(DY)
    tiny = TINY[dtype]
    for gd in {dtype, "float32"}:
        dx, dxbuf = c.outputs(inner)
        dw, dwbuf = stack(c.experts, cols, inner, gd, c.rng, pad, shift)
        db, dbbuf = make((c.experts, cols), gd, c.rng, pad, shift)
        for t in (dwbuf, dbbuf):
            t.fill_(7.0)
        B.bytecomp_grouped_linear_backward(dy, z, c.x, c.source, c.offsets, c.w, act, dx, dw, db, ws)
        want, slack = np.zeros((c.total, inner)), np.zeros((c.total, inner))
        ww, sw = np.zeros((c.experts, cols, inner)), np.zeros((c.experts, cols, inner))
        wb, sb = np.zeros((c.experts, cols)), np.zeros((c.experts, cols))
        for e, r in c.each():
            want[r] = dz[r] @ c.W[e]
            slack[r] = (A[r] * (each + cols * F32) + tiny + F32 * np.abs(DY[r])) @ np.abs(c.W[e])
            ww[e] = dz[r].T @ c.X[r]
            sw[e] = (A[r] * (each + len(r) * F32) + tiny + F32 * np.abs(DY[r])).T @ np.abs(c.X[r])
            wb[e] = dz[r].sum(0)
            sb[e] = (A[r] * (each - half + len(r) * F32) + F32 * np.abs(DY[r])).sum(0)
        if c.total:
            close(f64(dx)[c.own], want, dtype, slack)
        close(f64(dw), ww, gd, sw)
        close(f64(db), wb, gd, sb)
        c.check_outside(dxbuf, inner)
        rest = dwbuf.clone()
        rest.as_strided(dw.shape, dw.stride(), dw.storage_offset()).fill_(7.0)
        assert torch.equal(rest, torch.full_like(rest, 7.0))
    one = torch.empty_like(dw), torch.empty_like(dx), torch.empty_like(db)
    B.bytecomp_grouped_linear_backward(dy, z, c.x, c.source, c.offsets, c.w, act, None, one[0], None, ws)
    B.bytecomp_grouped_linear_backward(dy, z, c.x, c.source, c.offsets, c.w, act, one[1], None, None, ws)
    B.bytecomp_grouped_linear_backward(dy, z, c.x, c.source, c.offsets, c.w, act, None, None, one[2], ws)
    own = slice(before, before + c.total)
    assert torch.equal(one[0], dw) and torch.equal(one[1][own], dx[own]) and torch.equal(one[2], db)


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("counts", [[1], [2], [3], [4], [5], [0, 7, 2], [1] * 60])
@pytest.mark.parametrize("inner", [1, 7, 8, 511, 512, 520, 1600, 2049, 8200])
def test_tokens(counts, inner, dtype):
    """Few rows: those of a weight that end anywhere in a wave's pieces."""
    import torch
    from paper_2205_14465_amd import binding as B
    c = Case(counts, 0, 0, inner, 37, dtype, "none", True, 0, 0, inner)
    y = torch.empty(c.rows, 37, dtype=c.x.dtype, device="cuda")
    B.bytecomp_grouped_linear_forward(c.x, c.source, c.offsets, c.w, None, "none", y, None, None)
    for e, r in c.each():
        close(f64(y)[r], c.X[r] @ c.W[e].T, dtype, (inner + 6) * F32 * (np.abs(c.X[r]) @ np.abs(c.W[e]).T))


@pytest.mark.parametrize("inner,cols", [(640, 512), (264, 776), (1600, 320)])
@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
def test_tiles_of_every_size(inner, cols, dtype):
    """The same rows, alone and among so many that larger tiles take them: each row
    only depends on its own expert, up to the order of sums."""
    import torch
    from paper_2205_14465_amd import binding as B
    rng = np.random.default_rng(inner)
    w = make((3 * cols, inner), dtype, rng, scale=1 / math.sqrt(inner))[0].view(3, cols, inner)
    x, _ = make((9000, inner), dtype, rng)
    for counts in ([40, 30, 0], [300, 200, 100], [4000, 1000, 4000]):
        n = sum(counts)
        off = torch.from_numpy(np.cumsum([0] + counts).astype(np.int32)).cuda()
        y = torch.empty(n, cols, dtype=x.dtype, device="cuda")
        ws = B.alloc_grouped_linear_workspace(x, w, n, backward=True)
        B.bytecomp_grouped_linear_forward(x[:n], None, off, w, None, "none", y, None, ws)
        dx, dw = torch.empty(n, inner, dtype=x.dtype, device="cuda"), torch.empty_like(w)
        B.bytecomp_grouped_linear_backward(y, None, x[:n], None, off, w, "none", dx, dw, None, ws)
        e = np.repeat(np.arange(3), counts)
        pick = np.unique(np.concatenate([np.arange(0, n, max(1, n // 60)), np.cumsum(counts)[:2] - 1]))
        X, W, Y = f64(x[:n]), f64(w), f64(y)
        for i in range(3):
            r = pick[e[pick] == i]
            close(Y[r], X[r] @ W[i].T, dtype, (inner + 6) * F32 * (np.abs(X[r]) @ np.abs(W[i]).T))
            close(f64(dx)[r], Y[r] @ W[i], dtype, (cols + 6) * F32 * (np.abs(Y[r]) @ np.abs(W[i])))
            q = e == i
            close(f64(dw)[i][::37], Y[q][:, ::37].T @ X[q], dtype,
                  (max(1, q.sum()) + 6) * F32 * (np.abs(Y[q][:, ::37]).T @ np.abs(X[q])))


@pytest.mark.parametrize("act", ["none", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("counts", [[5, 0, 7], [100, 30, 1]])
def test_gradient_against_differences(counts, act):
    """As the linear layer's: central differences of the definition in 64 bits."""
    import torch
    from paper_2205_14465_amd import binding as B
    c = Case(counts, 0, 0, 70, 90, "float32", act, True, 0, 0, 5)
    rng, E = c.rng, c.experts
    b = rng.standard_normal((E, 90)).astype(np.float32)
    g = rng.standard_normal((c.rows, 90)).astype(np.float32)
    gy = torch.from_numpy(g).cuda()
    y, z = torch.empty_like(gy), torch.empty_like(gy)
    dx, dw, db = torch.empty(c.rows, 70, device="cuda"), torch.empty(c.w.shape, device="cuda"), torch.empty(E, 90, device="cuda")
    ws = B.alloc_grouped_linear_workspace(c.x, c.w, c.rows, backward=True)
    B.bytecomp_grouped_linear_forward(c.x, c.source, c.offsets, c.w, torch.from_numpy(b).cuda(), act, y, z, ws)
    B.bytecomp_grouped_linear_backward(gy, z, c.x, c.source, c.offsets, c.w, act, dx, dw, db, ws)
    u, v, t = rng.standard_normal(c.X.shape), rng.standard_normal(c.W.shape), rng.standard_normal(b.shape)
    e = 1e-4

    def loss(s):
        return sum((g[r] * act_ref(act, (c.X[r] + s * u[r]) @ (c.W[i] + s * v[i]).T + b[i] + s * t[i])).sum()
                   for i, r in c.each())
    slope = (loss(e) - loss(-e)) / (2 * e)
    got = (f64(dx) * u).sum() + (f64(dw) * v).sum() + (f64(db) * t).sum()
    size = math.sqrt(sum((f64(d) ** 2).sum() for d in (dx, dw, db)))
    assert abs(got - slope) <= 1e-4 * size


def test_special_values_stay_with_their_rows_and_experts():
    import torch
    from paper_2205_14465_amd import binding as B
    nan, inf = float("nan"), float("inf")
    for counts in ([3, 2, 1], [30, 30, 40], [100, 130, 60], [400, 700, 60]):
        for dtype in (torch.float16, torch.float32):
            n, off = sum(counts), torch.from_numpy(np.cumsum([0] + counts).astype(np.int32)).cuda()
            x = torch.randn(n, 64, device="cuda").to(dtype)
            w = torch.randn(3, 96, 64, device="cuda").to(dtype)
            x[1, 5] = nan
            w[1, 7, 3] = inf
            y, ws = torch.empty(n, 96, dtype=dtype, device="cuda"), None
            if n > 64 and dtype == torch.float32:
                ws = B.alloc_grouped_linear_workspace(x, w, n, backward=True)
            B.bytecomp_grouped_linear_forward(x, None, off, w, None, "relu", y, None, ws)
            a, b = counts[0], counts[0] + counts[1]
            assert y[1].isnan().all() and y[0].isfinite().all() and y[2:a].isfinite().all() and y[b:].isfinite().all()
            assert y[a:b, :7].isfinite().all() and y[a:b, 8:].isfinite().all() and not (y[a:b, 7] > 0).isfinite().logical_not().any()
            assert ((y[a:b, 7] == inf) | (y[a:b, 7] == 0)).all()
            # a gradient's NaN reaches its row of dx, its expert's column of dw
            dy = torch.randn(n, 96, device="cuda").to(dtype)
            dy[a, 9] = nan
            x[1, 5], w[1, 7, 3] = 1, 1
            dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty(3, 96, dtype=dtype, device="cuda")
            ws = B.alloc_grouped_linear_workspace(x, w, n, backward=True)
            B.bytecomp_grouped_linear_backward(dy, None, x, None, off, w, "none", dx, dw, db, ws)
            ok = torch.ones(n, dtype=torch.bool)
            ok[a] = False
            assert dx[a].isnan().all() and dx[ok.cuda()].isfinite().all()
            assert dw[1, 9].isnan().all() and dw[0].isfinite().all() and dw[2].isfinite().all()
            assert dw[1, :9].isfinite().all() and db[1, 9].isnan() and db.isnan().sum() == 1


def test_empty():
    import torch
    from paper_2205_14465_amd import binding as B
    off = torch.zeros(4, dtype=torch.int32, device="cuda")
    # no rows at all: dw and dbias are zero
    x, w = torch.empty(0, 40, device="cuda"), torch.randn(3, 30, 40, device="cuda")
    dw, db = torch.ones_like(w), torch.ones(3, 30, device="cuda")
    e = torch.empty(0, 30, device="cuda")
    B.bytecomp_grouped_linear_backward(e, None, x, None, off, w, "none", torch.empty_like(x), dw, db, None)
    assert not dw.any() and not db.any()
    # rows gathered from a matrix without any are zeros
    off = torch.tensor([0, 50, 50, 100], dtype=torch.int32, device="cuda")
    for n, o in ((100, off), (10, (off // 10).int())):
        src, b = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.randn(3, 30, device="cuda")
        y = torch.empty(n, 30, device="cuda")
        B.bytecomp_grouped_linear_forward(x, src, o, w, b, "none", y, None, torch.empty(1 << 22, dtype=torch.uint8,
                                                                                       device="cuda"))
        assert torch.equal(y, b[[0, 2]].repeat_interleave(n // 2, 0))
        # no inner axis: the bias
        x0, w0 = torch.empty(n, 0, device="cuda"), torch.empty(3, 30, 0, device="cuda")
        y.zero_()
        B.bytecomp_grouped_linear_forward(x0, None, o, w0, b, "none", y, None, None)
        assert torch.equal(y, b[[0, 2]].repeat_interleave(n // 2, 0))


def test_offsets_that_do_not_ascend_stay_within_the_tensors():
    """The library cannot see them: results are unspecified, places are not."""
    import torch
    from paper_2205_14465_amd import binding as B
    w = torch.randn(3, 64, 64, device="cuda").half()
    for n in (20, 300):
        for values in ([5, 2, 9, 1], [0, 1 << 30, 3, 10], [-7, -3, 5, 1 << 30], [300, 200, 100, 0]):
            off = torch.tensor(values, dtype=torch.int32, device="cuda")
            x = torch.randn(n, 64, device="cuda").half()
            buf = torch.full((n + 40, 64), 7.0, device="cuda", dtype=torch.float16)
            y, dx = buf[20:20 + n], torch.empty_like(x)
            ws = B.alloc_grouped_linear_workspace(x, w, n, backward=True)
            B.bytecomp_grouped_linear_forward(x, None, off, w, None, "none", y, None, ws)
            src = torch.randint(0, n, (n,), device="cuda").int()
            B.bytecomp_grouped_linear_backward(x, x, x, src, off, w, "silu", dx, torch.empty_like(w),
                                               torch.empty(3, 64, device="cuda").half(), ws)
            torch.cuda.synchronize()
            assert (buf[:20] == 7).all() and (buf[20 + n:] == 7).all()


def test_other_stream_and_graph():
    """Captured once, replayed with other inputs, offsets and an eager call between."""
    import torch
    from paper_2205_14465_amd import binding as B
    n, dt = 700, torch.bfloat16
    w = torch.randn(4, 200, 96, device="cuda").to(dt)
    x, dy, z = (torch.randn(n, c, device="cuda").to(dt) for c in (96, 200, 200))
    src, off = torch.randint(0, n, (n,), device="cuda").int(), torch.tensor([0, 100, 100, 500, 650], device="cuda").int()
    ws = B.alloc_grouped_linear_workspace(x, w, n, backward=True)

    def outputs():
        return (torch.zeros(n, 200, device="cuda", dtype=dt), torch.zeros(n, 96, device="cuda", dtype=dt),
                torch.zeros_like(w), torch.zeros(4, 200, device="cuda", dtype=dt))

    def calls(o, ws):
        B.bytecomp_grouped_linear_forward(x, src, off, w, None, "silu", o[0], None, ws)
        B.bytecomp_grouped_linear_backward(dy, z, x, src, off, w, "gelu", o[1], o[2], o[3], ws)
    got = outputs()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        calls(got, ws)
    torch.cuda.current_stream().wait_stream(s)
    want = outputs()
    calls(want, torch.empty_like(ws))
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls(got, ws)
    for values in ([0, 1, 2, 3, 700], [300, 301, 302, 303, 304], [0, 175, 350, 525, 700]):
        off.copy_(torch.tensor(values))
        src.copy_(torch.randint(0, n, (n,)))
        x.copy_(torch.randn(n, 96))
        for t in got + want:
            t.zero_()
        graph.replay()
        calls(want, torch.empty_like(ws))
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)


def test_wrong_tensors_raise():
    import torch
    from paper_2205_14465_amd import binding as B
    x, w = torch.randn(700, 64, device="cuda"), torch.randn(3, 32, 64, device="cuda")
    y, off = torch.empty(700, 32, device="cuda"), torch.tensor([0, 1, 2, 3], dtype=torch.int32, device="cuda")
    ws = B.alloc_grouped_linear_workspace(x, w, 700)

    def f(x=x, src=None, off=off, w=w, b=None, act="none", y=y, z=None, ws=ws):
        B.bytecomp_grouped_linear_forward(x, src, off, w, b, act, y, z, ws)
    f()
    for bad in (dict(w=w.half()), dict(w=w[:, :, :60]), dict(w=w[0]), dict(w=w.transpose(1, 2).contiguous().transpose(1, 2)),
                dict(w=w[:1].expand(3, 32, 64)), dict(x=x[:699]), dict(off=off[:3]), dict(off=off.long()), dict(act="swish"),
                dict(src=off), dict(b=torch.zeros(3, 31, device="cuda")), dict(w=w.cpu()), dict(y=y.half())):
        with pytest.raises(ValueError):
            f(**bad)
    with pytest.raises(B.BytecompError) as err:  # rows that are laid out first
        f(x=x.half()[:, :60], w=w.half()[:, :, :60], y=y.half(), ws=None)
    assert err.value.code == -7
