"""Orthogonalised updates and the optimizer step around them, against the
formulas in 64 bits: square, wide, tall and one-row matrices, ragged lists,
strides, types, dominant directions, extreme scales, special values.

Tolerance: the factors are held to 22 bits, so the reference is run a second
time with every stored factor (X, A, B) off by a random 2^-22 of itself at most;
a result may be 8 times as far (2-norm) from the first run as that, plus what
one rounding to its type costs.  The chain of fp32 additions (2^-24 each, on
sums whose terms have mixed signs) stays below those roundings."""
import numpy as np
import pytest

from tests.test_gpu_layernorm import UNIT, f64, make

pytestmark = pytest.mark.gpu
ABC = (3.4445, -4.7750, 2.0315)


def reference(u, steps=5, abc=ABC, eps=1e-7, noise=None):
    def held(v):
        return v if noise is None else v * (1 + 2.0 ** -22 * noise.uniform(-1, 1, v.shape))
    x = u.T if u.shape[0] > u.shape[1] else u
    x = held(x / (np.sqrt((x * x).sum()) + eps))
    a, b, c = abc
    for _ in range(steps):
        g = held(x @ x.T)
        x = held(a * x + held(b * g + c * (g @ g)) @ x)
    return x.T if u.shape[0] > u.shape[1] else x


def near(got, u, dtype="float32", **kw):
    want = reference(u, **kw)
    size = np.linalg.norm(want)
    wobble = np.linalg.norm(reference(u, noise=np.random.default_rng(5), **kw) - want)
    off = np.linalg.norm(got - want)
    assert off <= 8 * wobble + (UNIT[dtype] + 2.0 ** -23) * size, (off / size, wobble / size)


def gradient(shape, rng, kind="plain"):
    r, c = shape
    g = rng.standard_normal(shape)
    if kind == "directions":  # a few dominate
        g = 0.03 * g + rng.standard_normal((r, 3)) @ rng.standard_normal((3, c))
    if kind == "uneven":
        g = g * np.exp(rng.standard_normal((r, 1))) * np.exp(rng.standard_normal((1, c)))
    return g


SHAPES = [(1, 1), (1, 300), (300, 1), (7, 5), (64, 64), (65, 63), (64, 147), (128, 128), (129, 200), (200, 129),
          (256, 256), (257, 640), (640, 257), (31, 2000), (768, 768)]


@pytest.mark.parametrize("kind", ["plain", "directions", "uneven"])
@pytest.mark.parametrize("shape", SHAPES)
def test_one_matrix(shape, kind):
    import torch
    from paper_2205_14465_amd import binding as B
    rng = np.random.default_rng(shape[0] * 1000 + shape[1])
    u = torch.from_numpy(gradient(shape, rng, kind) * 1e-3).float().cuda()
    out = torch.full_like(u, 9.0)
    ws = B.alloc_orthogonalize_workspace([shape])
    ws.fill_(255)
    B.bytecomp_orthogonalize([u], [out], ws)
    near(f64(out), f64(u))
    B.bytecomp_orthogonalize([u], [u], ws)  # in place
    assert torch.equal(u, out)


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
def test_list(dtype):
    """Many shapes in one call, with strides and odd starts and empty matrices
    among them; rows of other tensors between them stay as they were."""
    import torch
    from paper_2205_14465_amd import binding as B
    rng = np.random.default_rng(3)
    shapes = SHAPES[:-1] + [(0, 5), (40, 40), (5, 0), (513, 70), (0, 0)]
    ups, outs, bufs = [], [], []
    for i, s in enumerate(shapes):
        pad, shift = (i % 3) * 5, i % 2
        ups.append(make(s, dtype, rng, pad, shift)[0])
        o, buf = make(s, dtype, rng, pad + 1, shift)
        buf.fill_(7.0)
        outs.append(o)
        bufs.append((buf, shift, pad + 1))
    ws = B.alloc_orthogonalize_workspace(shapes)
    ws.fill_(255)
    B.bytecomp_orthogonalize(ups, outs, ws)
    for s, u, o, (buf, shift, pad) in zip(shapes, ups, outs, bufs):
        if 0 not in s:
            near(f64(o), f64(u), dtype)
        outside = buf.clone()
        outside[shift:shift + s[0] * (s[1] + pad)].view(s[0], s[1] + pad)[:, :s[1]] = 7.0
        assert torch.equal(outside, torch.full_like(outside, 7.0))
    again = [torch.empty_like(o) for o in outs]
    B.bytecomp_orthogonalize(ups, again, ws)
    assert all(torch.equal(a, b) for a, b in zip(again, outs))


@pytest.mark.parametrize("shape", [(1600, 1664), (1700, 600), (700, 2300)])
def test_large_tiles(shape):
    import torch
    from paper_2205_14465_amd import binding as B
    rng = np.random.default_rng(9)
    T = 8
    ups = [torch.from_numpy(gradient(shape, rng)).float().cuda() for _ in range(T)]
    outs = [torch.empty_like(u) for u in ups]
    B.bytecomp_orthogonalize(ups, outs, B.alloc_orthogonalize_workspace([shape] * T))
    for i in (0, T - 1):
        near(f64(outs[i]), f64(ups[i]))


@pytest.mark.parametrize("steps,abc", [(1, ABC), (2, ABC), (5, (1.875, -1.25, 0.375)), (8, (1.5, -0.5, 0.0)),
                                       (3, (4.0848, -6.8946, 2.9270)), (6, (1.0, 0.0, 0.0))])
def test_steps_and_coefficients(steps, abc):
    import torch
    from paper_2205_14465_amd import binding as B
    rng = np.random.default_rng(steps)
    u = torch.from_numpy(gradient((90, 160), rng)).float().cuda()
    out = torch.empty_like(u)
    B.bytecomp_orthogonalize([u], [out], B.alloc_orthogonalize_workspace([(90, 160)]), steps=steps, coefficients=abc)
    near(f64(out), f64(u), steps=steps, abc=abc)


def test_scales_and_special_values():
    """The result does not depend on the update's scale, from the smallest
    normal numbers to the largest; a zero matrix gives zero; a NaN or an
    infinity spoils its own matrix only."""
    import torch
    from paper_2205_14465_amd import binding as B
    rng = np.random.default_rng(2)
    shape = (50, 70)
    base = torch.from_numpy(gradient(shape, rng)).float().cuda()
    # powers of two: the same bits without eps
    ups = [base, base * 2.0 ** 100, base * 2.0 ** -100, torch.zeros_like(base), base.clone(), base.clone(), base]
    ups[4][3, 4] = float("nan")
    ups[5][0, 0] = float("inf")
    outs = [torch.empty_like(u) for u in ups]
    ws = B.alloc_orthogonalize_workspace([shape] * len(ups))
    B.bytecomp_orthogonalize(ups, outs, ws, eps=0.0)
    near(f64(outs[0]), f64(base), eps=0.0)
    assert torch.equal(outs[1], outs[0]) and torch.equal(outs[2], outs[0]) and torch.equal(outs[6], outs[0])
    assert outs[3].isnan().all()  # 0 / 0
    assert outs[4].isnan().any() and outs[5].isnan().any()
    B.bytecomp_orthogonalize(ups, outs, ws)
    assert not outs[3].any()


@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("wdtype,gdtype", [("float32", "float32"), ("float32", "float16"), ("bfloat16", "bfloat16"),
                                           ("float16", "float32")])
def test_muon_step(wdtype, gdtype, nesterov):
    import torch
    from paper_2205_14465_amd import binding as B
    rng = np.random.default_rng(4)
    shapes = [(64, 147), (300, 1), (129, 200), (513, 70), (3, 0)]
    lr, mu, wd = 0.02, 0.95, 0.1
    ws_, gs, ms = [], [], []
    for i, s in enumerate(shapes):
        ws_.append(make(s, wdtype, rng, i, i % 2, scale=0.1)[0])
        gs.append(make(s, gdtype, rng, 2, 1, scale=0.01)[0])
        ms.append(make(s, "float32", rng, 3, 0, scale=0.1)[0])
    scales = [1.0, 0.3, 2.0, max(1.0, 513 / 70) ** 0.5, 1.0]
    call = B.MuonCall(ws_, gs, ms, B.alloc_orthogonalize_workspace(shapes), momentum=mu, nesterov=nesterov,
                      weight_decay=wd, scales=scales)
    for step in range(2):
        before = [(f64(w), f64(g), m.clone()) for w, g, m in zip(ws_, gs, ms)]
        call(lr)
        for (w, g, m), w2, m2, sc, g2 in zip(before, ws_, ms, scales, gs):
            if 0 in w.shape:
                continue
            mf = m * mu + g2.float()  # the momentum's two roundings, exactly
            assert torch.equal(m2, mf)
            u = f64(mf * mu + g2.float()) if nesterov else f64(mf)
            want = (1 - lr * wd) * w - lr * sc * reference(u)
            noisy = (1 - lr * wd) * w - lr * sc * reference(u, noise=np.random.default_rng(1))
            off, size = np.linalg.norm(f64(w2) - want), np.linalg.norm(want)
            assert off <= 8 * np.linalg.norm(noisy - want) + (UNIT[wdtype] + 2.0 ** -22) * size


def test_other_stream_and_wrong_tensors():
    import torch
    from paper_2205_14465_amd import binding as B
    u = torch.randn(300, 400, device="cuda")
    a, b = torch.empty_like(u), torch.empty_like(u)
    ws, ws2 = (B.alloc_orthogonalize_workspace([(300, 400)]) for _ in range(2))
    s = torch.cuda.Stream()
    B.bytecomp_orthogonalize([u], [a], ws)
    s.wait_stream(torch.cuda.current_stream())
    B.bytecomp_orthogonalize([u], [b], ws2, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(a, b)
    B.bytecomp_orthogonalize([], [], None)
    for bad in (lambda: B.bytecomp_orthogonalize([u], [], ws), lambda: B.bytecomp_orthogonalize([u], [a.half()], ws),
                lambda: B.bytecomp_orthogonalize([u, u.half()], [a, b], ws),
                lambda: B.bytecomp_orthogonalize([u.t()], [a.t()], ws),
                lambda: B.MuonCall([u], [u], [u.half()], ws), lambda: B.MuonCall([u], [u], [a], ws, scales=[])):
        with pytest.raises(ValueError):
            bad()


@pytest.mark.parametrize("shapes", [[(70, 6011)], [(4099, 180)], [(33, 1023)], [(17, 5000), (150, 150)],
                                    [(512, 4608)] * 3 + [(2048, 512)]])
def test_long_axes(shapes):
    """Few tiles and many steps along the longer axis: the result is the formula's
    and every run's the same, whichever workgroup comes last."""
    import torch
    from paper_2205_14465_amd import binding as B
    rng = np.random.default_rng(21)
    ups = [torch.from_numpy(gradient(s, rng, "uneven")).float().cuda() for s in shapes]
    outs = [torch.empty_like(u) for u in ups]
    ws = B.alloc_orthogonalize_workspace(shapes)
    ws.fill_(255)
    B.bytecomp_orthogonalize(ups, outs, ws)
    for u, o in zip(ups, outs):
        near(f64(o), f64(u))
    for _ in range(3):
        again = [torch.empty_like(u) for u in ups]
        B.bytecomp_orthogonalize(ups, again, ws)
        assert all(torch.equal(a, b) for a, b in zip(again, outs))
