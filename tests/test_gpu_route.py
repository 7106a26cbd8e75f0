"""The router and the combination of a block of experts, against plain
implementations in 64 bits: every number of lanes that a row of logits takes, one
and several workgroups, ties, masks that leave few or no experts, NaN and
infinities, strides.

Tolerances: choices, slots and offsets are exact (the logits are compared as they
are).  A weight is an exponential (within 2 units) over a sum of at most 1024 of
them, each addition off by half a unit of 2^-23, and a division: (1024/G + 16)
units of 2^-24 with G >= 8 lanes.  Sums of k terms: k units of 2^-24 of the sum of
magnitudes, a result rounded once to its type."""
import numpy as np
import pytest

from tests.test_gpu_layernorm import F32, TINY, UNIT, close, f64, make

pytestmark = pytest.mark.gpu
WEIGHT = 160 * F32


def route_ref(x, k, normalise):
    """weight, expert, slot, source, offsets of logits in 64 bits."""
    n, experts = x.shape
    weight, expert, slot = np.zeros((n, k)), np.full((n, k), -1), np.full((n, k), -1)
    with np.errstate(invalid="ignore", over="ignore"):
        for r in range(n):
            live = [e for e in range(experts) if not x[r, e] == -np.inf]
            order = sorted(live, key=lambda e: (0 if np.isnan(x[r, e]) else 1, 0 if np.isnan(x[r, e]) else -x[r, e], e))[:k]
            if not order:
                continue
            top = x[r, order[0]]
            p = {e: np.exp(x[r, e] - top) for e in live}
            by = sum(p[e] for e in (order if normalise else live))
            expert[r, :len(order)] = order
            weight[r, :len(order)] = [p[e] / by for e in order]
    source, offsets = [], [0]
    for e in range(experts):
        for r, j in zip(*np.nonzero(expert == e)):
            slot[r, j] = len(source)
            source.append(r)
        offsets.append(len(source))
    return weight, expert, slot, np.array(source, dtype=int), np.array(offsets)


def route(x, k, normalise, ws_fill=255, stream=None):
    import torch
    from paper_2205_14465_amd import binding as B
    n, experts = x.shape
    weight = torch.full((n, k), 7.0, device="cuda")
    ints = [torch.full(s, -5, dtype=torch.int32, device="cuda") for s in ((n, k), (n, k), (n * k,), (experts + 1,))]
    ws = B.alloc_route_workspace(n, experts, k)
    ws.fill_(ws_fill)
    B.bytecomp_route_forward(x, weight, *ints, ws, normalise=normalise, stream=stream)
    return weight, *ints


CASES = [  # rows, experts, k, dtype, normalise, pad
    (1, 1, 1, "float32", True, 0), (1, 64, 8, "bfloat16", True, 0), (1, 2, 2, "float16", False, 3),
    (5, 8, 8, "float32", False, 0), (63, 7, 2, "float16", True, 1), (64, 9, 3, "bfloat16", False, 0),
    (65, 16, 1, "float32", True, 0), (130, 31, 5, "bfloat16", True, 5), (200, 33, 32, "float32", True, 0),
    (333, 64, 2, "bfloat16", True, 0), (257, 65, 4, "float16", False, 0), (129, 129, 4, "float32", False, 1),
    (100, 300, 6, "bfloat16", True, 0), (70, 513, 8, "float32", False, 0), (150, 1024, 32, "float16", True, 0),
    (20000, 8, 2, "bfloat16", True, 0), (40000, 24, 1, "float16", False, 0),
]


@pytest.mark.parametrize("rows,experts,k,dtype,normalise,pad", CASES)
def test_forward(rows, experts, k, dtype, normalise, pad):
    rng = np.random.default_rng(rows * 3 + experts)
    x, _ = make((rows, experts), dtype, rng, pad, 0)
    # masks: some logits, some rows down to fewer than k, some whole rows
    mask = rng.random((rows, experts)) < 0.2
    mask[rng.random(rows) < 0.1] = True
    few = rng.random(rows) < 0.1
    mask[few, experts // 3:] = True
    import torch
    x[torch.from_numpy(mask).cuda()] = float("-inf")
    got = route(x, k, normalise)
    want = route_ref(f64(x), k, normalise)
    weight, expert, slot, source, offsets = (t.cpu().numpy() for t in got)
    assert np.array_equal(expert, want[1]) and np.array_equal(slot, want[2]) and np.array_equal(offsets, want[4])
    n = len(want[3])
    assert np.array_equal(source[:n], want[3]) and np.all(source[n:] == -5)
    assert np.all(np.abs(weight - want[0]) <= WEIGHT * want[0]), np.max(np.abs(weight - want[0]))
    # the same again, whatever the workspace holds
    for a, b in zip(got, route(x, k, normalise, ws_fill=0)):
        assert torch.equal(a, b)


def test_special_logits():
    """NaN is the largest, +-0 are equal, the type's lowest value is no mask."""
    import torch
    inf, nan = float("inf"), float("nan")
    low = torch.finfo(torch.float32).min
    x = torch.tensor([[1.0, nan, 3.0, nan], [0.0, -0.0, 0.0, -1.0], [inf, 1.0, 2.0, inf], [low, low, low, low],
                      [-inf, low, -inf, -inf], [-inf, -inf, -inf, -inf], [3.4e38, -3.4e38, 0.0, 1.0],
                      [1e-40, 2e-40, 0.0, -1e-40]], device="cuda")
    for normalise in (True, False):
        weight, expert, slot, source, offsets = (t.cpu().numpy() for t in route(x, 2, normalise))
        assert expert.tolist() == [[1, 3], [0, 1], [0, 3], [0, 1], [1, -1], [-1, -1], [0, 3], [1, 0]]
        assert np.isnan(weight[0]).all() and np.isnan(weight[2]).all()
        assert weight[5].tolist() == [0, 0] and weight[4].tolist() == [1, 0]
        assert weight[3].tolist() == ([0.5, 0.5] if normalise else [0.25, 0.25])
        assert weight[6].tolist() == [1, 0]
        want = route_ref(x.double().cpu().numpy(), 2, normalise)
        assert np.array_equal(slot, want[2]) and np.array_equal(offsets, want[4])
        assert np.array_equal(source[:len(want[3])], want[3])


def test_ties_go_to_the_lower_expert():
    import torch
    x = torch.randint(0, 3, (500, 40), device="cuda").to(torch.float16)
    _, expert, _, _, _ = route(x, 7, True)
    order = torch.sort(x.float(), dim=1, descending=True, stable=True).indices[:, :7]
    assert torch.equal(expert.long(), order)


def test_no_rows_and_other_stream():
    import torch
    out = route(torch.empty(0, 5, device="cuda"), 2, True)
    assert out[4].tolist() == [0] * 6
    x = torch.randn(3000, 12, device="cuda")
    want = route(x, 3, True)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = route(x, 3, True)
    torch.cuda.current_stream().wait_stream(s)
    for a, b in zip(want, got):
        assert torch.equal(a, b)


def grad_ref(x, weight, expert, dweight, normalise):
    n, experts = x.shape
    up, p = np.zeros((n, experts)), np.zeros((n, experts))
    for r in range(n):
        for j, e in enumerate(expert[r]):
            if e >= 0:
                up[r, e], p[r, e] = dweight[r, j], weight[r, j]
    if not normalise:
        top = np.where(np.isinf(x.max(1)), 0, x.max(1))[:, None]
        ex = np.exp(x - top)
        p = ex / np.maximum(ex.sum(1, keepdims=True), 1e-300)
    return p, up, p * (up - (p * up).sum(1, keepdims=True))


@pytest.mark.parametrize("rows,experts,k,dtype,normalise,pad", CASES)
def test_backward(rows, experts, k, dtype, normalise, pad):
    import torch
    from paper_2205_14465_amd import binding as B
    rng = np.random.default_rng(rows + experts)
    x, _ = make((rows, experts), dtype, rng, pad, 0)
    mask = rng.random((rows, experts)) < 0.2
    mask[rng.random(rows) < 0.1] = True
    x[torch.from_numpy(mask).cuda()] = float("-inf")
    weight, expert = route(x, k, normalise)[:2]
    dweight = torch.from_numpy(rng.standard_normal((rows, k)).astype(np.float32)).cuda()
    d, buf = make((rows, experts), dtype, rng, pad + 1, 1)
    buf.fill_(7.0)
    B.bytecomp_route_backward(x, weight, expert, dweight, d, normalise=normalise)
    p, up, want = grad_ref(f64(x), f64(weight), expert.cpu().numpy(), f64(dweight), normalise)
    # terms: the chance (WEIGHT), the sum of k products and one subtraction
    slack = (WEIGHT + (k + 3) * F32) * p * (np.abs(up) + (p * np.abs(up)).sum(1, keepdims=True))
    close(f64(d), want, dtype, slack)
    assert not f64(d)[mask].any()
    outside = buf.clone()
    outside[1:1 + rows * (experts + pad + 1)].view(rows, experts + pad + 1)[:, :experts] = 7.0
    assert torch.equal(outside, torch.full_like(outside, 7.0))


@pytest.mark.parametrize("normalise", [True, False])
def test_gradient_against_differences(normalise):
    """The weights' derivative along a direction by central differences in 64 bits
    (a step of 1e-5, no choice changes): off by under 1e-8 of the scale."""
    import torch
    from paper_2205_14465_amd import binding as B
    rng = np.random.default_rng(3)
    X = rng.standard_normal((40, 11)).astype(np.float32)
    x = torch.from_numpy(X).cuda()
    weight, expert = route(x, 3, normalise)[:2]
    g, u = rng.standard_normal((40, 3)).astype(np.float32), rng.standard_normal(X.shape)
    d = torch.empty_like(x)
    B.bytecomp_route_backward(x, weight, expert, torch.from_numpy(g).cuda(), d, normalise=normalise)

    def loss(s):
        w, e = route_ref(X + s * u, 3, normalise)[:2]
        assert np.array_equal(e, expert.cpu().numpy())
        return (g * w).sum()
    slope = (loss(1e-5) - loss(-1e-5)) / 2e-5
    assert abs((f64(d) * u).sum() - slope) <= 1e-5 * np.sqrt((f64(d) ** 2).sum())


def test_infinite_gradients_stay_with_the_chosen():
    import torch
    from paper_2205_14465_amd import binding as B
    x = torch.tensor([[1.0, 2.0, 3.0, float("-inf")]], device="cuda")
    weight, expert = route(x, 2, True)[:2]
    d = torch.empty_like(x)
    B.bytecomp_route_backward(x, weight, expert, torch.tensor([[float("inf"), 1.0]], device="cuda"), d, normalise=True)
    assert d[0, 0] == 0 and d[0, 3] == 0 and not d[0, 1:3].isfinite().all()


# ------------------------------------------------------------ combination

COMBINE = [  # rows, cols, k, slots, dtype, weighted, residual, pad, shift
    (1, 1, 1, 1, "float32", True, False, 0, 0), (1, 1600, 2, 2, "float16", True, True, 0, 0),
    (3, 7, 2, 6, "bfloat16", False, True, 1, 1), (70, 65, 4, 250, "float32", True, True, 3, 1),
    (129, 768, 8, 1100, "float16", False, False, 0, 0), (200, 1001, 2, 390, "float16", True, False, 0, 0),
    (64, 2056, 3, 200, "bfloat16", True, True, 8, 0), (33, 5000, 32, 1056, "float32", True, False, 0, 0),
    (4100, 40, 2, 8200, "bfloat16", True, True, 0, 0),
]


def slots_of(rows, k, slots, rng):
    """Slots in any order, each at most once, some missing or out of range."""
    s = np.full(rows * k, -1)
    n = min(rows * k, slots)
    s[rng.permutation(rows * k)[:n]] = rng.permutation(slots)[:n]
    s[rng.random(rows * k) < 0.15] = -1
    s[rng.random(rows * k) < 0.05] = slots + 3
    return s.reshape(rows, k).astype(np.int32)


@pytest.mark.parametrize("rows,cols,k,slots,dtype,weighted,residual,pad,shift", COMBINE)
def test_combine(rows, cols, k, slots, dtype, weighted, residual, pad, shift):
    import torch
    from paper_2205_14465_amd import binding as B
    rng = np.random.default_rng(rows + cols)
    y, _ = make((slots, cols), dtype, rng, pad, shift)
    S = slots_of(rows, k, slots, rng)
    slot = torch.from_numpy(S).cuda()
    weight = torch.from_numpy(rng.random((rows, k)).astype(np.float32)).cuda()
    res = make((rows, cols), dtype, rng, pad, shift)[0] if residual else None
    out, buf = make((rows, cols), dtype, rng, pad + 1, shift)
    buf.fill_(7.0)
    B.bytecomp_combine_forward(y, slot, weight if weighted else None, res, out)
    Y, W = f64(y), f64(weight) if weighted else np.ones((rows, k))
    R = f64(res) if residual else np.zeros((rows, cols))
    want, size = R.copy(), np.abs(R)
    for j in range(k):
        ok = (S[:, j] >= 0) & (S[:, j] < slots)
        want[ok] += W[ok, j, None] * Y[S[ok, j]]
        size[ok] += np.abs(W[ok, j, None] * Y[S[ok, j]])
    close(f64(out), want, dtype, (k + 2) * F32 * size)
    outside = buf.clone()
    outside[shift:shift + rows * (cols + pad + 1)].view(rows, cols + pad + 1)[:, :cols] = 7.0
    assert torch.equal(outside, torch.full_like(outside, 7.0))
    if residual:
        B.bytecomp_combine_forward(y, slot, weight if weighted else None, res, res)
        assert torch.equal(res, out)


@pytest.mark.parametrize("rows,cols,k,slots,dtype,weighted,residual,pad,shift", COMBINE)
def test_combine_backward(rows, cols, k, slots, dtype, weighted, residual, pad, shift):
    import torch
    from paper_2205_14465_amd import binding as B
    rng = np.random.default_rng(rows + 2 * cols)
    y, _ = make((slots, cols), dtype, rng, pad, shift)
    dout, _ = make((rows, cols), dtype, rng, pad, shift)
    S = slots_of(rows, k, slots, rng)
    slot = torch.from_numpy(S).cuda()
    weight = torch.from_numpy(rng.random((rows, k)).astype(np.float32)).cuda() if weighted else None
    dy, buf = make((slots, cols), dtype, rng, pad, shift)
    buf.fill_(7.0)
    dweight = torch.full((rows, k), 9.0, device="cuda")
    B.bytecomp_combine_backward(dout, y, slot, weight, dy, dweight)
    D, Y, W = f64(dout), f64(y), f64(weight) if weighted else np.ones((rows, k))
    want, dw, size = np.full((slots, cols), 7.0), np.zeros((rows, k)), np.zeros((rows, k))
    for r in range(rows):
        for j in range(k):
            if 0 <= S[r, j] < slots:
                want[S[r, j]] = W[r, j] * D[r]
                dw[r, j] = D[r] @ Y[S[r, j]]
                size[r, j] = np.abs(D[r]) @ np.abs(Y[S[r, j]])
    close(f64(dy), want, dtype, 2 * F32 * np.abs(want))
    close(f64(dweight), dw, "float32", (cols / 64 + 12) * F32 * size)
    used = torch.zeros(slots, dtype=torch.bool)
    used[torch.from_numpy(S[(S >= 0) & (S < slots)]).long()] = True
    assert (dy[~used.cuda()] == 7).all()
    # either alone
    only, alone = torch.full_like(dy, 7.0), torch.empty_like(dweight)
    B.bytecomp_combine_backward(dout, None, slot, weight, only, None)
    B.bytecomp_combine_backward(dout, y, slot, weight, None, alone)
    assert torch.equal(only, dy) and torch.equal(alone, dweight)


def test_wrong_tensors_raise():
    import torch
    from paper_2205_14465_amd import binding as B
    x = torch.randn(10, 4, device="cuda")
    w, i = torch.empty(10, 2, device="cuda"), torch.empty(10, 2, dtype=torch.int32, device="cuda")
    src, off = (torch.empty(n, dtype=torch.int32, device="cuda") for n in (20, 5))
    y = torch.randn(20, 8, device="cuda")
    out = torch.empty(10, 8, device="cuda")
    for bad in (lambda: B.bytecomp_route_forward(x, w.half(), i, i, src, off, None),
                lambda: B.bytecomp_route_forward(x, w, i.long(), i, src, off, None),
                lambda: B.bytecomp_route_forward(x, w, i, i, src[:19], off, None),
                lambda: B.bytecomp_route_forward(x, w, i, i, src, off[:4], None),
                lambda: B.bytecomp_route_forward(x.t().contiguous().t(), w, i, i, src, off, None),
                lambda: B.bytecomp_route_backward(x, w, i, w, x[:, :3]),
                lambda: B.bytecomp_combine_forward(y, i[:, :1], w, None, out),
                lambda: B.bytecomp_combine_forward(y, i, w, out.half(), out),
                lambda: B.bytecomp_combine_forward(y, i.cpu(), w, None, out),
                lambda: B.bytecomp_combine_backward(out, y, i, w, y[:19], w)):
        with pytest.raises(ValueError):
            bad()
