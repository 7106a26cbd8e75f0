"""A block of experts where its sizes end: the largest tiles with rows and columns that
fill only a part of them, rows gathered from more than 2 GB, experts and rows further
apart than 32 bits reach, 1024 experts, and captured graphs that share workspaces.
Against plain products in 64 bits on the device, tolerances as in
tests/test_gpu_grouped.py."""
import numpy as np
import pytest

from tests.test_gpu_layernorm import F32, close, f64

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def seeded():
    import torch
    torch.manual_seed(17)


def tensors(experts, n, inner, cols, dtype, seed, x_rows=None):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = getattr(torch, dtype)

    def normal(*shape, scale=1.0):
        return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dt)
    return (normal(x_rows or n, inner), normal(experts, cols, inner, scale=inner ** -0.5), normal(n, cols), dt)


def offsets_of(counts):
    import torch
    return torch.from_numpy(np.cumsum([0] + counts).astype(np.int32)).cuda()


def check_product(got, a, b, dtype):
    """got [m, n] against a [m, k] b [k, n], all of it, k 2^-24 of the magnitudes."""
    a, b = a.double(), b.double()
    close(f64(got), f64(a @ b), dtype, f64((a.shape[1] + 6) * F32 * (a.abs() @ b.abs())))


# sizes where the largest tile takes the forward pass, dx, dw, and both gradients in one
# launch; the last rows and columns fill less than half of a tile, or a little of it
@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("counts,inner,cols,what", [
    ([1400, 1285, 1409, 1347], 264, 2568, "y"), ([3000, 2951, 3000], 1544, 264, "dx"),
    ([300, 10, 0, 972], 1920, 1800, "dw"), ([257, 384, 385, 511, 512, 513, 0, 327], 1800, 376, "dx dw"),
    ([257, 384, 385, 511, 512, 513, 0, 327], 1800, 376, "dx dw gather"), ([9000, 1, 127, 128, 129], 520, 640, "y dx dw")])
def test_largest_tiles_in_part(counts, inner, cols, what, dtype):
    import torch
    from paper_2205_14465_amd import binding as B
    n, off = sum(counts), offsets_of(counts)
    gather = "gather" in what
    x, w, dy, dt = tensors(len(counts), n, inner, cols, dtype, inner, n // 2 if gather else None)
    src = torch.randint(0, n // 2, (n,), device="cuda").int() if gather else None
    y = torch.empty(n, cols, dtype=dt, device="cuda") if "y" in what else None
    dx = torch.empty(n, inner, dtype=dt, device="cuda") if "dx" in what else None
    dw = torch.empty_like(w) if "dw" in what else None
    ws = B.alloc_grouped_linear_workspace(x, w, n, backward=True)
    ws.fill_(255)
    if y is not None:
        B.bytecomp_grouped_linear_forward(x, src, off, w, None, "none", y, None, ws)
    B.bytecomp_grouped_linear_backward(dy, None, x, src, off, w, "none", dx, dw, None, ws)
    X = x[src.long()] if gather else x
    at = 0
    for e, c in enumerate(counts):
        r = slice(at, at + c)
        at += c
        if y is not None and c:
            check_product(y[r], X[r], w[e].T, dtype)
        if dx is not None and c:
            check_product(dx[r], dy[r], w[e], dtype)
        if dw is not None:
            check_product(dw[e], dy[r].T, X[r], dtype)


@pytest.mark.parametrize("dtype", ["float16", "float32"])
def test_rows_from_more_than_2gb(dtype):
    """Offsets of gathered rows no longer fit 32 bits: the rows are laid out first."""
    import torch
    from paper_2205_14465_amd import binding as B
    counts, inner, cols = [150, 0, 170, 130], 264, 72
    n, dt = sum(counts), getattr(torch, dtype)
    x_rows = (5 << 30) // (inner * dt.itemsize)
    x = torch.empty(x_rows, inner, dtype=dt, device="cuda")
    src = torch.randint(0, x_rows, (n,), device="cuda")
    src[:3] = torch.tensor([x_rows - 1, 0, x_rows // 2])
    rows = torch.randn(n, inner, device="cuda").to(dt)
    x[src] = rows
    X = x[src]
    src, off = src.int(), offsets_of(counts)
    w = torch.randn(4, cols, inner, device="cuda").mul(inner ** -0.5).to(dt)
    y, dy = torch.empty(n, cols, dtype=dt, device="cuda"), torch.randn(n, cols, device="cuda").to(dt)
    dx, dw = torch.empty(n, inner, dtype=dt, device="cuda"), torch.empty_like(w)
    ws = B.alloc_grouped_linear_workspace(x, w, n, backward=True)
    B.bytecomp_grouped_linear_forward(x, src, off, w, None, "none", y, None, ws)
    B.bytecomp_grouped_linear_backward(dy, None, x, src, off, w, "none", dx, dw, None, ws)
    at = 0
    for e, c in enumerate(counts):
        r = slice(at, at + c)
        at += c
        if c:
            check_product(y[r], X[r], w[e].T, dtype)
            check_product(dx[r], dy[r], w[e], dtype)
        check_product(dw[e], dy[r].T, X[r], dtype)


@pytest.mark.parametrize("dtype", ["float16", "bfloat16", "float32"])
@pytest.mark.parametrize("counts", [[25, 0, 40], [60, 1, 27]])
def test_some_rows_from_more_than_2gb(counts, dtype):
    """So few (65, and 64 + 8 experts) that the forward pass asks for no workspace."""
    import torch
    from paper_2205_14465_amd import binding as B
    inner, cols, n, dt = 264, 72, sum(counts), getattr(torch, dtype)
    x_rows = (5 << 30) // (inner * dt.itemsize)
    x = torch.empty(x_rows, inner, dtype=dt, device="cuda")
    src = torch.randint(0, x_rows, (n,), device="cuda")
    src[:3] = torch.tensor([x_rows - 1, 0, x_rows // 2])
    x[src] = torch.randn(n, inner, device="cuda").to(dt)
    X = x[src]
    w = torch.randn(3, cols, inner, device="cuda").mul(inner ** -0.5).to(dt)
    y = torch.empty(n, cols, dtype=dt, device="cuda")
    ws = B.alloc_grouped_linear_workspace(x, w, n)
    assert ws.numel() == 0
    B.bytecomp_grouped_linear_forward(x, src.int(), offsets_of(counts), w, None, "none", y, None, ws)
    at = 0
    for e, c in enumerate(counts):
        if c:
            check_product(y[at:at + c], X[at:at + c], w[e].T, dtype)
        at += c


@pytest.mark.parametrize("dtype,counts", [("float16", [3, 2, 4]), ("float32", [20, 31, 200]), ("bfloat16", [700, 1, 300])])
def test_experts_further_apart_than_32_bits(dtype, counts):
    import torch
    from paper_2205_14465_amd import binding as B
    inner, cols, apart = 200, 136, (1 << 31) + 64
    n, off, dt = sum(counts), offsets_of(counts), getattr(torch, dtype)

    def far():
        return torch.empty(2 * apart + inner * cols, dtype=dt, device="cuda").as_strided((3, cols, inner), (apart, inner, 1))
    x, _, dy, _ = tensors(3, n, inner, cols, dtype, 5)
    w, dw = far(), far()
    for e in range(3):
        w[e].normal_()
    y, dx = torch.empty(n, cols, dtype=dt, device="cuda"), torch.empty(n, inner, dtype=dt, device="cuda")
    ws = B.alloc_grouped_linear_workspace(x, w, n, backward=True)
    B.bytecomp_grouped_linear_forward(x, None, off, w, None, "none", y, None, ws)
    B.bytecomp_grouped_linear_backward(dy, None, x, None, off, w, "none", dx, dw, None, ws)
    at = 0
    for e, c in enumerate(counts):
        r = slice(at, at + c)
        at += c
        check_product(y[r], x[r], w[e].T, dtype)
        check_product(dx[r], dy[r], w[e], dtype)
        check_product(dw[e], dy[r].T, x[r], dtype)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows,k", [(1, 8), (500, 2), (9000, 4)])
def test_1024_experts(rows, k, dtype):
    """Routed and grouped, with runs of none to some rows."""
    import torch
    from paper_2205_14465_amd import binding as B
    experts, inner, cols, n = 1024, 72, 40, rows * k
    x, w, dy, dt = tensors(experts, n, inner, cols, dtype, rows, rows)
    logits = torch.randn(rows, experts, device="cuda").to(dt)
    weight = torch.empty(rows, k, device="cuda")
    expert, slot = (torch.empty(rows, k, dtype=torch.int32, device="cuda") for _ in range(2))
    src, off = torch.empty(n, dtype=torch.int32, device="cuda"), torch.empty(experts + 1, dtype=torch.int32, device="cuda")
    B.bytecomp_route_forward(logits, weight, expert, slot, src, off, B.alloc_route_workspace(rows, experts, k))
    of = torch.empty(n, dtype=torch.int64, device="cuda")
    of[slot.view(-1).long()] = expert.view(-1).long()
    assert torch.equal(off[1:].long(), torch.bincount(of, minlength=experts).cumsum(0)) and int(off[0]) == 0
    assert torch.equal(of, of.sort()[0])
    y, dx, dw = torch.empty(n, cols, dtype=dt, device="cuda"), torch.empty(n, inner, dtype=dt, device="cuda"), torch.empty_like(w)
    db = torch.empty(experts, cols, dtype=dt, device="cuda")
    ws = B.alloc_grouped_linear_workspace(x, w, n, backward=True)
    B.bytecomp_grouped_linear_forward(x, src, off, w, None, "none", y, None, ws)
    B.bytecomp_grouped_linear_backward(dy, None, x, src, off, w, "none", dx, dw, db, ws)
    X, W, D = x.double()[src.long()], w.double(), dy.double()

    def rowwise(got, a, b, k):  # [n, 1, k] [n, k, c]
        close(f64(got), f64((a[:, None] @ b)[:, 0]), dtype, f64((k + 6) * F32 * (a.abs()[:, None] @ b.abs())[:, 0]))
    for r in torch.arange(n, device="cuda").split(4000):
        rowwise(y[r], X[r], W[of[r]].transpose(1, 2).contiguous(), inner)
        rowwise(dx[r], D[r], W[of[r]], cols)
    outer, size = (torch.zeros(experts, cols, inner, dtype=torch.float64, device="cuda") for _ in range(2))
    for r in torch.arange(n, device="cuda").split(4000):
        one = D[r][:, :, None] * X[r][:, None, :]
        outer.index_add_(0, of[r], one)
        size.index_add_(0, of[r], one.abs())
    most = int(torch.bincount(of).max()) + 6
    close(f64(dw), f64(outer), dtype, f64(most * F32 * size))
    want = torch.zeros(experts, cols, dtype=torch.float64, device="cuda").index_add_(0, of, D)
    size = torch.zeros_like(want).index_add_(0, of, D.abs())
    close(f64(db), f64(want), dtype, f64(most * F32 * size))


def test_combination_past_32_bits():
    """Rows of y so far apart that their offsets, in elements, take 34 bits."""
    import torch
    from paper_2205_14465_amd import binding as B
    rows, cols, k, slots, ld = 40, 100, 2, 80, 1 << 27

    def far():
        return torch.empty((slots - 1) * ld + cols, dtype=torch.float16, device="cuda").as_strided((slots, cols), (ld, 1))
    y, dy = far(), far()
    y.normal_()
    slot = torch.randperm(slots, device="cuda").int().view(rows, k)
    weight = torch.rand(rows, k, device="cuda")
    out, dweight = torch.empty(rows, cols, dtype=torch.float16, device="cuda"), torch.empty(rows, k, device="cuda")
    B.bytecomp_combine_forward(y, slot, weight, None, out)
    Y = y.double()[slot.long()]  # [rows, k, cols]
    want, size = (weight.double()[:, :, None] * Y).sum(1), (weight.double()[:, :, None] * Y.abs()).sum(1)
    close(f64(out), f64(want), "float16", f64((k + 1) * F32 * size))
    dout = torch.randn(rows, cols, device="cuda").half()
    B.bytecomp_combine_backward(dout, y, slot, weight, dy, dweight)
    D = dout.double()[:, None, :]
    close(f64(dweight), f64((D * Y).sum(2)), "float32", f64((cols + 6) * F32 * (D * Y).abs().sum(2)))
    close(f64(dy[slot.long()]), f64(weight.double()[:, :, None] * D), "float16", 0.0)


def test_router_past_32_bits():
    import torch
    from paper_2205_14465_amd import binding as B
    rows, experts, k, ld = 70, 12, 2, 1 << 26

    def far():
        return torch.empty((rows - 1) * ld + experts, dtype=torch.bfloat16, device="cuda").as_strided((rows, experts), (ld, 1))
    logits, dlogits = far(), far()
    logits.normal_()
    near, dnear = logits.contiguous(), torch.empty(rows, experts, dtype=torch.bfloat16, device="cuda")
    results = []
    for x, d in ((logits, dlogits), (near, dnear)):
        weight, dweight = torch.empty(rows, k, device="cuda"), torch.ones(rows, k, device="cuda")
        dweight[:, 0] = 2.0
        expert, slot = (torch.empty(rows, k, dtype=torch.int32, device="cuda") for _ in range(2))
        src, off = (torch.empty(m, dtype=torch.int32, device="cuda") for m in (rows * k, experts + 1))
        B.bytecomp_route_forward(x, weight, expert, slot, src, off, B.alloc_route_workspace(rows, experts, k), False)
        B.bytecomp_route_backward(x, weight, expert, dweight, d, False)
        results.append((weight, expert, slot, src, off, d))
    for a, b in zip(*results):
        assert torch.equal(a, b)


def test_graphs_that_share_workspaces():
    """Two graphs of the same calls on other tensors and one workspace of each kind,
    replayed in turn, with eager calls on it between: each as by itself."""
    import torch
    from paper_2205_14465_amd import binding as B
    rows, experts, k, inner, cols = 900, 12, 2, 264, 392
    n = rows * k
    like = torch.empty(rows, inner, dtype=torch.float16, device="cuda")
    w = torch.randn(experts, cols, inner, device="cuda").mul(inner ** -0.5).half()
    shared = (B.alloc_route_workspace(rows, experts, k), B.alloc_grouped_linear_workspace(like, w, n, backward=True),
              B.alloc_grad_norm_workspace([w, w]))

    class Side:
        def __init__(self):
            self.x, self.dy = torch.empty_like(like), torch.empty(n, cols, dtype=torch.float16, device="cuda")
            self.logits = torch.empty(rows, experts, device="cuda")
            self.out = (torch.zeros(rows, k, device="cuda"),
                        *(torch.zeros(s, dtype=torch.int32, device="cuda") for s in ((rows, k), (rows, k), n, experts + 1)),
                        torch.zeros(n, cols, dtype=torch.float16, device="cuda"), torch.zeros(n, inner, dtype=torch.float16, device="cuda"),
                        torch.zeros(w.shape, device="cuda"), torch.zeros(experts, cols, device="cuda"),
                        torch.zeros(1, dtype=torch.float64, device="cuda"))

        def fill(self, seed):
            g = torch.Generator(device="cuda").manual_seed(seed)
            for t in (self.x, self.dy, self.logits):
                t.copy_(torch.randn(t.shape, generator=g, device="cuda"))

        def run(self, ws):
            weight, expert, slot, src, off, y, dx, dw, db, norm = self.out
            B.bytecomp_route_forward(self.logits, weight, expert, slot, src, off, ws[0])
            B.bytecomp_grouped_linear_forward(self.x, src, off, w, None, "silu", y, None, ws[1])
            B.bytecomp_grouped_linear_backward(self.dy, None, self.x, src, off, w, "none", dx, dw, db, ws[1])
            B.bytecomp_clip_grads([dw, db], [dw, db], 3.0, ws[2], norm=norm)
    sides, graphs, alone = [Side(), Side()], [], Side()
    for i, s in enumerate(sides):
        s.fill(i)
        s.run(shared)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            s.run(shared)
        graphs.append(graph)
    own = tuple(torch.empty_like(t) for t in shared)
    for i in (0, 1, 1, 0, 1, 0):
        for s, seed in ((sides[0], 10 + i), (sides[1], 20 + i)):
            s.fill(seed)
        graphs[i].replay()
        graphs[1 - i].replay()
        for j in (0, 1):
            alone.fill((10, 20)[j] + i)
            for t in alone.out:
                t.zero_()
            alone.run(own)
            torch.cuda.synchronize()
            for a, b in zip(sides[j].out, alone.out):
                assert torch.equal(a, b)
        alone.run(shared)


@pytest.mark.parametrize("rows,experts,k", [(65, 5, 5), (100, 512, 8), (128, 300, 32), (190, 257, 3), (1000, 64, 2), (1024, 64, 8),
                                            (1025, 64, 2), (4000, 64, 1), (5000, 3, 2)])
def test_order_of_the_choices(rows, experts, k):
    """Blocks of rows few enough that the last launch adds their counts up, and more:
    the slots are a stable sort by expert of the choices that there are."""
    import torch
    from paper_2205_14465_amd import binding as B
    logits = torch.randn(rows, experts, device="cuda")
    logits[torch.rand(rows, experts, device="cuda") < 0.3] = -torch.inf
    weight = torch.empty(rows, k, device="cuda")
    expert, slot = (torch.empty(rows, k, dtype=torch.int32, device="cuda") for _ in range(2))
    src = torch.full((rows * k,), -7, dtype=torch.int32, device="cuda")
    off = torch.empty(experts + 1, dtype=torch.int32, device="cuda")
    ws = B.alloc_route_workspace(rows, experts, k)
    ws.fill_(255)
    B.bytecomp_route_forward(logits, weight, expert, slot, src, off, ws)
    e = expert.view(-1).long().cpu()
    there = (e >= 0).nonzero()[:, 0]
    order = there[torch.sort(e[there], stable=True)[1]]
    want = torch.full_like(e, -1)
    want[order] = torch.arange(len(order))
    assert torch.equal(slot.view(-1).long().cpu(), want)
    assert torch.equal(src[:len(order)].long().cpu(), order // k) and bool((src[len(order):] == -7).all())
    counts = torch.bincount(e[there], minlength=experts)
    assert torch.equal(off.long().cpu(), torch.cat([torch.zeros(1, dtype=torch.long), counts.cumsum(0)]))
    best = [t[:, :k] for t in logits.sort(dim=1, descending=True, stable=True)]  # of equals the lower
    assert torch.equal(expert, torch.where(best[0] == -torch.inf, -1, best[1]).int())


@pytest.mark.parametrize("inner,cols,n", [(264, 392, 900), (1800, 376, 2889)])
def test_two_calls_at_once(inner, cols, n):
    """The same calls on two streams, on other tensors and workspaces of their own, with
    nothing between them: each as by itself."""
    import torch
    from paper_2205_14465_amd import binding as B
    counts = [n // 8 + (i == 3) * 50 - (i == 4) * 50 for i in range(8)]
    counts[7] += n - sum(counts)
    off, sides = offsets_of(counts), []
    for i in range(2):
        x, w, dy, dt = tensors(8, n, inner, cols, "bfloat16", 40 + i)
        out = (torch.empty(n, cols, dtype=dt, device="cuda"), torch.empty(n, inner, dtype=dt, device="cuda"), torch.empty_like(w),
               torch.empty(8, cols, dtype=dt, device="cuda"), torch.empty(1, dtype=torch.float64, device="cuda"))
        sides.append((x, w, dy, out, B.alloc_grouped_linear_workspace(x, w, n, backward=True),
                      B.alloc_grad_norm_workspace([w, w]), torch.cuda.Stream()))

    def run(x, w, dy, out, ws, norm_ws, stream):
        y, dx, dw, db, norm = out
        B.bytecomp_grouped_linear_forward(x, None, off, w, None, "gelu", y, None, ws, stream=stream)
        B.bytecomp_grouped_linear_backward(dy, None, x, None, off, w, "none", dx, dw, db, ws, stream=stream)
        B.bytecomp_grad_norm([dw, db], norm, norm_ws, stream=stream)
    want = []
    for s in sides:
        run(*s)
        torch.cuda.synchronize()
        want.append([t.clone() for t in s[3]])
        for t in s[3]:
            t.zero_()
    torch.cuda.synchronize()
    for _ in range(5):
        for s in sides:
            run(*s)
    torch.cuda.synchronize()
    for s, ws in zip(sides, want):
        for a, b in zip(s[3], ws):
            assert torch.equal(a, b)


# few rows, small tiles of both kinds, rows that are laid out, and the sizes above at
# which the largest tiles take the forward pass, dx and both gradients
@pytest.mark.parametrize("experts,n,inner,cols,dtype", [
    (3, 20, 64, 64, "float32"), (70, 900, 64, 72, "float32"), (200, 1700, 33, 19, "float32"), (200, 2100, 40, 24, "float16"),
    (130, 1900, 33, 19, "bfloat16"), (4, 5441, 264, 2568, "bfloat16"), (3, 8951, 1544, 264, "float16"),
    (8, 2889, 1800, 376, "bfloat16"), (300, 9257, 520, 640, "float16")])
def test_offsets_of_any_kind_leave_what_is_beside(experts, n, inner, cols, dtype):
    """Offsets that do not ascend or pass the rows: results are unspecified, but nothing
    around an output or the workspace is written."""
    import torch
    from paper_2205_14465_amd import binding as B
    beside = 1 << 16
    bufs = []

    def guarded(*shape, of):
        size = int(np.prod(shape))
        buf = torch.full((size + 2 * beside,), 7, dtype=of, device="cuda")
        bufs.append((buf, size))
        return buf[beside:beside + size].view(shape)
    x, w, dy, dt = tensors(experts, n, inner, cols, dtype, n)
    src = torch.randint(-2, n + 2, (n,), device="cuda").int()
    y, z, dx = (guarded(n, c, of=dt) for c in (cols, cols, inner))
    dw, db = guarded(experts, cols, inner, of=dt), guarded(experts, cols, of=dt)
    sizes = [B.alloc_grouped_linear_workspace(x, w, n, backward=b).numel() for b in (False, True)]
    ws = [guarded(size, of=torch.uint8) for size in sizes]
    rng = np.random.default_rng(n)
    up = np.sort(rng.integers(0, n + 1, experts + 1))
    ends = np.array([-(1 << 31), (1 << 31) - 1, 0, n, n - 1, 1, n // 2])
    for values in (up[::-1], rng.permutation(up), rng.integers(-5, n + 6, experts + 1), rng.choice(ends, experts + 1)):
        off = torch.from_numpy(values.astype(np.int32)).cuda()
        for source in (src, None):
            B.bytecomp_grouped_linear_forward(x, source, off, w, None, "gelu_tanh", y, z, ws[0] if sizes[0] else None)
            for act, pre in (("none", None), ("silu", z)):
                B.bytecomp_grouped_linear_backward(dy, pre, x, source, off, w, act, dx, dw, db, ws[1])
                B.bytecomp_grouped_linear_backward(dy, pre, x, source, off, w, act, dx, None, None, ws[1])
                B.bytecomp_grouped_linear_backward(dy, pre, x, source, off, w, act, None, dw, db, ws[1])
        torch.cuda.synchronize()
        for buf, size in bufs:
            assert bool((buf[:beside] == 7).all()) and bool((buf[beside + size:] == 7).all())
