"""Rows so far apart that their offsets pass 32 bits (in elements): every
operator gives the same bits as on close rows, and writes only its own."""
import pytest

pytestmark = pytest.mark.gpu
LD, ROWS = (1 << 26) + 8, 70


@pytest.fixture(scope="module")
def space():
    import torch
    buf = torch.empty((ROWS - 1) * LD + 4096, dtype=torch.float16, device="cuda")
    assert (ROWS - 1) * LD > 1 << 32
    yield buf
    del buf
    torch.cuda.empty_cache()


def far(space, at, like):
    """A view with rows LD apart that holds what `like` does."""
    v = space.as_strided(like.shape, (LD, 1), at)
    v.copy_(like)
    return v


def near(rows, cols, seed):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(rows, cols, generator=g, device="cuda").half()


def test_layer_norm(space):
    import torch
    from paper_2205_14465_amd import binding as B
    x, dy, w = near(ROWS, 328, 1), near(ROWS, 328, 2), torch.randn(328, device="cuda")
    out = []
    for spread in (False, True):
        place = (lambda at, t: far(space, at, t)) if spread else (lambda at, t: t.clone())
        a, d, y, dx = place(0, x), place(512, dy), place(1024, torch.zeros_like(x)), place(1536, torch.zeros_like(x))
        mean, rstd = torch.empty(ROWS, device="cuda"), torch.empty(ROWS, device="cuda")
        dw, db = torch.empty_like(w), torch.empty_like(w)
        B.bytecomp_layernorm_forward(a, w, None, 1e-5, y, mean, rstd)
        B.bytecomp_layernorm_backward(d, a, w, mean, rstd, dx, dw, db, B.alloc_layernorm_workspace(ROWS, 328))
        out.append([t.clone() for t in (y, dx, dw, db, mean, rstd)])
    assert all(torch.equal(p, q) for p, q in zip(*out))


@pytest.mark.parametrize("rows", [3, 40, 70])
def test_linear(space, rows):
    import torch
    from paper_2205_14465_amd import binding as B
    x, w, dy, res = near(rows, 128, 1), near(ROWS, 128, 2), near(rows, ROWS, 3), near(rows, ROWS, 4)
    out = []
    for spread in (False, True):
        place = (lambda at, t: far(space, at, t)) if spread else (lambda at, t: t.clone())
        a, b, d, r = place(0, x), place(256, w), place(512, dy), place(768, res)
        y, z = place(1024, torch.zeros_like(res)), place(1280, torch.zeros_like(res))
        dx, dw = place(1536, torch.zeros_like(x)), place(1792, torch.zeros_like(w))
        B.bytecomp_linear_forward(a, b, None, r, "silu", y, z, B.alloc_linear_workspace(a, b))
        B.bytecomp_linear_backward(d, z, a, b, "silu", dx, dw, None, B.alloc_linear_workspace(a, b, backward=True))
        out.append([t.clone() for t in (y, z, dx, dw)])
    assert all(torch.equal(p, q) for p, q in zip(*out))


def test_orthogonalize(space):
    import torch
    from paper_2205_14465_amd import binding as B
    u = near(ROWS, 300, 5)
    got = torch.empty_like(u)
    ws = B.alloc_orthogonalize_workspace([u.shape])
    B.bytecomp_orthogonalize([u], [got], ws)
    a, o = far(space, 0, u), far(space, 512, torch.zeros_like(u))
    B.bytecomp_orthogonalize([a], [o], ws)
    assert torch.equal(o, got)
