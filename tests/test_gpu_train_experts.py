"""The block of experts and the clipping as the training example runs them:
forward, gradients and a whole step against the same in plain torch with
autograd, in 64 bits; the gradients against differences; captured and replayed."""
import pytest

pytestmark = pytest.mark.gpu

WIDTH, HIDDEN = 96, 160


@pytest.fixture(autouse=True)
def seeded():
    import torch
    torch.manual_seed(17)


def plain(params, x, expert):
    """The block's output in 64 bits, each row's experts given."""
    import torch
    p = {k: v.double().clone().requires_grad_() for k, v in params.items()}
    x = x.double()
    h = torch.nn.functional.layer_norm(x, x.shape[1:], p["norm_weight"], p["norm_bias"], 1e-5)
    logits = h.matmul(p["gate"].mT)
    weight = logits.gather(1, expert.long()).softmax(1)
    y = x
    for j in range(expert.shape[1]):
        out = torch.zeros_like(x)
        for e in range(logits.shape[1]):
            rows = (expert[:, j] == e).nonzero()[:, 0]
            u = torch.nn.functional.gelu(h[rows].matmul(p["w1"][e].mT) + p["b1"][e], approximate="tanh")
            out = out.index_add(0, rows, u.matmul(p["w2"][e].mT) + p["b2"][e])
        y = y + weight[:, j:j + 1] * out
    return p, logits, y


def largest(t):
    return float(t.detach().abs().max()) if t.numel() else 0.0


def close(got, want, name):
    """fp32: a chain of at most seven products of sums of n <= 640 random terms,
    each product off by n^0.5 2^-24 of its terms' magnitudes, themselves n^0.5 of
    the sum: 7 x 640 x 2^-24 = 2.7e-4 of the largest."""
    off = largest(got.double() - want)
    assert off <= 3e-4 * largest(want), (name, off, largest(want))


def block_of(rows, experts, choices, seed, dtype="float32"):
    import torch
    from paper_2205_14465_amd import train_mlp as M
    params = M.expert_parameters(WIDTH, HIDDEN, experts, seed)
    block = M.ExpertBlock(params, rows, getattr(torch, dtype), choices)
    g = torch.Generator(device="cuda").manual_seed(seed + 100)
    block.x.copy_(torch.randn(rows, WIDTH, generator=g, device="cuda"))
    block.dy.copy_(torch.randn(rows, WIDTH, generator=g, device="cuda"))
    return params, block


@pytest.mark.parametrize("rows,experts,choices", [(1, 4, 2), (3, 8, 8), (70, 8, 2), (300, 5, 1), (129, 64, 4)])
def test_against_autograd(rows, experts, choices):
    import torch
    params, block = block_of(rows, experts, choices, seed=rows)
    block.forward()
    block.backward()
    p, logits, y = plain(params, block.x, block.expert)
    # the choices: no logit left out is above one chosen, but by the logits' error
    chosen = logits.detach().gather(1, block.expert.long())
    rest = logits.detach().scatter(1, block.expert.long(), -torch.inf)
    assert float((rest.amax(1) - chosen.amin(1)).amax()) <= 3e-4 * largest(logits)
    close(block.y, y.detach(), "y")
    y.backward(block.dy.double())
    for k in params:
        close(block.grads[k], p[k].grad, k)


def test_gradient_against_differences():
    """Of L = sum of dy y along one direction of the experts' weights (which choices
    do not depend on).  Two fp32 losses of rows x width = 6720 terms of about 1 are
    off by 6720^0.5 2^-22 = 2e-5 each, over 2 h = 0.1: 4e-4; the third derivative
    adds h^2 / 6 of its own size, under 1e-3 of the slope's for these scales."""
    import torch
    h, names = 0.05, ("w1", "b1", "w2", "b2")
    params, block = block_of(70, 8, 2, seed=7)
    block.forward()
    block.backward()
    g = torch.Generator(device="cuda").manual_seed(1)
    way = {k: torch.randn(params[k].shape, generator=g, device="cuda") for k in names}
    norm = sum(float(v.square().sum()) for v in way.values()) ** 0.5
    slope = sum(float((block.grads[k].double() * way[k] / norm).sum()) for k in names)
    size = sum(float(block.grads[k].double().square().sum()) for k in names) ** 0.5
    start = {k: params[k].clone() for k in names}
    loss = []
    for sign in (1, -1):
        for k in names:
            params[k].copy_(start[k] + sign * h / norm * way[k])
        block.refresh()
        block.forward()
        loss.append(float((block.y.double() * block.dy.double()).sum()))
    assert abs((loss[0] - loss[1]) / (2 * h) - slope) <= 4e-4 + 1e-3 * size, (loss, slope, size)


@pytest.mark.parametrize("clip", [1e-3, 1e3])
def test_one_step_against_autograd(clip):
    """fp32, every entry sent, two workers: the step is that of the clipped mean
    gradient (the vectors' part shows the clipping; the matrices' update has no scale)."""
    import torch
    from paper_2205_14465_amd import train_mlp as M
    from tests.test_gpu_orthogonalize import reference
    rows, experts, choices, lr, vector_lr = 70, 4, 2, 0.02, 0.5
    params = M.expert_parameters(WIDTH, HIDDEN, experts, 5)
    batches = [(torch.randn(rows, WIDTH, device="cuda"), torch.randn(rows, WIDTH, device="cuda")) for _ in range(2)]
    block = M.ExpertBlock({k: v.clone() for k, v in params.items()}, rows, torch.float32, choices)
    chosen = []
    for x, _ in batches:
        block.x.copy_(x)
        block.forward()
        chosen.append(block.expert.clone())
    trainer = M.Trainer(block, workers=2, kind="topk", ratio=1.0, clip=clip)
    loss = float(trainer.step(batches, lr, vector_lr, seed=1))
    want_loss, grad = 0.0, {k: 0.0 for k in params}
    for (x, target), expert in zip(batches, chosen):
        p, _, y = plain(params, x, expert)
        one = (y - target.double()).square().mean() / 2
        one.backward()
        want_loss += float(one.detach())
        grad = {k: grad[k] + (p[k].grad if p[k].grad is not None else 0.0) for k in params}
    assert abs(loss - want_loss) <= 1e-5 * want_loss
    norm = sum(float(v.square().sum()) for v in grad.values()) ** 0.5
    assert clip == 1e3 or norm > 10 * clip
    c = min(1.0, clip / norm)
    for k in M.VECTORS:
        moved = block.params[k].double() - params[k].double()
        # the weights are rounded to 24 bits
        off = largest(moved + vector_lr * c * grad[k])
        assert off <= 3e-4 * vector_lr * c * largest(grad[k]) + 2 * 2.0 ** -24 * largest(params[k]), (k, off)
    for k in block.matrices:
        for i, m in enumerate(grad[k] if grad[k].dim() == 3 else grad[k][None]):
            w = params[k][i] if grad[k].dim() == 3 else params[k]
            got = block.params[k][i] if grad[k].dim() == 3 else block.params[k]
            u = torch.from_numpy(reference((1.95 * c * m).cpu().numpy())).cuda()
            want = w.double() - lr * max(1.0, m.shape[0] / m.shape[1]) ** 0.5 * u
            assert largest(got.double() - want) <= 1e-4 * largest(want), (k, i)


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
def test_captured_and_replayed(dtype):
    """Forward, backward and clipping in one graph, replayed on other batches with
    eager work between: every replay as the eager pass, bit for bit."""
    import torch
    from paper_2205_14465_amd import binding as B
    from paper_2205_14465_amd import train_mlp as M
    rows, experts, choices = 200, 8, 2
    params = M.expert_parameters(WIDTH, HIDDEN, experts, 11)
    stream = torch.cuda.Stream()
    eager = M.ExpertBlock(params, rows, getattr(torch, dtype), choices)
    graph = torch.cuda.CUDAGraph()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        block = M.ExpertBlock(params, rows, getattr(torch, dtype), choices)
        grads = list(block.grads.values())
        clipped = [torch.zeros_like(v) for v in grads]
        norm = torch.zeros(1, dtype=torch.float64, device="cuda")
        clip = B.ClipGradsCall(grads, clipped, 2.0, B.alloc_grad_norm_workspace(grads), norm=norm)

        def run():
            block.forward()
            block.backward()
            clip()
        for t in (block.x, block.dy):
            t.normal_()
        run()
        stream.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            run()
    out, want_norm = [torch.zeros_like(v) for v in grads], torch.zeros_like(norm)
    theirs = list(eager.grads.values())
    ws = B.alloc_grad_norm_workspace(theirs)
    for i in range(4):
        g = torch.Generator(device="cuda").manual_seed(i)
        x, dy = (torch.randn(rows, WIDTH, generator=g, device="cuda") for _ in range(2))
        for b in (block, eager):
            b.x.copy_(x)
            b.dy.copy_(dy)
        eager.forward()
        eager.backward()
        B.ClipGradsCall(theirs, out, 2.0, ws, norm=want_norm)()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(block.y, eager.y) and torch.equal(block.dx, eager.dx)
        assert torch.equal(norm, want_norm) and float(norm) > 2.0
        for got, want in zip(clipped, out):
            assert torch.equal(got, want)


@pytest.mark.parametrize("kind,dtype", [("topk", "float16"), ("sign", "bfloat16")])
def test_the_command_runs(kind, dtype):
    from paper_2205_14465_amd import train_mlp as M
    losses = M.main(["--width", "128", "--hidden", "256", "--rows", "256", "--workers", "2", "--kind", kind, "--ratio",
                     "0.05", "--dtype", dtype, "--steps", "5", "--experts", "8", "--choices", "2", "--clip", "0.1"])
    assert len(losses) == 5 and all(v == v and v < 1e3 for v in losses), losses
