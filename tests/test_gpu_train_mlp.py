"""The training example: one step without loss in the compression against the
same step in plain torch with autograd, in 64 bits, and a short run whose loss
has to fall under lossy compression."""
import pytest

pytestmark = pytest.mark.gpu


def plain_step(params, batches, lr, vector_lr, momentum):
    import torch
    from tests.test_gpu_orthogonalize import reference
    p = {k: v.double().clone().requires_grad_() for k, v in params.items()}
    loss = 0.0
    for x, target in batches:
        x = x.double()
        h = torch.nn.functional.layer_norm(x, x.shape[1:], p["norm_weight"], p["norm_bias"], 1e-5)
        u = torch.nn.functional.gelu(h.matmul(p["w1"].mT) + p["b1"], approximate="tanh")
        y = x + u.matmul(p["w2"].mT) + p["b2"]
        loss = loss + (y - target.double()).square().mean() / len(batches)
    loss.backward()
    out = {}
    for k, v in p.items():
        if v.dim() == 1:
            out[k] = v.detach() - vector_lr * v.grad
        else:  # the first step's momentum is the gradient
            u = ((1 + momentum) * v.grad).cpu().numpy()
            out[k] = v.detach() - lr * max(1.0, v.shape[0] / v.shape[1]) ** 0.5 * torch.from_numpy(reference(u)).cuda()
    return float(loss.detach()), out


def test_one_step_against_autograd():
    """fp32, every entry sent: the step's error is that of fp32 products and of
    the orthogonalised update (tests/test_gpu_orthogonalize.py), under 1e-4 of the
    largest weight by far."""
    import torch
    from paper_2205_14465_amd import train_mlp as M
    params = M.parameters(96, 160, 5)
    batches = [(torch.randn(70, 96, device="cuda"), torch.randn(70, 96, device="cuda")) for _ in range(3)]
    block = M.Block({k: v.clone() for k, v in params.items()}, 70, torch.float32)
    trainer = M.Trainer(block, workers=3, kind="topk", ratio=1.0)
    loss = float(trainer.step(batches, 0.02, 0.5, seed=1))
    want_loss, want = plain_step(params, batches, 0.02, 0.5, 0.95)
    assert abs(loss - want_loss) <= 1e-5 * want_loss
    for k in params:
        off = (block.params[k].double() - want[k]).abs().max()
        assert off <= 1e-4 * want[k].abs().max(), (k, float(off))
        assert not torch.equal(block.params[k], params[k])


@pytest.mark.parametrize("kind,ratio,dtype", [("topk", 0.05, "float16"), ("sign", 0.0, "bfloat16"),
                                              ("randk", 0.2, "float32")])
def test_training_reduces_the_loss(kind, ratio, dtype):
    from paper_2205_14465_amd import train_mlp as M
    losses = M.main(["--width", "128", "--hidden", "256", "--rows", "256", "--workers", "4", "--kind", kind, "--ratio",
                     str(ratio), "--dtype", dtype, "--steps", "60"])
    assert sum(losses[-5:]) < 0.35 * sum(losses[:5]), losses
