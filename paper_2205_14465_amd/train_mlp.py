"""A data-parallel training step around the compression path, on one GPU.

A residual MLP block as transformers have it,

    y = x + W2 act(W1 layernorm(x) + b1) + b2,

is trained by W workers (taken in turn here; one process per GPU in earnest)
to imitate another such block.  Each step runs, for every worker, the layers'
forward and backward passes, whose parameter gradients come out in fp32, and
the compression with error feedback; then the aggregate of the workers'
payloads and the optimizer step: Muon for the two matrices, plain descent for
the vectors.  Nothing between the batch and the new weights is computed by
PyTorch but the loss.

    python -m paper_2205_14465_amd.train_mlp [--kind topk --ratio 0.05 ...]
"""
from __future__ import annotations

import argparse
import time

import torch

from . import binding as B

VECTORS = ("norm_weight", "norm_bias", "b1", "b2")
MATRICES = ("w1", "w2")
EPS = 1e-5


def parameters(width, hidden, seed, device="cuda"):
    """fp32 parameters of one block."""
    g = torch.Generator(device=device).manual_seed(seed)

    def normal(*shape, scale):
        return torch.randn(*shape, generator=g, device=device) * scale
    return {"norm_weight": 1 + normal(width, scale=0.1), "norm_bias": normal(width, scale=0.1),
            "w1": normal(hidden, width, scale=width ** -0.5), "b1": normal(hidden, scale=0.1),
            "w2": normal(width, hidden, scale=hidden ** -0.5), "b2": normal(width, scale=0.1)}


class Block:
    """The block's forward and backward passes for batches of `rows` rows:
    buffers and marshalled calls, made once.  x, y and dy hold a batch's input,
    output and the output's gradient; grads the parameters' gradients in fp32.
    The layers compute with a copy of the weights in `dtype`."""

    def __init__(self, params, rows, dtype, activation="gelu_tanh"):
        hidden, width = params["w1"].shape
        self.params = params
        # layer norm keeps its fp32 weights, the linear layers have theirs in dtype
        self.low = {k: params[k] if k.startswith("norm") else params[k].to(dtype) for k in params}
        self.grads = {k: torch.zeros_like(p) for k, p in params.items()}

        def buf(cols):
            return torch.empty(rows, cols, dtype=dtype, device=params["w1"].device)
        self.x, self.h, self.y, self.dy, self.dh, self.dx = (buf(width) for _ in range(6))
        self.z, self.u, self.du = (buf(hidden) for _ in range(3))
        mean, rstd = (torch.empty(rows, device=self.x.device) for _ in range(2))
        p, g = self.low, self.grads
        ln_ws = B.alloc_layernorm_workspace(rows, width)
        ws = [B.alloc_linear_workspace(a, p[w], backward=b) for a, w in ((self.h, "w1"), (self.u, "w2"))
              for b in (False, True)]
        self.forward_calls = [
            B.LayerNormCall(self.x, p["norm_weight"], p["norm_bias"], EPS, self.h, mean, rstd),
            B.LinearCall(self.h, p["w1"], p["b1"], None, activation, self.u, self.z, ws[0]),
            B.LinearCall(self.u, p["w2"], p["b2"], self.x, "none", self.y, None, ws[2])]
        self.backward_calls = [
            B.LinearGradCall(self.dy, None, self.u, p["w2"], "none", self.du, g["w2"], g["b2"], ws[3]),
            B.LinearGradCall(self.du, self.z, self.h, p["w1"], activation, self.dh, g["w1"], g["b1"], ws[1]),
            # the input's gradient by way of the layers; the residual adds dy to it
            B.LayerNormGradCall(self.dh, self.x, p["norm_weight"], mean, rstd, self.dx, g["norm_weight"],
                                g["norm_bias"], ln_ws)]

    def refresh(self):
        """The weights' copies after an optimizer step."""
        for k, p in self.params.items():
            if self.low[k] is not p:
                self.low[k].copy_(p)

    def forward(self):
        for call in self.forward_calls:
            call()

    def backward(self):
        for call in self.backward_calls:
            call()


class Trainer:
    """W workers' error feedback and payloads, the aggregate, and the
    optimizer step on one block's parameters."""

    def __init__(self, block, workers=4, kind="topk", ratio=0.05, momentum=0.95, weight_decay=0.0):
        self.block, self.workers = block, workers
        self.names = list(block.grads)
        ns = [block.grads[k].numel() for k in self.names]
        flat = [block.grads[k].view(-1) for k in self.names]
        ws = B.alloc_workspace(kind, ratio, ns, W=workers)
        self.payloads = [B.alloc_payload(kind, ratio, ns) for _ in range(workers)]
        self.residuals = [[torch.zeros(n, device=block.x.device) for n in ns] for _ in range(workers)]
        B.bytecomp_workspace_init(ws)
        self.compress = [B.CompressCall(kind, ratio, flat, self.residuals[w], self.payloads[w], ws)
                         for w in range(workers)]
        self.mean = {k: torch.empty_like(block.grads[k]) for k in self.names}
        self.aggregate = B.AggregateCall(kind, ratio, self.payloads, ns, [self.mean[k].view(-1) for k in self.names],
                                         1.0 / workers, ws)
        self.momenta = [torch.zeros_like(block.params[k]) for k in MATRICES]
        muon_ws = B.alloc_orthogonalize_workspace([tuple(block.params[k].shape) for k in MATRICES])
        self.muon = B.MuonCall([block.params[k] for k in MATRICES], [self.mean[k] for k in MATRICES], self.momenta,
                               muon_ws, momentum=momentum, weight_decay=weight_decay)

    def step(self, batches, lr, vector_lr, seed):
        """One step on a batch (x, target) per worker; returns the mean loss
        (a device tensor) before the step."""
        b, loss = self.block, 0.0
        for w, (x, target) in enumerate(batches):
            b.x.copy_(x)
            b.forward()
            error = b.y.float() - target
            loss = loss + error.square().mean() / self.workers
            b.dy.copy_(error * (2.0 / error.numel()) * self.loss_scale())
            b.backward()
            self.compress[w](seed)
        self.aggregate()
        self.muon(lr)  # the update has no scale: the gradients' does not matter
        for k in VECTORS:
            b.params[k].sub_(self.mean[k], alpha=vector_lr / self.loss_scale())
        b.refresh()
        return loss

    def loss_scale(self):
        """Keeps a mean loss's gradients in fp16's range."""
        return float(self.block.x.numel())


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--width", type=int, default=768)
    ap.add_argument("--hidden", type=int, default=1600)
    ap.add_argument("--rows", type=int, default=2048, help="rows of a worker's batch")
    ap.add_argument("--workers", type=int, default=4)
    ap.add_argument("--kind", default="topk", choices=sorted(B.KIND))
    ap.add_argument("--ratio", type=float, default=0.05)
    ap.add_argument("--dtype", default="float16", choices=["float32", "float16", "bfloat16"])
    ap.add_argument("--steps", type=int, default=100)
    ap.add_argument("--lr", type=float, default=0.02)
    ap.add_argument("--vector-lr", type=float, default=4.0)
    a = ap.parse_args(argv)
    dtype = getattr(torch, a.dtype)
    teacher = Block(parameters(a.width, a.hidden, 1), a.rows, torch.float32)
    student = Block(parameters(a.width, a.hidden, 2), a.rows, dtype)
    trainer = Trainer(student, a.workers, a.kind, a.ratio)
    gen = torch.Generator(device="cuda").manual_seed(3)
    losses = []
    for step in range(a.steps):
        batches = []
        for _ in range(a.workers):
            teacher.x.copy_(torch.randn(a.rows, a.width, generator=gen, device="cuda"))
            teacher.forward()
            batches.append((teacher.x.clone(), teacher.y.clone()))
        torch.cuda.synchronize()
        began = time.perf_counter()
        # falling to a tenth, as the update does not shrink with the gradient
        loss = trainer.step(batches, a.lr * (1 - 0.9 * step / a.steps), a.vector_lr, seed=step)
        torch.cuda.synchronize()
        losses.append(float(loss))
        if step % max(1, a.steps // 10) == 0 or step == a.steps - 1:
            print(f"step {step:4d}  loss {losses[-1]:.5f}  {1e3 * (time.perf_counter() - began):.2f} ms", flush=True)
    return losses


if __name__ == "__main__":
    main()
