"""A data-parallel training step around the compression path, on one GPU.

A residual MLP block as transformers have it,

    y = x + W2 act(W1 layernorm(x) + b1) + b2,

is trained by W workers (taken in turn here; one process per GPU in earnest)
to imitate another such block.  Each step runs, for every worker, the layers'
forward and backward passes, whose parameter gradients come out in fp32, and
the compression with error feedback; then the aggregate of the workers'
payloads and the optimizer step: Muon for the two matrices, plain descent for
the vectors.  Nothing between the batch and the new weights is computed by
PyTorch but the loss.  With experts, the layers between the norm and the sum are
a block of them: each row goes through the k that a router of its own chooses,

    y = x + sum over j of weight_j (W2_e act(W1_e h + b1_e) + b2_e), e = expert_j

and with clipping the aggregate is scaled down to a largest norm before the step.

    python -m paper_2205_14465_amd.train_mlp [--kind topk --ratio 0.05 ...]
    python -m paper_2205_14465_amd.train_mlp --experts 8 --choices 2 --clip 0.1
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


def expert_parameters(width, hidden, experts, seed, device="cuda"):
    """fp32 parameters of a block of experts, each expert's along the first axis."""
    each = [parameters(width, hidden, seed + i, device) for i in range(experts)]
    out = {k: torch.stack([p[k] for p in each]) for k in ("w1", "b1", "w2", "b2")}
    g = torch.Generator(device=device).manual_seed(seed + experts)
    return {"norm_weight": each[0]["norm_weight"], "norm_bias": each[0]["norm_bias"],
            "gate": torch.randn(experts, width, generator=g, device=device) * width ** -0.5, **out}


class Block:
    """The block's forward and backward passes for batches of `rows` rows:
    buffers and marshalled calls, made once.  x, y and dy hold a batch's input,
    output and the output's gradient; grads the parameters' gradients in fp32.
    The layers compute with a copy of the weights in `dtype`."""
    matrices = MATRICES

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


class ExpertBlock(Block):
    """Block with a block of experts in the layers' place (expert_parameters); each
    row's `choices` experts are weighted by their softmax among themselves."""
    matrices = ("gate",) + MATRICES

    def __init__(self, params, rows, dtype, choices=2, activation="gelu_tanh"):
        experts, hidden, width = params["w1"].shape
        device, slots = params["w1"].device, rows * choices
        self.params = params
        self.low = {k: params[k] if k.startswith("norm") else params[k].to(dtype) for k in params}
        self.grads = {k: torch.zeros_like(p) for k, p in params.items()}

        def buf(n, cols, of=dtype):
            return torch.empty(n, cols, dtype=of, device=device)
        self.x, self.h, self.y, self.dy, self.dh, self.dx, self.dh_gate = (buf(rows, width) for _ in range(7))
        self.logits, self.dlogits = (buf(rows, experts) for _ in range(2))
        self.weight, self.dweight = (buf(rows, choices, torch.float32) for _ in range(2))
        self.expert, self.slot = (buf(rows, choices, torch.int32) for _ in range(2))
        self.source = torch.empty(slots, dtype=torch.int32, device=device)
        self.offsets = torch.empty(experts + 1, dtype=torch.int32, device=device)
        # in the order of the slots: an expert's rows one after another
        self.z, self.u, self.du = (buf(slots, hidden) for _ in range(3))
        self.ys, self.dys, self.dhs = (buf(slots, width) for _ in range(3))
        mean, rstd = (torch.empty(rows, device=device) for _ in range(2))
        p, g = self.low, self.grads
        ln_ws = B.alloc_layernorm_workspace(rows, width)
        gate_ws = [B.alloc_linear_workspace(self.h, p["gate"], backward=b) for b in (False, True)]
        ws = [B.alloc_grouped_linear_workspace(a, p[w], slots, backward=b)
              for a, w in ((self.h, "w1"), (self.u, "w2")) for b in (False, True)]
        route_ws = B.alloc_route_workspace(rows, experts, choices)
        self.forward_calls = [
            B.LayerNormCall(self.x, p["norm_weight"], p["norm_bias"], EPS, self.h, mean, rstd),
            B.LinearCall(self.h, p["gate"], None, None, "none", self.logits, None, gate_ws[0]),
            B.RouteCall(self.logits, self.weight, self.expert, self.slot, self.source, self.offsets, route_ws),
            B.GroupedLinearCall(self.h, self.source, self.offsets, p["w1"], p["b1"], activation, self.u, self.z, ws[0]),
            B.GroupedLinearCall(self.u, None, self.offsets, p["w2"], p["b2"], "none", self.ys, None, ws[2]),
            B.CombineCall(self.ys, self.slot, self.weight, self.x, self.y)]
        self.backward_calls = [
            B.CombineGradCall(self.dy, self.ys, self.slot, self.weight, self.dys, self.dweight),
            B.GroupedLinearGradCall(self.dys, None, self.u, None, self.offsets, p["w2"], "none", self.du, g["w2"],
                                    g["b2"], ws[3]),
            B.GroupedLinearGradCall(self.du, self.z, self.h, self.source, self.offsets, p["w1"], activation, self.dhs,
                                    g["w1"], g["b1"], ws[1]),
            B.RouteGradCall(self.logits, self.weight, self.expert, self.dweight, self.dlogits),
            B.LinearGradCall(self.dlogits, None, self.h, p["gate"], "none", self.dh_gate, g["gate"], None, gate_ws[1]),
            # a row's gradient: of its choices' rows and of its logits
            B.CombineCall(self.dhs, self.slot, None, self.dh_gate, self.dh),
            B.LayerNormGradCall(self.dh, self.x, p["norm_weight"], mean, rstd, self.dx, g["norm_weight"],
                                g["norm_bias"], ln_ws)]


class Trainer:
    """W workers' error feedback and payloads, the aggregate, and the
    optimizer step on one block's parameters.  clip: the largest norm of the
    aggregate (None: any)."""

    def __init__(self, block, workers=4, kind="topk", ratio=0.05, momentum=0.95, weight_decay=0.0, clip=None):
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
        self.clip = None
        if clip is not None:
            means = list(self.mean.values())
            self.clip = B.ClipGradsCall(means, means, clip * self.loss_scale(), B.alloc_grad_norm_workspace(means))

        def matrices(of):  # each expert's by itself
            return [m for k in block.matrices for m in (of[k].unbind() if of[k].dim() == 3 else [of[k]])]
        weights = matrices(block.params)
        self.momenta = [torch.zeros_like(w) for w in weights]
        muon_ws = B.alloc_orthogonalize_workspace([tuple(w.shape) for w in weights])
        self.muon = B.MuonCall(weights, matrices(self.mean), self.momenta, muon_ws, momentum=momentum,
                               weight_decay=weight_decay)

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
        if self.clip:
            self.clip()
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
    ap.add_argument("--experts", type=int, default=0, help="of the student; 0: two layers for every row")
    ap.add_argument("--choices", type=int, default=2, help="experts a row")
    ap.add_argument("--clip", type=float, help="largest norm of the aggregate (default: any)")
    a = ap.parse_args(argv)
    dtype = getattr(torch, a.dtype)
    teacher = Block(parameters(a.width, a.hidden, 1), a.rows, torch.float32)
    if a.experts:
        student = ExpertBlock(expert_parameters(a.width, a.hidden, a.experts, 2), a.rows, dtype, a.choices)
    else:
        student = Block(parameters(a.width, a.hidden, 2), a.rows, dtype)
    trainer = Trainer(student, a.workers, a.kind, a.ratio, clip=a.clip)
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
