"""A block of experts around the compression path, as calls to measure: the
router (softmax gate, choice of experts, order of the rows by expert), the
linear layer grouped by expert over ragged runs of rows, the combination of a
row's experts, each with its gradients; and the global norm of a list of
gradients with clipping, between the aggregate and the optimizer step.

A case names an operator and its sizes.  `prepare` makes what a training or
serving program has in hand before the call, `run` makes one call: with `own`
false in elementary torch operations in 32 bits (sums of squares over whole
models in 64), with `own` true through the library's entry points.  `exact`
gives the same results from the operators' definitions in 64 bits, `work` the
bytes and operations of one call that no implementation can do without.
"""
import math

import torch

own = False

DTYPE = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
ACTIVATIONS = ("none", "relu", "gelu", "gelu_tanh", "silu")

# Parameter tensors as "rows x columns" or a length, "*n" n of them: GPT-2-XL, and the
# 161 tensors of ResNet-50 (convolutions and the head as matrices, two vectors for
# each norm).
GPT2XL = "50257x1600,1024x1600,1600*2," + ",".join(
    ["1600*2,1600x4800,4800,1600x1600,1600,1600*2,1600x6400,6400,6400x1600,1600"] * 48)
RESNET50 = ("64x147,64*2,64x64,64*2,64x576*3,64*6,256x64*4,256*8,64x256*2,64*4,128x256,128*2,128x1152*4,128*8,"
            "512x128*4,512*8,512x256,512*2,128x512*3,128*6,256x512,256*2,256x2304*6,256*12,1024x256*6,1024*12,"
            "1024x512,1024*2,256x1024*5,256*10,512x1024,512*2,512x4608*3,512*6,2048x512*3,2048*6,2048x1024,2048*2,"
            "512x2048*2,512*4,1000x2048,1000")


def listed():
    return [
        # one token of a decoder through the router of 64 experts: nothing but latency
        {"name": "route_fwd_1x64_k8_bf16", "op": "route_forward", "dtype": "bf16", "tokens": 1, "masked": 0,
         "experts": 64, "k": 8, "normalise": True},
        # a training batch of 16 x 1024 tokens, the last sequences padded
        {"name": "route_fwd_16384x64_k2_bf16", "op": "route_forward", "dtype": "bf16", "tokens": 16384, "masked": 700,
         "experts": 64, "k": 2, "normalise": True},
        # the router's gradient over a ragged batch, gate weights as the softmax has them
        {"name": "route_bwd_8191x129_k4_f32", "op": "route_backward", "dtype": "f32", "tokens": 8191, "masked": 63,
         "experts": 129, "k": 4, "normalise": False},
        # a GPT-2-XL-wide batch of 8 x 1024 tokens: the experts' results and the residual
        {"name": "combine_fwd_8192x1600_k2_bf16", "op": "combine_forward", "dtype": "bf16", "tokens": 8192, "masked": 0,
         "experts": 16, "k": 2, "cols": 1600, "weighted": True, "residual": True},
        # its gradient, an odd width and a padded batch
        {"name": "combine_bwd_8000x1001_k2_f16", "op": "combine_backward", "dtype": "f16", "tokens": 8000, "masked": 321,
         "experts": 16, "k": 2, "cols": 1001},
        # one token through the second projections of two of eight experts: their
        # 41 MB of weights are what has to be read
        {"name": "grouped_fwd_1x6400x1600_k2_f16", "op": "grouped_forward", "dtype": "f16", "tokens": 1, "masked": 0,
         "experts": 8, "k": 2, "inner": 6400, "cols": 1600, "act": "none", "gather": False, "save": False},
        # the first projections over a training batch, rows gathered from the tokens
        {"name": "grouped_fwd_16384x1600x6400_e16_bf16", "op": "grouped_forward", "dtype": "bf16", "tokens": 8192,
         "masked": 0, "experts": 16, "k": 2, "inner": 1600, "cols": 6400, "act": "gelu_tanh", "gather": True,
         "save": True},
        # fp32 experts of odd sizes on a ragged, padded batch
        {"name": "grouped_fwd_2474x1001x515_e5_f32", "op": "grouped_forward", "dtype": "f32", "tokens": 1237,
         "masked": 37, "experts": 5, "k": 2, "inner": 1001, "cols": 515, "act": "relu", "gather": True, "save": True},
        # the gradients of the first projections
        {"name": "grouped_bwd_16384x1600x6400_e16_bf16", "op": "grouped_backward", "dtype": "bf16", "tokens": 8192,
         "masked": 0, "experts": 16, "k": 2, "inner": 1600, "cols": 6400, "act": "gelu_tanh", "gather": True},
        # the gradients of eight BERT-base-wide experts in fp32, eight sequences of 128
        {"name": "grouped_bwd_2048x768x768_e8_f32", "op": "grouped_backward", "dtype": "f32", "tokens": 1024,
         "masked": 0, "experts": 8, "k": 2, "inner": 768, "cols": 768, "act": "none", "gather": True},
        # ResNet-50's gradients as most steps find them, under the threshold: read, not written
        {"name": "clip_resnet50_f32", "op": "clip", "dtype": "f32", "list": RESNET50, "kind": "l2", "over": 0.5,
         "apart": False},
        # GPT-2-XL's aggregate clipped into the buffers that the optimizer reads: the largest call
        {"name": "clip_gpt2xl_f32", "op": "clip", "dtype": "f32", "list": GPT2XL, "kind": "l2", "over": 3.0,
         "apart": True},
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm, odd as often as even."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["route_forward", "route_backward", "combine_forward", "combine_backward", "grouped_forward",
                     "grouped_backward", "clip"])
    case = {"op": op, "dtype": rng.choice(["f32", "f16", "bf16"])}
    if op == "clip":
        tensors, left = [], 1 << 29
        for _ in range(_log(rng, 1, 24)):
            n = rng.choice([1, 1, 2, 5, 12])
            rows, cols = _log(rng, 1, 8192), _log(rng, 1, 8192)
            while rows * cols * n > left:
                rows, cols = max(1, rows // 2), max(1, cols // 2)
            left -= rows * cols * n
            tensors.append(("%dx%d" % (rows, cols) if rng.random() < 0.7 else "%d" % (rows * cols)) + "*%d" % n)
        # (clipped in place, a second pass would find other gradients)
        over = rng.choice([0.5, 3.0])
        return case | {"list": ",".join(tensors), "kind": rng.choice(["l2", "l2", "max"]), "over": over,
                       "apart": over > 1 or rng.random() < 0.5}
    tokens = _log(rng, 1, 16384)
    case |= {"tokens": tokens, "masked": rng.choice([0, 0, tokens // 5])}
    if op.startswith("route"):
        experts = _log(rng, 2, 256)
        return case | {"experts": experts, "k": rng.randint(1, min(8, experts)), "normalise": rng.random() < 0.5}
    experts = _log(rng, 2, 64)
    case |= {"experts": experts, "k": rng.randint(1, min(4, experts))}
    if op.startswith("combine"):
        case["cols"] = _log(rng, 16, min(8192, (1 << 26) // (tokens * case["k"])))
        if op == "combine_forward":
            case |= {"weighted": rng.random() < 0.7, "residual": rng.random() < 0.5}
        return case
    # widths from a small head to GPT-2-XL's MLP, half of them multiples of 64 as
    # models have them, half of any value
    snap = 64 if rng.random() < 0.5 else 1
    inner, cols = (max(snap, snap * (_log(rng, 64, 6400) // snap)) for _ in range(2))
    case["experts"] = max(2, min(experts, (1 << 27) // (inner * cols)))
    case["k"] = min(case["k"], case["experts"])
    most = (1 << 37) // (inner * cols * case["k"])
    case["tokens"] = max(1, min(tokens, 8192, most))
    case["masked"] = min(case["masked"], case["tokens"] // 5)
    case |= {"inner": inner, "cols": cols, "act": rng.choice(ACTIVATIONS), "gather": rng.random() < 0.5}
    if op == "grouped_forward":
        case["save"] = rng.random() < 0.5
    return case


def _shapes(text):
    out = []
    for part in text.split(","):
        shape, _, n = part.partition("*")
        out += [tuple(int(v) for v in shape.split("x"))] * int(n or 1)
    return out


# ------------------------------------------------------------------- inputs

def _logits(case, g):
    """Gate logits: some experts are liked more than others; the padding's rows are
    masked out, at the batch's end."""
    n, e = case["tokens"], case["experts"]
    x = torch.randn(n, e, generator=g, device="cuda") + 0.5 * torch.randn(e, generator=g, device="cuda")
    x[n - case["masked"]:] = float("-inf")
    return x


def _routing(case, g):
    """What the router leaves for the calls behind it."""
    r = _plain_route(_logits(case, g), case["k"], True)
    return r | {"counts": (r["offsets"][1:] - r["offsets"][:-1]).tolist()}


def _flat(shapes, dtype):
    """A zeroed buffer and the tensors that lie in it one after the other, each at a multiple of 64 elements."""
    sizes = [-(-math.prod(shape) // 64) * 64 for shape in shapes]
    flat = torch.zeros(sum(sizes), dtype=dtype, device="cuda")
    return flat, [t[:math.prod(shape)].view(shape) for t, shape in zip(flat.split(sizes), shapes)]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = DTYPE[case["dtype"]]

    def normal(*shape, scale=1.0, dtype=dt):
        return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)

    op, s = case["op"], {"case": case}
    if op == "clip":
        shapes = _shapes(case["list"])
        # gradients of tensors whose sizes differ by orders of magnitude
        scale = (1e-3 * torch.exp(torch.randn(len(shapes), generator=g, device="cuda"))).tolist()
        # views of one flat buffer, as a data-parallel program keeps them
        flat, s["grad"] = _flat(shapes, dt)
        for t, c in zip(s["grad"], scale):
            t.copy_(normal(*t.shape, scale=c))
        s["flat"], s["out"] = _flat(shapes, dt) if case["apart"] else (flat, s["grad"])
        # about what the norm will be, and the threshold in its proportion
        if case["kind"] == "l2":
            near = math.sqrt(sum(c * c * math.prod(shape) for shape, c in zip(shapes, scale)))
        else:
            near = max(c * math.sqrt(2 * math.log(math.prod(shape) + 1)) for shape, c in zip(shapes, scale))
        s["max_norm"] = near / case["over"]
        s["norm"] = torch.zeros(1, dtype=torch.float64, device="cuda")
        s["factor"] = torch.zeros(1, device="cuda")
        return s
    n, k = case["tokens"], case["k"]
    if op.startswith("route"):
        s["logits"] = _logits(case, g).to(dt)
        if op == "route_forward":
            def ints(*shape):
                return torch.zeros(*shape, dtype=torch.int32, device="cuda")
            s |= {"weight": torch.zeros(n, k, device="cuda"), "expert": ints(n, k), "slot": ints(n, k),
                  "source": ints(n * k), "offsets": ints(case["experts"] + 1)}
        else:
            s |= _plain_route(s["logits"], k, case["normalise"])
            s["dweight"] = normal(n, k, scale=0.05, dtype=torch.float32)
            s["dlogits"] = torch.empty_like(s["logits"])
        return s
    s |= _routing(case, g)
    rows = n * k
    if op.startswith("combine"):
        cols = case["cols"]
        s["y"] = normal(rows, cols)
        if op == "combine_forward":
            s["residual"] = normal(n, cols) if case["residual"] else None
            s["out"] = torch.empty(n, cols, dtype=dt, device="cuda")
        else:
            s["dout"] = normal(n, cols, scale=0.05)
            s["dy"] = torch.zeros(rows, cols, dtype=dt, device="cuda")
            s["dweight"] = torch.empty(n, k, device="cuda")
        return s
    inner, cols, experts = case["inner"], case["cols"], case["experts"]
    s["x"] = normal(n if case["gather"] else rows, inner)
    s["w"] = normal(experts, cols, inner, scale=1 / math.sqrt(inner))
    if op == "grouped_forward":
        s["bias"] = normal(experts, cols, scale=0.1)
        s["y"] = torch.zeros(rows, cols, dtype=dt, device="cuda")
        s["z"] = torch.zeros_like(s["y"]) if case["save"] else None
    else:
        s["z"] = normal(rows, cols) if case["act"] != "none" else None
        s["dy"] = normal(rows, cols, scale=0.05)
        s["dx"] = torch.zeros(rows, inner, dtype=dt, device="cuda")
        s["dw"] = torch.empty_like(s["w"])
        s["dbias"] = torch.empty(experts, cols, dtype=dt, device="cuda")
    return s


# --------------------------------------------------------------- plain forms

def _act(name, z):
    if name == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if name == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if name == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))
    if name == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _act_slope(name, z):
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    if name == "gelu_tanh":
        c = math.sqrt(2 / math.pi)
        t = torch.tanh(c * (z + 0.044715 * z * z * z))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 3 * 0.044715 * z * z)
    if name == "silu":
        p = 1 / (1 + torch.exp(-z))
        return p * (1 + z * (1 - p))
    return torch.ones_like(z)


def _chances(x):
    """Softmax over the rows; rows masked out whole have none."""
    top = x.max(1, keepdim=True).values
    e = torch.exp(x - torch.where(top == float("-inf"), torch.zeros_like(top), top))
    total = e.sum(1, keepdim=True)
    return e / torch.where(total == 0, torch.ones_like(total), total)


def _plain_route(logits, k, normalise):
    n, experts = logits.shape
    x = logits.float()
    value, order = torch.sort(x, dim=1, descending=True, stable=True)
    value, order = value[:, :k], order[:, :k]
    there = value > float("-inf")
    weight = torch.where(there, torch.gather(_chances(x), 1, order), torch.zeros_like(value))
    if normalise:
        total = weight.sum(1, keepdim=True)
        weight = weight / torch.where(total == 0, torch.ones_like(total), total)
    expert = torch.where(there, order, torch.full_like(order, -1))
    # choices in the order of their experts, rows in their own within each
    place = torch.where(there, order, torch.full_like(order, experts)).view(-1)
    by = torch.sort(place, stable=True).indices
    total = there.sum()
    slot = torch.empty_like(by)
    slot[by] = torch.arange(n * k, device=by.device)
    source = torch.where(torch.arange(n * k, device=by.device) < total, by // k, torch.zeros_like(by))
    each = (place[:, None] == torch.arange(experts, device=by.device)).sum(0)
    offsets = torch.cat([each.new_zeros(1), torch.cumsum(each, 0)])
    return {"weight": weight, "expert": expert.int(), "slot": torch.where(there, slot.view(n, k), -1).int(),
            "source": source.int(), "offsets": offsets.int()}


def _plain_route_backward(s):
    chosen = (s["expert"] >= 0).float()
    at = s["expert"].clamp(min=0).long()
    if s["case"]["normalise"]:
        dot = (s["weight"] * s["dweight"]).sum(1, keepdim=True)
        d = torch.zeros(s["logits"].shape, device="cuda")
        d.scatter_add_(1, at, chosen * s["weight"] * (s["dweight"] - dot))
    else:
        p = _chances(s["logits"].float())
        d = torch.zeros_like(p).scatter_add_(1, at, chosen * s["dweight"])
        d = p * (d - (p * d).sum(1, keepdim=True))
    return {"dlogits": d.to(s["logits"].dtype)}


def _plain_combine(s):
    case = s["case"]
    there = (s["slot"] >= 0)[:, :, None]
    at = s["slot"].clamp(min=0).long()
    out = s["residual"].float() if case.get("residual") else torch.zeros(s["out"].shape, device="cuda")
    for j in range(case["k"]):
        part = torch.where(there[:, j], s["y"][at[:, j]].float(), torch.zeros((), device="cuda"))
        out = out + (part * s["weight"][:, j, None] if case["weighted"] else part)
    return {"out": out.to(s["y"].dtype)}


def _plain_combine_backward(s):
    dout = s["dout"].float()
    dy = torch.zeros(s["y"].shape, device="cuda")
    dweight = torch.zeros(s["slot"].shape, device="cuda")
    for j in range(s["case"]["k"]):
        rows = torch.nonzero(s["slot"][:, j] >= 0)[:, 0]
        at = s["slot"][rows, j].long()
        dy[at] = dout[rows] * s["weight"][rows, j, None]
        dweight[rows, j] = (dout[rows] * s["y"][at].float()).sum(1)
    return {"dy": dy.to(s["y"].dtype), "dweight": dweight}


def _plain_grouped(s):
    case = s["case"]
    y = torch.zeros(s["y"].shape, device="cuda")
    z = torch.zeros_like(y)
    at = 0
    for e, n in enumerate(s["counts"]):
        x = s["x"][s["source"][at:at + n].long()] if case["gather"] else s["x"][at:at + n]
        z[at:at + n] = x.float() @ s["w"][e].float().t() + s["bias"][e].float()
        at += n
    y[:at] = _act(case["act"], z[:at])
    dt = s["x"].dtype
    return {"y": y.to(dt), "z": z.to(dt)} if case["save"] else {"y": y.to(dt)}


def _plain_grouped_backward(s):
    case = s["case"]
    dx = torch.zeros(s["dx"].shape, device="cuda")
    dw = torch.zeros(s["dw"].shape, device="cuda")
    dbias = torch.zeros(s["dbias"].shape, device="cuda")
    dz = s["dy"].float()
    if case["act"] != "none":
        dz = dz * _act_slope(case["act"], s["z"].float())
    at = 0
    for e, n in enumerate(s["counts"]):
        x = s["x"][s["source"][at:at + n].long()] if case["gather"] else s["x"][at:at + n]
        d = dz[at:at + n]
        dx[at:at + n] = d @ s["w"][e].float()
        dw[e] = d.t() @ x.float()
        dbias[e] = d.sum(0)
        at += n
    dt = s["x"].dtype
    return {"dx": dx.to(dt), "dw": dw.to(dt), "dbias": dbias.to(dt)}


def _plain_clip(s):
    if s["case"]["kind"] == "l2":
        norm = torch.stack([g.double().square().sum() for g in s["grad"]]).sum().sqrt()
    else:
        norm = torch.stack([g.abs().max() for g in s["grad"]]).max().double()
    factor = torch.where(norm > s["max_norm"], s["max_norm"] / norm, torch.ones_like(norm)).float()
    for g, o in zip(s["grad"], s["out"]):
        if g.dtype == torch.float32:
            torch.mul(g, factor, out=o)
        else:
            o.copy_(g.float() * factor)
    return {"flat": s["flat"], "norm": norm.view(1), "factor": factor.view(1)}


def _plain(s):
    op = s["case"]["op"]
    if op == "route_forward":
        return _plain_route(s["logits"], s["case"]["k"], s["case"]["normalise"])
    return {"route_backward": _plain_route_backward, "combine_forward": _plain_combine,
            "combine_backward": _plain_combine_backward, "grouped_forward": _plain_grouped,
            "grouped_backward": _plain_grouped_backward, "clip": _plain_clip}[op](s)


# ---------------------------------------------------------- the library's calls

def _call(s):
    """The call with its arguments marshalled once and its workspace, as a program keeps it for a layer."""
    from paper_2205_14465_amd import binding as B
    case, op = s["case"], s["case"]["op"]
    if op == "route_forward":
        ws = B.alloc_route_workspace(case["tokens"], case["experts"], case["k"])
        return B.RouteCall(s["logits"], s["weight"], s["expert"], s["slot"], s["source"], s["offsets"], ws,
                           normalise=case["normalise"])
    if op == "route_backward":
        return B.RouteGradCall(s["logits"], s["weight"], s["expert"], s["dweight"], s["dlogits"],
                               normalise=case["normalise"])
    if op == "combine_forward":
        return B.CombineCall(s["y"], s["slot"], s["weight"] if case["weighted"] else None, s["residual"], s["out"])
    if op == "combine_backward":
        return B.CombineGradCall(s["dout"], s["y"], s["slot"], s["weight"], s["dy"], s["dweight"])
    if op == "clip":
        ws = B.alloc_grad_norm_workspace(s["grad"])
        return B.ClipGradsCall(s["grad"], s["out"], s["max_norm"], ws, kind=case["kind"], norm=s["norm"],
                               factor=s["factor"])
    source = s["source"] if case["gather"] else None
    ws = B.alloc_grouped_linear_workspace(s["x"], s["w"], case["tokens"] * case["k"],
                                          backward=op == "grouped_backward")
    if op == "grouped_forward":
        return B.GroupedLinearCall(s["x"], source, s["offsets"], s["w"], s["bias"], case["act"], s["y"], s["z"], ws)
    return B.GroupedLinearGradCall(s["dy"], s["z"], s["x"], source, s["offsets"], s["w"], case["act"], s["dx"], s["dw"],
                                   s["dbias"], ws)


OUTPUTS = {"route_forward": ("weight", "expert", "slot", "source", "offsets"), "route_backward": ("dlogits",),
           "combine_forward": ("out",), "combine_backward": ("dy", "dweight"), "grouped_forward": ("y", "z"),
           "grouped_backward": ("dx", "dw", "dbias"), "clip": ("flat", "norm", "factor")}


def _own(s):
    if "call" not in s:
        s["call"] = _call(s)
    s["call"]()
    return {k: s[k] for k in OUTPUTS[s["case"]["op"]] if s[k] is not None}


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------------ bytes, operations

def work(case):
    op, e = case["op"], SIZE[case["dtype"]]
    if op == "clip":
        n = sum(math.prod(shape) for shape in _shapes(case["list"]))
        return {"bytes": n * e * (2 if case["apart"] or case["over"] > 1 else 1) + 12, "flops": 3 * n}
    n, k, experts = case["tokens"], case["k"], case["experts"]
    rows = (n - case["masked"]) * k  # that an expert has
    if op == "route_forward":
        return {"bytes": n * experts * e + 12 * n * k + 4 * rows + 4 * (experts + 1), "flops": n * experts * (4 + k)}
    if op == "route_backward":
        return {"bytes": n * experts * e * (1 if case["normalise"] else 2) + 12 * n * k,
                "flops": 6 * n * (k if case["normalise"] else experts)}
    if op.startswith("combine"):
        cols = case["cols"]
        if op == "combine_forward":
            return {"bytes": e * cols * (rows + n * (1 + int(case["residual"]))) + n * k * (4 + 4 * int(case["weighted"])),
                    "flops": 2 * rows * cols}
        return {"bytes": e * cols * (2 * rows + n) + 12 * n * k, "flops": 3 * rows * cols}
    inner, cols = case["inner"], case["cols"]
    # experts that some row goes to, if it went to any with the same chance
    busy = min(experts, max(k, round(experts * (1 - (1 - 1 / experts) ** rows))))
    x = (n - case["masked"] if case["gather"] else rows) * inner
    if op == "grouped_forward":
        return {"bytes": e * (x + busy * cols * (inner + 1) + rows * cols * (1 + int(case["save"]))) + 4 * rows,
                "flops": 2 * rows * inner * cols}
    return {"bytes": e * (x + busy * cols * inner + experts * cols * (inner + 1) + rows * inner +
                          rows * cols * (1 + int(case["act"] != "none"))) + 4 * rows,
            "flops": 4 * rows * inner * cols}


# --------------------------------------------------------- definitions in 64 bits

def _exact_act(name, z):
    """The activation and its derivative."""
    if name == "none":
        return z, torch.ones_like(z)
    if name == "relu":
        return z.clamp(min=0), torch.heaviside(z, torch.zeros_like(z))
    if name == "silu":
        p = torch.sigmoid(z)
        return z * p, p + z * p * (1 - p)
    if name == "gelu":
        p = torch.special.ndtr(z)
        return z * p, p + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    # 0.5 (1 + tanh v) is the logistic function of 2 v
    v = 2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)
    p = torch.sigmoid(v)
    return z * p, p + z * p * (1 - p) * 2 * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * z ** 2)


def _exact_route(s):
    case, x = s["case"], s["logits"].double()
    n, experts, k = case["tokens"], case["experts"], case["k"]
    # one choice after the other: the largest that is left, the first of equals
    left, here = x.clone(), torch.arange(experts, device=x.device)
    expert, value = [], []
    for _ in range(k):
        top = left.amax(1, keepdim=True)
        first = torch.where(left == top, here, experts).amin(1, keepdim=True)
        left.scatter_(1, first, float("-inf"))
        none = top == float("-inf")
        expert.append(torch.where(none, -1, first))
        value.append(top)
    expert, value = torch.cat(expert, 1), torch.cat(value, 1)
    among = torch.logsumexp(value if case["normalise"] else x, 1, keepdim=True)
    weight = torch.where(expert < 0, 0.0, torch.exp(value - among)).nan_to_num(0.0)
    chosen = [torch.nonzero(expert == e)[:, 0] for e in range(experts)]
    source = torch.zeros(n * k, dtype=torch.long, device=x.device)
    slot, at, offsets = torch.full((n, k), -1, device=x.device), 0, [0]
    for e, rows in enumerate(chosen):
        source[at:at + len(rows)] = rows
        slot[expert == e] = torch.arange(at, at + len(rows), device=x.device)
        at += len(rows)
        offsets.append(at)
    return {"weight": weight, "expert": expert.int(), "slot": slot.int(), "source": source.int(),
            "offsets": torch.tensor(offsets, dtype=torch.int32, device=x.device)}


def _exact_route_backward(s):
    case, x = s["case"], s["logits"].double()
    n, experts = x.shape
    # the choices as a 0/1 matrix; the derivative of softmax by its quotient rule
    picks = torch.nn.functional.one_hot(s["expert"].long() + 1, experts + 1)[:, :, 1:].double()
    up = (s["dweight"].double()[:, :, None] * picks).sum(1)
    if case["normalise"]:
        p = (s["weight"].double()[:, :, None] * picks).sum(1)
    else:
        p = torch.softmax(x, 1).nan_to_num(0.0)
    return {"dlogits": torch.addcmul(p * up, p, (p * up).sum(1, keepdim=True), value=-1)}


def _exact_combine(s):
    case = s["case"]
    y = s["y"].double()
    at = s["slot"].flatten().long()
    parts = torch.cat([y, y.new_zeros(1, y.shape[1])])[at].unflatten(0, tuple(s["slot"].shape))
    w = s["weight"].double() if case["weighted"] else torch.ones(s["slot"].shape, dtype=torch.float64, device="cuda")
    out = (w[:, :, None] * parts).sum(1)
    return {"out": out + s["residual"].double() if case["residual"] else out}


def _exact_combine_backward(s):
    n, k = s["slot"].shape
    y, dout = s["y"].double(), s["dout"].double()
    at = s["slot"].flatten().long()
    row = torch.arange(n * k, device="cuda") // k
    there = at >= 0
    dy = torch.zeros_like(y)
    dy.index_add_(0, at[there], s["weight"].double().flatten()[there, None] * dout[row[there]])
    dweight = torch.zeros(n * k, dtype=torch.float64, device="cuda")
    dweight[there] = torch.linalg.vecdot(dout[row[there]], y[at[there]])
    return {"dy": dy, "dweight": dweight.view(n, k)}


def _exact_rows(s):
    """(expert, its slots, its rows of x in 64 bits) of every expert."""
    offsets = s["offsets"].tolist()
    for e, (a, b) in enumerate(zip(offsets, offsets[1:])):
        slots = torch.arange(a, b, device="cuda")
        yield e, slots, s["x"].double().index_select(0, s["source"][slots].long() if s["case"]["gather"] else slots)


def _exact_grouped(s):
    case = s["case"]
    z = torch.zeros(s["y"].shape, dtype=torch.float64, device="cuda")
    y = torch.zeros_like(z)
    for e, slots, x in _exact_rows(s):
        z[slots] = torch.addmm(s["bias"][e].double(), x, s["w"][e].double().mT)
        y[slots] = _exact_act(case["act"], z[slots])[0]
    return {"y": y, "z": z} if case["save"] else {"y": y}


def _exact_grouped_backward(s):
    case = s["case"]
    dx, dw, dbias = (torch.zeros(s[k].shape, dtype=torch.float64, device="cuda") for k in ("dx", "dw", "dbias"))
    for e, slots, x in _exact_rows(s):
        dz = s["dy"][slots].double()
        if case["act"] != "none":
            dz *= _exact_act(case["act"], s["z"][slots].double())[1]
        dx[slots] = dz.matmul(s["w"][e].double())
        dw[e] = x.mT.matmul(dz).mT
        dbias[e] = torch.ones(1, len(slots), dtype=torch.float64, device="cuda").matmul(dz)[0]
    return {"dx": dx, "dw": dw, "dbias": dbias}


def _exact_clip(s):
    if s["case"]["kind"] == "l2":
        norm = math.sqrt(math.fsum(float(torch.linalg.vector_norm(g.flatten(), dtype=torch.float64)) ** 2
                                   for g in s["grad"]))
    else:
        norm = max(float(torch.linalg.vector_norm(g.flatten(), ord=math.inf)) for g in s["grad"])
    factor = s["max_norm"] / norm if norm > s["max_norm"] else 1.0
    flat, out = _flat(_shapes(s["case"]["list"]), torch.float64)
    for o, g in zip(out, s["grad"]):
        torch.mul(g, factor, out=o)
    return {"flat": flat,
            "norm": torch.tensor([norm], dtype=torch.float64), "factor": torch.tensor([factor], dtype=torch.float64)}


def exact(case, seed):
    s = prepare(case, seed)
    return {"route_forward": _exact_route, "route_backward": _exact_route_backward, "combine_forward": _exact_combine,
            "combine_backward": _exact_combine_backward, "grouped_forward": _exact_grouped,
            "grouped_backward": _exact_grouped_backward, "clip": _exact_clip}[case["op"]](s)
