"""The operators beside the compression path, as calls to measure: the layers
whose gradients the path compresses (layer norm and the linear layer, forward
and backward) and the optimizer step that takes the aggregate (an update
orthogonalised by Newton-Schulz products).

A case names an operator and its sizes.  `prepare` makes what a training or
serving program has in hand before the call, `run` makes one call: with `own`
false in elementary torch operations in 32 bits, with `own` true through the
library's entry points.  `exact` gives the same results from the operators'
definitions in 64 bits, `work` the bytes and operations of one call that no
implementation can do without.
"""
import math

import torch

own = False

DTYPE = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
ACTIVATIONS = ("none", "relu", "gelu", "gelu_tanh", "silu")
LN_EPS = 1e-5
NS_COEFFICIENTS = (3.4445, -4.7750, 2.0315)
NS_STEPS = 5
NS_EPS = 1e-7
MUON = {"lr": 0.02, "momentum": 0.95, "weight_decay": 0.01}

# The matrices (rows x columns) of one GPT-2-XL block and of ResNet-50 (each
# convolution as output channels x inputs of one output), "*n" n of them.
GPT2XL_BLOCK = "1600x4800,1600x1600,1600x6400,6400x1600"
RESNET50 = ("64x147,64x64,64x576*3,256x64*4,64x256*2,128x256,128x1152*4,512x128*4,512x256,128x512*3,256x512,"
            "256x2304*6,1024x256*6,1024x512,256x1024*5,512x1024,512x4608*3,2048x512*3,2048x1024,512x2048*2,"
            "1000x2048")


def listed():
    return [
        # layer norm of one BERT-base token, as a decoder or a small batch's head
        # calls it: nothing but latency
        {"name": "ln_fwd_1x768_f16", "op": "layernorm_forward", "dtype": "f16", "wdtype": "f16", "rows": 1, "cols": 768},
        # the forward pass over a GPT-2-XL batch of 8 x 1024 tokens
        {"name": "ln_fwd_8192x1600_bf16", "op": "layernorm_forward", "dtype": "bf16", "wdtype": "f32", "rows": 8192,
         "cols": 1600},
        # the backward pass over the same batch: fp32 gradients of the weights, as
        # the compression path takes them
        {"name": "ln_bwd_8192x1600_f16", "op": "layernorm_backward", "dtype": "f16", "wdtype": "f32", "rows": 8192,
         "cols": 1600},
        # a ragged batch at an odd width, fp32 throughout
        {"name": "ln_bwd_1237x1001_f32", "op": "layernorm_backward", "dtype": "f32", "wdtype": "f32", "rows": 1237,
         "cols": 1001},
        # one token through the second projection of GPT-2-XL's MLP: the weight's
        # 20 MB are what has to be read
        {"name": "linear_fwd_1x6400x1600_f16", "op": "linear_forward", "dtype": "f16", "rows": 1, "inner": 6400,
         "cols": 1600, "act": "none", "residual": True, "save": False},
        # the first projection of that MLP over a training batch
        {"name": "linear_fwd_8192x1600x6400_bf16", "op": "linear_forward", "dtype": "bf16", "rows": 8192,
         "inner": 1600, "cols": 6400, "act": "gelu_tanh", "residual": False, "save": True},
        # an fp32 layer of odd sizes on a ragged batch
        {"name": "linear_fwd_777x1001x515_f32", "op": "linear_forward", "dtype": "f32", "rows": 777, "inner": 1001,
         "cols": 515, "act": "relu", "residual": True, "save": True},
        # the backward pass of the first projection: the largest call
        {"name": "linear_bwd_8192x1600x6400_bf16", "op": "linear_backward", "dtype": "bf16", "rows": 8192,
         "inner": 1600, "cols": 6400, "act": "gelu_tanh"},
        # the backward pass of a BERT-base projection in fp32, eight sequences of 128
        {"name": "linear_bwd_1024x768x768_f32", "op": "linear_backward", "dtype": "f32", "rows": 1024, "inner": 768,
         "cols": 768, "act": "none"},
        # one BERT-base projection's gradient orthogonalised alone: fifteen
        # dependent small products
        {"name": "orthogonalize_768x768_f32", "op": "orthogonalize", "dtype": "f32", "mats": "768x768"},
        # every matrix of ResNet-50 in one call, bfloat16 gradients: odd and
        # ragged shapes
        {"name": "orthogonalize_resnet50_bf16", "op": "orthogonalize", "dtype": "bf16", "mats": RESNET50},
        # the optimizer step of two GPT-2-XL blocks: momentum, products, weights
        {"name": "muon_gpt2xl_2blocks_f32", "op": "muon_step", "dtype": "f32", "mats": GPT2XL_BLOCK + "," + GPT2XL_BLOCK},
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm, odd as often as even."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["layernorm_forward", "layernorm_backward", "linear_forward", "linear_backward", "orthogonalize",
                     "muon_step"])
    dtype = rng.choice(["f32", "f16", "bf16"])
    case = {"op": op, "dtype": dtype}
    if op.startswith("layernorm"):
        cols = _log(rng, 16, 16384)
        case |= {"wdtype": rng.choice([dtype, "f32"]), "cols": cols, "rows": _log(rng, 1, min(32768, (1 << 25) // cols))}
    elif op.startswith("linear"):
        # widths from a small head to GPT-2-XL's MLP, half of them multiples of 64 as
        # models have them, half of any value
        snap = 64 if rng.random() < 0.5 else 1
        inner, cols = (max(snap, snap * (_log(rng, 64, 6400) // snap)) for _ in range(2))
        case |= {"inner": inner, "cols": cols, "rows": _log(rng, 1, min(8192, (1 << 36) // (inner * cols))),
                 "act": rng.choice(ACTIVATIONS)}
        if op == "linear_forward":
            case |= {"residual": rng.random() < 0.5, "save": rng.random() < 0.5}
    else:
        mats, left = [], 1.2e12  # operations: six large squares would be past the largest listed case
        for _ in range(rng.randint(1, 6)):
            r, c, n = _log(rng, 16, 6400), _log(rng, 16, 6400), rng.choice([1, 1, 1, 2, 4])
            while (cost := 15 * n * min(r, c) ** 2 * (r + c)) > left:
                r, c = max(16, r * 2 // 3), max(16, c * 2 // 3)
            left -= cost
            mats.append("%dx%d" % (r, c) + ("*%d" % n if n > 1 else ""))
        case["mats"] = ",".join(mats)
    return case


def _mats(text):
    out = []
    for part in text.split(","):
        shape, _, n = part.partition("*")
        out += [tuple(int(v) for v in shape.split("x"))] * int(n or 1)
    return out


# ------------------------------------------------------------------- inputs

def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = DTYPE[case["dtype"]]

    def normal(*shape, scale=1.0, dtype=dt):
        return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)

    op, s = case["op"], {"case": case}
    if op.startswith("layernorm"):
        rows, cols, wdt = case["rows"], case["cols"], DTYPE[case["wdtype"]]
        # activations of a residual stream: a scale of its own for every feature and a
        # common offset, so that rows have means to subtract
        x = torch.randn(rows, cols, generator=g, device="cuda")
        x = x * torch.exp(0.5 * torch.randn(cols, generator=g, device="cuda")) + 0.25
        s["x"] = x.to(dt)
        s["weight"] = (1 + 0.1 * torch.randn(cols, generator=g, device="cuda")).to(wdt)
        s["bias"] = normal(cols, scale=0.1, dtype=wdt)
        s["mean"] = torch.empty(rows, device="cuda")
        s["rstd"] = torch.empty(rows, device="cuda")
        if op == "layernorm_forward":
            s["y"] = torch.empty_like(s["x"])
        else:
            x = s["x"].double()
            m = x.mean(1)
            s["mean"].copy_(m)
            s["rstd"].copy_(((x - m[:, None]).square().mean(1) + LN_EPS).rsqrt())
            # gradients of a mean loss, kept in range by loss scaling as fp16 training does
            s["dy"] = normal(rows, cols, scale=0.05)
            s["dx"] = torch.empty_like(s["x"])
            s["dweight"], s["dbias"] = torch.empty_like(s["weight"]), torch.empty_like(s["bias"])
    elif op.startswith("linear"):
        rows, inner, cols, act = case["rows"], case["inner"], case["cols"], case["act"]
        s["x"] = normal(rows, inner)  # a layer norm's output
        s["w"] = normal(cols, inner, scale=1 / math.sqrt(inner))
        if op == "linear_forward":
            s["bias"] = normal(cols, scale=0.1)
            s["residual"] = normal(rows, cols) if case["residual"] else None
            s["y"] = torch.empty(rows, cols, dtype=dt, device="cuda")
            s["z"] = torch.empty_like(s["y"]) if case["save"] else None
        else:
            s["z"] = normal(rows, cols) if act != "none" else None
            s["dy"] = normal(rows, cols, scale=0.05)
            s["dx"], s["dw"] = torch.empty_like(s["x"]), torch.empty_like(s["w"])
            s["dbias"] = torch.empty(cols, dtype=dt, device="cuda")
    else:
        def gradient(r, c):
            # unequal rows and columns, and one direction that most examples share, as the
            # sum over a batch of tokens has them
            a = torch.randn(r, c, generator=g, device="cuda")
            a *= torch.exp(0.5 * torch.randn(r, 1, generator=g, device="cuda"))
            a *= torch.exp(0.5 * torch.randn(1, c, generator=g, device="cuda"))
            a += torch.randn(r, 1, generator=g, device="cuda") * torch.randn(1, c, generator=g, device="cuda")
            return a * 1e-3
        shapes = _mats(case["mats"])
        if op == "orthogonalize":
            s["update"] = [gradient(r, c).to(dt) for r, c in shapes]
            s["out"] = [torch.empty_like(u) for u in s["update"]]
        else:
            s["grad"] = [gradient(r, c).to(dt) for r, c in shapes]
            s["momentum"] = [10 * gradient(r, c) for r, c in shapes]
            s["weight"] = [normal(r, c, scale=0.02, dtype=torch.float32) for r, c in shapes]
    return s


def _muon_scale(r, c):
    return math.sqrt(max(1.0, r / c))


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


def _plain_orthogonalize(u):
    x = u.t() if u.shape[0] > u.shape[1] else u
    x = x / (x.square().sum().sqrt() + NS_EPS)
    a, b, c = NS_COEFFICIENTS
    for _ in range(NS_STEPS):
        p = x @ x.t()
        x = a * x + (b * p + c * (p @ p)) @ x
    return x.t() if u.shape[0] > u.shape[1] else x


def _plain(s):
    case = s["case"]
    op = case["op"]
    if op == "layernorm_forward":
        x = s["x"].float()
        mean = x.mean(1)
        d = x - mean[:, None]
        rstd = 1 / (d.square().mean(1) + LN_EPS).sqrt()
        y = d * rstd[:, None] * s["weight"].float() + s["bias"].float()
        return {"y": y.to(s["x"].dtype), "mean": mean, "rstd": rstd}
    if op == "layernorm_backward":
        x, dy = s["x"].float(), s["dy"].float()
        xhat = (x - s["mean"][:, None]) * s["rstd"][:, None]
        h = dy * s["weight"].float()
        dx = s["rstd"][:, None] * (h - h.mean(1, keepdim=True) - xhat * (h * xhat).mean(1, keepdim=True))
        return {"dx": dx.to(s["x"].dtype), "dweight": (dy * xhat).sum(0).to(s["weight"].dtype),
                "dbias": dy.sum(0).to(s["bias"].dtype)}
    if op == "linear_forward":
        dt = s["x"].dtype
        z = s["x"].float() @ s["w"].float().t() + s["bias"].float()
        y = _act(case["act"], z)
        if s["residual"] is not None:
            y = y + s["residual"].float()
        return {"y": y.to(dt), "z": z.to(dt)} if case["save"] else {"y": y.to(dt)}
    if op == "linear_backward":
        dt = s["x"].dtype
        dz = s["dy"].float()
        if case["act"] != "none":
            dz = dz * _act_slope(case["act"], s["z"].float())
        return {"dx": (dz @ s["w"].float()).to(dt), "dw": (dz.t() @ s["x"].float()).to(dt), "dbias": dz.sum(0).to(dt)}
    if op == "orthogonalize":
        return [_plain_orthogonalize(u.float()).to(u.dtype) for u in s["update"]]
    for w, g, m in zip(s["weight"], s["grad"], s["momentum"]):
        m.mul_(MUON["momentum"]).add_(g.float())
        o = _plain_orthogonalize(m * MUON["momentum"] + g.float())
        w.mul_(1 - MUON["lr"] * MUON["weight_decay"]).sub_(o, alpha=MUON["lr"] * _muon_scale(*w.shape))
    return {"weight": s["weight"], "momentum": s["momentum"]}


# ---------------------------------------------------------- the library's calls

def _call(s):
    """The call with its arguments marshalled once and its workspace, as a program keeps it for a layer."""
    from paper_2205_14465_amd import binding as B
    case, op = s["case"], s["case"]["op"]
    if op == "layernorm_forward":
        return B.LayerNormCall(s["x"], s["weight"], s["bias"], LN_EPS, s["y"], s["mean"], s["rstd"])
    if op == "layernorm_backward":
        ws = B.alloc_layernorm_workspace(case["rows"], case["cols"])
        return B.LayerNormGradCall(s["dy"], s["x"], s["weight"], s["mean"], s["rstd"], s["dx"], s["dweight"],
                                   s["dbias"], ws)
    if op == "linear_forward":
        ws = B.alloc_linear_workspace(s["x"], s["w"], backward=False)
        return B.LinearCall(s["x"], s["w"], s["bias"], s["residual"], case["act"], s["y"], s["z"], ws)
    if op == "linear_backward":
        ws = B.alloc_linear_workspace(s["x"], s["w"], backward=True)
        return B.LinearGradCall(s["dy"], s["z"], s["x"], s["w"], case["act"], s["dx"], s["dw"], s["dbias"], ws)
    shapes = _mats(case["mats"])
    ws = B.alloc_orthogonalize_workspace(shapes)
    if op == "orthogonalize":
        return B.OrthogonalizeCall(s["update"], s["out"], ws, steps=NS_STEPS, coefficients=NS_COEFFICIENTS, eps=NS_EPS)
    return B.MuonCall(s["weight"], s["grad"], s["momentum"], ws, momentum=MUON["momentum"], nesterov=True,
                      weight_decay=MUON["weight_decay"], scales=[_muon_scale(r, c) for r, c in shapes],
                      steps=NS_STEPS, coefficients=NS_COEFFICIENTS, eps=NS_EPS)


def _own(s):
    if "call" not in s:
        s["call"] = _call(s)
    case, call = s["case"], s["call"]
    if case["op"] == "muon_step":
        call(MUON["lr"])
        return {"weight": s["weight"], "momentum": s["momentum"]}
    call()
    if case["op"] == "layernorm_forward":
        return {"y": s["y"], "mean": s["mean"], "rstd": s["rstd"]}
    if case["op"] == "layernorm_backward":
        return {"dx": s["dx"], "dweight": s["dweight"], "dbias": s["dbias"]}
    if case["op"] == "linear_forward":
        return {"y": s["y"], "z": s["z"]} if case["save"] else {"y": s["y"]}
    if case["op"] == "linear_backward":
        return {"dx": s["dx"], "dw": s["dw"], "dbias": s["dbias"]}
    return s["out"]


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------------ bytes, operations

def work(case):
    op, e = case["op"], SIZE[case["dtype"]]
    if op.startswith("layernorm"):
        rows, cols, we = case["rows"], case["cols"], SIZE[case["wdtype"]]
        if op == "layernorm_forward":
            return {"bytes": 2 * rows * cols * e + 2 * cols * we + 8 * rows, "flops": 8 * rows * cols}
        return {"bytes": 3 * rows * cols * e + 3 * cols * we + 8 * rows, "flops": 14 * rows * cols}
    if op.startswith("linear"):
        m, k, n = case["rows"], case["inner"], case["cols"]
        if op == "linear_forward":
            out = 1 + int(case["residual"]) + int(case["save"])
            return {"bytes": e * (m * k + n * k + n + out * m * n), "flops": 2 * m * k * n}
        out = 1 + int(case["act"] != "none")
        return {"bytes": e * (2 * m * k + 2 * n * k + n + out * m * n), "flops": 4 * m * k * n}
    b = f = 0
    for r, c in _mats(case["mats"]):
        m, n = min(r, c), max(r, c)
        # the two products with a symmetric result cost half
        f += NS_STEPS * (m * m * n + m * m * m + 2 * m * m * n)
        b += r * c * (2 * e if op == "orthogonalize" else e + 16)
    return {"bytes": b, "flops": f}


# --------------------------------------------------------- definitions in 64 bits

def _exact_orthogonal(u):
    """Newton-Schulz in the left Gram matrix: X_k = Q_k X_0 with Q_k = P_k ... P_1, each
    P a polynomial of the Gram matrix that the last one left."""
    r, c = u.shape
    x = u if r <= c else u.mT
    x = x / (torch.linalg.matrix_norm(x) + NS_EPS)
    eye = torch.eye(x.shape[0], dtype=torch.float64, device=x.device)
    gram, q = x.matmul(x.mT), eye
    a, b, c2 = NS_COEFFICIENTS
    for _ in range(NS_STEPS):
        p = a * eye + b * gram + c2 * gram.matmul(gram)
        q = p.matmul(q)
        gram = p.matmul(gram).matmul(p)
    o = q.matmul(x)
    return o if r <= c else o.mT


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


def exact(case, seed):
    s = prepare(case, seed)
    d = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor)}
    op = case["op"]
    if op == "layernorm_forward":
        var, mean = torch.var_mean(d["x"], dim=1, correction=0)
        y = torch.addcmul(d["bias"], d["x"].sub(mean[:, None]).div((var + LN_EPS).sqrt()[:, None]), d["weight"])
        return {"y": y, "mean": mean, "rstd": (var + LN_EPS).pow(-0.5)}
    if op == "layernorm_backward":
        # dx is rstd times the part of weight * dy that is orthogonal to the constant row and to xhat
        n = case["cols"]
        xhat = d["rstd"][:, None] * d["x"] - (d["rstd"] * d["mean"])[:, None]
        h = d["dy"] * d["weight"]
        along = torch.stack([h.sum(1), torch.linalg.vecdot(h, xhat)], 1) / n
        dx = (h - along[:, :1] - along[:, 1:] * xhat) * d["rstd"][:, None]
        return {"dx": dx, "dweight": torch.linalg.vecdot(d["dy"], xhat, dim=0), "dbias": d["dy"].sum(0)}
    if op == "linear_forward":
        z = torch.addmm(d["bias"], d["x"], d["w"].mT)
        y = _exact_act(case["act"], z)[0] + (d["residual"] if case["residual"] else 0)
        return {"y": y, "z": z} if case["save"] else {"y": y}
    if op == "linear_backward":
        dz = d["dy"] if case["act"] == "none" else d["dy"] * _exact_act(case["act"], d["z"])[1]
        return {"dx": dz.matmul(d["w"]), "dw": d["x"].mT.matmul(dz).mT, "dbias": dz.sum(0)}
    if op == "orthogonalize":
        return [_exact_orthogonal(u.double()) for u in s["update"]]
    mu, weights, momenta = MUON["momentum"], [], []
    for w, g, m in zip(s["weight"], s["grad"], s["momentum"]):
        m = mu * m.double() + g.double()
        o = _exact_orthogonal(g.double() + mu * m)
        momenta.append(m)
        weights.append((1 - MUON["lr"] * MUON["weight_decay"]) * w.double() - MUON["lr"] * _muon_scale(*w.shape) * o)
    return {"weight": weights, "momentum": momenta}
