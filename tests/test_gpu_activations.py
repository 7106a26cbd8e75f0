"""The linear layer's activations and their slopes alone, over all sizes of
their argument: a layer whose product is its input, and dbias of one row of
ones.

Tolerance: fp32 tensors, activations and slopes as exact as the formulas in
fp32: the exponential's argument t is rounded a few times, which moves the
exponential by 4 |t| 2^-24 of itself, and the logistic function by at most a
quarter of that (1 / 4 bounds u / (1 + u)^2 for any u), with |t| under 90 wherever
it is not 0 or 1; times |z| in the slope.  Otherwise the hardware's exponential
the same way.  All of it is under 2^-18 (1 + |z|) for |z| <= 12, and past
that the functions are z or 0 and the slopes 1 or 0 to within 2^-18.  The
result is rounded once to its type."""
import math

import numpy as np
import pytest

from tests.test_gpu_layernorm import TINY, UNIT, f64

pytestmark = pytest.mark.gpu
NAMES = ["none", "relu", "gelu", "gelu_tanh", "silu"]


def value_and_slope(name, z):
    import torch
    z = torch.from_numpy(z)
    if name == "none":
        return z.numpy(), np.ones(len(z))
    if name == "relu":
        return z.clamp(min=0).numpy(), (z > 0).double().numpy()
    if name == "gelu":
        p = torch.special.ndtr(z)
        q = torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    elif name == "silu":
        p = torch.sigmoid(z)
        q = p * torch.sigmoid(-z)
    else:
        c = 2 * math.sqrt(2 / math.pi)
        v = c * (z + 0.044715 * z ** 3)
        p = torch.sigmoid(v)
        q = p * torch.sigmoid(-v) * c * (1 + 3 * 0.044715 * z * z)
    return (z * p).numpy(), (p + z * q).numpy()


def arguments(dtype):
    import torch
    most = {"float16": 65504.0, "bfloat16": 3.38e38, "float32": 3.4e38}[dtype]
    z = np.concatenate([[0.0], np.geomspace(1e-4, 1, 90), np.linspace(1, 12, 200), [15, 20, 40, 80, 90, 105, 1000, 6e4],
                        [v for v in (1e6, 1e9, 1e12, 1e13, 1e18, 2e19, 1e25, 1e38, most) if v <= most]])
    return torch.from_numpy(np.concatenate([z, -z])).to(getattr(torch, dtype)).cuda()


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
def test_values(dtype, name):
    import torch
    from paper_2205_14465_amd import binding as B
    z = arguments(dtype)
    want, _ = value_and_slope(name, f64(z))
    for rows in (1, 7, 70):  # dot products, few rows, tiles
        w = torch.zeros(len(z), 64, dtype=z.dtype, device="cuda")
        w[:, 0] = z
        x = torch.zeros(rows, 64, dtype=z.dtype, device="cuda")
        x[:, 0] = 1
        y = torch.empty(rows, len(z), dtype=z.dtype, device="cuda")
        B.bytecomp_linear_forward(x, w, None, None, name, y, None, B.alloc_linear_workspace(x, w))
        got = f64(y)
        slack = 2.0 ** -18 * (1 + np.minimum(np.abs(f64(z)), 12)) if name not in ("none", "relu") else 0
        assert np.all(np.abs(got - want) <= slack + UNIT[dtype] * np.abs(want) * 1.01 + TINY[dtype]), (rows, name)


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
def test_slopes(dtype, name):
    import torch
    from paper_2205_14465_amd import binding as B
    z = arguments(dtype)
    _, want = value_and_slope(name, f64(z))
    x, w = torch.zeros(1, 3, dtype=z.dtype, device="cuda"), torch.zeros(len(z), 3, dtype=z.dtype, device="cuda")
    db = torch.empty(len(z), device="cuda")
    dy = torch.ones(1, len(z), dtype=z.dtype, device="cuda")
    B.bytecomp_linear_backward(dy, z[None], x, w, name, None, None, db, B.alloc_linear_workspace(x, w, backward=True))
    slack = 2.0 ** -18 * (1 + np.minimum(np.abs(f64(z)), 12)) if name not in ("none", "relu") else 0
    off = np.abs(f64(db) - want)
    assert np.all(off <= slack + 2.0 ** -24), (name, f64(z)[~(off <= slack + 2.0 ** -24)])
