"""The residual MLP block's operators written out in 64 bits, on the CPU, for the tests."""
import math

import torch

D = torch.float64
U = 2.0 ** -24  # fp32's rounding
B = 2.0 ** -8   # bf16's rounding (8 significant bits)


def act(z, name):
    """The activation and its derivative."""
    if name == "relu":
        return z.clamp_min(0), (z > 0).to(z.dtype)
    if name == "gelu":
        cdf = 0.5 * torch.erfc(-z / math.sqrt(2.0))
        return z * cdf, cdf + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    if name == "gelu_tanh":
        a, b = math.sqrt(2 / math.pi), 0.044715
        t = torch.tanh(a * (z + b * z ** 3))
        return 0.5 * z * (1 + t), 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * a * (1 + 3 * b * z * z)
    if name == "silu":
        s = torch.sigmoid(z)
        return z * s, s * (1 + z * (1 - s))
    return z.clone(), torch.ones_like(z)


def close(got, ref, bound, what):
    """Every element of got within bound (a tensor or a number) of ref; an empty tensor is."""
    got, ref = got.detach().cpu().to(D), ref.to(D)
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    off = (got - ref).abs() - bound
    bad = ~(off <= 0)
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst by {float(off.max()):.3g}"


def layer_norm(x, gamma, beta, eps):
    mean = x.mean(1)
    rstd = 1 / torch.sqrt(((x - mean[:, None]) ** 2).mean(1) + eps)
    return (x - mean[:, None]) * rstd[:, None] * gamma + beta, mean, rstd


def layer_norm_grads(dy, x, mean, rstd, gamma):
    xh = (x - mean[:, None]) * rstd[:, None]
    h = dy * gamma
    dx = rstd[:, None] * (h - h.mean(1, keepdim=True) - xh * (h * xh).mean(1, keepdim=True))
    return dx, (dy * xh).sum(0), dy.sum(0)
