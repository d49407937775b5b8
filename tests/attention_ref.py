"""The residual attention block's operators written out in 64 bits, on the CPU, for the tests."""
import math

import torch

from mlp_ref import D


def group_norm(x, n, groups, gamma, beta, eps):
    """x: [n m][c].  xh, t = gamma xh + beta, mean and rstd [n][groups]."""
    c = x.shape[1]
    v = x.reshape(n, -1, groups, c // groups)
    mean = v.mean((1, 3))
    rstd = 1 / torch.sqrt(((v - mean[:, None, :, None]) ** 2).mean((1, 3)) + eps)
    xh = ((v - mean[:, None, :, None]) * rstd[:, None, :, None]).reshape(x.shape)
    return xh, xh * gamma + beta, mean, rstd


def spread(t, m, c):
    """A value [n][groups] of each image's group at every row and channel: [n m][c]."""
    return t.repeat_interleave(c // t.shape[1], 1).repeat_interleave(m, 0)


def group_mean(t, n, groups):
    """The means over an image's group, at every element."""
    c = t.shape[1]
    return spread(t.reshape(n, -1, groups, c // groups).mean((1, 3)), t.shape[0] // n, c)


def rotary(x, heads, positions, pairs, base, layout, shared, inverse):
    """x: [m][heads d], positions [m][axes]; by complex numbers."""
    m, total = x.shape[0], sum(pairs)
    x = x.reshape(m, heads, -1)
    y = x.clone()
    j = 0
    for axis, p in enumerate(pairs):
        for i in range(p):
            t = positions[:, axis].to(D) * base ** -((j / total) if shared else (i / p)) * (-1 if inverse else 1)
            a, b = (j, j + total) if layout == "halves" else (2 * j, 2 * j + 1)
            z = torch.complex(x[..., a], x[..., b]) * torch.complex(torch.cos(t), torch.sin(t))[:, None]
            y[..., a], y[..., b] = z.real, z.imag
            j += 1
    return y.reshape(m, -1)


def grid_positions(m, extents):
    r, cols = torch.arange(m), []
    for e in reversed(extents):
        cols.insert(0, r % e)
        r = r // e
    return torch.stack(cols, 1)


def split(t, batch, heads):
    """[batch rows][heads d] as [batch][heads][rows][d]."""
    return t.reshape(batch, t.shape[0] // batch if batch else 0, heads, t.shape[1] // heads).transpose(1, 2)


def join(t):
    return t.transpose(1, 2).reshape(t.shape[0] * t.shape[2], -1)


def visible(batch, q_len, kv_len, q_lengths, kv_lengths, causal):
    """[batch][1][q_len][kv_len]: the keys that each query sees."""
    ql = torch.as_tensor(q_lengths if q_lengths is not None else [q_len] * batch).clamp(0, q_len)[:, None, None]
    kl = torch.as_tensor(kv_lengths if kv_lengths is not None else [kv_len] * batch).clamp(0, kv_len)[:, None, None]
    i, j = torch.arange(q_len)[None, :, None], torch.arange(kv_len)[None, None, :]
    see = (i < ql) & (j < kl)
    if causal:
        see = see & (j <= i + (kl - ql))
    return see[:, None]


def attention(q, k, v, see, scale):
    """q, k, v: [batch][heads][rows][d] (k's and v's heads repeated).  y, lse, p; zeros and minus infinity where a
    query sees nothing.  What is not seen counts for nothing, whatever it holds."""
    s = (q @ k.transpose(2, 3) * scale).masked_fill(~see, -math.inf)
    lse = torch.logsumexp(s, -1)
    p = torch.exp(s - lse[..., None]).masked_fill(~see, 0.0)
    return p @ v, lse, p


def attention_grads(dy, q, k, v, y, p, scale):
    """Of the repeated heads: dq, dk, dv, and ds."""
    ds = p * (dy @ v.transpose(2, 3) - (dy * y).sum(-1, keepdim=True))
    return scale * ds @ k, scale * ds.transpose(2, 3) @ q, p.transpose(2, 3) @ dy, ds


def fold(t, kv_heads):
    """The sums over the heads that share a head of k and v."""
    b, h, n, d = t.shape
    return t.reshape(b, kv_heads, h // kv_heads, n, d).sum(2)
