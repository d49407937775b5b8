"""The residual attention block's operators written out in 64 bits, on the CPU, for the tests."""
import math

import torch

from mlp_ref import B, D, U


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


def weight_error(q, k, see, scale, lse):
    """Of exp(s - lse), relative, before it is rounded to bf16: a score is off by (d + 8) 2^-24 of the sum of its
    products' sizes, the exponential by 2^-20, its argument's two roundings by 2^-23 of their size."""
    s_off = (q.shape[-1] + 8) * U * scale * (q.abs() @ k.abs().transpose(2, 3))
    s = scale * q @ k.transpose(2, 3)
    arg = 2 * U * (s.abs() + lse[..., None].abs().clamp(max=1e30)) + 2 * U * (s - lse[..., None].clamp(min=-1e30)).abs()
    return torch.where(see, s_off + arg + 2 ** -20, torch.zeros((), dtype=D))


def forward_bounds(q, k, v, p, lse, y, see, scale):
    """How far y and lse may be off."""
    n, off = k.shape[2], weight_error(q, k, see, scale, lse)
    lse_off = (p * off).sum(-1) + (n + 8) * U + 4 * U * lse.abs()
    off = off + (p * off).sum(-1, keepdim=True)  # (of the sum that divides it too)
    return (p * (B + off + (n + 8) * 2 * U)) @ v.abs() + B * y.abs(), lse_off


def grad_bounds(dy, q, k, v, y, p, ds, dq, dk, dv, lse, see, scale, kv_heads):
    """How far dq, dk and dv may be off; dk and dv are the folded ones."""
    d, n, cols = q.shape[-1], k.shape[2], q.shape[2] * (q.shape[1] // kv_heads)
    off = weight_error(q, k, see, scale, lse)
    dp_size = dy.abs() @ v.abs().transpose(2, 3) + (dy.abs() * y.abs()).sum(-1, keepdim=True)
    ds_off = ds.abs() * (off + B + 4 * U) + p * (d + 16) * U * dp_size
    return (scale * (ds_off + (n + 8) * 2 * U * ds.abs()) @ k.abs() + B * dq.abs(),
            fold(scale * (ds_off + (cols + 8) * 2 * U * ds.abs()).transpose(2, 3) @ q.abs(), kv_heads) + B * dk.abs(),
            fold((p * (B + off + (cols + 8) * 2 * U)).transpose(2, 3) @ dy.abs(), kv_heads) + B * dv.abs())
