"""The residual attention block's step against the AdamW formula in 64 bits: parameters, moments in 32 and 8 bits,
the copies that the products read, decay of the matrices alone, the norm over all gradients and its clip; and that
the next forward is one with the new weights.

Bounds: an update is a dozen fp32 operations on values of its own size, 16 2^-24 of each term.  In 8 bits a moment's
root is rounded to one of 127 or 255 codes of its block's largest: |m| within u (q + 0.3) for a code q and unit u,
and v's root likewise, or within one unit where it is below it (it never rounds to zero)."""
import math

import pytest

from mlp_ref import D, U, close

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
if torch.cuda.is_available():
    from paper_2609_10632_amd.attention import AttentionBlock

B1, B2, EPS, BLOCK = 0.9, 0.95, 1e-8, 256
NAMES = ("wqkv", "bqkv", "wo", "bo", "gamma", "beta")


def d(t):
    return t.detach().cpu().to(D).flatten()


def rand(shape, seed, scale=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * scale).bfloat16().cuda()


def units(blk, name, unit):
    """A tensor's units, one for each of its elements.  (Every tensor starts a whole block of the flat state.)"""
    at = blk.m[name].data_ptr() - blk.m["wqkv"].data_ptr()
    assert at % BLOCK == 0
    n = blk.m[name].numel()
    return d(unit)[at // BLOCK:at // BLOCK + -(-n // BLOCK)].repeat_interleave(BLOCK)[:n]


def moments(blk, name):
    m, v = d(blk.m[name]), d(blk.v[name])
    if blk.state_bits == 32:
        return m, v
    return units(blk, name, blk.m_unit) * m * m.abs(), (units(blk, name, blk.v_unit) * v * v) ** 2


@pytest.mark.parametrize("bits", (32, 8))
@pytest.mark.parametrize("kv_heads,max_norm", [(3, 0.0), (1, 0.05), (3, 1e6)])
def test_step(bits, kv_heads, max_norm):
    blk = AttentionBlock(2, (5, 7), 72, 3, kv_heads, groups=9, act="silu", state_bits=bits, seed=2)
    x, decay, lr = rand((70, 72), 1), 0.1, 3e-3
    for t in (1, 2, 3):
        blk.forward(x)
        blk.backward(x, rand((70, 72), 10 + t, 0.1))
        old = {k: (d(blk.params[k]), *moments(blk, k)) for k in NAMES}
        grads = {k: d(blk.grads[k]) for k in NAMES}
        total = math.sqrt(sum(float((g ** 2).sum()) for g in grads.values()))
        clip = min(1.0, max_norm / (total + 1e-6)) if max_norm else 1.0
        assert all(float(g.abs().max()) > 0 for g in grads.values())
        got = blk.step(lr, weight_decay=decay, betas=(B1, B2), eps=EPS, max_norm=max_norm)
        if max_norm:
            close(got, torch.tensor([total], dtype=D), 2 * U * total, "norm")
        else:
            assert got is None
        for k in NAMES:
            w, m, v = old[k]
            g = grads[k] * clip
            em = 8 * U * (B1 * m.abs() + (1 - B1) * g.abs())
            m, v = B1 * m + (1 - B1) * g, B2 * v + (1 - B2) * g * g
            move = lr / (1 - B1 ** t) * m / (torch.sqrt(v / (1 - B2 ** t)) + EPS)
            off = 16 * U * (move.abs() + w.abs()) + lr / (1 - B1 ** t) * em / (torch.sqrt(v / (1 - B2 ** t)) + EPS)
            w = w * (1 - lr * (decay if k in ("wqkv", "wo") else 0.0)) - move
            close(d(blk.params[k]), w, off + 1e-40, k)
            assert torch.equal(blk.copies[k], blk.params[k].bfloat16()), k
            new_m, new_v = moments(blk, k)
            if bits == 32:
                close(new_m, m, em + 1e-40, "m of " + k)
                close(new_v, v, 12 * U * v + 1e-40, "v of " + k)
            else:
                u, r = units(blk, k, blk.m_unit), torch.sqrt(v)
                close(new_m, m, u * (torch.sqrt(m.abs() / u.clamp(min=1e-300)) + 0.3) + 16 * U * m.abs() + em, "m of " + k)
                u = units(blk, k, blk.v_unit)
                close(torch.sqrt(new_v), r, u * (torch.sqrt(r / u.clamp(min=1e-300)) + 1.0) + 16 * U * r, "root of v of " + k)
    other = AttentionBlock(2, (5, 7), 72, 3, kv_heads, groups=9, act="silu", seed=8)
    assert not torch.equal(other.forward(x), blk.forward(x))
    for k in NAMES:
        other.params[k].copy_(blk.params[k])
        other.copies[k].copy_(blk.params[k])
    assert torch.equal(other.forward(x), blk.forward(x))
