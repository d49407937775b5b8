"""The residual attention block (forward, backward, step) against the same block in 64 bits: maps and padded
sequences, a channel slice of a wider map, shared heads, smaller batches than the block has room for; captured
into a graph and replayed; on another stream than the current one.

Each stage is compared on the GPU's own inputs to it, so the bounds are those of one call: an fp32 sum of k
products is off by at most (k + 8) 2^-24 sum|products|, an output rounds by 2^-8 (bf16) of itself; a norm's
sums are at most 256 additions deep (test_gpu_group_norm.py); attention's bounds stand in attention_ref.py."""
import math

import pytest

from attention_ref import (attention, attention_grads, fold, forward_bounds, grad_bounds, grid_positions, group_mean,
                           group_norm, join, rotary, split, spread, visible)
from mlp_ref import B, D, U, act, close

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
if torch.cuda.is_available():
    from paper_2609_10632_amd.attention import AttentionBlock, main


def d(t):
    return t.detach().cpu().to(D)


def rand(shape, seed, scale=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * scale).bfloat16().cuda()


def scramble(blk, seed=6):
    g = torch.Generator().manual_seed(seed)
    blk.params["gamma"].copy_(torch.rand(blk.width, generator=g) + 0.5)
    blk.params["beta"].copy_(torch.randn(blk.width, generator=g) * 0.1)


def linear(got, left, w, bias, extra, what):
    ref = left @ w.t() + (0 if bias is None else bias) + (0 if extra is None else extra)
    size = left.abs() @ w.abs().t() + (0 if bias is None else bias.abs()) + (0 if extra is None else extra.abs())
    close(got, ref, (left.shape[1] + 8) * U * size + B * ref.abs(), what)


@pytest.mark.parametrize("images,extents,width,heads,kv_heads,groups,name,causal,lengths,spare,pitch", [
    (2, (10, 13), 96, 3, 3, 8, "none", False, None, 0, 0), (3, (7, 7), 128, 2, 1, 32, "silu", False, None, 2, 40),
    (4, (75,), 64, 4, 2, 4, "none", True, [75, 1, 0, 40], 0, 0), (1, (3, 6, 8), 192, 6, 2, 6, "gelu", False, [101], 0, 8),
    (2, (1,), 32, 1, 1, 1, "none", False, None, 0, 0)])
def test_block(images, extents, width, heads, kv_heads, groups, name, causal, lengths, spare, pitch):
    blk = AttentionBlock(images + spare, extents, width, heads, kv_heads, groups, act=name, causal=causal, seed=5)
    scramble(blk)
    n, feat = math.prod(extents), width // heads
    rows = images * n
    x, g = rand((rows, width + pitch), 1)[:, pitch:], rand((rows, width + pitch), 2, 0.1)[:, pitch:] if pitch == 8 else rand((rows, width), 2, 0.1)
    ln = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    y = blk.forward(x, lengths=ln)
    par = {k: d(v) for k, v in blk.params.items()}
    wqkv, wo = d(blk.copies["wqkv"]), d(blk.copies["wo"])
    xd, normed, mixed = d(x), d(blk.normed[:rows]), d(blk.mixed[:rows])
    xh, t, mean, rstd = group_norm(xd, images, groups, par["gamma"], par["beta"], blk.eps)
    size = spread((xd.abs().reshape(images, n, groups, -1).amax((1, 3)) * rstd), n, width)
    off = 512 * U * (size + xh.abs()) * par["gamma"].abs() * (1 + size)
    ref = act(t, name)[0]
    close(blk.normed[:rows], ref, 1.13 * off + 2 ** -20 * t.abs() + B * ref.abs(), "normed")
    # q, k and v as they were before they were turned
    pre = normed @ wqkv.t() + par["bqkv"]
    pre_off = (width + 8) * U * (normed.abs() @ wqkv.abs().t() + par["bqkv"].abs()) + B * pre.abs()
    turned = (heads + kv_heads) * feat
    at = grid_positions(n, extents).repeat(images, 1)
    ref = torch.cat((rotary(pre[:, :turned], heads + kv_heads, at, blk.pairs, blk.base, "halves", False, False), pre[:, turned:]), 1)
    p = sum(blk.pairs)
    e = pre_off[:, :turned].reshape(rows, heads + kv_heads, feat).clone()
    s = pre[:, :turned].abs().reshape(rows, heads + kv_heads, feat)
    for a, b in ((slice(0, p), slice(p, 2 * p)),):
        both, big = e[..., a] + e[..., b], s[..., a] + s[..., b]
        e[..., a] = e[..., b] = both + 8 * U * big
    e = torch.cat((e.reshape(rows, turned), pre_off[:, turned:]), 1)
    close(blk.qkv[:rows], ref, e + B * (ref.abs() + e), "qkv")
    # attention on the GPU's q, k and v
    qkv = d(blk.qkv[:rows])
    q, k, v = (split(t_, images, h) for t_, h in zip((qkv[:, :heads * feat], qkv[:, heads * feat:turned], qkv[:, turned:]),
                                                     (heads, kv_heads, kv_heads)))
    k, v = (t_.repeat_interleave(heads // kv_heads, 1) for t_ in (k, v))
    see, scale = visible(images, n, n, lengths, lengths, causal), feat ** -0.5
    out, lse, w = attention(q, k, v, see, scale)
    close(mixed, join(out), join(forward_bounds(q, k, v, w, lse, out, see, scale)[0]), "mixed")
    linear(y, mixed, wo, par["bo"], xd, "y")
    same = blk.forward(x, lengths=ln, keep=False).clone()
    assert torch.equal(same, blk.forward(x, lengths=ln))  # what serving computes is what training computes

    dx = blk.backward(x, g, lengths=ln)
    gd = d(g)
    linear(blk.dmixed[:rows], gd, wo.t(), None, None, "dmixed")
    dmixed = split(d(blk.dmixed[:rows]), images, heads)
    empty = ~see.any(-1)
    dmixed = dmixed * (~empty)[..., None].expand(dmixed.shape[:3] + (1,))
    klse = d(blk.lse[:rows * heads]).reshape(images, heads, n).masked_fill(empty.expand(images, heads, n), 0.0)
    w = torch.exp(scale * q @ k.transpose(2, 3) - klse[..., None]).masked_fill(~see, 0.0)
    dq, dk, dv, ds = attention_grads(dmixed, q, k, v, split(mixed, images, heads), w, scale)
    dk, dv = fold(dk, kv_heads), fold(dv, kv_heads)
    bounds = grad_bounds(dmixed, q, k, v, split(mixed, images, heads), w, ds, dq, dk, dv, klse, see, scale, kv_heads)
    pre, e = (torch.cat([join(t_) for t_ in ts], 1) for ts in ((dq, dk, dv), bounds))
    ref = torch.cat((rotary(pre[:, :turned], heads + kv_heads, at, blk.pairs, blk.base, "halves", False, True), pre[:, turned:]), 1)
    eh, s = e[:, :turned].reshape(rows, heads + kv_heads, feat).clone(), pre[:, :turned].abs().reshape(rows, heads + kv_heads, feat)
    both = eh[..., :p] + eh[..., p:2 * p] + 8 * U * (s[..., :p] + s[..., p:2 * p])
    eh[..., :p] = eh[..., p:2 * p] = both
    e = torch.cat((eh.reshape(rows, turned), e[:, turned:]), 1)
    close(blk.dqkv[:rows], ref, e + B * (ref.abs() + e), "dqkv")
    dqkv = d(blk.dqkv[:rows])
    linear(blk.dnormed[:rows], dqkv, wqkv.t(), None, None, "dnormed")
    for wn, bn, left, right in (("wo", "bo", gd, mixed), ("wqkv", "bqkv", dqkv, normed)):
        close(blk.grads[wn], left.t() @ right, (rows + 8) * U * (left.abs().t() @ right.abs()), "d" + wn)
        close(blk.grads[bn], left.sum(0), (rows + 8) * U * left.abs().sum(0), "d" + bn)
    # the norm's gradients on its own statistics
    mu, rs = spread(d(blk.mean[:images]), n, width), spread(d(blk.rstd[:images]), n, width)
    xh, dn = (xd - mu) * rs, d(blk.dnormed[:rows])
    t = xh * par["gamma"] + par["beta"]
    dt = dn * act(t, name)[1]
    h = dt * par["gamma"]
    gm = lambda v_: group_mean(v_, images, groups)  # noqa: E731
    ref = rs * (h - gm(h) - xh * gm(h * xh)) + gd
    xe = 4 * U * (xd.abs() + mu.abs()) * rs
    he = (dn.abs() * (2 ** -20 * (1 + t.abs()) + 1.2 * (xe + 4 * U) * (1 + par["gamma"].abs())) + 4 * U * dt.abs()) * par["gamma"].abs()
    big = h.abs() + gm(h.abs()) + xh.abs() * gm((h * xh).abs())
    off = rs * (he + gm(he) + xh.abs() * gm(he * xh.abs() + h.abs() * xe) + xe * gm((h * xh).abs()) + 256 * U * big) + 4 * U * gd.abs()
    close(dx, ref, off + B * ref.abs(), "dx")
    close(blk.grads["gamma"], (dt * xh).sum(0), (he / par["gamma"].abs() * xh.abs() + dt.abs() * xe).sum(0) + 256 * U * (dt * xh).abs().sum(0), "dgamma")
    close(blk.grads["beta"], dt.sum(0), (he / par["gamma"].abs()).sum(0) + 256 * U * dt.abs().sum(0), "dbeta")

    once = {k_: v_.clone() for k_, v_ in blk.grads.items()}
    blk.backward(x, g, lengths=ln, accumulate=True)
    for k_, v_ in once.items():
        close(blk.grads[k_], 2 * d(v_), 2 * U * d(v_).abs(), "twice d" + k_)  # the second time is added, one rounding


def test_other_extents():
    """A block made for larger maps gives smaller ones what a block of their own gives."""
    big, own = AttentionBlock(3, (12, 10), 64, 2, groups=8, seed=4), AttentionBlock(2, (5, 7), 64, 2, groups=8, seed=4)
    x, g = rand((70, 64), 1), rand((70, 64), 2)
    assert torch.equal(big.forward(x, (5, 7)), own.forward(x))
    assert torch.equal(big.backward(x, g, (5, 7)), own.backward(x, g))
    for k in own.grads:
        assert torch.equal(big.grads[k], own.grads[k])


def test_gradient_against_differences():
    """Along one direction in every parameter and in x: the block's gradient against the difference of
    sum(g y), in 64 bits, of the block's own formula."""
    images, extents, width, heads, kv_heads, groups = 2, (5, 6), 48, 2, 1, 4
    blk = AttentionBlock(images, extents, width, heads, kv_heads, groups, act="silu", seed=3)
    scramble(blk)
    n, feat, rows = 30, 24, 60
    x, g = rand((rows, width), 1), rand((rows, width), 2)
    blk.forward(x)
    dx = blk.backward(x, g)
    par = {k: d(v) for k, v in blk.params.items()}
    par["wqkv"], par["wo"], par["x"] = d(blk.copies["wqkv"]), d(blk.copies["wo"]), d(x)
    gen = torch.Generator().manual_seed(9)
    way = {k: torch.randn(v.shape, generator=gen, dtype=D) * (0.1 if k == "x" else 1.0) for k, v in par.items()}
    at = grid_positions(n, extents).repeat(images, 1)
    see = visible(images, n, n, None, None, False)

    def value(t):
        p = {k: v + t * way[k] for k, v in par.items()}
        a = act(group_norm(p["x"], images, groups, p["gamma"], p["beta"], blk.eps)[1], "silu")[0]
        qkv = a @ p["wqkv"].t() + p["bqkv"]
        turned = (heads + kv_heads) * feat
        qk = rotary(qkv[:, :turned], heads + kv_heads, at, blk.pairs, blk.base, "halves", False, False)
        q, k, v = split(qk[:, :heads * feat], images, heads), split(qk[:, heads * feat:], images, kv_heads), split(qkv[:, turned:], images, kv_heads)
        k, v = (t_.repeat_interleave(heads // kv_heads, 1) for t_ in (k, v))
        y = p["x"] + join(attention(q, k, v, see, feat ** -0.5)[0]) @ p["wo"].t() + p["bo"]
        return float((d(g) * y).sum())

    step = 1e-5  # central difference: error of the order of step^2 of the value's third derivative
    slope = (value(step) - value(-step)) / (2 * step)
    parts = [d(dx if k == "x" else blk.grads[k]) * way[k] for k in par]
    # each gradient holds a handful of bf16 roundings of independent signs in its chain: 2^-8 of the root of
    # the sum of squares would do; 2^-5 of the terms' root sum of squares is allowed
    terms = sum(float((t ** 2).sum()) for t in parts) ** 0.5
    assert abs(sum(float(t.sum()) for t in parts) - slope) <= 2 ** -5 * terms, (slope, terms)


def test_captured_and_replayed():
    """A forward and backward in a graph, replayed on changing inputs with eager work of another block between."""
    blk, other = (AttentionBlock(2, (9, 11), 96, 3, groups=8, act="silu", seed=7) for _ in range(2))
    x, g = rand((198, 96), 1), rand((198, 96), 2, 0.1)
    blk.forward(x)
    blk.backward(x, g)  # workspaces are there
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = blk.forward(x)
        dx = blk.backward(x, g)
    for i in range(4):
        x.copy_(rand((198, 96), 10 + i))
        g.copy_(rand((198, 96), 20 + i, 0.1))
        graph.replay()
        assert torch.equal(y, other.forward(x)) and torch.equal(dx, other.backward(x, g))
        for k in blk.grads:
            assert torch.equal(blk.grads[k], other.grads[k]), k
        torch.cuda.synchronize()


def test_on_another_stream():
    one, two = (AttentionBlock(2, (9, 11), 96, 3, groups=8, seed=7) for _ in range(2))
    x, g = rand((198, 96), 1), rand((198, 96), 2, 0.1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y1 = one.forward(x)
        dx1 = one.backward(x, g)
    y2, dx2 = two.forward(x), two.backward(x, g)  # at the same time, with a workspace of its own
    torch.cuda.synchronize()
    assert torch.equal(y1, y2) and torch.equal(dx1, dx2)


@pytest.mark.parametrize("bits", (32, 8))
def test_training_runs(bits):
    first, last = main(["--images", "2", "--side", "9", "--width", "64", "--heads", "2", "--groups", "8", "--steps", "20",
                        "--state-bits", str(bits)])
    assert math.isfinite(first) and math.isfinite(last)
