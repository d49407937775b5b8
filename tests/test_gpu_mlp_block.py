"""The residual MLP block (forward, backward, step) against the same block in 64 bits, on an odd
number of rows, on a channel slice of a map, and with fewer rows than the block has room for.

Each stage is compared on the GPU's own inputs to it, so the bounds are those of one call: an fp32
sum of k products is off by at most (k + 8) 2^-24 sum|products|, an activation (slope at most 1.13)
by 2^-20 of its argument besides, an output rounds by 2^-8 (bf16) of itself; a norm's outputs by
(c + 16) 2^-24 of the magnitudes that enter them and by 2^-8 of themselves."""
import pytest

from mlp_ref import B, D, U, act, close, layer_norm, layer_norm_grads

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
if torch.cuda.is_available():
    from paper_2609_10632_amd.mlp import MlpBlock, main


def d(t):
    return t.detach().cpu().to(D)


def rand(shape, seed, scale=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * scale).bfloat16().cuda()


def inputs(rows, width, kind):
    """x and g: dense, or channel slices of wider maps."""
    if kind == "dense":
        return rand((rows, width), 1), rand((rows, width), 2, 0.1)
    x = rand((1, rows, 1, 2 * width + 8), 1)
    g = rand((1, rows, 1, width + 24), 2, 0.1)
    return x[..., 8:8 + width].flatten(0, 2), g[..., 16:16 + width].flatten(0, 2)


@pytest.mark.parametrize("rows,spare,width,hidden,name,kind", [
    (100, 0, 192, 768, "silu", "maps"), (77, 300, 136, 264, "gelu", "dense"), (1, 63, 64, 256, "gelu_tanh", "dense"),
    (259, 0, 41, 83, "relu", "dense")])
def test_block(rows, spare, width, hidden, name, kind):
    blk = MlpBlock(rows + spare, width, hidden, name, seed=5)
    g0 = torch.Generator().manual_seed(6)
    blk.params["gamma"].copy_(torch.rand(width, generator=g0) + 0.5)
    blk.params["beta"].copy_(torch.randn(width, generator=g0) * 0.1)
    x, g = inputs(rows, width, kind)
    y = blk.forward(x)
    par = {k: d(v) for k, v in blk.params.items()}
    w1, w2 = d(blk.copies["w1"]), d(blk.copies["w2"])
    n, z, h, dx_ = d(blk.normed[:rows]), d(blk.z[:rows]), d(blk.wide[:rows]), d(x)

    ref, mean, rstd = layer_norm(dx_, par["gamma"], par["beta"], blk.eps)
    size = (dx_.abs() + mean.abs()[:, None] + dx_.abs().amax(1, keepdim=True)) * rstd[:, None] * par["gamma"].abs() + par["beta"].abs()
    close(blk.normed[:rows], ref, (width + 16) * U * size + B * ref.abs(), "norm")
    t = n @ w1.t() + par["b1"]
    off = (width + 8) * U * (n.abs() @ w1.abs().t() + par["b1"].abs())
    close(blk.z[:rows], t, off + B * t.abs(), "z")
    a = act(t, name)[0]
    close(blk.wide[:rows], a, 1.13 * off + 2 ** -20 * t.abs() + B * a.abs(), "wide")
    ref = h @ w2.t() + par["b2"] + dx_
    off = (hidden + 8) * U * (h.abs() @ w2.abs().t() + par["b2"].abs() + dx_.abs())
    close(y, ref, off + B * ref.abs(), "y")

    same = blk.forward(x, keep=False).clone()
    assert torch.equal(same, blk.forward(x))  # what serving computes is what training computes

    dx = blk.backward(x, g)
    gd, slope = d(g), act(z, name)[1]
    s = gd @ w2
    ref = s * slope
    off = ((width + 8) * U * (gd.abs() @ w2.abs())) * slope.abs() + 2 ** -20 * s.abs() * (1 + z.abs())
    close(blk.dwide[:rows], ref, off + B * ref.abs(), "dz")
    dz = d(blk.dwide[:rows])
    for w, b, left, right in (("w2", "b2", gd, h), ("w1", "b1", dz, n)):
        close(blk.grads[w], left.t() @ right, (rows + 8) * U * (left.abs().t() @ right.abs()), "d" + w)
        close(blk.grads[b], left.sum(0), (rows + 8) * U * left.abs().sum(0), "d" + b)
    ref = dz @ w1
    close(blk.dnormed[:rows], ref, (hidden + 8) * U * (dz.abs() @ w1.abs()) + B * ref.abs(), "dnormed")
    dn, mean, rstd = d(blk.dnormed[:rows]), d(blk.mean[:rows]), d(blk.rstd[:rows])
    ref, dgamma, dbeta = layer_norm_grads(dn, dx_, mean, rstd, par["gamma"])
    ref = ref + gd
    hh, xh = (dn * par["gamma"]).abs(), ((dx_ - mean[:, None]) * rstd[:, None]).abs()
    size = rstd[:, None] * (hh + hh.mean(1, keepdim=True) + xh * (hh * xh).mean(1, keepdim=True)) + gd.abs()
    close(dx, ref, (width + 16) * U * size + B * ref.abs(), "dx")
    close(blk.grads["gamma"], dgamma, (rows + 16) * U * (dn.abs() * xh).sum(0), "dgamma")
    close(blk.grads["beta"], dbeta, (rows + 16) * U * dn.abs().sum(0), "dbeta")

    once = {k: v.clone() for k, v in blk.grads.items()}
    blk.backward(x, g, accumulate=True)
    for k, v in once.items():
        close(blk.grads[k], 2 * d(v), 2 * U * d(v).abs(), "twice d" + k)  # the second time is added, one rounding


def test_gradient_against_differences():
    """Along one direction in every parameter: the block's gradient against the difference of sum(g y),
    in 64 bits, of the block's own formula."""
    rows, width, hidden = 40, 48, 96
    blk = MlpBlock(rows, width, hidden, "gelu", seed=3)
    x, g = rand((rows, width), 1), rand((rows, width), 2)
    blk.forward(x)
    blk.backward(x, g)
    par = {k: d(v) for k, v in blk.params.items()}
    par["w1"], par["w2"] = d(blk.copies["w1"]), d(blk.copies["w2"])
    gen = torch.Generator().manual_seed(9)
    way = {k: torch.randn(v.shape, generator=gen, dtype=D) for k, v in par.items()}

    def value(t):
        p = {k: v + t * way[k] for k, v in par.items()}
        n = layer_norm(d(x), p["gamma"], p["beta"], blk.eps)[0]
        return float((d(g) * (d(x) + act(n @ p["w1"].t() + p["b1"], "gelu")[0] @ p["w2"].t() + p["b2"])).sum())

    step = 1e-4  # central difference: error of the order of step^2 of the value's third derivative
    slope = (value(step) - value(-step)) / (2 * step)
    got = sum(float((d(blk.grads[k]) * way[k]).sum()) for k in par)
    # each gradient holds four bf16 roundings of independent signs in its chain: 2^-8 of the root of
    # the sum of squares would do; 2^-6 of the terms' root sum of squares is allowed
    terms = sum(float(((d(blk.grads[k]) * way[k]) ** 2).sum()) for k in par) ** 0.5
    assert abs(got - slope) <= 2 ** -6 * max(abs(slope), terms), (got, slope, terms)


@pytest.mark.parametrize("bits", (32, 8))
def test_training_follows_its_goal(bits):
    first, last = main(["--rows", "500", "--width", "64", "--hidden", "136", "--steps", "60", "--state-bits", str(bits)])
    assert last < 0.5 * first


def test_refusals():
    blk = MlpBlock(10, 16, 32)
    with pytest.raises(ValueError):
        blk.forward(rand((11, 16), 1))
    with pytest.raises(ValueError):
        blk.forward(rand((10, 24), 1))
    with pytest.raises(ValueError):
        blk.forward(rand((10, 16), 1).float())
    with pytest.raises(ValueError):
        blk.backward(rand((10, 16), 1), rand((9, 16), 1))
