"""Group norm with an activation (numbat_group_norm_*) against the formulas in 64 bits: both types on each
side, odd channels, rows and strides, groups of one channel and of all, one row, long maps, a mean far from
zero, in place.

Bounds.  A thread adds at most 64 rows after a shift that lies within their spread (twice the centred squares
at most), at most 128 sums are joined one after another, then lanes, channels and ranges: sums are at
most 256 additions deep, so a mean is off by 256 2^-24 of the values' size and a variance by 512 2^-24 of
itself.  Activations: 2^-20 of their argument, slopes 2^-20 (1 + |t|), and a change of t enters by a
slope of at most 1.13 (a second derivative of at most 1.2)."""
import pytest

from attention_ref import group_mean, group_norm, spread
from mlp_ref import B, D, U, act, close

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
if torch.cuda.is_available():
    from paper_2609_10632_amd import blocks
    from paper_2609_10632_amd import numbat as nb

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
DEEP = 256 * U
# images, rows, channels, groups
SIZES = [(1, 1, 8, 1), (1, 1, 6, 2), (2, 3, 7, 7), (1, 400, 576, 32), (2, 1600, 96, 32), (3, 77, 327, 3), (2, 6400, 48, 8),
         (1, 130, 2056, 257), (1, 9, 4104, 1), (2, 50, 24, 24), (1, 5000, 9, 1), (5, 31, 40, 5), (1, 25600, 16, 2),
         (70, 2, 64, 4), (1, 33, 5000, 4), (1, 1601, 384, 32), (3, 6500, 192, 32),
         # held: one row of threads' registers after another full, slabs of several groups, groups that are no whole
         # vectors, and the sizes past which the passes take over
         (1, 170, 24, 2), (1, 171, 24, 2), (1, 2040, 24, 2), (1, 2050, 24, 2), (1, 2720, 24, 2), (1, 2721, 24, 2),
         (40, 200, 96, 24), (2, 500, 54, 3), (2, 700, 15, 1), (33, 16, 2048, 1), (3, 10, 2056, 1),
         # passes: groups over several slabs, groups too many to join in every block, many images
         (2, 3000, 4100, 2), (1, 6000, 2048, 2048), (65, 1300, 40, 1)]


def matrix(rows, c, seed, dtype, pitch=0, scale=1.0, mean=1.0, ends=float("nan")):
    """Channels of different means and spreads; what lies between the rows is no number."""
    g = torch.Generator().manual_seed(seed)
    t = torch.randn((rows, c), generator=g) * (0.5 + torch.rand(c, generator=g)) + mean * torch.randn(c, generator=g)
    full = torch.full((rows, c + pitch), ends, dtype=dtype, device="cuda")
    full[:, :c] = (t * scale).to(dtype).cuda()
    return full[:, :c]


def vec(c, seed, lo):
    return (lo + torch.rand(c, generator=torch.Generator().manual_seed(seed))).cuda()


def d(t):
    return t.detach().cpu().to(D)


def problem(n, m, c, groups, name, xt, yt, pitch, eps):
    code = {"bf16": nb.BF16, "f32": nb.F32}
    return nb.group_norm_problem(n, m, c, groups, act=getattr(nb, "ACT_" + name.upper()), eps=eps, x_type=code[xt],
                                 y_type=code[yt], x_row_stride=c + pitch, y_row_stride=c + pitch,
                                 r_row_stride=c + pitch, dx_row_stride=c + pitch)


def space(op, p):
    return blocks.workspace(nb.numbat_workspace_size(op, p))


def forward(n, m, c, groups, name="silu", xt="bf16", yt="bf16", pitch=0, affine=True, eps=1e-5, mean=1.0, seed=0):
    x = matrix(n * m, c, seed, TYPES[xt], pitch, mean=mean)
    gamma, beta = (vec(c, seed + 1, 0.5), vec(c, seed + 2, -0.5)) if affine else (None, None)
    y = torch.full((n * m, c + pitch), 7.0, dtype=TYPES[yt], device="cuda")
    mu, rs = torch.full((n, groups), 7.0, device="cuda"), torch.full((n, groups), 7.0, device="cuda")
    p = problem(n, m, c, groups, name, xt, yt, pitch, eps)
    ws = space(nb.OP_GROUP_NORM_FWD, p)
    print("group norm", n, m, c, groups, name, xt, yt, pitch, flush=True)
    nb.numbat_group_norm_fwd(p, x, gamma, beta, y[:, :c], mu, rs, ws)
    xd = d(x)
    ga, be = (d(gamma), d(beta)) if affine else (torch.ones(c, dtype=D), torch.zeros(c, dtype=D))
    xh, t, mean_, rstd = group_norm(xd, n, groups, ga, be, eps)
    size = xd.abs().reshape(n, m, groups, -1).amax((1, 3))
    # (the statistics of a mean that is off by e are off by e^2 besides: nothing beside these)
    close(mu, mean_, DEEP * size + 1e-30, "mean")
    # the mean's own error enters the variance squared, its rounding in x - mean by 2^-24 of x
    slack = (DEEP * size * rstd) ** 2 + 4 * U * size * rstd
    close(rs, rstd, rstd * (DEEP + slack), "rstd")
    m_off, r_off = spread(DEEP * size * rstd, m, c), spread(DEEP + slack, m, c)
    off = (m_off + r_off * xh.abs() + 4 * U * (xh.abs() + spread(size * rstd, m, c))) * ga.abs() + 2 * U * be.abs()
    ref = act(t, name)[0]
    bound = 1.13 * off + 2 ** -20 * t.abs() + (B if yt == "bf16" else U) * ref.abs()
    close(y[:, :c], ref, bound, "y")
    if pitch:
        assert bool((y[:, c:] == 7).all())
    same = torch.full_like(y, 7.0)
    nb.numbat_group_norm_fwd(p, x, gamma, beta, same[:, :c], None, None, ws)
    assert torch.equal(same, y)  # again, and without the statistics
    if xt == yt:
        nb.numbat_group_norm_fwd(p, x, gamma, beta, x, None, None, ws)
        assert torch.equal(x, y[:, :c])  # in place
    return p


@pytest.mark.parametrize("size", SIZES)
def test_forward(size):
    forward(*size)


@pytest.mark.parametrize("name", ("none", "relu", "gelu", "gelu_tanh", "silu"))
@pytest.mark.parametrize("xt,yt", [("bf16", "f32"), ("f32", "bf16"), ("f32", "f32")])
def test_forward_types(name, xt, yt):
    forward(2, 77, 48, 6, name, xt, yt)
    forward(1, 130, 45, 3, name, xt, yt, pitch=3)


@pytest.mark.parametrize("pitch", (1, 8, 192))
def test_forward_strides(pitch):
    forward(2, 300, 96, 32, pitch=pitch)
    forward(2, 30, 51, 3, pitch=pitch, affine=False)


def test_forward_far_mean():
    """Means a thousand times the spread: nothing but x's own rounding is lost."""
    forward(2, 900, 64, 8, "none", "f32", "f32", mean=1000.0)
    forward(1, 6400, 24, 4, "none", "f32", "f32", mean=1000.0)


def test_forward_without_spread():
    x = torch.full((50, 16), 3.25, dtype=torch.bfloat16, device="cuda")
    p = problem(1, 50, 16, 2, "none", "bf16", "f32", 0, 1e-5)
    y, mu, rs = torch.empty((50, 16), device="cuda"), torch.empty((1, 2), device="cuda"), torch.empty((1, 2), device="cuda")
    nb.numbat_group_norm_fwd(p, x, None, None, y, mu, rs, space(nb.OP_GROUP_NORM_FWD, p))
    assert bool((y == 0).all()) and bool((mu == 3.25).all())
    close(rs, torch.full((1, 2), 1e-5 ** -0.5, dtype=D), 2 * U * 317, "rstd")


@pytest.mark.parametrize("m", (40, 20000))  # held, in passes
def test_numbers_that_are_none_stay_in_their_group(m):
    n, c, groups = 2, 32, 4
    x = matrix(n * m, c, 3, torch.bfloat16)
    p = problem(n, m, c, groups, "silu", "bf16", "bf16", 0, 1e-5)
    clean, y = (torch.empty((n * m, c), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    mu, rs = torch.zeros((n, groups), device="cuda"), torch.zeros((n, groups), device="cuda")
    ws = space(nb.OP_GROUP_NORM_FWD, p)
    nb.numbat_group_norm_fwd(p, x, None, None, clean, None, None, ws)
    x[5, 9] = float("nan")  # image 0, group 1
    x[m + 7, 30] = float("inf")  # image 1, group 3
    nb.numbat_group_norm_fwd(p, x, None, None, y, mu, rs, ws)
    bad = torch.zeros((n * m, c), dtype=torch.bool, device="cuda")
    bad[:m, 8:16] = bad[m:, 24:] = True
    assert torch.equal(y[~bad], clean[~bad]) and bool(y[bad].isnan().all())
    which = torch.tensor([[False, True, False, False], [False, False, False, True]], device="cuda")
    assert torch.equal(rs.isnan(), which) and bool((~mu[which].isfinite()).all()) and bool(mu[~which].isfinite().all())


def backward(n, m, c, groups, name="silu", xt="bf16", yt="bf16", pitch=0, affine=True, seed=0, wanted="xgb"):
    x = matrix(n * m, c, seed, TYPES[xt], pitch)
    dy = matrix(n * m, c, seed + 5, TYPES[yt], pitch, scale=0.1)
    gamma, beta = (vec(c, seed + 1, 0.5), vec(c, seed + 2, -0.5)) if affine else (None, None)
    ga, be = (d(gamma), d(beta)) if affine else (torch.ones(c, dtype=D), torch.zeros(c, dtype=D))
    _, _, mean, rstd = group_norm(d(x), n, groups, ga, be, 1e-5)
    mu, rs = mean.float().cuda(), rstd.float().cuda()
    p = problem(n, m, c, groups, name, xt, yt, pitch, 1e-5)
    ws = space(nb.OP_GROUP_NORM_BWD, p)
    dx = torch.full((n * m, c + pitch), 7.0, dtype=TYPES[xt], device="cuda")
    dg, db = torch.full((c,), 7.0, device="cuda"), torch.full((c,), 7.0, device="cuda")
    print("group norm grads", n, m, c, groups, name, xt, yt, pitch, wanted, flush=True)
    args = (dx[:, :c] if "x" in wanted else None, dg if "g" in wanted else None, db if "b" in wanted else None)
    nb.numbat_group_norm_bwd(p, dy, x, mu, rs, gamma, beta, *args, False, ws)

    xd, g, mean, rstd = d(x), d(dy), spread(d(mu), m, c), spread(d(rs), m, c)
    xh = (xd - mean) * rstd
    t = xh * ga + be
    xh_off = 2 * U * (xd.abs() + mean.abs()) * rstd + 2 * U * xh.abs()
    t_off = xh_off * ga.abs() + 2 * U * (t.abs() + be.abs())
    slope = act(t, name)[1]
    dt = g * slope
    dt_off = g.abs() * (2 ** -20 * (1 + t.abs()) + 1.2 * t_off) if name != "none" else 0 * g
    if name == "relu":  # the kink: either side may be taken within t's error
        dt_off = dt_off + torch.where(t.abs() <= t_off, g.abs(), 0 * g)
    h, h_off = dt * ga, dt_off * ga.abs() + U * (dt * ga).abs()
    hx_off = h_off * xh.abs() + h.abs() * xh_off
    gm = lambda v: group_mean(v, n, groups)  # noqa: E731
    dx_ref = rstd * (h - gm(h) - xh * gm(h * xh))
    size = h.abs() + gm(h.abs()) + xh.abs() * gm((h * xh).abs())
    off = h_off + gm(h_off) + DEEP * gm(h.abs()) + xh.abs() * (gm(hx_off) + DEEP * gm((h * xh).abs())) \
        + xh_off * gm((h * xh).abs()) + 4 * U * size
    sum_off = DEEP + n * U  # (images are added in turn)
    if "x" in wanted:
        close(dx[:, :c], dx_ref, rstd * off + (B if xt == "bf16" else U) * dx_ref.abs(), "dx")
        if pitch:
            assert bool((dx[:, c:] == 7).all())
    if "g" in wanted:
        bound = (dt_off * xh.abs() + dt.abs() * xh_off).sum(0) + sum_off * (dt * xh).abs().sum(0)
        close(dg, (dt * xh).sum(0), bound, "dgamma")
    if "b" in wanted:
        close(db, dt.sum(0), dt_off.sum(0) + sum_off * dt.abs().sum(0), "dbeta")
    if wanted == "xgb":
        once = dx.clone(), dg.clone(), db.clone()
        nb.numbat_group_norm_bwd(p, dy, x, mu, rs, gamma, beta, *args, True, ws)
        assert torch.equal(dx, once[0]) and torch.equal(dg, 2 * once[1]) and torch.equal(db, 2 * once[2])
        res = matrix(n * m, c, seed + 9, TYPES[xt], pitch)
        nb.numbat_group_norm_bwd(p, dy, x, mu, rs, gamma, beta, dx[:, :c], None, None, False, ws, residual_grad=res)
        both = dx_ref + d(res)  # the sum is rounded once
        close(dx[:, :c], both, rstd * off + 2 * U * (dx_ref.abs() + d(res).abs()) + (B if xt == "bf16" else U) * both.abs(), "dx + residual")
        mine = torch.empty_strided(res.shape, (c + pitch, 1), dtype=res.dtype, device="cuda").copy_(res)
        nb.numbat_group_norm_bwd(p, dy, x, mu, rs, gamma, beta, mine, None, None, False, ws, residual_grad=mine)
        assert torch.equal(mine, dx[:, :c])
        for buf in ((x,) if xt != yt else (x, dy)):  # in the buffer of either operand
            mine = torch.empty_strided(buf.shape, (c + pitch, 1), dtype=buf.dtype, device="cuda").copy_(buf)
            nb.numbat_group_norm_bwd(p, mine if buf is dy else dy, mine if buf is x else x, mu, rs, gamma, beta, mine, None,
                                     None, False, ws)
            assert torch.equal(mine, once[0][:, :c])


@pytest.mark.parametrize("size", SIZES)
def test_backward(size):
    backward(*size)


@pytest.mark.parametrize("name", ("none", "relu", "gelu", "gelu_tanh", "silu"))
@pytest.mark.parametrize("xt,yt", [("bf16", "f32"), ("f32", "bf16"), ("f32", "f32")])
def test_backward_types(name, xt, yt):
    backward(2, 77, 48, 6, name, xt, yt)
    backward(1, 130, 45, 3, name, xt, yt, pitch=3)


@pytest.mark.parametrize("wanted", ("x", "g", "b", "xb"))
def test_backward_of_some(wanted):
    backward(2, 60, 48, 4, pitch=8, wanted=wanted, affine=False)
    backward(2, 1700, 96, 4, wanted=wanted)


def test_gradients_against_differences():
    """Along one direction in x, gamma and beta: the gradient against the central difference, in 64 bits, of
    sum(dy y)."""
    n, m, c, groups = 2, 45, 24, 3
    x, dy = matrix(n * m, c, 1, torch.float32), matrix(n * m, c, 2, torch.float32, scale=0.1)
    gamma, beta = vec(c, 3, 0.5), vec(c, 4, -0.5)
    p = problem(n, m, c, groups, "gelu", "f32", "f32", 0, 1e-5)
    mu, rs, y = torch.empty((n, groups), device="cuda"), torch.empty((n, groups), device="cuda"), torch.empty_like(x)
    nb.numbat_group_norm_fwd(p, x, gamma, beta, y, mu, rs, space(nb.OP_GROUP_NORM_FWD, p))
    dx, dg, db = torch.empty_like(x), torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
    nb.numbat_group_norm_bwd(p, dy, x, mu, rs, gamma, beta, dx, dg, db, False, space(nb.OP_GROUP_NORM_BWD, p))
    gen = torch.Generator().manual_seed(9)
    way = [torch.randn(t.shape, generator=gen, dtype=D) for t in (x, gamma, beta)]

    def value(step):
        a, b, e = (d(t) + step * w for t, w in zip((x, gamma, beta), way))
        return float((d(dy) * act(group_norm(a, n, groups, b, e, 1e-5)[1], "gelu")[0]).sum())

    step = 1e-4
    slope = (value(step) - value(-step)) / (2 * step)
    parts = [d(g) * w for g, w in zip((dx, dg, db), way)]
    # the gradients are within 2^-14 of the terms they are sums of, the difference within step^2 of them
    assert abs(sum(float(t.sum()) for t in parts) - slope) <= 2 ** -14 * sum(float(t.abs().sum()) for t in parts)


def test_no_rows():
    p = problem(0, 50, 16, 2, "silu", "bf16", "bf16", 0, 1e-5)
    dg, db = torch.full((16,), 7.0, device="cuda"), torch.full((16,), 7.0, device="cuda")
    nb.numbat_group_norm_bwd(p, None, None, None, None, None, None, None, dg, db, True)
    assert bool((dg == 7).all())
    nb.numbat_group_norm_bwd(p, None, None, None, None, None, None, None, dg, db, False)
    assert bool((dg == 0).all()) and bool((db == 0).all())
