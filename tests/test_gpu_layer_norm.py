"""Layer norm (numbat_layer_norm_*) against the formulas in 64 bits: both types on each side, odd
and strided rows, one feature, one row, no row, long rows, rows without spread.

Bounds: a row's sums are at most 64 additions deep (per lane, across the wave, across the waves),
so a mean is off by at most 64 2^-24 of the mean magnitude; past the longest row that registers
hold, lanes add c / 1024 values in turn."""
import pytest

from mlp_ref import B, D, U, close, layer_norm, layer_norm_grads

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
if torch.cuda.is_available():
    from paper_2609_10632_amd import blocks
    from paper_2609_10632_amd import numbat as nb

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
# rows, features: around every group width, odd, long
SIZES = [(1, 1), (3, 7), (5, 8), (300, 64), (33, 128), (17, 129), (1000, 192), (9, 255), (64, 256), (31, 257), (12, 512),
         (7, 1003), (20, 1024), (3, 2048), (5, 2049), (4, 4096), (3, 5000), (2, 8192), (3, 8200), (2, 16384), (3, 16385),
         (2, 20008)]


def rows(m, c, seed, dtype, pitch=0, spread=True):
    g = torch.Generator().manual_seed(seed)
    t = torch.randn((m, c), generator=g)
    if spread:
        t = t * (0.5 + torch.rand((m, 1), generator=g)) + torch.randn((m, 1), generator=g)
    full = torch.full((m, c + pitch), float("nan"), dtype=dtype, device="cuda")
    full[:, :c] = t.to(dtype).cuda()
    return full[:, :c]


def vec(c, seed, lo):
    return (lo + torch.rand(c, generator=torch.Generator().manual_seed(seed))).cuda()


def code(t):
    return nb.F32 if t == "f32" else nb.BF16


def deep(c):
    return (64 + c // 1024) * U


def check_forward(m, c, xt, yt, pitch=0, affine=True, eps=1e-5, seed=0):
    x = rows(m, c, seed, TYPES[xt], pitch)
    gamma, beta = (vec(c, seed + 1, 0.5), vec(c, seed + 2, -0.5)) if affine else (None, None)
    y = torch.full((m, c + pitch), 7.0, dtype=TYPES[yt], device="cuda")
    mean, rstd = torch.empty(m, device="cuda"), torch.empty(m, device="cuda")
    p = nb.layer_norm_problem(m, c, eps, code(xt), code(yt), x_row_stride=c + pitch, y_row_stride=c + pitch)
    nb.numbat_layer_norm_fwd(p, x, gamma, beta, y, mean, rstd)
    y2 = y.clone()
    nb.numbat_layer_norm_fwd(p, x, gamma, beta, y2, None, None)
    torch.cuda.synchronize()
    xd = x.cpu().to(D)
    gd, bd = (gamma.cpu().to(D), beta.cpu().to(D)) if affine else (torch.ones(c, dtype=D), torch.zeros(c, dtype=D))
    ry, rm, rr = layer_norm(xd, gd, bd, eps)
    big = xd.abs().mean(1)
    close(mean, rm, deep(c) * big + 1e-30, f"mean {m}x{c}")
    # the mean's error shifts every centred value; the variance's relative error follows
    shift = deep(c) * big * rr
    rel = deep(c) + 2 * shift + shift * shift + 4 * U
    close(rstd, rr, rel * rr, "rstd")
    xh = (xd - rm[:, None]) * rr[:, None]
    off = (gd.abs() * (shift[:, None] + xh.abs() * (rel[:, None] + 4 * U) + 2 * U * (rr * big)[:, None])) + 2 * U * bd.abs()
    rnd = U if yt == "f32" else B
    close(y[:, :c], ry, off + rnd * (ry.abs() + off) + 1e-30, f"y {m}x{c}")
    assert bool((y[:, c:] == 7).all()) and torch.equal(y, y2)


@pytest.mark.parametrize("m,c", SIZES)
def test_forward(m, c):
    for xt, yt in (("bf16", "bf16"), ("f32", "bf16")):
        check_forward(m, c, xt, yt, seed=c)


@pytest.mark.parametrize("xt", TYPES)
@pytest.mark.parametrize("yt", TYPES)
def test_forward_types_and_strides(xt, yt):
    for m, c in ((19, 192), (5, 1000), (3, 33), (2, 4104)):
        for pitch, affine in ((0, True), (8, False), (24, True), (5, True)):
            check_forward(m, c, xt, yt, pitch, affine, seed=3)


def check_backward(m, c, xt, yt, pitch=0, affine=True, res=True, accumulate=False, seed=0):
    x, dy = rows(m, c, seed, TYPES[xt], pitch), rows(m, c, seed + 1, TYPES[yt], pitch, spread=False)
    gamma = vec(c, seed + 2, 0.5) if affine else None
    r = rows(m, c, seed + 3, TYPES[xt], pitch, spread=False) if res else None
    xd, dyd = x.cpu().to(D), dy.cpu().to(D)
    gd = gamma.cpu().to(D) if affine else torch.ones(c, dtype=D)
    _, rm, rr = layer_norm(xd, gd, 0.0, 1e-5)
    mean, rstd = rm.float().cuda(), rr.float().cuda()
    rm, rr = mean.cpu().to(D), rstd.cpu().to(D)
    dx = torch.full((m, c + pitch), 7.0, dtype=TYPES[xt], device="cuda")
    start = 3.0 if accumulate else float("nan")
    dg, db = torch.full((c,), start, device="cuda"), torch.full((c,), start, device="cuda")
    p = nb.layer_norm_problem(m, c, 1e-5, code(xt), code(yt), x_row_stride=c + pitch, y_row_stride=c + pitch,
                              r_row_stride=c + pitch, dx_row_stride=c + pitch)
    ws = blocks.workspace(nb.numbat_workspace_size(nb.OP_LAYER_NORM_BWD, p))
    ws[256:] = 255
    nb.numbat_layer_norm_bwd(p, dy, x, mean, rstd, gamma, r, dx, dg, db, accumulate, ws)
    torch.cuda.synchronize()
    rdx, rdg, rdb = layer_norm_grads(dyd, xd, rm, rr, gd)
    xh = ((xd - rm[:, None]) * rr[:, None]).abs()
    exh = 4 * U * (xh + (rm.abs() * rr)[:, None])  # error of a normalised value
    h = (dyd * gd).abs()
    sums = deep(c) * (h.mean(1, keepdim=True) + xh * (h * xh).mean(1, keepdim=True))
    off = rr[:, None] * (sums + 8 * U * (h + h.mean(1, keepdim=True) + xh * (h * xh).mean(1, keepdim=True))
                         + exh * (h * xh).mean(1, keepdim=True) + xh * (h * exh).mean(1, keepdim=True))
    full = rdx + (r.cpu().to(D) if res else 0)
    rnd = 2 * U if xt == "f32" else B + U
    close(dx[:, :c], full, off + rnd * (full.abs() + off) + 1e-30, f"dx {m}x{c}")
    add = 3.0 if accumulate else 0.0
    close(dg, rdg + add, (m + 8) * U * (dyd.abs() * xh).sum(0) + (dyd.abs() * exh).sum(0) + 2 * U * (rdg.abs() + add) + 1e-30, "dgamma")
    close(db, rdb + add, (m + 8) * U * dyd.abs().sum(0) + 2 * U * (rdb.abs() + add) + 1e-30, "dbeta")
    assert bool((dx[:, c:] == 7).all())
    # each output alone is the same
    only = torch.empty_like(dg)
    nb.numbat_layer_norm_bwd(p, dy, x, mean, rstd, gamma, None, None, only, None, False, ws)
    dx2 = torch.full_like(dx, 7.0)
    nb.numbat_layer_norm_bwd(p, dy, x, mean, rstd, gamma, r, dx2, None, None, False, ws)
    torch.cuda.synchronize()
    assert torch.equal(dx, dx2)
    if not accumulate:
        assert torch.equal(only, dg)


@pytest.mark.parametrize("m,c", SIZES)
def test_backward(m, c):
    check_backward(m, c, "bf16", "bf16", seed=c)
    check_backward(m, c, "f32", "bf16", res=False, accumulate=True, seed=c)


@pytest.mark.parametrize("xt", TYPES)
@pytest.mark.parametrize("yt", TYPES)
def test_backward_types_and_strides(xt, yt):
    for m, c in ((19, 192), (5, 1000), (3, 33), (2, 4104)):
        for pitch, affine in ((0, True), (8, False), (24, True), (5, True)):
            check_backward(m, c, xt, yt, pitch, affine, res=pitch != 8, seed=3)


@pytest.mark.parametrize("m,c", [(5000, 192), (20000, 40), (3000, 1032)])
def test_backward_many_rows(m, c):
    check_backward(m, c, "bf16", "bf16", seed=5)


def test_backward_against_differences():
    """d/dx of sum(g * layer_norm(x)) by central differences of the forward in fp32."""
    m, c, h = 4, 24, 2.0 ** -6
    x, g = rows(m, c, 1, torch.float32), rows(m, c, 2, torch.float32, spread=False)
    gamma, beta = vec(c, 3, 0.5), vec(c, 4, -0.5)
    p = nb.layer_norm_problem(m, c, 1e-5, nb.F32, nb.F32)
    mean, rstd, y = torch.empty(m, device="cuda"), torch.empty(m, device="cuda"), torch.empty((m, c), device="cuda")

    def loss(xv):
        nb.numbat_layer_norm_fwd(p, xv, gamma, beta, y, mean, rstd)
        return float((y.cpu().to(D) * g.cpu().to(D)).sum())

    direction = rows(m, c, 6, torch.float32, spread=False).sign()
    want = (loss(x + h * direction) - loss(x - h * direction)) / (2 * h)
    loss(x)
    dx, dg, db = torch.empty_like(x), torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
    ws = blocks.workspace(nb.numbat_workspace_size(nb.OP_LAYER_NORM_BWD, p))
    nb.numbat_layer_norm_bwd(p, g, x, mean, rstd, gamma, None, dx, dg, db, False, ws)
    got = float((dx.cpu().to(D) * direction.cpu().to(D)).sum())
    # the second-order remainder h^2 / 6 |f'''| with |f'''| below 50 rstd^3 sum|g gamma|, and the
    # forward's fp32 rounding over 2 h
    size = float((g.abs() * gamma.abs()).sum())
    bound = h * h / 6 * 50 * float(rstd.max()) ** 3 * size + 64 * U * 4 * size / h
    assert abs(got - want) <= bound, (got, want, bound)


def test_no_rows_and_rows_without_spread():
    p = nb.layer_norm_problem(0, 40)
    e = torch.empty((0, 40), dtype=torch.bfloat16, device="cuda")
    nb.numbat_layer_norm_fwd(p, e, None, None, e, None, None)
    dg, db = torch.ones(40, device="cuda"), torch.ones(40, device="cuda")
    nb.numbat_layer_norm_bwd(p, e, e, None, None, None, None, e, dg, db, True, None)
    assert bool((dg == 1).all() and (db == 1).all())
    nb.numbat_layer_norm_bwd(p, e, e, None, None, None, None, e, dg, db, False, None)
    assert bool((dg == 0).all() and (db == 0).all())
    # equal values: the variance is exactly 0, y is beta
    for c in (24, 1003, 4096):
        x = torch.full((3, c), 3.0, dtype=torch.bfloat16, device="cuda")
        beta = vec(c, 1, 0.0)
        y, mean, rstd = torch.empty((3, c), device="cuda"), torch.empty(3, device="cuda"), torch.empty(3, device="cuda")
        nb.numbat_layer_norm_fwd(nb.layer_norm_problem(3, c, 1e-5, nb.BF16, nb.F32), x, vec(c, 2, 0.0), beta, y, mean, rstd)
        close(mean, torch.full((3,), 3.0, dtype=D), deep(c) * 3.0, "mean")
        shift = deep(c) * 3.0 / 1e-5 ** 0.5
        close(y, beta.cpu().to(D).expand(3, c), shift + 2 * U, "y")


def test_large_offsets_do_not_cancel():
    """Rows far from zero: the spread survives a mean 1000 times as large."""
    m, c = 8, 1024
    g = torch.Generator().manual_seed(1)
    x = (1000.0 + torch.randn((m, c), generator=g)).cuda()
    y, mean, rstd = torch.empty((m, c), device="cuda"), torch.empty(m, device="cuda"), torch.empty(m, device="cuda")
    nb.numbat_layer_norm_fwd(nb.layer_norm_problem(m, c, 0.0, nb.F32, nb.F32), x, None, None, y, mean, rstd)
    ry, _, rr = layer_norm(x.cpu().to(D), 1.0, 0.0, 0.0)
    close(rstd, rr, 1e-4 * rr, "rstd")  # the mean is off by at most 64 2^-24 1000 = 0.004 of a spread
    close(y, ry, 64 * U * 1000 * 1.1 + 1e-4 * ry.abs(), "y")


def test_bad_row_stays_alone():
    for c in (192, 1003, 4096):
        x = rows(9, c, 1, torch.bfloat16)
        p = nb.layer_norm_problem(9, c)
        y, base = torch.empty((9, c), dtype=torch.bfloat16, device="cuda"), torch.empty((9, c), dtype=torch.bfloat16, device="cuda")
        nb.numbat_layer_norm_fwd(p, x, None, None, base)
        for bad in (float("nan"), float("inf")):
            x2 = x.clone()
            x2[4, c // 2] = bad
            nb.numbat_layer_norm_fwd(p, x2, None, None, y)
            keep = [0, 1, 2, 3, 5, 6, 7, 8]
            assert torch.equal(y[keep], base[keep]) and bool(torch.isnan(y[4].float()).all())


def test_in_place_streams_and_graph():
    m, c = 500, 192
    x, dy, res = rows(m, c, 1, torch.bfloat16), rows(m, c, 2, torch.bfloat16), rows(m, c, 3, torch.bfloat16)
    gamma, beta = vec(c, 4, 0.5), vec(c, 5, -0.5)
    p = nb.layer_norm_problem(m, c)
    mean, rstd, y = torch.empty(m, device="cuda"), torch.empty(m, device="cuda"), torch.empty_like(x)
    dx, dg, db = torch.empty_like(x), torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
    ws = blocks.workspace(nb.numbat_workspace_size(nb.OP_LAYER_NORM_BWD, p))

    def step(stream=None):
        nb.numbat_layer_norm_fwd(p, x, gamma, beta, y, mean, rstd, stream=stream)
        nb.numbat_layer_norm_bwd(p, dy, x, mean, rstd, gamma, res, dx, dg, db, False, ws, stream=stream)

    step()
    torch.cuda.synchronize()
    want = [t.clone() for t in (y, dx, dg, db)]
    inplace = res.clone()
    nb.numbat_layer_norm_bwd(p, dy, x, mean, rstd, gamma, inplace, inplace, None, None, False, ws)
    assert torch.equal(inplace, want[1])
    x2 = x.clone()
    nb.numbat_layer_norm_fwd(p, x2, gamma, beta, x2)
    assert torch.equal(x2, want[0])
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    step(other)
    other.synchronize()
    for a, b in zip(want, (y, dx, dg, db)):
        assert torch.equal(a, b)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for i in range(3):
        x.copy_(rows(m, c, 20 + i, torch.bfloat16))
        step()
        torch.cuda.synchronize()
        want = [t.clone() for t in (y, dx, dg, db)]
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, (y, dx, dg, db)):
            assert torch.equal(a, b)


def test_forward_of_more_rows_than_one_launch():
    """2^31 threads a launch: 2^27 rows of at most 128 features."""
    m, c = (1 << 27) + 21, 2
    x = torch.randint(-8, 8, (m, c), device="cuda", dtype=torch.int16).bfloat16()
    x[-3:] = torch.tensor([[1.0, 3.0], [5.0, 5.0], [-2.0, 6.0]])
    y = torch.full_like(x, float("nan"))
    mean, rstd = (torch.full((m,), float("nan"), device="cuda") for _ in range(2))
    nb.numbat_layer_norm_fwd(nb.layer_norm_problem(m, c, eps=1.0), x, None, None, y, mean, rstd)
    assert mean[-3:].tolist() == [2.0, 5.0, 2.0]
    # half-sums of small integers and their squares are exact; a root and a quotient round once or twice
    half = (x[:, 0].float() - x[:, 1].float()) * 0.5
    assert torch.equal(mean, (x[:, 0].float() + x[:, 1].float()) * 0.5)
    want = 1.0 / torch.sqrt(half * half + 1.0)
    assert bool(((rstd - want).abs() <= 2 ** -22 * want).all())
    half *= want
    assert bool(((y[:, 0].float() - half).abs() <= (2 ** -8 + 2 ** -20) * half.abs()).all())
    assert bool(((y[:, 1].float() + half).abs() <= (2 ** -8 + 2 ** -20) * half.abs()).all())
