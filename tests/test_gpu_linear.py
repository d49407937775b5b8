"""Linear layers (numbat_linear_*) against the same products in 64 bits: every activation, output
type and direction, odd sizes and strides, one row, no row, values that are not finite, streams
and graphs.

Bounds, from the arithmetic: a sum of k exact products of bf16 values added in fp32 in any order is
off by at most (k + 8) 2^-24 sum|products| (the 8: bias, split ranges, residual); an activation's
slope is at most 1.13 and its own evaluation good to 2^-20 of its argument; an output rounds by
2^-8 (bf16) or 2^-24 of itself."""
import pytest

from mlp_ref import B, D, U, act, close

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
if torch.cuda.is_available():
    from paper_2609_10632_amd import blocks
    from paper_2609_10632_amd import numbat as nb

ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")
# m, k, n: one row; a few; ragged on every side; past one tile of every kernel; long reductions
SIZES = [(1, 64, 64), (1, 2048, 520), (1, 9, 1), (3, 8, 8), (16, 256, 1024), (17, 72, 40), (24, 1024, 136), (33, 1003, 65),
         (64, 4096, 64), (65, 33, 257), (100, 192, 768), (129, 4160, 72), (257, 136, 264), (300, 520, 1000),
         (513, 96, 513), (1, 1, 1), (2, 1, 3), (5, 16384, 16)]


def act_id(name):
    return ACTS.index(name)


def rand(shape, seed, scale=1.0, dtype=torch.bfloat16, pitch=0):
    """On the GPU, rows `pitch` elements further apart than they are long, the gap filled with NaN."""
    g = torch.Generator().manual_seed(seed)
    t = (torch.randn(shape, generator=g) * scale).to(dtype)
    full = torch.full((shape[0], shape[1] + pitch), float("nan"), dtype=dtype, device="cuda")
    full[:, :shape[1]] = t.cuda()
    return full[:, :shape[1]]


def out(shape, dtype=torch.bfloat16, pitch=0):
    """An output with guard rows before and after and a guard gap in each row."""
    full = torch.full((shape[0] + 2, shape[1] + pitch), 7.0, dtype=dtype, device="cuda")
    return full, full[1:-1, :shape[1]]


def guards_kept(full, shape):
    inner = full[1:-1]
    assert bool((full[0] == 7).all() and (full[-1] == 7).all() and (inner[:, shape[1]:] == 7).all())


def workspace(op, p):
    n = nb.numbat_workspace_size(op, p)
    ws = blocks.workspace(n)
    if ws is not None:
        ws[256:] = 255  # NaNs: nothing may rely on what a workspace held
    return ws


def aligned_rows(w, pitch, size):
    """Elements per guard row that keep the inner rows' first address 16-byte aligned."""
    return (w + pitch) * size % 16 == 0


def forward(m, k, n, name, y_type="bf16", bias=True, res=False, keep=False, pitch=0, seed=0):
    dt = torch.float32 if y_type == "f32" else torch.bfloat16
    x, w = rand((m, k), seed, pitch=pitch), rand((n, k), seed + 1, k ** -0.5)
    b = torch.randn(n, generator=torch.Generator().manual_seed(seed + 2)).cuda() * 0.5 if bias else None
    r = rand((m, n), seed + 3, dtype=dt, pitch=pitch) if res else None
    full, y = out((m, n), dt, pitch)
    if not aligned_rows(n, pitch, dt.itemsize):  # the guard row before would misalign the first row
        full = torch.full((m, n + pitch), 7.0, dtype=dt, device="cuda")
        y = full[:, :n]
    z = torch.empty((m, n), dtype=torch.bfloat16, device="cuda") if keep else None
    p = nb.linear_problem(m, n, k, act=act_id(name), y_type=nb.F32 if y_type == "f32" else nb.BF16,
                          x_row_stride=k + pitch, y_row_stride=n + pitch, r_row_stride=n + pitch)
    nb.numbat_linear_fwd(p, x, w, b, r, z, y, workspace(nb.OP_LINEAR_FWD, p))
    torch.cuda.synchronize()
    xd, wd = x.cpu().to(D), w.cpu().to(D)
    t = xd @ wd.t() + (b.cpu().to(D) if bias else 0)
    sums = xd.abs() @ wd.abs().t() + (b.cpu().to(D).abs() if bias else 0)
    off = (k + 8) * U * sums
    ref = act(t, name)[0] + (r.cpu().to(D) if res else 0)
    rnd = U if y_type == "f32" else B
    close(y, ref, 1.13 * off + 2.0 ** -20 * t.abs() + (rnd + 2 * U) * (ref.abs() + 1.13 * off) + 1e-30, f"y {m}x{k}x{n} {name}")
    if keep:
        close(z, t, off + B * (t.abs() + off) + 1e-30, "z")
    if full.shape[0] == m + 2:
        guards_kept(full, (m, n))
    else:
        assert bool((full[:, n:] == 7).all())


@pytest.mark.parametrize("m,k,n", SIZES)
def test_forward_sizes(m, k, n):
    forward(m, k, n, "silu", keep=True, seed=m)
    forward(m, k, n, "gelu", "f32", res=True, seed=m + 1)


@pytest.mark.parametrize("name", ACTS)
@pytest.mark.parametrize("y_type", ("bf16", "f32"))
def test_forward_epilogues(name, y_type):
    for bias, res, keep, pitch in ((True, True, True, 0), (False, False, False, 8), (True, True, False, 24), (False, True, True, 3)):
        forward(70, 200, 144, name, y_type, bias, res, keep, pitch, seed=11)
        forward(1, 200, 144, name, y_type, bias, res, keep, pitch, seed=12)
        forward(9, 640, 136, name, y_type, bias, res, keep, pitch, seed=13)


@pytest.mark.parametrize("m,k,n", [(1024, 128, 1100), (2100, 72, 2056), (4000, 520, 264), (8200, 64, 520), (700, 2048, 1032)])
def test_forward_many_tiles(m, k, n):
    forward(m, k, n, "gelu_tanh", res=True, keep=True, seed=k)


def backward(m, k, n, name, accumulate=False, pitch=0, seed=0, db=True):
    dy, w = rand((m, n), seed, 0.1, pitch=pitch), rand((n, k), seed + 1, k ** -0.5)
    x, z = rand((m, k), seed + 2, pitch=pitch), rand((m, k), seed + 3, 2.0, pitch=pitch)
    full = torch.full((m, k + pitch), 7.0, dtype=torch.bfloat16, device="cuda")
    dx = full[:, :k]
    if accumulate:
        dx.copy_(rand((m, k), seed + 4))
    dw = rand((n, k), seed + 5, dtype=torch.float32) if accumulate else torch.full((n, k), float("nan"), device="cuda")
    dbv = rand((1, n), seed + 6, dtype=torch.float32)[0] if accumulate else torch.full((n,), float("nan"), device="cuda")
    dx0, dw0, db0 = (t.clone().cpu().to(D) if accumulate else 0 for t in (dx, dw, dbv))
    p = nb.linear_problem(m, n, k, act=act_id(name), x_row_stride=k + pitch, y_row_stride=n + pitch,
                          z_row_stride=k + pitch)
    nb.numbat_linear_bwd_data(p, dy, w, z if name != "none" else None, dx, accumulate, workspace(nb.OP_LINEAR_BWD_DATA, p))
    nb.numbat_linear_bwd_weight(p, x, dy, dw, dbv if db else None, accumulate, workspace(nb.OP_LINEAR_BWD_WEIGHT, p))
    torch.cuda.synchronize()
    dyd, wd, xd, zd = (t.cpu().to(D) for t in (dy, w, x, z))
    slope = act(zd, name)[1]
    ref = dyd @ wd
    off = (n + 8) * U * (dyd.abs() @ wd.abs())
    got = ref * slope + dx0
    close(dx, got, off * 1.13 + 2.0 ** -20 * ref.abs() * (1 + zd.abs()) + B * (got.abs() + 1.13 * off) + 1e-30, "dx")
    rw = dyd.t() @ xd
    sw = dyd.abs().t() @ xd.abs()
    close(dw, rw + dw0, (m + 8) * U * sw + 2 * U * (rw.abs() + (dw0.abs() if accumulate else 0)) + 1e-30, "dw")
    if db:
        rb = dyd.sum(0)
        close(dbv, rb + db0, (m + 8) * U * dyd.abs().sum(0) + 2 * U * (rb.abs() + (db0.abs() if accumulate else 0)) + 1e-30, "db")
    assert bool((full[:, k:] == 7).all())


@pytest.mark.parametrize("m,k,n", SIZES)
def test_backward_sizes(m, k, n):
    backward(m, k, n, "silu", seed=m)
    backward(m, k, n, "none", accumulate=True, seed=m, db=m % 2 == 0)


@pytest.mark.parametrize("name", ACTS)
def test_backward_epilogues(name):
    for acc, pitch in ((False, 0), (True, 8), (False, 5), (True, 24)):
        backward(150, 264, 136, name, acc, pitch, seed=21)


@pytest.mark.parametrize("m,k,n", [(8192, 264, 72), (3001, 1032, 520), (40000, 40, 136)])
def test_backward_long_sums(m, k, n):
    backward(m, k, n, "gelu", seed=k)


def test_gradients_against_differences():
    """d/dx, d/dw and d/db of sum(g * act(x w^T + b)) from the forward's own fp32 results: central
    differences of step h in one direction; x and w stay exact in bf16 (steps of their grid)."""
    m, k, n, h = 6, 16, 24, 2.0 ** -4
    g = torch.Generator().manual_seed(5)
    grid = lambda *s: torch.randint(-16, 17, s, generator=g).to(D) * 2.0 ** -7  # noqa: E731
    x, w, b, gy = grid(m, k), grid(n, k), grid(n), grid(m, n)
    dirs = {"x": grid(m, k).sign(), "w": grid(n, k).sign(), "b": grid(n).sign()}
    p = nb.linear_problem(m, n, k, act=nb.ACT_GELU, y_type=nb.F32)

    def loss(xv, wv, bv):
        y = torch.empty((m, n), device="cuda")
        z = torch.empty((m, n), dtype=torch.bfloat16, device="cuda")
        nb.numbat_linear_fwd(p, xv.bfloat16().cuda(), wv.bfloat16().cuda(), bv.float().cuda(), None, z, y,
                             workspace(nb.OP_LINEAR_FWD, p))
        return float((y.cpu().to(D) * gy).sum())

    t = x @ w.t() + b
    dz = gy * act(t, "gelu")[1]
    dzb = dz.bfloat16().cuda()
    q = nb.linear_problem(m, n, k)
    dx = torch.empty((m, k), dtype=torch.bfloat16, device="cuda")
    dw, db = torch.empty((n, k), device="cuda"), torch.empty(n, device="cuda")
    nb.numbat_linear_bwd_data(q, dzb, w.bfloat16().cuda(), None, dx, False, workspace(nb.OP_LINEAR_BWD_DATA, q))
    nb.numbat_linear_bwd_weight(q, x.bfloat16().cuda(), dzb, dw, db, False, workspace(nb.OP_LINEAR_BWD_WEIGHT, q))
    for which, grad in (("x", dx), ("w", dw), ("b", db)):
        hi, lo = ({"x": x, "w": w, "b": b} for _ in range(2))
        hi[which], lo[which] = hi[which] + h * dirs[which], lo[which] - h * dirs[which]
        got = (loss(hi["x"], hi["w"], hi["b"]) - loss(lo["x"], lo["w"], lo["b"])) / (2 * h)
        want = float((grad.cpu().to(D) * dirs[which]).sum())
        # third derivative of gelu below 2, inner steps of at most sum|direction| |operand|; bf16
        # rounding of dz and dx on the analytic side
        inner = {"x": w.abs().sum(1).expand(m, n), "w": x.abs().sum(1, keepdim=True).expand(m, n),
                 "b": torch.ones(m, n, dtype=D)}[which]
        bound = float((gy.abs() * 2 * inner ** 3 * h * h / 6).sum()) + 2 * B * float((grad.cpu().to(D).abs()).sum()) + \
            B * float((dz.abs() * inner).sum()) + 1e-3
        assert abs(got - want) <= bound, (which, got, want, bound)


def test_no_rows():
    p = nb.linear_problem(0, 24, 40)
    e = torch.empty((0, 40), dtype=torch.bfloat16, device="cuda")
    w = rand((24, 40), 1)
    nb.numbat_linear_fwd(p, e, w, None, None, None, e, None)
    nb.numbat_linear_bwd_data(p, e, w, None, e, False, None)
    dw, db = torch.ones((24, 40), device="cuda"), torch.ones(24, device="cuda")
    nb.numbat_linear_bwd_weight(p, e, e, dw, db, True, None)
    assert bool((dw == 1).all() and (db == 1).all())
    nb.numbat_linear_bwd_weight(p, e, e, dw, db, False, None)
    assert bool((dw == 0).all() and (db == 0).all())


@pytest.mark.parametrize("m,k,n", [(1, 72, 40), (20, 1003, 65), (300, 264, 264)])
def test_values_that_are_not_finite_stay_in_their_row(m, k, n):
    """A NaN or infinity in one row of x reaches that row of y alone, and one in a row of w that
    column alone, whatever lies next to them in memory."""
    x, w = rand((m, k), 1), rand((n, k), 2, k ** -0.5)
    p = nb.linear_problem(m, n, k, act=nb.ACT_RELU)
    y = torch.empty((m, n), dtype=torch.bfloat16, device="cuda")
    base = torch.empty_like(y)
    ws = workspace(nb.OP_LINEAR_FWD, p)
    nb.numbat_linear_fwd(p, x, w, None, None, None, base, ws)
    assert bool(torch.isfinite(base.float()).all())
    x2, w2 = x.clone(), w.clone()
    x2[m - 1, k - 1] = float("nan")
    nb.numbat_linear_fwd(p, x2, w, None, None, None, y, ws)
    assert bool(torch.isnan(y[m - 1].float()).all()) and torch.equal(y[:m - 1], base[:m - 1])
    w2[n - 1, 0] = float("inf")
    nb.numbat_linear_fwd(p, x, w2, None, None, None, y, ws)
    col = y[:, n - 1].float()
    assert bool(((x[:, 0] > 0) == torch.isinf(col)).all()) and torch.equal(y[:, :n - 1], base[:, :n - 1])


def test_same_bits_every_time_and_on_another_stream():
    m, k, n = 1000, 1032, 520
    x, w, dy = rand((m, k), 1), rand((n, k), 2, 0.03), rand((m, n), 3)
    p = nb.linear_problem(m, n, k, act=nb.ACT_GELU)

    def all_three(stream):
        y, z = (torch.empty((m, n), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        dx = torch.empty((m, k), dtype=torch.bfloat16, device="cuda")
        dw, db = torch.empty((n, k), device="cuda"), torch.empty(n, device="cuda")
        wss = [workspace(o, p) for o in (nb.OP_LINEAR_FWD, nb.OP_LINEAR_BWD_DATA, nb.OP_LINEAR_BWD_WEIGHT)]
        stream.wait_stream(torch.cuda.current_stream())
        nb.numbat_linear_fwd(p, x, w, None, None, z, y, wss[0], stream=stream)
        nb.numbat_linear_bwd_data(p, dy, w, x, dx, False, wss[1], stream=stream)
        nb.numbat_linear_bwd_weight(p, x, dy, dw, db, False, wss[2], stream=stream)
        stream.synchronize()
        return y, z, dx, dw, db

    first = all_three(torch.cuda.current_stream())
    for _ in range(2):
        for a, b in zip(first, all_three(torch.cuda.Stream())):
            assert torch.equal(a, b)


def test_graph_replays_equal_eager():
    """One token, an odd batch with padded operands, a split reduction: captured and replayed."""
    for m, k, n in ((1, 512, 264), (19, 515, 77), (128, 4096, 128)):
        x, w, dy = rand((m, k), 1), rand((n, k), 2, 0.05), rand((m, n), 3)
        p = nb.linear_problem(m, n, k, act=nb.ACT_SILU)
        y, z = (torch.empty((m, n), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        dx, dw = torch.empty((m, k), dtype=torch.bfloat16, device="cuda"), torch.empty((n, k), device="cuda")
        db = torch.empty(n, device="cuda")
        wss = [workspace(o, p) for o in (nb.OP_LINEAR_FWD, nb.OP_LINEAR_BWD_DATA, nb.OP_LINEAR_BWD_WEIGHT)]

        def step():
            nb.numbat_linear_fwd(p, x, w, None, None, z, y, wss[0])
            nb.numbat_linear_bwd_data(p, dy, w, x, dx, False, wss[1])
            nb.numbat_linear_bwd_weight(p, x, dy, dw, db, False, wss[2])

        step()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
        for i in range(4):
            x.copy_(rand((m, k), 10 + i))
            step()
            torch.cuda.synchronize()
            want = [t.clone() for t in (y, z, dx, dw, db)]
            for t in (y, z, dx, dw, db):
                t.zero_()
            g.replay()
            torch.cuda.synchronize()
            for a, b in zip(want, (y, z, dx, dw, db)):
                assert torch.equal(a, b)
