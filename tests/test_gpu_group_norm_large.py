"""Group norm (numbat_group_norm_*) where its sizes are large: more groups in all than a launch has waves, rows that lie
past 2^32 elements, and long sums of one thread.  The references are formed on the GPU in 64 bits, a part at a
time, or known in closed form; bounds as in test_gpu_group_norm.py."""
import pytest

from mlp_ref import B, D, U, close

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
if torch.cuda.is_available():
    from paper_2609_10632_amd import blocks
    from paper_2609_10632_amd import numbat as nb

DEEP = 256 * U


def space(op, p):
    return blocks.workspace(nb.numbat_workspace_size(op, p))


def within(got, ref, bound, what):
    off = (got.double() - ref).abs() - bound
    assert bool((off <= 0).all()), f"{what}: worst by {float(off.max()):.3g}"


def test_groups_past_the_waves_of_a_launch():
    """8192 images of 8192 groups of 8 channels, one row each: 2^26 groups, a wave for each of which would be 2^32
    threads."""
    n, c, groups = 8192, 65536, 8192
    g = torch.Generator(device="cuda").manual_seed(0)
    x = torch.randn((n, c), generator=g, device="cuda", dtype=torch.bfloat16)
    y = torch.empty_like(x)
    mean, rstd = torch.empty((n, groups), device="cuda"), torch.empty((n, groups), device="cuda")
    p = nb.group_norm_problem(n, 1, c, groups)
    print("group norm", n, 1, c, groups, flush=True)
    nb.numbat_group_norm_fwd(p, x, None, None, y, mean, rstd, space(nb.OP_GROUP_NORM_FWD, p))
    dy = torch.randn((n, c), generator=g, device="cuda", dtype=torch.bfloat16)
    dx, dg, db = torch.empty_like(x), torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
    nb.numbat_group_norm_bwd(p, dy, x, mean, rstd, None, None, dx, dg, db, False, space(nb.OP_GROUP_NORM_BWD, p))
    torch.cuda.synchronize()
    dg_ref, db_ref, dg_size, db_size = (torch.zeros(c, dtype=D, device="cuda") for _ in range(4))
    step = 256
    for i in range(0, n, step):
        cut = slice(i, i + step)
        v = x[cut].double().view(step, groups, 8)
        size = v.abs().amax(2)
        m = v.mean(2)
        r = 1 / torch.sqrt(((v - m[..., None]) ** 2).mean(2) + 1e-5)
        within(mean[cut], m, DEEP * size, "mean")
        off = DEEP + (DEEP * size * r) ** 2 + 4 * U * size * r
        within(rstd[cut], r, r * off, "rstd")
        xh = (v - m[..., None]) * r[..., None]
        bound = (DEEP + 4 * U) * (size * r)[..., None] + (off[..., None] + 4 * U) * xh.abs() + B * xh.abs()
        within(y[cut].view(step, groups, 8), xh, bound, "y")
        # the gradients on the statistics that the call was given
        xh = (v - mean[cut].double()[..., None]) * rstd[cut].double()[..., None]
        xh_off = 4 * U * (size * r)[..., None] + 2 * U * xh.abs()
        h = dy[cut].double().view(step, groups, 8)
        h1, h2 = h.mean(2, keepdim=True), (h * xh).mean(2, keepdim=True)
        big = h.abs() + h.abs().mean(2, keepdim=True) + xh.abs() * (h * xh).abs().mean(2, keepdim=True)
        bound = r[..., None] * (DEEP * big + xh_off * h2.abs() + xh.abs() * (h.abs() * xh_off).mean(2, keepdim=True))
        ref = rstd[cut].double()[..., None] * (h - h1 - xh * h2)
        within(dx[cut].view(step, groups, 8), ref, bound + B * ref.abs(), "dx")
        dg_ref += (h * xh).sum(0).view(-1)
        dg_size += ((h * xh).abs() * (DEEP + n * U) + h.abs() * xh_off).sum(0).view(-1)
        db_ref += h.sum(0).view(-1)
        db_size += h.abs().sum(0).view(-1) * (DEEP + n * U)
    within(dg, dg_ref, dg_size, "dgamma")
    within(db, db_ref, db_size, "dbeta")


def long_rows(pattern, c, dtype):
    """Rows of a constant each, `pattern` over and over in ranges."""
    return pattern.to(dtype).cuda().repeat(256)[:, None].expand(-1, c).contiguous()


# one image of 1032 channels: 256 ranges at most, a thread down a slab, so 4000 rows of each thread.  Numbers just
# above one by half of what a sum in the thousands can hold: added one after another every addition is off to the
# same side (a thousand times 2^-24 of the sum)
C, RANGE, ODD = 1032, 4000, 0.49 * 2.0 ** -12


def test_long_sums_of_squares():
    v = (1 + ODD) ** 0.5
    pattern = torch.tensor([0.0] * 8 + [v, -v] * (RANGE // 2 - 4))
    x = long_rows(pattern, C, torch.float32)
    m = x.shape[0]
    p = nb.group_norm_problem(1, m, C, 3, x_type=nb.F32)
    y = torch.empty((m, C), dtype=torch.bfloat16, device="cuda")
    mean, rstd = torch.empty((1, 3), device="cuda"), torch.empty((1, 3), device="cuda")
    print("group norm", 1, m, C, 3, flush=True)
    nb.numbat_group_norm_fwd(p, x, None, None, y, mean, rstd, space(nb.OP_GROUP_NORM_FWD, p))
    exact = pattern.double()
    ref = 1 / torch.sqrt((exact ** 2).mean() + 1e-5)
    close(mean, torch.zeros((1, 3), dtype=D), DEEP * v, "mean")
    close(rstd, ref.expand(1, 3), ref * (DEEP + (DEEP * v * ref) ** 2 + 4 * U * v * ref), "rstd")
    ref = (exact * ref)[:, None].expand(RANGE, C)
    close(y[-RANGE:], ref, (2 * DEEP + 8 * U) * (1 + ref.abs()) + B * ref.abs(), "y")


def test_long_sums():
    pattern = torch.tensor([0.0] * 8 + [1 + ODD] * (RANGE - 8))
    x = long_rows(pattern, C, torch.float32)
    m = x.shape[0]
    p = nb.group_norm_problem(1, m, C, 3, x_type=nb.F32, y_type=nb.F32)
    mean, rstd, one = torch.empty((1, 3), device="cuda"), torch.empty((1, 3), device="cuda"), float(pattern[-1])
    out = torch.empty_like(x)
    print("group norm", 1, m, C, 3, flush=True)
    nb.numbat_group_norm_fwd(p, x, None, None, out, mean, rstd, space(nb.OP_GROUP_NORM_FWD, p))
    close(mean, pattern.double().mean().expand(1, 3), DEEP * one, "mean")
    # x as a gradient: dbeta is its sum, dgamma that of its products with a norm of one
    mean.zero_()
    rstd.fill_(1.0)
    xh = torch.ones_like(x)
    dg, db = torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    nb.numbat_group_norm_bwd(p, x, xh, mean, rstd, None, None, out, dg, db, False, space(nb.OP_GROUP_NORM_BWD, p))
    total = 256 * pattern.double().sum()
    for name, got in (("dgamma", dg), ("dbeta", db)):
        close(got, total.expand(C), (DEEP + U) * total, name)
    # dx = dy - mean(dy) - xh mean(dy xh), with xh = 1
    ref = (pattern.double() - 2 * pattern.double().mean())[:, None].expand(RANGE, C)
    close(out[-RANGE:], ref, 2 * (DEEP + 4 * U) * one + U * ref.abs(), "dx")


@pytest.mark.parametrize("n,m,c,groups", [(2, 1100, 24, 3),     # held
                                          (1, 2200, 40, 1),     # in passes
                                          (3, 740, 45, 3)])     # rows that are no whole vectors
def test_offsets_past_32_bits(n, m, c, groups):
    """Rows 2^21 elements apart: elements and bytes pass 2^32.  The same bits as from dense rows."""
    stride = 1 << 21
    wide = torch.empty((n * m, stride), dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    outs = []
    gamma, beta = (torch.rand(c, generator=g, device="cuda") for _ in range(2))
    x, dy, res = (torch.randn((n * m, c), generator=g, device="cuda").bfloat16() for _ in range(3))
    print("group norm far rows", n, m, c, groups, flush=True)
    for far in (False, True):
        # (all of them beside each other in one matrix)
        at = (lambda i: wide[:, 64 * i:64 * i + c]) if far else (lambda i: torch.empty((n * m, c), dtype=torch.bfloat16, device="cuda"))  # noqa: E731
        y, dx, mine = at(0), at(1), [at(i + 2).copy_(t) for i, t in enumerate((x, dy, res))]
        s = stride if far else 0
        p = nb.group_norm_problem(n, m, c, groups, act=nb.ACT_SILU, x_row_stride=s, y_row_stride=s, r_row_stride=s, dx_row_stride=s)
        mean, rstd = torch.empty((n, groups), device="cuda"), torch.empty((n, groups), device="cuda")
        dg, db = torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
        nb.numbat_group_norm_fwd(p, mine[0], gamma, beta, y, mean, rstd, space(nb.OP_GROUP_NORM_FWD, p))
        nb.numbat_group_norm_bwd(p, mine[1], mine[0], mean, rstd, gamma, beta, dx, dg, db, False, space(nb.OP_GROUP_NORM_BWD, p),
                                 residual_grad=mine[2])
        outs.append([t.contiguous() for t in (y, mean, rstd, dx, dg, db)])
    for a, b, name in zip(*outs, ("y", "mean", "rstd", "dx", "dgamma", "dbeta")):
        assert torch.equal(a, b), name


@pytest.mark.parametrize("m", (40, 20000))  # held, in passes
@pytest.mark.parametrize("bad", (float("nan"), float("inf")))
def test_gradients_that_are_no_numbers_stay_in_their_group(m, bad):
    n, c, groups = 2, 32, 4
    g = torch.Generator().manual_seed(5)
    x, dy = (torch.randn((n * m, c), generator=g).bfloat16().cuda() for _ in range(2))
    p = nb.group_norm_problem(n, m, c, groups, act=nb.ACT_SILU)
    mean, rstd = torch.zeros((n, groups), device="cuda"), torch.ones((n, groups), device="cuda")
    ws = space(nb.OP_GROUP_NORM_BWD, p)

    def call():
        dx, dg, db = torch.empty_like(x), torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
        nb.numbat_group_norm_bwd(p, dy, x, mean, rstd, None, None, dx, dg, db, False, ws)
        return dx, dg, db

    clean = call()
    for t, row, channel, image in ((dy, 5, 9, 0), (x, m + 7, 30, 1)):
        was = t[row, channel].clone()
        t[row, channel] = bad
        got = call()
        t[row, channel] = was
        hit = torch.zeros((n * m, c), dtype=torch.bool, device="cuda")
        hit[image * m:(image + 1) * m, channel // 8 * 8:channel // 8 * 8 + 8] = True
        assert torch.equal(got[0][~hit], clean[0][~hit]) and not bool(got[0][hit].isfinite().any())
        for now, then in zip(got[1:], clean[1:]):
            own = torch.arange(c, device="cuda") == channel
            assert torch.equal(now[~own], then[~own]) and not bool(now[own].isfinite().any())
