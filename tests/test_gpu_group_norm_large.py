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
