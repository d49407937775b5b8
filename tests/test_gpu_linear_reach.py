"""Linear layers on every kernel that a size can choose: each tile, whole and with a split reduction, in
each direction and type, results on whole cache lines (which go past the caches), on whole vectors and on
odd rows, with everything their epilogues read and write.  Against the products in 64 bits on the GPU.

Bounds as for other sizes: an fp32 sum of k products, and of split ranges of it, is off by at most (k + 8)
2^-24 sum|products|; an activation's slope is at most 1.13, its own evaluation good to 2^-20 of its
argument; a result rounds by 2^-8 (bf16) or 2^-24 of itself."""
import pytest

import linear_plan as lp
from mlp_ref import B, D, U, act

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
if torch.cuda.is_available():
    from paper_2609_10632_amd import numbat as nb
    from test_gpu_linear_tiles import close, guards_kept, out, prod, rand, workspace


def place(whole, width):
    """Pitch and lead of a matrix's rows: dense from a line's start, or apart and off it (odd ones dense)."""
    return (0, 64) if whole else (40 if width % 8 == 0 else 0, 8)


def forward(m, k, n, whole, f32):
    dt = torch.float32 if f32 else torch.bfloat16
    pitch, lead = place(whole, n)
    x, w = rand((m, k), 1, pitch=pitch if k % 8 == 0 else 0), rand((n, k), 2, k ** -0.5)
    bias = rand((1, n), 3, dtype=torch.float32, lead=3)[0]
    res = rand((m, n), 4, dtype=dt, pitch=pitch, lead=lead)
    flat, y = out((m, n), dt, pitch, lead)
    zflat, z = out((m, n), torch.bfloat16, 2 * pitch, lead)
    p = nb.linear_problem(m, n, k, act=nb.ACT_SILU, y_type=nb.F32 if f32 else nb.BF16, x_row_stride=x.stride(0),
                          y_row_stride=n + pitch, r_row_stride=n + pitch, z_row_stride=n + 2 * pitch)
    nb.numbat_linear_fwd(p, x, w, bias, res, z, y, workspace(nb.OP_LINEAR_FWD, p))
    t = prod(x, w) + bias.to(D)
    off = (k + 8) * U * (prod(x.abs(), w.abs()) + bias.to(D).abs())
    close(z, t, off + B * t.abs(), "z")
    ref = act(t, "silu")[0] + res.to(D)
    close(y, ref, 1.13 * off + 2 ** -20 * (t.abs() + res.to(D).abs()) + (U if f32 else B) * ref.abs(), "y")
    guards_kept(flat, y)
    guards_kept(zflat, z)
    # in the residual's place, and without what is optional, the same
    nb.numbat_linear_fwd(p, x, w, bias, res, None, res, workspace(nb.OP_LINEAR_FWD, p))
    assert torch.equal(res, y)


@pytest.mark.parametrize("m,k,n,whole", lp.sizes(lp.FORWARD_BF16))
def test_forward_bf16(m, k, n, whole):
    forward(m, k, n, whole, False)


@pytest.mark.parametrize("m,k,n,whole", lp.sizes(lp.FORWARD_F32))
def test_forward_fp32(m, k, n, whole):
    forward(m, k, n, whole, True)


@pytest.mark.parametrize("f32", (False, True))
@pytest.mark.parametrize("m,k,n", lp.ROWS)
def test_forward_few_rows(m, k, n, f32):
    forward(m, k, n, False, f32)


@pytest.mark.parametrize("accumulate", (False, True))
@pytest.mark.parametrize("m,k,n,whole", lp.sizes(lp.DATA_GRADIENT))
def test_data_gradient(m, k, n, whole, accumulate):
    pitch, lead = place(whole, k)
    dy, w = rand((m, n), 1, pitch=pitch if n % 8 == 0 else 0), rand((n, k), 2, n ** -0.5)
    z = rand((m, k), 3, pitch=2 * pitch, lead=lead)
    flat, dx = out((m, k), torch.bfloat16, pitch, lead)
    start = rand((m, k), 4)
    if accumulate:
        dx.copy_(start)
    p = nb.linear_problem(m, n, k, act=nb.ACT_GELU, x_row_stride=k + pitch, y_row_stride=dy.stride(0),
                          z_row_stride=k + 2 * pitch)
    nb.numbat_linear_bwd_data(p, dy, w, z, dx, accumulate, workspace(nb.OP_LINEAR_BWD_DATA, p))
    wt = w.t().contiguous()
    s, slope = prod(dy, wt), act(z.to(D), "gelu")[1]
    was = start.to(D) if accumulate else torch.zeros_like(s)
    ref = s * slope + was
    off = (n + 8) * U * prod(dy.abs(), wt.abs()) * slope.abs() + 2 ** -20 * (s.abs() * (1 + z.to(D).abs()) + was.abs())
    close(dx, ref, off + B * ref.abs(), "dx")
    guards_kept(flat, dx)


@pytest.mark.parametrize("accumulate", (False, True))
@pytest.mark.parametrize("m,k,n,whole", lp.sizes(lp.WEIGHT_GRADIENT))
def test_weight_gradient(m, k, n, whole, accumulate):
    pitch = 40 if not whole and k % 8 == 0 and n % 8 == 0 else 0
    x, dy = rand((m, k), 1, pitch=pitch), rand((m, n), 2, m ** -0.5, pitch=pitch)
    flat, dw = out((n, k), torch.float32, 0, 64 if whole else 4)
    bflat, db = out((1, n), torch.float32, 0, 1)
    start, bstart = rand((n, k), 3, dtype=torch.float32), rand((1, n), 4, dtype=torch.float32)
    if accumulate:
        dw.copy_(start)
        db.copy_(bstart)
    p = nb.linear_problem(m, n, k, x_row_stride=k + pitch, y_row_stride=n + pitch)
    nb.numbat_linear_bwd_weight(p, x, dy, dw, db, accumulate, workspace(nb.OP_LINEAR_BWD_WEIGHT, p))
    xt, dyt = x.t().contiguous(), dy.t().contiguous()
    keep = 1.0 if accumulate else 0.0
    close(dw, prod(dyt, xt) + keep * start.to(D), (m + 8) * U * (prod(dyt.abs(), xt.abs()) + keep * start.to(D).abs()), "dw")
    close(db[0], dy.to(D).sum(0) + keep * bstart[0].to(D), (m + 8) * U * (dy.to(D).abs().sum(0) + keep * bstart[0].to(D).abs()), "db")
    guards_kept(flat, dw)
    guards_kept(bflat, db)
    alone = torch.full_like(dw, float("nan"))
    nb.numbat_linear_bwd_weight(p, x, dy, alone, None, False, workspace(nb.OP_LINEAR_BWD_WEIGHT, p))
    if not accumulate:
        assert torch.equal(alone, dw)
