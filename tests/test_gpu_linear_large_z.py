"""Activations of large finite pre-activations, up to the largest that bf16 holds: the activation is z
or 0 there and its slope 1 or 0, though the formula's powers of z pass fp32's range.

Bounds: past |z| = 128 the values and slopes are those to within 1e-50, which fp32 holds as zero; what
is left is a product with a factor good to 2^-22, and bf16's rounding of results it can hold exactly."""
import pytest

from mlp_ref import D, act

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
if torch.cuda.is_available():
    from paper_2609_10632_amd import blocks
    from paper_2609_10632_amd import numbat as nb

ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")
SIZES = (128.0, 1e4, 1e9, 1.8e19, 2.0e19, 6.0e19, 1e25, 1e38, 3.3e38)


def large(m, n):
    """bf16 [m][n] of both signs."""
    v = torch.tensor([s * z for z in SIZES for s in (1.0, -1.0)]).bfloat16()
    return v.repeat(m * n // v.numel() + 1)[:m * n].view(m, n)


@pytest.mark.parametrize("name", ACTS)
@pytest.mark.parametrize("m,k", [(3, 8), (70, 40), (300, 264)])
def test_slopes(name, m, k):
    """dx = act'(z) where dy and w make every sum 1."""
    z, n = large(m, k), 8
    dy, w = torch.zeros((m, n)).bfloat16(), torch.zeros((n, k)).bfloat16()
    dy[:, 0] = w[0] = 1.0
    dx = torch.full((m, k), float("nan"), dtype=torch.bfloat16, device="cuda")
    p = nb.linear_problem(m, n, k, act=ACTS.index(name))
    nb.numbat_linear_bwd_data(p, dy.cuda(), w.cuda(), z.cuda(), dx, False,
                              blocks.workspace(nb.numbat_workspace_size(nb.OP_LINEAR_BWD_DATA, p)))
    want = act(z.to(D), name)[1]
    assert bool(((want - want.round()).abs() < 1e-50).all())  # 0 or 1
    bad = ~((dx.cpu().to(D) - want).abs() <= 2.0 ** -20)
    assert not bool(bad.any()), sorted(set(z[bad].tolist()))


@pytest.mark.parametrize("name", ACTS)
@pytest.mark.parametrize("m,n", [(3, 8), (70, 40), (300, 264)])
def test_values(name, m, n):
    z, k = large(m, n).t().contiguous(), 8  # as wide as a row of x is long: z [n][m]
    x, w = torch.zeros((m, k)).bfloat16(), torch.zeros((n, k)).bfloat16()
    x[:, 0] = z[0]
    w[:, 0] = 1.0
    y = torch.full((m, n), float("nan"), device="cuda")
    p = nb.linear_problem(m, n, k, act=ACTS.index(name), y_type=nb.F32)
    nb.numbat_linear_fwd(p, x.cuda(), w.cuda(), None, None, None, y,
                         blocks.workspace(nb.numbat_workspace_size(nb.OP_LINEAR_FWD, p)))
    want = act(x[:, :1].to(D), name)[0].expand(m, n)
    bad = ~((y.cpu().to(D) - want).abs() <= 2.0 ** -20 * want.abs() + 1e-37)
    assert not bool(bad.any()), (sorted(set(x[:, 0][bad.any(1)].tolist())))
