"""AdamW with second moments below fp32's normal numbers and an eps far below their roots: the step
divides by the root of what is stored, which the formula gives in 64 bits.

Bounds: those of a step of ordinary values, a dozen fp32 operations on values of its own size, 16 2^-24
of each term; a stored moment below the normal numbers is off by half its spacing, 2^-150, after each of
the three operations that form it."""
import pytest

from mlp_ref import D, U

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
if torch.cuda.is_available():
    from paper_2609_10632_amd import blocks
    from paper_2609_10632_amd import numbat as nb

LR, B1, B2, EPS = 2.0 ** -10, 0.9, 0.95, 1e-30


@pytest.mark.parametrize("n", (5, 300, 5000))
@pytest.mark.parametrize("step", (1, 50))
def test_small_second_moments(n, step):
    g = torch.Generator().manual_seed(n)
    # roots from 2^-73 (the smallest v that is not zero is 2^-149) to 2^-40: across the normal numbers' start (2^-63)
    # and the range where the hardware's root is good by itself; m of the roots' size, so that steps are of lr's
    root = torch.exp2(torch.rand(n, generator=g) * 33 - 73)
    e = {"w": torch.zeros(n), "grad": torch.zeros(n), "m": root * (1 + torch.rand(n, generator=g)), "v": root * root,
         "group": 0}
    old = {k: t.to(D) for k, t in e.items() if k != "group"}
    d = {k: t.cuda() if torch.is_tensor(t) else t for k, t in e.items()}
    table = torch.frombuffer(bytearray(nb.adamw_table([d])), dtype=torch.uint8).cuda()
    ws = blocks.workspace(nb.numbat_workspace_size(nb.OP_ADAMW, None))
    nb.numbat_adamw_step(table, 1, [(LR, 0.0)], 32, B1, B2, EPS, step, 0.0, None, ws)
    torch.cuda.synchronize()
    # the update divides by the root of the new v, which is itself rounded; from the v that is stored the
    # step follows without that rounding
    v = d["v"].cpu().to(D)
    assert bool(((v - B2 * old["v"]).abs() <= 4 * U * v + 3 * 2.0 ** -150).all())
    assert bool((v > 0).all()) and bool((v < 2.0 ** -126).any()) and bool((n < 100) | (v > 2.0 ** -96).any())
    want = -LR / (1 - B1 ** step) * (B1 * old["m"]) / (torch.sqrt(v / (1 - B2 ** step)) + EPS)
    off = (d["w"].cpu().to(D) - want).abs() / want.abs()
    print("largest relative error of a step:", float(off.max()))
    assert bool((off <= 16 * U).all()), float(off.max())
