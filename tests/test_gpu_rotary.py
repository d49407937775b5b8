"""Rotary positions (numbat_rotary) against complex rotations in 64 bits: grids and given positions, one to
four axes, both layouts and ladders, both types, odd features, rows and strides, far positions, in place, and
the inverse as the gradient.

Bounds: turns are exact to 2^-52 of the position's turns, what is left of a turn is rounded to fp32 (an
angle within pi 2^-24), cosine and sine within 2 2^-24: together 6 2^-24; two products and a sum add 2 2^-24."""
import pytest

from attention_ref import grid_positions, rotary
from mlp_ref import B, D, U, close

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
if torch.cuda.is_available():
    from paper_2609_10632_amd import numbat as nb

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def check(m, heads, d, pairs, extents=None, positions=None, layout="halves", shared=False, inverse=False, kind="bf16",
          base=10000.0, rest=0, ypitch=0, seed=0):
    g = torch.Generator().manual_seed(seed)
    width = heads * d
    full = torch.full((m, width + rest), float("nan"), dtype=TYPES[kind], device="cuda")
    full[:, :width] = torch.randn((m, width), generator=g).to(TYPES[kind]).cuda()
    x = full[:, :width]
    y = torch.full((m, width + ypitch), 7.0, dtype=TYPES[kind], device="cuda")
    make = lambda ys: nb.rotary_problem(m, heads, d, pairs, extents=extents, base=base, shared=shared, inverse=inverse,  # noqa: E731
                                        layout=nb.ROTARY_HALVES if layout == "halves" else nb.ROTARY_PAIRS,
                                        type=nb.BF16 if kind == "bf16" else nb.F32, x_row_stride=width + rest,
                                        y_row_stride=ys)
    pos = None if positions is None else positions.to(torch.int32).cuda()
    print("rotary", m, heads, d, pairs, extents, layout, shared, inverse, kind, rest, ypitch, flush=True)
    nb.numbat_rotary(make(width + ypitch), x, pos, y[:, :width])
    at = grid_positions(m, extents) if positions is None else positions
    xd = x.cpu().to(D)
    ref = rotary(xd, heads, at, pairs, base, layout, shared, inverse)
    pair = (rotary(xd.abs(), heads, 0 * at, pairs, base, layout, shared, False)).reshape(m, heads, d)
    p = sum(pairs)
    size = torch.zeros_like(pair)
    a, b = (slice(0, p), slice(p, 2 * p)) if layout == "halves" else (slice(0, 2 * p, 2), slice(1, 2 * p, 2))
    size[..., a] = size[..., b] = pair[..., a] + pair[..., b]
    close(y[:, :width], ref, 8 * U * size.reshape(m, width) + (B if kind == "bf16" else U) * ref.abs(), "y")
    same = y[:, :width].reshape(m, heads, d)[..., 2 * p:]
    assert torch.equal(same, x.reshape(m, heads, d)[..., 2 * p:])  # features that do not turn
    if ypitch:
        assert bool((y[:, width:] == 7).all())
    nb.numbat_rotary(make(width + rest), x, pos, x)
    assert torch.equal(x, y[:, :width])  # in place
    assert bool(full[:, width:].isnan().all())


@pytest.mark.parametrize("layout", ("halves", "pairs"))
@pytest.mark.parametrize("kind", ("bf16", "f32"))
@pytest.mark.parametrize("m,heads,d,pairs,extents", [
    (1, 1, 2, (1,), (1,)), (400, 6, 64, (16, 16), (20, 20)), (77, 3, 32, (8, 8), (7, 11)), (300, 2, 128, (16, 24, 24), (3, 10, 10)),
    (50, 5, 40, (3, 2, 4, 5), (2, 3, 2, 5)), (33, 1, 30, (7,), (100,)), (9, 7, 11, (2, 3), (3, 2)), (5000, 3, 16, (4, 4), (50, 50)),
    (3, 2, 512, (256,), (3,)), (2, 300, 64, (32,), (2,))])
def test_grids(m, heads, d, pairs, extents, layout, kind):
    check(m, heads, d, pairs, extents, layout=layout, kind=kind)
    check(m, heads, d, pairs, extents, layout=layout, kind=kind, shared=True, inverse=True, rest=8 * heads, ypitch=16, seed=1)
    check(m, heads, d, pairs, extents, layout=layout, kind=kind, rest=3, ypitch=1, seed=2)


@pytest.mark.parametrize("layout", ("halves", "pairs"))
@pytest.mark.parametrize("kind", ("bf16", "f32"))
def test_positions(layout, kind):
    g = torch.Generator().manual_seed(4)
    check(1, 40, 128, (64,), positions=torch.tensor([[987_654]]), layout=layout, kind=kind, rest=1024)
    check(60, 4, 96, (16, 16, 16), positions=torch.randint(0, 1000, (60, 3), generator=g), layout=layout, kind=kind)
    # as far as they go, before zero too, and the same position twice
    far = torch.tensor([[2**31 - 1], [-2**31], [0], [-1], [5], [5], [2**30 + 12345]])
    check(7, 3, 64, (32,), positions=far, layout=layout, kind=kind, base=1e6)


def test_the_inverse_is_the_gradient():
    """<R x, g> = <x, R^-1 g>, and both against central differences of <R x, g>, which is linear in x."""
    m, heads, d, pairs, extents = 60, 3, 48, (10, 12), (6, 10)
    g = torch.Generator().manual_seed(3)
    x, dy, way = (torch.randn((m, heads * d), generator=g) for _ in range(3))
    dx = torch.empty((m, heads * d), device="cuda")
    nb.numbat_rotary(nb.rotary_problem(m, heads, d, pairs, extents=extents, inverse=True, type=nb.F32), dy.cuda(), None, dx)
    at = grid_positions(m, extents)
    value = lambda t: float((rotary((x + t * way).to(D), heads, at, pairs, 10000.0, "halves", False, False) * dy.to(D)).sum())  # noqa: E731
    slope = (value(0.5) - value(-0.5)) / 1.0
    terms = dx.cpu().to(D) * way.to(D)
    assert abs(float(terms.sum()) - slope) <= 16 * U * float(terms.abs().sum()) + 16 * U * float((dy.abs() * way.abs()).sum())


def test_no_rows():
    nb.numbat_rotary(nb.rotary_problem(0, 2, 8, (4,), extents=(3,)), None, None, None)
