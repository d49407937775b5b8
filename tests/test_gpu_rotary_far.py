"""Rotary positions (numbat_rotary) of rows so far apart that elements and bytes pass 2^32: the same bits as from dense
rows, in place too."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
if torch.cuda.is_available():
    from paper_2609_10632_amd import numbat as nb


@pytest.mark.parametrize("layout", ("HALVES", "PAIRS"))
@pytest.mark.parametrize("heads,d,pairs", [(3, 32, (8, 8)), (1, 45, (7, 9))])
def test_offsets_past_32_bits(heads, d, pairs, layout):
    m, stride, width = 2200, 1 << 21, heads * d
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn((m, width), generator=g, device="cuda").bfloat16()
    wide = torch.empty((m, stride), dtype=torch.bfloat16, device="cuda")
    far_x, far_y, y = wide[:, :width].copy_(x), wide[:, 128:128 + width], torch.empty_like(x)
    make = lambda s: nb.rotary_problem(m, heads, d, pairs, extents=(44, 50), layout=getattr(nb, "ROTARY_" + layout),  # noqa: E731
                                       x_row_stride=s, y_row_stride=s)
    print("rotary far rows", heads, d, pairs, layout, flush=True)
    nb.numbat_rotary(make(0), x, None, y)
    nb.numbat_rotary(make(stride), far_x, None, far_y)
    assert torch.equal(far_y, y)
    nb.numbat_rotary(make(stride), far_x, None, far_x)
    assert torch.equal(far_x, y)
