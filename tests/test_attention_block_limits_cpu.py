"""What the residual attention block refuses when it is made, not in its first forward; without a GPU."""
import pytest

torch = pytest.importorskip("torch")

from paper_2609_10632_amd import attention  # noqa: E402


def make(**kw):
    return attention.AttentionBlock(**{"images": 2, "extents": (4, 5), "width": 64, "heads": 2, "groups": 8, "device": "cpu", **kw})


@pytest.mark.parametrize("kw", [
    {"width": 272, "heads": 2}, {"width": 264, "heads": 1},  # heads of 136 and of 264 features
    {"pairs": (16, 1)}, {"pairs": (0, 16)}, {"pairs": (16, 0)}, {"pairs": (-1, 4)},
    {"extents": (1,) * 5}, {"extents": (2, 2, 2, 2, 2), "pairs": (1,) * 5}, {"extents": (4, 0)}, {"extents": (-4, -5)},
    {"extents": ()}, {"extents": (), "pairs": ()},
    {"heads": 0}, {"kv_heads": 0}, {"groups": 0}, {"width": 0}])
def test_refused(kw):
    with pytest.raises(ValueError):
        make(**kw)


@pytest.mark.parametrize("kw", [{"width": 256}, {"pairs": (8, 8)}, {"pairs": (1, 15)}, {"pairs": ()}, {"extents": (1, 2, 3, 4)},
                                {"extents": (1,) * 5, "pairs": ()}, {"extents": (1,)}])
def test_taken(kw):
    make(**kw)


def test_extents_of_a_batch():
    with pytest.raises(ValueError):
        make().forward(torch.zeros((20, 64), dtype=torch.bfloat16), (-4, -5))
