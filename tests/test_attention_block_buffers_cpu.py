"""The residual attention block given its own buffers as operands, without a GPU: what a call would write over
before it has read it for the last time is refused."""
import pytest

torch = pytest.importorskip("torch")

from paper_2609_10632_amd import attention  # noqa: E402
from test_attention_block_cpu import CALLS  # noqa: E402

ROWS = 40


@pytest.fixture
def block(monkeypatch):
    for name in CALLS:
        monkeypatch.setattr(attention.nb, name, lambda *a, **k: None)
    return attention.AttentionBlock(2, (4, 5), 64, 2, groups=8, device="cpu")


def rows():
    return torch.zeros((ROWS, 64), dtype=torch.bfloat16)


@pytest.mark.parametrize("name", ("y", "normed", "qkv", "mixed"))
def test_a_forward_of_its_activations(block, name):
    x = getattr(block, name)[:, :64]
    for keep in (True, False):
        with pytest.raises(ValueError):
            block.forward(x, keep=keep)
    with pytest.raises(ValueError):
        block.forward(getattr(block, name)[20:, :64])
    assert block.kept is None


@pytest.mark.parametrize("name", ("dnormed", "dqkv", "dmixed"))
def test_of_its_activations_gradients(block, name):
    t = getattr(block, name)[:, :64]
    with pytest.raises(ValueError):
        block.forward(t)
    block.forward(t, keep=False)  # (nothing of it is read later)
    block.forward(rows())
    with pytest.raises(ValueError):
        block.backward(rows(), t)
    with pytest.raises(ValueError):
        block.backward(t, rows())
    block.backward(rows(), rows())


def test_of_the_returned_gradient(block):
    x, g = rows(), rows()
    block.forward(x)
    dx = block.backward(x, g)
    block.backward(x, dx)
    block.backward(x, g)  # x is what it was
    block.forward(dx)
    block.backward(dx, g)
    with pytest.raises(RuntimeError):
        block.backward(dx, g)  # it has become its own gradient


def test_no_rows(block):
    none = torch.zeros((0, 64), dtype=torch.bfloat16)
    block.forward(none)
    block.backward(none, none)
