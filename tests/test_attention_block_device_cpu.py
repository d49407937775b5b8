"""The residual attention block and devices, without a GPU: operands elsewhere are refused, and a block whose device is
not the current one makes its own current while it calls the library."""
import contextlib

import pytest

torch = pytest.importorskip("torch")

from paper_2609_10632_amd import attention  # noqa: E402
from test_attention_block_cpu import CALLS  # noqa: E402


@pytest.fixture
def block(monkeypatch):
    for name in CALLS:
        monkeypatch.setattr(attention.nb, name, lambda *a, **k: None)
    return attention.AttentionBlock(2, (4, 5), 64, 2, groups=8, device="cpu")


def rows(device="cpu"):
    return torch.zeros((40, 64), dtype=torch.bfloat16, device=device)


def test_operands_elsewhere(block):
    with pytest.raises(ValueError):
        block.forward(rows("meta"))
    with pytest.raises(ValueError):
        block.forward(rows(), lengths=torch.zeros(2, dtype=torch.int32, device="meta"))
    lengths = torch.zeros(2, dtype=torch.int32)
    block.forward(rows(), lengths=lengths)
    for x, g, n in ((rows("meta"), rows(), lengths), (rows(), rows("meta"), lengths), (rows(), rows(), lengths.to("meta"))):
        with pytest.raises(ValueError):
            block.backward(x, g, lengths=n)
    block.backward(rows(), rows(), lengths=lengths)


def test_the_current_device(block, monkeypatch):
    """A block on the second of two cards; the calls note which is current when they are made."""
    current, seen = [0], []

    @contextlib.contextmanager
    def device(d):
        was, current[0] = current[0], torch.device(d).index
        yield
        current[0] = was

    monkeypatch.setattr(attention.torch.cuda, "current_device", lambda: current[0])
    monkeypatch.setattr(attention.torch.cuda, "device", device)
    for name in CALLS:
        monkeypatch.setattr(attention.nb, name, lambda *a, **k: seen.append(current[0]))
    x, g = rows(), rows()
    block.place = torch.device("cuda", 1)
    monkeypatch.setattr(block, "_check", lambda *a, **k: 64)
    block.forward(x)
    block.backward(x, g)
    block.step(1e-3)
    assert len(seen) == 5 + 7 + 1 and set(seen) == {1} and current == [0]
    seen.clear()
    current[0] = 1
    block.step(1e-3)
    block.place = torch.device("cuda", 0)
    block.step(1e-3)
    assert seen == [1, 0] and current == [1]
