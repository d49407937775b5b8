"""The residual attention block's own bookkeeping, without a GPU: its calls into the library are replaced by
ones that compute nothing, and what it refuses is looked at."""
import pytest

torch = pytest.importorskip("torch")

from paper_2609_10632_amd import attention  # noqa: E402

CALLS = ("numbat_group_norm_fwd", "numbat_group_norm_bwd", "numbat_linear_fwd", "numbat_linear_bwd_data",
         "numbat_linear_bwd_weight", "numbat_rotary", "numbat_attention_fwd", "numbat_attention_bwd", "numbat_adamw_step")


@pytest.fixture
def block(monkeypatch):
    for name in CALLS:
        monkeypatch.setattr(attention.nb, name, lambda *a, **k: None)
    return attention.AttentionBlock(3, (4, 5), 64, 2, groups=8, device="cpu")


def rows(n, width=64):
    return torch.zeros((n, width), dtype=torch.bfloat16)


def test_backward_takes_what_a_forward_has_kept(block):
    with pytest.raises(RuntimeError):
        block.backward(rows(60), rows(60))  # no forward yet
    block.forward(rows(60))
    block.backward(rows(60), rows(60))
    block.backward(rows(60), rows(60), accumulate=True)  # as often as wanted
    with pytest.raises(RuntimeError):
        block.backward(rows(60), rows(60), (5, 4))
    with pytest.raises(RuntimeError):
        block.backward(rows(60), rows(60), lengths=torch.zeros(3, dtype=torch.int32))
    block.forward(rows(60), keep=False)  # the buffers now hold another input's activations
    with pytest.raises(RuntimeError):
        block.backward(rows(60), rows(60))
    block.forward(rows(60))
    block.forward(rows(24), (2, 4))
    with pytest.raises(RuntimeError):
        block.backward(rows(60), rows(60))
    block.backward(rows(24), rows(24), (2, 4))
    block.step(1e-3)  # the weights are no longer those of the forward
    with pytest.raises(RuntimeError):
        block.backward(rows(24), rows(24), (2, 4))


def test_a_forward_that_fails_keeps_nothing(block, monkeypatch):
    block.forward(rows(60))

    def fail(*a, **k):
        raise ValueError

    monkeypatch.setattr(attention.nb, "numbat_attention_fwd", fail)
    with pytest.raises(ValueError):
        block.forward(rows(60))
    with pytest.raises(RuntimeError):
        block.backward(rows(60), rows(60))


def test_refusals(block):
    for x, extents in ((rows(80), None), (rows(61), None), (rows(60, 72), None), (rows(60).float(), None), (rows(60), (4, 5, 1)),
                       (rows(64), (4, 4)), (rows(60), (0, 5)), (torch.zeros((64, 60), dtype=torch.bfloat16).t(), None)):
        with pytest.raises(ValueError):
            block.forward(x, extents)
    for lengths in (torch.zeros(3), torch.zeros(2, dtype=torch.int32), torch.zeros((3, 1), dtype=torch.int32),
                    torch.zeros(6, dtype=torch.int32)[::2]):
        with pytest.raises(ValueError):
            block.forward(rows(60), lengths=lengths)
    with pytest.raises(ValueError):
        block.forward(block.y)
    block.forward(rows(60))
    with pytest.raises(ValueError):
        block.backward(rows(60), rows(59))
    for kw in ({"heads": 3}, {"heads": 16}, {"kv_heads": 3}, {"groups": 7}, {"pairs": (3,)}):
        with pytest.raises(ValueError):
            attention.AttentionBlock(**{"images": 3, "extents": (4, 5), "width": 64, "heads": 2, "groups": 8, "device": "cpu", **kw})


def test_pairs(block):
    assert block.pairs == (8, 8)
    assert attention.AttentionBlock(1, (2, 3, 4), 64, 1, groups=8, device="cpu").pairs == (12, 10, 10)
    assert attention.AttentionBlock(1, (7,), 64, 1, groups=8, pairs=(), device="cpu").pairs == ()
