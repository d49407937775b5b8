"""The residual MLP block's own bookkeeping, without a GPU: its calls into the library are replaced by
ones that compute nothing, and what it refuses is looked at."""
import pytest

torch = pytest.importorskip("torch")

from paper_2609_10632_amd import mlp  # noqa: E402

CALLS = ("numbat_linear_fwd", "numbat_linear_bwd_data", "numbat_linear_bwd_weight", "numbat_layer_norm_fwd",
         "numbat_layer_norm_bwd", "numbat_adamw_step")


@pytest.fixture
def block(monkeypatch):
    for name in CALLS:
        monkeypatch.setattr(mlp.nb, name, lambda *a, **k: None)
    return mlp.MlpBlock(10, 16, 32, device="cpu")


def rows(n):
    return torch.zeros((n, 16), dtype=torch.bfloat16)


def test_backward_takes_what_a_forward_has_kept(block):
    with pytest.raises(RuntimeError):
        block.backward(rows(10), rows(10))  # no forward yet
    block.forward(rows(10))
    block.backward(rows(10), rows(10))
    block.backward(rows(10), rows(10), accumulate=True)  # as often as wanted
    block.forward(rows(10), keep=False)  # the buffers now hold another input's activations
    with pytest.raises(RuntimeError):
        block.backward(rows(10), rows(10))
    block.forward(rows(10))
    block.forward(rows(7))
    with pytest.raises(RuntimeError):
        block.backward(rows(10), rows(10))
    block.backward(rows(7), rows(7))
    block.step(1e-3)  # the weights are no longer those of the forward
    with pytest.raises(RuntimeError):
        block.backward(rows(7), rows(7))


def test_a_forward_that_fails_keeps_nothing(block, monkeypatch):
    block.forward(rows(10))

    def fail(*a, **k):
        raise ValueError

    monkeypatch.setattr(mlp.nb, "numbat_linear_fwd", fail)
    with pytest.raises(ValueError):
        block.forward(rows(10))
    with pytest.raises(RuntimeError):
        block.backward(rows(10), rows(10))


def test_a_step_that_is_refused_is_not_counted(block, monkeypatch):
    took = []
    monkeypatch.setattr(mlp.nb, "numbat_adamw_step", lambda *a, **k: took.append(a[7]))
    block.step(1e-3)

    def refuse(*a, **k):
        raise mlp.nb.NumbatError(mlp.nb.ERR_BAD_DESC, "bad", "detail", "numbat_adamw_step")

    block.forward(rows(10))
    with monkeypatch.context() as m:
        m.setattr(mlp.nb, "numbat_adamw_step", refuse)
        with pytest.raises(mlp.nb.NumbatError):
            block.step(float("nan"))
    block.backward(rows(10), rows(10))  # nor has it changed the weights
    block.step(1e-3)
    assert took == [1, 2]  # the bias corrections go by the steps taken


def test_a_step_without_a_clip_has_no_norm(block):
    assert block.step(1e-3, max_norm=1.0) is block.norm
    assert block.step(1e-3, max_norm=0.0) is None  # not that of an earlier step


def test_a_forward_over_its_own_output_keeps_nothing(block):
    """Its last call writes y over the rows that a backward would read as x."""
    y = block.forward(rows(10))
    with pytest.raises(ValueError):
        block.forward(y)
    with pytest.raises(ValueError):
        block.forward(y[2:7])
    block.forward(y, keep=False)  # serving: nothing reads x afterwards
    with pytest.raises(ValueError):
        block.forward(y[2:7], keep=False)  # but each row of it has to lie where its result goes
    mlp.MlpBlock(0, 16, 32, device="cpu").forward(rows(0))
    block.forward(y.clone())
    block.backward(rows(10), rows(10))
