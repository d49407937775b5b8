"""The AdamW table's entries name types and pointers that the kernels take at their word: what they would
misread is refused where the table is made."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

from paper_2609_10632_amd import numbat as nb  # noqa: E402


def entry(n=300, grad=torch.float32, bits=32, **change):
    blocks = -(-n // 256)
    e = {"w": torch.zeros(n), "grad": torch.zeros(n, dtype=grad), "group": 1}
    if bits == 32:
        e.update(m=torch.zeros(n), v=torch.zeros(n))
    else:
        e.update(m=torch.zeros(n, dtype=torch.int8), v=torch.zeros(n, dtype=torch.uint8), m_unit=torch.zeros(blocks),
                 v_unit=torch.zeros(blocks))
    e.update(change)
    return {k: v for k, v in e.items() if v is not None}


@pytest.mark.parametrize("bits", (32, 8))
def test_entries(bits):
    given = [entry(bits=bits), entry(5, torch.bfloat16, bits, w_copy=torch.zeros(5, dtype=torch.bfloat16))]
    raw = nb.adamw_table(given)
    got = (nb.numbat_adamw_tensor * 2).from_buffer_copy(raw)
    assert ctypes.sizeof(got) == len(raw)
    assert [e.grad_type for e in got] == [nb.F32, nb.BF16] and [e.n for e in got] == [300, 5]
    for e, d in zip(got, given):
        for f in ("w", "grad", "m", "v", "m_unit", "v_unit", "w_copy"):
            assert getattr(e, f) == (d[f].data_ptr() if f in d else None), f


@pytest.mark.parametrize("dtype", (torch.float16, torch.float64, torch.int16))
def test_gradients_of_other_types(dtype):
    with pytest.raises(TypeError):
        nb.adamw_table([entry(), entry(grad=dtype)])


@pytest.mark.parametrize("unit", ("m_unit", "v_unit"))
def test_8_bit_moments_without_units(unit):
    with pytest.raises(ValueError):
        nb.adamw_table([entry(bits=8, **{unit: None})])
