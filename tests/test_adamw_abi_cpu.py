"""AdamW's scalar arguments without a GPU: they are doubles that the kernels take as fp32, so what is
refused goes by the fp32 value."""
import pytest

from paper_2609_10632_amd import numbat as nb
from test_mlp_abi_cpu import P, status_of


def step(eps=1e-8, max_norm=0.0, norm=None):
    # (no workspace: a call that passes the checks before it is refused for that)
    return status_of(nb.numbat_adamw_step, P, 1, ((1e-3, 0.1),), 32, 0.9, 0.95, eps, 1, max_norm, norm, None)


@pytest.mark.parametrize("tiny", (1e-46, 1e-45, 1e-39, 1.17e-38))
def test_values_that_fp32_does_not_hold(tiny):
    """An eps of zero or below the normal numbers has no finite reciprocal, and a parameter whose moments are zero
    would become NaN; a max_norm of zero would not clip, nor write the norm."""
    assert step(eps=tiny) == nb.ERR_BAD_DESC
    assert step(max_norm=tiny) == step(max_norm=tiny, norm=P) == nb.ERR_BAD_DESC


def test_the_smallest_and_largest():
    smallest = 2.0 ** -126
    assert step(eps=smallest) == step(max_norm=smallest) == step(max_norm=smallest, norm=P) == nb.ERR_WORKSPACE
    assert step(eps=2e38, max_norm=2e38) == nb.ERR_WORKSPACE
