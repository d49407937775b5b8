"""Results that take an operand's buffer (the linear forward's residual, layer norm's x and residual
gradient) without a GPU: rows that the result would move within the buffer are refused, before a
launch, since one block's rows would overwrite what another has yet to read."""
import pytest

from paper_2609_10632_amd import numbat as nb
from test_mlp_abi_cpu import P, status_of


def test_linear_residual():
    # (sizes that need a workspace: without one, a call that passes the checks before it is refused for it)
    def call(residual, m=20001, **strides):
        p = nb.linear_problem(m, 2049, 1025, **strides)
        return status_of(nb.numbat_linear_fwd, p, 2 * P, 3 * P, None, residual, None, P)

    for strides in ({"y_row_stride": 2056}, {"r_row_stride": 2056}, {"y_row_stride": 2064, "r_row_stride": 2056}):
        assert status_of(nb.numbat_workspace_size, nb.OP_LINEAR_FWD, nb.linear_problem(20001, 2049, 1025, **strides)) == nb.OK
        assert call(P, **strides) == nb.ERR_BAD_DESC, strides
        assert call(4 * P, **strides) == nb.ERR_WORKSPACE, strides
    assert call(P) == call(P, y_row_stride=2056, r_row_stride=2056) == call(P, r_row_stride=2049) == nb.ERR_WORKSPACE


@pytest.mark.parametrize("kw", ({"x_row_stride": 24}, {"y_row_stride": 24}, {"x_type": nb.F32},
                                {"y_type": nb.F32, "x_row_stride": 16}))
def test_layer_norm_x(kw):
    p = nb.layer_norm_problem(8, 16, **kw)
    assert status_of(nb.numbat_layer_norm_fwd, p, P, None, None, P) == nb.ERR_BAD_DESC


def test_layer_norm_residual_gradient():
    def call(res, dx, **strides):
        p = nb.layer_norm_problem(8, 16, **strides)
        return status_of(nb.numbat_layer_norm_bwd, p, 2 * P, 3 * P, 4 * P, 5 * P, None, res, dx, None, None, False, None)

    for strides in ({"r_row_stride": 24}, {"dx_row_stride": 24}, {"r_row_stride": 24, "dx_row_stride": 32}):
        assert call(P, P, **strides) == nb.ERR_BAD_DESC, strides
        assert call(P, 6 * P, **strides) == nb.ERR_WORKSPACE, strides
    assert call(P, P) == call(P, P, r_row_stride=24, dx_row_stride=24) == call(None, P, dx_row_stride=24) == nb.ERR_WORKSPACE
