"""The functions of include/numbat_mlp.h without a GPU: exported, bound, and refusing every bad
argument with its own status before anything is launched."""
import ctypes
import os
import re

import pytest

from paper_2609_10632_amd import numbat as nb

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 1 << 20  # an aligned address that is never touched


def status_of(fn, *a, **k):
    try:
        fn(*a, **k)
    except nb.NumbatError as e:
        assert e.detail
        return e.status
    return nb.OK


def test_header_binding_and_library_agree():
    text = open(os.path.join(ROOT, "include", "numbat_mlp.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = set(re.findall(r"\b(numbat_[a-z0-9_]+)\s*\(", text))
    assert names == set(nb.EXPORTED_MLP)
    for n in names:
        assert getattr(nb.load(), n) is not None and callable(getattr(nb, n))
    assert ctypes.sizeof(nb.numbat_linear_problem) == 64
    assert ctypes.sizeof(nb.numbat_layer_norm_problem) == 64
    assert ctypes.sizeof(nb.numbat_adamw_tensor) == 72


def test_kernel_classes():
    names = [nb.numbat_kernel_class_name(i) for i in nb.MLP_KERNEL_CLASSES]
    assert all(names) and len(set(names)) == len(names)
    assert nb.numbat_kernel_class_name(nb.MLP_KERNEL_CLASSES.stop) == ""
    nb.numbat_timing_enable(True)
    assert all(nb.numbat_timing_read(i) == (0.0, 0) for i in nb.MLP_KERNEL_CLASSES)
    nb.numbat_timing_enable(False)


LINEAR = {
    "fwd": lambda p, x=P, w=P, y=P, ws=None, b=0, bias=None, res=None, z=None:
        nb.numbat_linear_fwd(p, x, w, bias, res, z, y, ws, ws_bytes=b),
    "data": lambda p, x=P, w=P, y=P, ws=None, b=0, z=P: nb.numbat_linear_bwd_data(p, x, w, z, y, False, ws, ws_bytes=b),
    "weight": lambda p, x=P, w=P, y=P, ws=None, b=0: nb.numbat_linear_bwd_weight(p, x, w, y, None, False, ws, ws_bytes=b),
}


@pytest.mark.parametrize("which", LINEAR)
def test_linear_refusals(which):
    call = LINEAR[which]
    ok = nb.linear_problem(8, 16, 24)
    bad = nb.linear_problem(8, 16, 24)
    bad.struct_size -= 8
    assert status_of(call, bad) == nb.ERR_VERSION
    for kw in ({"m": -1}, {"n": 0}, {"k": 0}, {"act": 5}, {"act": -1}, {"y_type": 2}, {"x_row_stride": 23},
               {"y_row_stride": 15}, {"r_row_stride": 8}, {"z_row_stride": 7}, {"x_row_stride": (1 << 21) + 8},
               {"y_row_stride": -16}):
        assert status_of(call, nb.linear_problem(**{"m": 8, "n": 16, "k": 24, **kw})) == nb.ERR_BAD_DESC, kw
    for kw in ({"m": 1 << 31}, {"n": (1 << 21) + 1}, {"k": (1 << 21) + 1}):
        assert status_of(call, nb.linear_problem(**{"m": 8, "n": 16, "k": 24, **kw})) == nb.ERR_UNSUPPORTED, kw
    bad = nb.linear_problem(8, 16, 24)
    bad.reserved = 1
    assert status_of(call, bad) == nb.ERR_BAD_DESC
    for arg in ("x", "w", "y"):
        assert status_of(call, ok, **{arg: None}) == nb.ERR_NULL, arg
        if which != "weight" or arg != "y":
            assert status_of(call, ok, **{arg: P + 8}) == nb.ERR_ALIGN, arg
    # large operands with odd rows are padded in the workspace
    op = {"fwd": nb.OP_LINEAR_FWD, "data": nb.OP_LINEAR_BWD_DATA, "weight": nb.OP_LINEAR_BWD_WEIGHT}[which]
    odd = nb.linear_problem(20001, 2049, 1025)
    need = nb.numbat_workspace_size(op, odd)
    assert need >= 256 + 20001 * 1032 * 2
    assert status_of(call, odd) == nb.ERR_WORKSPACE
    assert status_of(call, odd, ws=P, b=need - 1) == nb.ERR_WORKSPACE
    assert status_of(call, odd, ws=P + 4, b=need) == nb.ERR_ALIGN


def test_linear_fine_points():
    call = LINEAR["fwd"]
    ok = nb.linear_problem(8, 16, 24)
    assert status_of(call, ok, res=P + 2) == nb.ERR_ALIGN
    assert status_of(call, ok, z=P + 2) == nb.ERR_ALIGN
    assert status_of(LINEAR["data"], nb.linear_problem(8, 16, 24, act=nb.ACT_SILU), z=None) == nb.ERR_NULL
    # a strided z is as wide as the output forward and as the input backward
    assert status_of(call, nb.linear_problem(8, 16, 24, z_row_stride=16), x=None) == nb.ERR_NULL
    assert status_of(LINEAR["data"], nb.linear_problem(8, 16, 24, z_row_stride=16)) == nb.ERR_BAD_DESC
    # no rows: nothing to do, and nothing is needed
    empty = nb.linear_problem(0, 16, 24)
    assert status_of(call, empty, None, None, None) == nb.OK
    assert status_of(LINEAR["data"], empty, None, None, None) == nb.OK
    for op in (nb.OP_LINEAR_FWD, nb.OP_LINEAR_BWD_DATA, nb.OP_LINEAR_BWD_WEIGHT):
        assert nb.numbat_workspace_size(op, empty) == 0
    assert status_of(nb.numbat_workspace_size, nb.OP_LINEAR_FWD, nb.linear_problem(8, 0, 24)) == nb.ERR_BAD_DESC


def test_layer_norm_refusals():
    fwd = lambda p, x=P, y=P: nb.numbat_layer_norm_fwd(p, x, None, None, y)  # noqa: E731

    def bwd(p, dy=P, x=P, mean=P, rstd=P, res=None, dx=P, dg=P, ws=P, b=1 << 30):
        nb.numbat_layer_norm_bwd(p, dy, x, mean, rstd, None, res, dx, dg, None, False, ws, ws_bytes=b)

    for call in (fwd, bwd):
        bad = nb.layer_norm_problem(8, 16)
        bad.struct_size += 8
        assert status_of(call, bad) == nb.ERR_VERSION
        for kw in ({"m": -1}, {"c": 0}, {"eps": -1.0}, {"eps": float("nan")}, {"eps": float("inf")}, {"x_type": 2},
                   {"y_type": -1}, {"x_row_stride": 8}, {"y_row_stride": 15}, {"r_row_stride": 1}, {"dx_row_stride": -16}):
            assert status_of(call, nb.layer_norm_problem(**{"m": 8, "c": 16, **kw})) == nb.ERR_BAD_DESC, kw
        for kw in ({"m": 1 << 31}, {"c": (1 << 21) + 1}):
            assert status_of(call, nb.layer_norm_problem(**{"m": 8, "c": 16, **kw})) == nb.ERR_UNSUPPORTED, kw
    p = nb.layer_norm_problem(8, 16)
    for arg in ("x", "y"):
        assert status_of(fwd, p, **{arg: None}) == nb.ERR_NULL
        assert status_of(fwd, p, **{arg: P + 2}) == nb.ERR_ALIGN
    for arg in ("dy", "x", "mean", "rstd"):
        assert status_of(bwd, p, **{arg: None}) == nb.ERR_NULL
    assert status_of(bwd, p, dx=None, dg=None) == nb.ERR_NULL
    assert status_of(bwd, p, dx=None, res=P) == nb.ERR_NULL
    for arg in ("dy", "x", "res", "dx"):
        assert status_of(bwd, p, **{arg: P + 8}) == nb.ERR_ALIGN
    assert status_of(bwd, p, ws=None) == nb.ERR_WORKSPACE
    assert status_of(bwd, p, b=nb.numbat_workspace_size(nb.OP_LAYER_NORM_BWD, p) - 1) == nb.ERR_WORKSPACE
    assert nb.numbat_workspace_size(nb.OP_LAYER_NORM_BWD, nb.layer_norm_problem(0, 16)) == 0
    assert status_of(fwd, nb.layer_norm_problem(0, 16), None, None) == nb.OK


def test_adamw_refusals():
    def step(tensors=P, count=1, groups=((1e-3, 0.1),), bits=32, b1=0.9, b2=0.95, eps=1e-8, t=1, max_norm=0.0, norm=None,
             ws=P, b=1 << 20):
        nb.numbat_adamw_step(tensors, count, groups, bits, b1, b2, eps, t, max_norm, norm, ws, ws_bytes=b)

    inf, nan = float("inf"), float("nan")
    assert status_of(step, tensors=None) == nb.ERR_NULL
    assert status_of(step, tensors=P + 4) == nb.ERR_ALIGN
    assert status_of(step, max_norm=1.0, norm=P + 2) == nb.ERR_ALIGN
    assert status_of(step, bits=16) == nb.ERR_UNSUPPORTED
    for kw in ({"count": 0}, {"count": 1025}, {"groups": ()}, {"groups": ((1e-3, 0.0),) * 9}, {"b1": 1.0}, {"b1": -0.1},
               {"b2": nan}, {"eps": 0.0}, {"eps": inf}, {"t": 0}, {"max_norm": -1.0}, {"max_norm": inf}, {"norm": P},
               {"groups": ((nan, 0.0),)}, {"groups": ((1e-3, -1.0),)}, {"groups": ((1e-3, inf),)}):
        assert status_of(step, **kw) == nb.ERR_BAD_DESC, kw
    assert status_of(step, ws=None) == nb.ERR_WORKSPACE
    need = nb.numbat_workspace_size(nb.OP_ADAMW, None)
    assert status_of(step, b=need - 1) == nb.ERR_WORKSPACE
    values = nb.numbat_adamw_state_values
    assert status_of(values, -1, P, P, P, P, P, P) == nb.ERR_BAD_DESC
    assert status_of(values, 0, None, None, None, None, None, None) == nb.OK
    for i in range(6):
        args = [P] * 6
        args[i] = None
        assert status_of(values, 8, *args) == nb.ERR_NULL


def test_products_past_one_launch_are_refused():
    """A launch takes fewer than 2^32 threads: a 64 x 64 tile's 256 threads, 2^24 tiles."""
    big = nb.linear_problem((1 << 31) - 1, 8, 8)
    for op, which in ((nb.OP_LINEAR_FWD, "fwd"), (nb.OP_LINEAR_BWD_DATA, "data")):
        assert status_of(nb.numbat_workspace_size, op, big) == nb.ERR_UNSUPPORTED
        assert status_of(LINEAR[which], big, ws=P, b=1 << 40) == nb.ERR_UNSUPPORTED
    wide = nb.linear_problem(8, 1 << 21, 1 << 21)
    assert status_of(LINEAR["weight"], wide, ws=P, b=1 << 62) == nb.ERR_UNSUPPORTED
    # the sums over as many rows are few tiles
    assert nb.numbat_workspace_size(nb.OP_LINEAR_BWD_WEIGHT, big) > 0
