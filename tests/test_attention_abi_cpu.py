"""The residual attention block's entry points without a GPU: header, binding and library agree, and every
refusal comes with its status before anything is enqueued."""
import ctypes
import os
import re

import pytest

from paper_2609_10632_amd import numbat as nb

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 0x1000  # an aligned address that is never followed


def status_of(fn, *a, **k):
    try:
        fn(*a, **k)
    except nb.NumbatError as e:
        assert e.detail
        return e.status
    return nb.OK


def test_header_binding_and_library_agree():
    text = open(os.path.join(ROOT, "include", "numbat_attention.h")).read()
    first, count = (int(re.search(rf"NUMBAT_ATTENTION_KERNEL_CLASS_{w} (\d+)", text).group(1)) for w in ("FIRST", "COUNT"))
    assert nb.ATTENTION_KERNEL_CLASSES == range(first, first + count)
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = set(re.findall(r"\b(numbat_[a-z0-9_]+)\s*\(", text))
    assert names == set(nb.EXPORTED_ATTENTION)
    for n in names:
        assert getattr(nb.load(), n) is not None and callable(getattr(nb, n))
    # uint32, int32, int64, 3 int32, float, 2 int32, 4 int64
    assert ctypes.sizeof(nb.numbat_group_norm_problem) == 72
    # uint32, 3 int32, int64, 8 int32, 4 int32, double, 2 int64
    assert ctypes.sizeof(nb.numbat_rotary_problem) == 96
    # uint32, 7 int32, float, int32, 4 int64
    assert ctypes.sizeof(nb.numbat_attention_problem) == 72


def test_kernel_classes():
    names = [nb.numbat_kernel_class_name(i) for i in nb.ATTENTION_KERNEL_CLASSES]
    assert all(names) and len(set(names)) == len(names)
    assert nb.numbat_kernel_class_name(nb.ATTENTION_KERNEL_CLASSES.stop) == ""
    assert nb.numbat_kernel_class_name(nb.ATTENTION_KERNEL_CLASSES.start - 1) == ""
    nb.numbat_timing_enable(True)
    assert all(nb.numbat_timing_read(i) == (0.0, 0) for i in nb.ATTENTION_KERNEL_CLASSES)
    nb.numbat_timing_enable(False)


def gn_fwd(p, x=P, y=P + 64, gamma=None, beta=None, mean=None, rstd=None, ws=P, b=1 << 40):
    nb.numbat_group_norm_fwd(p, x, gamma, beta, y, mean, rstd, ws, ws_bytes=b)


def gn_bwd(p, dy=P, x=P, mean=P, rstd=P, gamma=None, beta=None, res=None, dx=P + 64, dg=P, db=None, ws=P, b=1 << 40):
    nb.numbat_group_norm_bwd(p, dy, x, mean, rstd, gamma, beta, dx, dg, db, False, ws, residual_grad=res, ws_bytes=b)


@pytest.mark.parametrize("call,op", [(gn_fwd, nb.OP_GROUP_NORM_FWD), (gn_bwd, nb.OP_GROUP_NORM_BWD)])
def test_group_norm_refusals(call, op):
    make = lambda **kw: nb.group_norm_problem(**{"n": 2, "m": 50000, "c": 24, "groups": 3, **kw})  # noqa: E731
    bad = make()
    bad.struct_size += 8
    assert status_of(call, bad) == nb.ERR_VERSION
    for kw in ({"n": -1}, {"m": -1}, {"c": 0}, {"groups": 0}, {"groups": 5}, {"groups": 25}, {"act": 5}, {"act": -1},
               {"eps": -1.0}, {"eps": float("nan")}, {"eps": float("inf")}, {"x_type": 2}, {"y_type": -1},
               {"x_row_stride": 23}, {"y_row_stride": -24}, {"r_row_stride": 8}, {"dx_row_stride": (1 << 21) + 8}):
        assert status_of(call, make(**kw)) == nb.ERR_BAD_DESC, kw
        assert status_of(nb.numbat_workspace_size, op, make(**kw)) == nb.ERR_BAD_DESC, kw
    for kw in ({"n": 65536}, {"c": 65544, "groups": 3}, {"m": 1 << 31}):
        assert status_of(call, make(**kw)) == nb.ERR_UNSUPPORTED, kw
    p = make()
    for arg in ("x", "y", "mean", "rstd", "dy") if call is gn_bwd else ("x", "y"):
        if call is gn_bwd and arg == "y":
            continue
        assert status_of(call, p, **{arg: None}) == nb.ERR_NULL, arg
    for arg in ("x", "dy", "dx", "res") if call is gn_bwd else ("x", "y"):
        assert status_of(call, p, **{arg: P + 8}) == nb.ERR_ALIGN, arg
    for arg in ("gamma", "beta", "mean", "rstd"):
        assert status_of(call, p, **{arg: P + 2}) == nb.ERR_ALIGN, arg
    need = nb.numbat_workspace_size(op, p)
    assert need > 256
    assert status_of(call, p, ws=None) == nb.ERR_WORKSPACE
    assert status_of(call, p, b=need - 1) == nb.ERR_WORKSPACE
    assert status_of(call, p, ws=P + 4) == nb.ERR_ALIGN
    for kw in ({"n": 0}, {"m": 0}):
        assert nb.numbat_workspace_size(op, make(**kw)) == 0
    assert status_of(gn_fwd, make(n=0), None, None, ws=None, b=0) == nb.OK


def test_group_norm_in_place():
    make = lambda **kw: nb.group_norm_problem(2, 50, 24, 3, **kw)  # noqa: E731
    assert status_of(gn_fwd, make(y_type=nb.F32), y=P) == nb.ERR_BAD_DESC
    assert status_of(gn_fwd, make(x_row_stride=32), y=P) == nb.ERR_BAD_DESC
    assert status_of(gn_bwd, make(dx_row_stride=32), dx=P, dy=P + 64) == nb.ERR_BAD_DESC
    assert status_of(gn_bwd, make(y_row_stride=32), dx=P, x=P + 64) == nb.ERR_BAD_DESC
    assert status_of(gn_bwd, make(y_type=nb.F32), dx=P, x=P + 64) == nb.ERR_BAD_DESC
    assert status_of(gn_bwd, make(r_row_stride=32), dx=P, res=P, x=P + 64, dy=P + 64) == nb.ERR_BAD_DESC
    assert status_of(gn_bwd, make(), dx=None, dg=None) == nb.ERR_NULL
    assert status_of(gn_bwd, make(), dx=None, res=P) == nb.ERR_NULL


def test_rotary_refusals():
    def call(p, x=P, pos=None, y=P + 64):
        nb.numbat_rotary(p, x, pos, y)

    make = lambda **kw: nb.rotary_problem(**{"m": 8, "heads": 2, "d": 16, "pairs": (4, 4), "extents": (2, 4), **kw})  # noqa: E731
    bad = make()
    bad.struct_size -= 4
    assert status_of(call, bad) == nb.ERR_VERSION
    for kw in ({"m": -1}, {"heads": 0}, {"d": 1}, {"pairs": (4, 0)}, {"pairs": (4, 5)}, {"pairs": (-1, 4)}, {"extents": (2, 0)},
               {"extents": None}, {"layout": 2}, {"type": 2}, {"base": 1.0}, {"base": float("nan")}, {"base": 1e31},
               {"x_row_stride": 31}, {"y_row_stride": -32}, {"x_row_stride": (1 << 21) + 8}):
        assert status_of(call, make(**kw)) == nb.ERR_BAD_DESC, kw
    for field, value in (("axes", 0), ("axes", 5), ("shared", 2), ("inverse", -1)):
        bad = make()
        setattr(bad, field, value)
        assert status_of(call, bad) == nb.ERR_BAD_DESC, field
    bad = make()
    bad.axes = 1  # the second axis' pairs belong to none
    assert status_of(call, bad) == nb.ERR_BAD_DESC
    for kw in ({"m": 1 << 31}, {"d": 1024, "pairs": (200, 57)}, {"heads": 1 << 18}):
        assert status_of(call, make(**kw)) == nb.ERR_UNSUPPORTED, kw
    p = make()
    assert status_of(call, p, x=None) == nb.ERR_NULL
    assert status_of(call, p, y=None) == nb.ERR_NULL
    for kw in ({"x": P + 8}, {"y": P + 2}, {"pos": P + 2}):
        assert status_of(call, p, **kw) == nb.ERR_ALIGN, kw
    assert status_of(call, make(x_row_stride=40), y=P) == nb.ERR_BAD_DESC
    assert status_of(call, make(m=0), None, None, None) == nb.OK
    with pytest.raises(ValueError):
        nb.rotary_problem(8, 2, 16, (4, 4), extents=(2,))
    with pytest.raises(ValueError):
        nb.rotary_problem(8, 2, 16, ())


def attn_fwd(p, q=P, k=P, v=P, ql=None, kl=None, y=P, lse=None, ws=P, b=1 << 40):
    nb.numbat_attention_fwd(p, q, k, v, ql, kl, y, lse, ws, ws_bytes=b)


def attn_bwd(p, dy=P, q=P, k=P, v=P, y=P, lse=P, ql=None, kl=None, dq=P, dk=P, dv=P, ws=P, b=1 << 40):
    nb.numbat_attention_bwd(p, dy, q, k, v, y, lse, ql, kl, dq, dk, dv, ws, ws_bytes=b)


@pytest.mark.parametrize("call,op", [(attn_fwd, nb.OP_ATTENTION_FWD), (attn_bwd, nb.OP_ATTENTION_BWD)])
def test_attention_refusals(call, op):
    make = lambda **kw: nb.attention_problem(**{"batch": 2, "q_len": 1, "kv_len": 20000, "q_heads": 4, "kv_heads": 2,  # noqa: E731
                                                "d": 64, **kw})
    bad = make()
    bad.struct_size += 8
    assert status_of(call, bad) == nb.ERR_VERSION
    for kw in ({"batch": -1}, {"q_len": -1}, {"kv_len": -1}, {"q_heads": 0}, {"kv_heads": 0}, {"kv_heads": 3}, {"d": 0},
               {"scale": 0.0}, {"scale": -1.0}, {"scale": float("nan")}, {"scale": float("inf")}, {"scale": 2e38}, {"q_row_stride": 248},
               {"y_row_stride": -256}, {"k_row_stride": 64}, {"v_row_stride": (1 << 21) + 8}):
        assert status_of(call, make(**kw)) == nb.ERR_BAD_DESC, kw
        assert status_of(nb.numbat_workspace_size, op, make(**kw)) == nb.ERR_BAD_DESC, kw
    for field, value in (("reserved", 1), ("causal", 2)):
        bad = make()
        setattr(bad, field, value)
        assert status_of(call, bad) == nb.ERR_BAD_DESC
    for kw in ({"d": 60}, {"d": 136}, {"batch": 65536}, {"q_len": (1 << 29) + 1}, {"kv_len": (1 << 30) + 1},
               {"batch": 65535, "kv_len": 1 << 20}, {"batch": 65535, "q_len": 1 << 20}):
        assert status_of(call, make(**kw)) == nb.ERR_UNSUPPORTED, kw
    for kw in ({"q_row_stride": 260}, {"k_row_stride": 132}, {"v_row_stride": 129}, {"y_row_stride": 257}):
        assert status_of(call, make(**kw)) == nb.ERR_ALIGN, kw
    p = make()
    for arg in ("q", "k", "v", "y") if call is attn_fwd else ("dy", "q", "k", "v", "y", "lse", "dq", "dk", "dv"):
        assert status_of(call, p, **{arg: None}) == nb.ERR_NULL, arg
        if arg != "lse":
            assert status_of(call, p, **{arg: P + 8}) == nb.ERR_ALIGN, arg
    for arg in ("ql", "kl", "lse"):
        assert status_of(call, p, **{arg: P + 2}) == nb.ERR_ALIGN, arg
    need = nb.numbat_workspace_size(op, p)
    assert need > 256
    assert status_of(call, p, ws=None) == nb.ERR_WORKSPACE
    assert status_of(call, p, b=need - 1) == nb.ERR_WORKSPACE
    assert status_of(call, p, ws=P + 4) == nb.ERR_ALIGN
    # nothing to do, and nothing is needed
    assert nb.numbat_workspace_size(op, make(batch=0)) == 0
    assert status_of(call, make(batch=0), *[None] * 3, ws=None, b=0) == nb.OK
    if call is attn_fwd:
        assert status_of(call, make(q_len=0), None, None, None, ws=None, b=0) == nb.OK
