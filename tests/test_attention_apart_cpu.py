"""Attention's results in its operands' buffers are refused, before anything is enqueued."""
import pytest

from paper_2609_10632_amd import numbat as nb

AT = {n: 0x1000 * (i + 1) for i, n in enumerate(("q", "k", "v", "y", "dy", "lse", "ql", "kl", "dq", "dk", "dv", "ws"))}


def problem(**kw):
    return nb.attention_problem(**{"batch": 2, "q_len": 30, "kv_len": 50, "q_heads": 4, "kv_heads": 2, "d": 64, **kw})


def refusal(fn, *a, **k):
    with pytest.raises(nb.NumbatError) as e:
        fn(*a, **k)
    assert e.value.detail
    return e.value.status


def forward(p, **kw):
    t = {**AT, **kw}
    nb.numbat_attention_fwd(p, t["q"], t["k"], t["v"], t["ql"], t["kl"], t["y"], t["lse"], t["ws"], ws_bytes=1 << 40)


def backward(p, **kw):
    t = {**AT, **kw}
    nb.numbat_attention_bwd(p, t["dy"], t["q"], t["k"], t["v"], t["y"], t["lse"], t["ql"], t["kl"], t["dq"], t["dk"], t["dv"],
                            t["ws"], ws_bytes=1 << 40)


@pytest.mark.parametrize("result", ("y", "lse"))
@pytest.mark.parametrize("operand", ("q", "k", "v", "ql", "kl"))
def test_forward(result, operand):
    assert refusal(forward, problem(), **{result: AT[operand]}) == nb.ERR_BAD_DESC


@pytest.mark.parametrize("result", ("dq", "dk", "dv"))
@pytest.mark.parametrize("operand", ("dy", "q", "k", "v", "y", "lse", "ql", "kl"))
def test_backward(result, operand):
    assert refusal(backward, problem(), **{result: AT[operand]}) == nb.ERR_BAD_DESC


def test_two_results_in_one():
    assert refusal(forward, problem(), y=AT["lse"]) == nb.ERR_BAD_DESC
    for a, b in (("dq", "dk"), ("dk", "dv"), ("dq", "dv")):
        assert refusal(backward, problem(), **{a: AT[b]}) == nb.ERR_BAD_DESC


def test_what_is_not_there_lies_nowhere():
    """No queries: nothing of theirs is given, and the address that is missing is not one that they share."""
    p = problem(q_len=0)
    gone = dict.fromkeys(("dy", "q", "y", "lse", "ql", "kl", "dq"))
    assert refusal(backward, p, **gone, dk=AT["k"]) == nb.ERR_BAD_DESC
    assert refusal(backward, p, **gone, dk=AT["dv"]) == nb.ERR_BAD_DESC
