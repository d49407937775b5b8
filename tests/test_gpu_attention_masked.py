"""Attention (numbat_attention_*) with numbers that are none: what queries that see no key hold reaches nothing, and
what counts reaches all that it belongs to and nothing else."""
import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
if torch.cuda.is_available():
    from paper_2609_10632_amd import blocks
    from paper_2609_10632_amd import numbat as nb

NAN = math.nan


def inputs(batch, q_len, kv_len, heads, kv_heads, feat, seed=0):
    g = torch.Generator().manual_seed(seed)
    new = lambda n, w: torch.randn((n, w), generator=g).bfloat16().cuda()  # noqa: E731
    return {"q": new(batch * q_len, heads * feat), "k": new(batch * kv_len, kv_heads * feat),
            "v": new(batch * kv_len, kv_heads * feat), "dy": new(batch * q_len, heads * feat)}


def run(t, batch, q_len, kv_len, heads, kv_heads, feat, causal=False, y=None):
    print("attention with numbers that are none", batch, q_len, kv_len, heads, kv_heads, feat, flush=True)
    p = nb.attention_problem(batch, q_len, kv_len, heads, kv_heads, feat, causal=causal)
    out = {"y": torch.empty_like(t["q"]), "lse": torch.empty((batch, heads, q_len), device="cuda"),
           "dq": torch.empty_like(t["q"]), "dk": torch.empty_like(t["k"]), "dv": torch.empty_like(t["v"])}
    nb.numbat_attention_fwd(p, t["q"], t["k"], t["v"], None, None, out["y"], out["lse"],
                            blocks.workspace(nb.numbat_workspace_size(nb.OP_ATTENTION_FWD, p)))
    nb.numbat_attention_bwd(p, t["dy"], t["q"], t["k"], t["v"], out["y"] if y is None else y, out["lse"], None, None, out["dq"],
                            out["dk"], out["dv"], blocks.workspace(nb.numbat_workspace_size(nb.OP_ATTENTION_BWD, p)))
    return out


@pytest.mark.parametrize("size", [(2, 100, 37, 2, 2, 32), (1, 300, 90, 4, 2, 64), (1, 1500, 200, 3, 1, 128), (2, 65, 64, 2, 1, 96),
                                  (1, 700, 1, 1, 1, 8)])
@pytest.mark.parametrize("bad", (NAN, math.inf))
def test_queries_that_see_no_key(size, bad):
    """The first q_len - kv_len queries of a causal sequence: their q, dy and y are not taken in."""
    batch, q_len, kv_len = size[:3]
    t = inputs(*size)
    clean = run(t, *size, causal=True)
    none = (torch.arange(batch * q_len) % q_len < q_len - kv_len).cuda()
    for what in ("q", "dy"):
        t[what][none] = bad
    y = clean["y"].clone()
    y[none] = bad
    got = run(t, *size, causal=True, y=y)
    for name in clean:
        assert torch.equal(got[name], clean[name]), name
    assert bool((got["y"][none] == 0).all()) and bool((got["dq"][none] == 0).all())


@pytest.mark.parametrize("size", [(2, 40, 70, 4, 2, 32), (1, 3, 2000, 2, 1, 64), (1, 300, 300, 2, 2, 128)])
@pytest.mark.parametrize("bad", (NAN, math.inf))
def test_what_counts_spreads_as_far_as_it_belongs(size, bad):
    batch, q_len, kv_len, heads, kv_heads, feat = size
    clean = run(inputs(*size), *size)
    group = heads // kv_heads
    split = lambda u, n: u.reshape(batch, n, -1, feat)  # noqa: E731
    lens = {"y": q_len, "dq": q_len, "dk": kv_len, "dv": kv_len}
    b, h = batch - 1, kv_heads - 1  # the last sequence, the last head of k and v and the first of its heads of q

    def check(got, where):
        """where[name]: [batch][rows][heads][feat] of what cannot be a number; a feature that is finite in it is
        allowed where not all of them need be none."""
        for name, n in lens.items():
            none, was, now = where.get(name), split(clean[name], n), split(got[name], n)
            if none is None:
                none = torch.zeros(was.shape, dtype=torch.bool, device="cuda")
            assert torch.equal(now[~none], was[~none]), name
            assert not bool(now[none].isfinite().any()), name

    def marks(name):
        return torch.zeros(split(clean[name], lens[name]).shape, dtype=torch.bool, device="cuda")

    mine = slice(h * group, (h + 1) * group)
    # a value: its feature of every query of its heads; delta and dp with it, hence dq and dk of those rows
    t = inputs(*size)
    split(t["v"], kv_len)[b, 2, h, 5] = bad
    y, dq, dk = marks("y"), marks("dq"), marks("dk")
    y[b, :, mine, 5] = dq[b, :, mine] = dk[b, :, h] = True
    check(run(t, *size), {"y": y, "dq": dq, "dk": dk})
    # a gradient: its query's dq, and all of its head's dk; dv in its feature
    t = inputs(*size)
    split(t["dy"], q_len)[b, 1, h * group, 3] = bad
    dq, dk, dv = marks("dq"), marks("dk"), marks("dv")
    dq[b, 1, h * group] = dk[b, :, h] = dv[b, :, h, 3] = True
    check(run(t, *size), {"dq": dq, "dk": dk, "dv": dv})
    if bad == bad:
        return  # (an infinite score is a weight of one or of nothing)
    # a query: all that comes of it
    t = inputs(*size)
    split(t["q"], q_len)[b, 1, h * group, 3] = bad
    y, dq, dk, dv = (marks(n) for n in ("y", "dq", "dk", "dv"))
    y[b, 1, h * group] = dq[b, 1, h * group] = dk[b, :, h] = dv[b, :, h] = True
    got = run(t, *size)
    check(got, {"y": y, "dq": dq, "dk": dk, "dv": dv})
    assert bool(got["lse"][b, h * group, 1].isnan())
    # a key: every query of its heads
    t = inputs(*size)
    split(t["k"], kv_len)[b, 2, h, 7] = bad
    y, dq, dk, dv = (marks(n) for n in ("y", "dq", "dk", "dv"))
    y[b, :, mine] = dq[b, :, mine] = dk[b, :, h] = dv[b, :, h] = True
    check(run(t, *size), {"y": y, "dq": dq, "dk": dk, "dv": dv})
