"""Attention (numbat_attention_*) with rows of y and dy further apart than they are long, and otherwise than those of q:
the same bits as from dense rows, and what lies between them neither read nor written."""
import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
if torch.cuda.is_available():
    from paper_2609_10632_amd import blocks
    from paper_2609_10632_amd import numbat as nb


def spread(t, pitch):
    """The rows of t with `pitch` numbers that are none between them."""
    if pitch is None:
        return t.clone()
    wide = torch.full((t.shape[0], t.shape[1] + pitch), math.nan, dtype=t.dtype, device=t.device)
    wide[:, :t.shape[1]] = t
    return wide[:, :t.shape[1]]


def between(t):
    """What lies behind the rows' ends."""
    return t.as_strided((t.shape[0], t.stride(0) - t.shape[1]), (t.stride(0), 1), t.storage_offset() + t.shape[1])


def run(size, pitches, causal, lengths):
    """pitches: of y (and dy), q, k, v."""
    b, q_len, kv_len, heads, kv_heads, feat = size
    g = torch.Generator().manual_seed(3)
    new = lambda n, w: torch.randn((n, w), generator=g).bfloat16().cuda()  # noqa: E731
    q, k, v, dy = new(b * q_len, heads * feat), new(b * kv_len, kv_heads * feat), new(b * kv_len, kv_heads * feat), new(b * q_len, heads * feat)
    q, k, v, dy = spread(q, pitches[1]), spread(k, pitches[2]), spread(v, pitches[3]), spread(dy, pitches[0])
    y, dq, dk, dv = (spread(torch.full_like(t, 7.0).contiguous(), p) for t, p in ((dy, pitches[0]), (q, pitches[1]), (k, pitches[2]), (v, pitches[3])))
    lse = torch.empty((b, heads, q_len), device="cuda")
    ln = [None if n is None else torch.tensor(n, dtype=torch.int32, device="cuda") for n in lengths]
    print("attention rows", size, pitches, causal, lengths, flush=True)
    p = nb.attention_problem(*size, causal=causal, q_row_stride=q.stride(0), k_row_stride=k.stride(0), v_row_stride=v.stride(0),
                             y_row_stride=y.stride(0))
    nb.numbat_attention_fwd(p, q, k, v, *ln, y, lse, blocks.workspace(nb.numbat_workspace_size(nb.OP_ATTENTION_FWD, p)))
    nb.numbat_attention_bwd(p, dy, q, k, v, y, lse, *ln, dq, dk, dv, blocks.workspace(nb.numbat_workspace_size(nb.OP_ATTENTION_BWD, p)))
    for t in (y, dq, dk, dv):
        assert bool(between(t).isnan().all())
    return [t.contiguous() for t in (y, lse, dq, dk, dv)]


@pytest.mark.parametrize("size,causal,lengths", [
    ((1, 100, 130, 2, 2, 64), False, (None, None)),           # one range
    ((2, 400, 400, 9, 9, 64), False, ([400, 311], [400, 311])),
    ((2, 2, 3000, 4, 2, 128), False, (None, [3000, 1100])),   # ranges of keys, joined
    ((1, 3000, 40, 4, 2, 32), False, (None, None)),           # ranges of queries in dk and dv
    ((2, 260, 260, 6, 2, 96), True, (None, None)),            # shared heads
    ((1, 1, 2000, 8, 1, 40), True, (None, None)),
    ((1, 70, 33, 1, 1, 8), True, (None, None))])
def test_rows(size, causal, lengths):
    dense = run(size, (None,) * 4, causal, lengths)
    for pitches in ((8, None, None, None), (24, 8, None, 16), (None, 40, 8, None), (256, 16, 32, 48)):
        for a, b, name in zip(dense, run(size, pitches, causal, lengths), ("y", "lse", "dq", "dk", "dv")):
            assert torch.equal(a, b), (name, pitches)
