"""Attention (numbat_attention_*) against the formulas in 64 bits: one query and many, one key and many, odd
lengths, features that are no power of two, shared heads, padded batches, causal sequences of unequal lengths,
sequences without keys, q, k and v beside each other in one matrix, ranges of keys and queries.

Bounds (attention_ref.py): of a score, (d + 8) 2^-24 of the sum of its products' sizes, of a weight, relatively,
that and 2^-20 for the exponential with its argument's rounding, and 2^-8 where it is rounded to bf16 for a
product; of a sum of n products, (n + 8) 2^-24 of the sum of their sizes."""
import math

import pytest

from attention_ref import attention, attention_grads, fold, forward_bounds, grad_bounds, join, split, visible
from mlp_ref import D, close

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
if torch.cuda.is_available():
    from paper_2609_10632_amd import blocks
    from paper_2609_10632_amd import numbat as nb

# batch, queries, keys, heads, heads of k and v, features
SIZES = [(1, 1, 1, 1, 1, 8), (2, 1, 5, 2, 2, 32), (1, 3, 64, 2, 1, 64), (2, 33, 65, 3, 3, 40), (1, 64, 64, 2, 2, 128),
         (2, 100, 100, 4, 2, 96), (1, 129, 300, 2, 2, 64), (1, 400, 400, 3, 3, 64), (3, 20, 7, 8, 2, 24), (1, 5, 1000, 8, 1, 128),
         (2, 1, 1000, 8, 2, 128), (1, 260, 3, 2, 2, 72), (1, 1000, 77, 2, 1, 80), (2, 128, 128, 1, 1, 16), (1, 70, 513, 6, 2, 112),
         (4, 31, 640, 1, 1, 32), (1, 2, 2000, 3, 1, 8)]


def d(t):
    return t.detach().cpu().to(D)


class Case:
    """Inputs, the call's results, and the formulas' on the CPU.  What lies behind a sequence's length, and beside
    the heads of a row, is no number."""

    def __init__(self, batch, q_len, kv_len, heads, kv_heads, feat, causal=False, q_lengths=None, kv_lengths=None,
                 fused=False, seed=0, spread=1.5, scale=None):
        self.size = batch, q_len, kv_len, heads, kv_heads, feat
        self.scale = feat ** -0.5 if scale is None else scale
        g = torch.Generator().manual_seed(seed)
        nan = float("nan")
        if fused:
            assert q_len == kv_len
            rows = torch.full((batch * q_len, (heads + 2 * kv_heads) * feat + 8), nan, dtype=torch.bfloat16, device="cuda")
            cut = lambda t: (t[:, :heads * feat], t[:, heads * feat:(heads + kv_heads) * feat],  # noqa: E731
                             t[:, (heads + kv_heads) * feat:(heads + 2 * kv_heads) * feat])
            self.q, self.k, self.v = cut(rows)
            self.dq, self.dk, self.dv = cut(torch.full_like(rows, 7.0))
        else:
            new = lambda n, w: torch.full((n, w), nan, dtype=torch.bfloat16, device="cuda")  # noqa: E731
            self.q, self.k, self.v = new(batch * q_len, heads * feat), new(batch * kv_len, kv_heads * feat), new(batch * kv_len, kv_heads * feat)
            self.dq, self.dk, self.dv = (torch.full_like(t, 7.0) for t in (self.q, self.k, self.v))
        self.dy = torch.empty((batch * q_len, heads * feat), dtype=torch.bfloat16, device="cuda")
        for t, s in ((self.q, spread), (self.k, 1.0), (self.v, 1.0), (self.dy, 0.3)):
            t.copy_((torch.randn(t.shape, generator=g) * s).bfloat16())
        self.ql = None if q_lengths is None else torch.tensor(q_lengths, dtype=torch.int32, device="cuda")
        self.kl = None if kv_lengths is None else torch.tensor(kv_lengths, dtype=torch.int32, device="cuda")
        self.see = visible(batch, q_len, kv_len, q_lengths, kv_lengths, causal)
        # on the CPU zeros stand where no number will
        behind = lambda lengths, n: torch.zeros((batch, n), dtype=torch.bool) if lengths is None else \
            torch.arange(n)[None] >= torch.tensor(lengths).clamp(0, n)[:, None]  # noqa: E731
        gone_q, gone_k = behind(q_lengths, q_len).flatten(), behind(kv_lengths, kv_len).flatten()
        group = heads // kv_heads
        at = lambda t, gone, h: split(d(t).masked_fill(gone[:, None], 0.0), batch, h)  # noqa: E731
        self.rq, self.rdy = at(self.q, gone_q, heads), at(self.dy, gone_q, heads)
        self.rk, self.rv = (at(t, gone_k, kv_heads).repeat_interleave(group, 1) for t in (self.k, self.v))
        for t, gone in ((self.q, gone_q), (self.dy, gone_q), (self.k, gone_k), (self.v, gone_k)):
            t[gone.cuda()] = nan
        self.p = nb.attention_problem(batch, q_len, kv_len, heads, kv_heads, feat, causal=causal, scale=scale,
                                      q_row_stride=self.q.stride(0), k_row_stride=self.k.stride(0), v_row_stride=self.v.stride(0))
        self.y = torch.full((batch * q_len, heads * feat), 7.0, dtype=torch.bfloat16, device="cuda")
        self.lse = torch.full((batch, heads, q_len), 7.0, device="cuda")
        print("attention", self.size, "causal" if causal else "", q_lengths, kv_lengths, "fused" if fused else "", flush=True)
        self.ws = blocks.workspace(nb.numbat_workspace_size(nb.OP_ATTENTION_FWD, self.p))
        nb.numbat_attention_fwd(self.p, self.q, self.k, self.v, self.ql, self.kl, self.y, self.lse, self.ws)
        self.ry, self.rlse, self.rp = attention(self.rq, self.rk, self.rv, self.see, self.scale)
        self.empty = ~self.see.any(-1)[:, 0]  # [batch][q_len] or of one row for all sequences

    def check_forward(self):
        bound, lse_off = forward_bounds(self.rq, self.rk, self.rv, self.rp, self.rlse, self.ry, self.see, self.scale)
        close(self.y, join(self.ry), join(bound), "y")
        lse = d(self.lse)
        empty = self.empty[:, None].expand(lse.shape)
        assert bool((lse[empty] == -math.inf).all()) and bool((lse[~empty] > -math.inf).all())
        close(lse[~empty], self.rlse[~empty], lse_off[~empty], "lse")
        again = torch.full_like(self.y, 7.0)
        nb.numbat_attention_fwd(self.p, self.q, self.k, self.v, self.ql, self.kl, again, None, self.ws)
        assert torch.equal(again, self.y)

    def check_backward(self):
        batch, q_len, kv_len, heads, kv_heads, feat = self.size
        ws = blocks.workspace(nb.numbat_workspace_size(nb.OP_ATTENTION_BWD, self.p))
        for t, rows in ((self.y, self.ql), (self.lse, self.ql)):  # nothing is read behind a sequence's length
            if rows is not None:
                gone = torch.arange(q_len, device="cuda")[None] >= rows[:, None].clamp(0, q_len)
                if t is self.y:
                    t[gone.flatten()] = float("nan")
                else:
                    t.masked_fill_(gone[:, None], float("nan"))
        call = lambda: nb.numbat_attention_bwd(self.p, self.dy, self.q, self.k, self.v, self.y, self.lse, self.ql, self.kl,  # noqa: E731
                                               self.dq, self.dk, self.dv, ws)
        call()
        # the formulas on the y and lse that the call was given
        y = split(d(self.y).nan_to_num(0.0), batch, heads)
        lse = d(self.lse).masked_fill(self.empty[:, None].expand(self.lse.shape), 0.0)
        p = torch.exp(self.scale * self.rq @ self.rk.transpose(2, 3) - lse[..., None]).masked_fill(~self.see, 0.0)
        dq, dk, dv, ds = attention_grads(self.rdy, self.rq, self.rk, self.rv, y, p, self.scale)
        dk, dv = fold(dk, kv_heads), fold(dv, kv_heads)
        off = grad_bounds(self.rdy, self.rq, self.rk, self.rv, y, p, ds, dq, dk, dv, lse, self.see, self.scale, kv_heads)
        for name, got, ref, bound in zip(("dq", "dk", "dv"), (self.dq, self.dk, self.dv), (dq, dk, dv), off):
            close(got, join(ref), join(bound), name)
        once = [t.clone() for t in (self.dq, self.dk, self.dv)]
        call()
        assert all(torch.equal(a, b) for a, b in zip(once, (self.dq, self.dk, self.dv)))


def both(*a, **k):
    c = Case(*a, **k)
    c.check_forward()
    c.check_backward()
    return c


@pytest.mark.parametrize("size", SIZES)
def test_sizes(size):
    both(*size)


@pytest.mark.parametrize("size", [(1, 1, 1, 1, 1, 8), (1, 64, 64, 2, 2, 64), (2, 200, 200, 4, 2, 128), (1, 100, 333, 3, 1, 32),
                                  (1, 300, 100, 2, 2, 64), (2, 65, 64, 2, 1, 96), (1, 1, 700, 4, 2, 64), (1, 500, 500, 6, 2, 40)])
def test_causal(size):
    both(*size, causal=True)  # (more queries than keys: the first see nothing)


@pytest.mark.parametrize("feat", (32, 64, 96, 128))
@pytest.mark.parametrize("batch,length,heads,kv_heads,causal", [
    (4, 500, 16, 16, False),  # 256 blocks of four waves, one to a CU: as many waves as 512 of two, which cost more
    (4, 500, 32, 16, True),
    (3, 100, 24, 24, False),  # 72 blocks of four waves leave more of the card idle than 144 of two
    (3, 100, 24, 24, True)])
def test_waves_of_a_block(batch, length, heads, kv_heads, causal, feat):
    both(batch, length, length, heads, kv_heads, feat, causal=causal)


@pytest.mark.parametrize("causal", (False, True))
def test_a_batch_in_the_order_of_its_work(causal):
    """64 sequences of all lengths are taken longest first; 65 are not ordered."""
    g = torch.Generator().manual_seed(8)
    for batch in (64, 65):
        lengths = torch.randint(0, 41, (batch,), generator=g).tolist()
        both(batch, 40, 40, 2, 2, 32, causal=causal, q_lengths=lengths, kv_lengths=lengths[::-1])


@pytest.mark.parametrize("causal", (False, True))
@pytest.mark.parametrize("feat", (32, 64, 128))
def test_padded_batches(feat, causal):
    both(5, 150, 150, 4, 2, feat, causal=causal, q_lengths=[150, 0, 1, 149, 64], kv_lengths=[150, 70, 0, 65, 1])
    both(4, 1, 900, 4, 1, feat, causal=causal, q_lengths=[1, 1, 0, 1], kv_lengths=[900, 1, 5, 0])
    both(3, 700, 40, 2, 2, feat, causal=causal, q_lengths=[700, 3, 130], kv_lengths=[40, 40, 17])


def test_lengths_out_of_range_are_taken_into_it():
    both(3, 50, 60, 2, 1, 64, q_lengths=[90, -4, 20], kv_lengths=[2**31 - 1, 10, -2**31])


@pytest.mark.parametrize("size", [(2, 400, 400, 6, 6, 64), (1, 90, 90, 8, 2, 32), (2, 130, 130, 2, 1, 128)])
def test_side_by_side(size):
    both(*size, fused=True, q_lengths=[size[1] - 3] * size[0], kv_lengths=[size[1] - 3] * size[0])


def test_large_and_small_scores():
    both(1, 100, 200, 2, 2, 64, spread=40.0)  # one key takes all of a row's weight
    both(1, 100, 200, 2, 2, 64, spread=0.0)   # all keys the same
    both(1, 100, 200, 2, 2, 64, scale=1.0)


def test_rising_scores():
    """Every tile of keys raises the maximum, by a little and by much."""
    for step in (0.02, 0.5):
        c = Case(1, 40, 1000, 1, 1, 64, spread=0.0, seed=3)
        c.q.fill_(1.0)
        c.k.copy_((torch.arange(1000)[:, None] * step / 64).expand(1000, 64).bfloat16())
        c.rq, c.rk = split(d(c.q), 1, 1), split(d(c.k), 1, 1)
        nb.numbat_attention_fwd(c.p, c.q, c.k, c.v, None, None, c.y, c.lse, c.ws)
        c.ry, c.rlse, c.rp = attention(c.rq, c.rk, c.rv, c.see, c.scale)
        c.check_forward()
        c.check_backward()


def test_gradients_against_differences():
    """Along one direction in q, k and v: the gradients against the central difference, in 64 bits, of sum(dy y)."""
    c = Case(2, 60, 80, 4, 2, 32, causal=True, seed=5)
    ws = blocks.workspace(nb.numbat_workspace_size(nb.OP_ATTENTION_BWD, c.p))
    nb.numbat_attention_bwd(c.p, c.dy, c.q, c.k, c.v, c.y, c.lse, None, None, c.dq, c.dk, c.dv, ws)
    gen = torch.Generator().manual_seed(9)
    way = [torch.randn(t.shape, generator=gen, dtype=D) for t in (c.q, c.k, c.v)]

    def value(step):
        q, k, v = (d(t) + step * w for t, w in zip((c.q, c.k, c.v), way))
        k, v = (split(t, 2, 2).repeat_interleave(2, 1) for t in (k, v))
        return float((c.rdy * attention(split(q, 2, 4), k, v, c.see, c.scale)[0]).sum())

    step = 1e-4
    slope = (value(step) - value(-step)) / (2 * step)
    parts = [d(g) * w for g, w in zip((c.dq, c.dk, c.dv), way)]
    # each gradient's elements hold a few bf16 roundings of independent signs: 2^-6 of the root of their sum of squares
    # is several times what they can add up to
    assert abs(sum(float(t.sum()) for t in parts) - slope) <= 2 ** -6 * sum(float((t ** 2).sum()) for t in parts) ** 0.5


def test_offsets_past_32_bits():
    """Rows of k and v so far apart that bytes and elements pass 2^32: the same results as from dense rows."""
    n, stride, feat = 20000, 1 << 17, 64
    g = torch.Generator(device="cuda").manual_seed(1)
    q = torch.randn((3, 64), generator=g, device="cuda").bfloat16()
    wide = torch.empty((n, stride), dtype=torch.bfloat16, device="cuda")
    wide[:, :2 * feat] = torch.randn((n, 2 * feat), generator=g, device="cuda").bfloat16()
    outs = []
    for kv in (wide[:, :2 * feat], wide[:, :2 * feat].contiguous()):
        k, v = kv[:, :feat], kv[:, feat:]
        p = nb.attention_problem(1, 3, n, 1, 1, feat, k_row_stride=kv.stride(0), v_row_stride=kv.stride(0))
        y, lse = torch.empty_like(q), torch.empty((1, 1, 3), device="cuda")
        nb.numbat_attention_fwd(p, q, k, v, None, None, y, lse, blocks.workspace(nb.numbat_workspace_size(nb.OP_ATTENTION_FWD, p)))
        dq, dkv = torch.empty_like(q), torch.empty_strided(kv.shape, kv.stride(), dtype=kv.dtype, device="cuda")
        nb.numbat_attention_bwd(p, q, q, k, v, y, lse, None, None, dq, dkv[:, :feat], dkv[:, feat:],
                                blocks.workspace(nb.numbat_workspace_size(nb.OP_ATTENTION_BWD, p)))
        outs.append([y, lse, dq, dkv.contiguous()])
        del dkv
    assert all(torch.equal(a, b) for a, b in zip(*outs))


def test_no_keys_no_queries():
    q = torch.ones((6, 64), dtype=torch.bfloat16, device="cuda")
    y, lse, dq = torch.full_like(q, 7.0), torch.full((2, 1, 3), 7.0, device="cuda"), torch.full_like(q, 7.0)
    p = nb.attention_problem(2, 3, 0, 1, 1, 64)
    nb.numbat_attention_fwd(p, q, None, None, None, None, y, lse)
    assert bool((y == 0).all()) and bool((lse == -math.inf).all())
    ws = blocks.workspace(nb.numbat_workspace_size(nb.OP_ATTENTION_BWD, p))
    nb.numbat_attention_bwd(p, q, q, None, None, y, lse, None, None, dq, None, None, ws)
    assert bool((dq == 0).all())
    p = nb.attention_problem(2, 0, 3, 1, 1, 64)
    nb.numbat_attention_fwd(p, None, None, None, None, None, None, None)
    dk, dv = torch.full_like(q, 7.0), torch.full_like(q, 7.0)
    nb.numbat_attention_bwd(p, None, None, q, q, None, None, None, None, None, dk, dv)
    assert bool((dk == 0).all()) and bool((dv == 0).all())
