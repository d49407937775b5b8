"""Attention (numbat_attention_*) where the scores are far from zero: the largest key of a row has a weight of one at
any score, in one range of keys and in several, rising, falling, and with a scale that does what q and k do
not.

The scores here are exact in fp32 (a power of two times a small number, plus eighths where they are small enough for
them), so that only what follows them rounds.  With g = s - max s, a weight's argument is off by 4 2^-24 |g| and
its exponential by 2^-20 (twice where ranges are joined, whose logarithms are off by 2^-10 at most up to 2^14 and
by 2^-24 of a sum's logarithm past it); a sum of n terms by (n + 8) 2^-24; weights and y are rounded to bf16.
Of the gradients' weights: lse and its product with log2(e) are rounded five times between the forward's
logarithm and the backward's exponent, 5 2^-24 |lse| < 2^-21 |lse|."""
import math

import pytest

from mlp_ref import B, D, U, close

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
if torch.cuda.is_available():
    from paper_2609_10632_amd import blocks
    from paper_2609_10632_amd import numbat as nb

FEAT = 8
ODD = 161 / 128  # scores whose products with log2(e) round


def d(t):
    return t.detach().cpu().to(D)


def inputs(levels, small, rows, size, seed=0, feat=FEAT):
    """q, k, v of one head with q_i k_j = size levels[j] + small[j]."""
    n = len(levels)
    q, k = torch.zeros((rows, feat)), torch.zeros((n, feat))
    q[:, 0], q[:, 1] = size, 1.0
    k[:, 0], k[:, 1] = torch.as_tensor(levels), torch.as_tensor(small)
    v = torch.randn((n, feat), generator=torch.Generator().manual_seed(seed))
    q, k, v = (t.bfloat16().cuda() for t in (q, k, v))
    s = d(q) @ d(k).t()
    assert torch.equal(s, s.float().to(D))
    return q, k, v, s


def forward(q, k, v, s, scale, causal=False, batch=1, heads=1):
    """batch, heads: as many copies, which give the same results."""
    rows, n = s.shape
    feat = q.shape[1]
    p = nb.attention_problem(batch, rows, n, heads, heads, feat, causal=causal, scale=scale)
    y, lse = torch.empty((batch * rows, heads * feat), dtype=torch.bfloat16, device="cuda"), torch.empty((batch, heads, rows), device="cuda")
    print("attention of far scores", batch, heads, feat, rows, n, scale, float(s.min()), float(s.max()), flush=True)
    nb.numbat_attention_fwd(p, *(t.repeat(batch, heads) for t in (q, k, v)), None, None, y, lse,
                            blocks.workspace(nb.numbat_workspace_size(nb.OP_ATTENTION_FWD, p)))
    assert torch.equal(y, y[:rows, :feat].repeat(batch, heads)) and torch.equal(lse, lse[:1, :1].expand(batch, heads, rows))
    y, lse = y[:rows, :feat], lse[:1, :1]
    scale = float(torch.tensor(scale, dtype=torch.float32))
    t = s * scale
    if causal:
        t = t.masked_fill(torch.arange(n)[None] > torch.arange(rows)[:, None] + (n - rows), -math.inf)
    gap = t - t.amax(1, keepdim=True)
    w = torch.exp(gap)
    total = w.sum(1, keepdim=True)
    w = w / total
    off = torch.where(w > 0, 4 * U * gap.abs().clamp(max=1e3) + 2 * 2 ** -20 + 2 ** -10 * (n > 256), torch.zeros((), dtype=D))
    ref = w @ d(v)
    bound = (w * (B + off + (n + 8) * 2 * U)) @ d(v).abs() + (w * off).sum(1, keepdim=True) * ref.abs() + B * ref.abs()
    close(y, ref, bound, "y")
    ref = t.amax(1) + torch.log(total[:, 0])
    close(lse[0, 0], ref, 4 * U * ref.abs() + (w * off).sum(1) + (n + 8) * U, "lse")
    return p, y, lse, t


@pytest.mark.parametrize("rows,n", [(40, 200), (1, 4000), (3, 1000), (300, 77)])
@pytest.mark.parametrize("power", (10, 13, 14, 19, 20, 30, 37, 100))
@pytest.mark.parametrize("sign", (1, -1))
def test_one_key_takes_all(rows, n, power, sign):
    """Its value comes out as it is, wherever the key lies."""
    size = 2.0 ** power
    for at in (0, n // 2, n - 1):
        levels = torch.full((n,), ODD * (0.5 if sign > 0 else -1.0))
        levels[at] = ODD * (1.0 if sign > 0 else -0.5)
        q, k, v, s = inputs(levels, torch.zeros(n), rows, size)
        _, y, lse, _ = forward(q, k, v, s, 1.0)
        if power > 10:
            assert torch.equal(y, v[at].expand(rows, FEAT)) and bool((lse == float(s[0, at])).all())


@pytest.mark.parametrize("rows,n", [(40, 200), (1, 4000)])
@pytest.mark.parametrize("power", (13, 14, 19, 20, -20))
def test_near_the_largest(rows, n, power):
    """Keys within a few units of each other at a score of 2^power (beside 0 at -20)."""
    g = torch.Generator().manual_seed(power + 50)
    small = torch.randint(-32, 33, (n,), generator=g).float() / 8
    forward(*inputs(torch.full((n,), ODD), small, rows, 2.0 ** power if power > 0 else 0.0), 1.0)


@pytest.mark.parametrize("rows,n", [(40, 1000), (1, 4000)])
def test_scores_that_rise_and_fall(rows, n):
    """From one side of zero to the other, through all sizes, and ties a thousand keys apart."""
    steps = [-(2.0 ** e) for e in range(0, -40, -2)] + [0.0] + [2.0 ** e for e in range(-38, 1, 2)]
    levels = torch.tensor([ODD * steps[j * len(steps) // n] for j in range(n)])
    for size in (2.0 ** 37, 2.0 ** 20):
        for order in (levels, levels.flip(0)):
            forward(*inputs(order, torch.zeros(n), rows, size), 1.0)
    tie = torch.full((n,), ODD / 2)
    tie[3] = tie[n - 5] = ODD
    q, k, v, s = inputs(tie, torch.zeros(n), rows, 2.0 ** 40)
    y = forward(q, k, v, s, 1.0)[1]
    both = (d(v[3]) + d(v[n - 5])) / 2
    close(y, both.expand(rows, FEAT), B * both.abs() + 2 ** -18, "the mean of two values")


@pytest.mark.parametrize("scale", (1e38, 2.0 ** 60, 1e-30))
def test_scales(scale):
    for size in (2.0 ** -70, 1.0, 2.0 ** 90):
        levels = torch.full((300,), ODD / 2)
        levels[170] = ODD
        q, k, v, s = inputs(levels, torch.zeros(300), 5, size)
        if size * scale < 2e38:
            forward(q, k, v, s, scale)
        else:  # (lse passes fp32's range, the weights do not)
            p = nb.attention_problem(1, 5, 300, 1, 1, FEAT, scale=scale)
            y = torch.empty((5, FEAT), dtype=torch.bfloat16, device="cuda")
            nb.numbat_attention_fwd(p, q, k, v, None, None, y, None, blocks.workspace(nb.numbat_workspace_size(nb.OP_ATTENTION_FWD, p)))
            assert torch.equal(y, v[170].expand(5, FEAT))


def test_causal():
    levels = torch.tensor([(-1.0) ** j * ODD * 2.0 ** -(j % 7) for j in range(150)])
    forward(*inputs(levels, torch.zeros(150), 150, 2.0 ** 33), 1.0, causal=True)


@pytest.mark.parametrize("rows,n", [(40, 200), (1, 3000), (300, 77)])
@pytest.mark.parametrize("power", (10, 13, 16))
def test_gradients_as_far_as_lse_allows(rows, n, power):
    """A weight's exponent is off by 2^-21 |lse| where it is formed from an lse in fp32."""
    g = torch.Generator().manual_seed(power)
    small = torch.randint(-16, 17, (n,), generator=g).float() / 8
    q, k, v, s = inputs(torch.full((n,), ODD), small, rows, 2.0 ** power)
    p, y, lse, t = forward(q, k, v, s, 1.0)
    dy = torch.randn((rows, FEAT), generator=g).bfloat16().cuda()
    dq, dk, dv = (torch.full_like(a, 7.0) for a in (q, k, v))
    nb.numbat_attention_bwd(p, dy, q, k, v, y, lse, None, None, dq, dk, dv,
                            blocks.workspace(nb.numbat_workspace_size(nb.OP_ATTENTION_BWD, p)))
    q, k, v, y, dy = (d(a) for a in (q, k, v, y, dy))
    w = torch.softmax(t, 1)
    off = torch.expm1(2 ** -21 * torch.logsumexp(t, 1).abs())[:, None] + 2 ** -20
    ds = w * (dy @ v.t() - (dy * y).sum(1, keepdim=True))
    ds_off = ds.abs() * (off + B + 4 * U) + w * (1 + off) * (FEAT + 16) * U * (dy.abs() @ v.abs().t() + (dy * y).abs().sum(1, keepdim=True))
    for name, got, ref, bound in (
            ("dq", dq, ds @ k, (ds_off + (n + 8) * 2 * U * ds.abs()) @ k.abs()),
            ("dk", dk, ds.t() @ q, (ds_off + (rows + 8) * 2 * U * ds.abs()).t() @ q.abs()),
            ("dv", dv, w.t() @ dy, (w * (B + off + (rows + 8) * 2 * U)).t() @ dy.abs())):
        close(got, ref, bound * (1 + B) + B * ref.abs(), name)


@pytest.mark.parametrize("feat", (32, 40, 64, 96, 128))
@pytest.mark.parametrize("batch,heads,rows,n", [(1, 1, 1, 4000), (1, 1, 70, 90), (3, 24, 100, 100), (4, 16, 500, 500)])
@pytest.mark.parametrize("causal", (False, True))
def test_widths_of_heads_and_blocks(feat, batch, heads, rows, n, causal):
    """Every width of a head, in blocks of one, two and four waves; scores on both sides of where the maximum is taken off
    first, with ties and contenders."""
    g = torch.Generator().manual_seed(feat)
    steps = torch.tensor([-1.0, -2.0 ** -6, 0.0, 2.0 ** -20, 2.0 ** -6, 0.5, 1.0])
    levels = ODD * steps[torch.randint(0, 7, (n,), generator=g)]
    small = torch.where(levels.abs() < 2.0 ** -10, torch.randint(-32, 33, (n,), generator=g).float() / 8, torch.zeros(n))
    small = torch.where(levels == 0, small, torch.zeros(n))
    for size in (2.0 ** 35, 2.0 ** 21):
        for order in (slice(None), torch.arange(n - 1, -1, -1)):
            forward(*inputs(levels[order], small[order], rows, size, feat=feat), 1.0, causal=causal, batch=batch, heads=heads)
