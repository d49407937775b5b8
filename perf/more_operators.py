"""Cases of the residual attention block's operators: group norm with an activation over NHWC maps,
rotary positions along several axes, and attention over the pixels of maps or over tokens, each
forward and backward.

``own`` chooses between the operators written out in elementary torch operations (fp32 whatever the
inputs' type, angles in 64 bits, rounded once at the end) and the framework's entry points.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
GN_EPS = 1e-5
BASE = 10000.0

# no case costs more than the largest listed ones
MOST_ELEMENTS = 51200 * 4096
MOST_PAIRS = 2 * 32 * 8192 * 8192 * 128 // 2   # (query, key) pairs times features, forward
MOST_PAIRS_BWD = 2 * 16 * 8192 * 8192 * 128 // 2
SCORES = 1 << 28                               # scores that the plain forms hold at a time


def listed():
    return [
        # serving: the coarsest map of one image, the detector's widest layer, 18 channels a group; latency
        {"name": "group norm 20x20 map", "op": "group_norm", "n": 1, "m": 400, "c": 576, "groups": 32, "act": "silu",
         "x": "bf16", "y": "bf16", "keep": False, "pitch": 0},
        # training on the 80x80 maps at batch 16, 192 channels of a 384-channel concatenation buffer
        {"name": "group norm 80x80 maps", "op": "group_norm", "n": 16, "m": 6400, "c": 192, "groups": 32, "act": "silu",
         "x": "bf16", "y": "bf16", "keep": True, "pitch": 192},
        # its gradients on the 40x40 maps at batch 16
        {"name": "group norm grads 40x40 maps", "op": "group_norm_grads", "n": 16, "m": 1600, "c": 384, "groups": 32,
         "act": "silu", "x": "bf16", "y": "bf16", "pitch": 0},
        # nothing a multiple of anything, fp32 maps
        {"name": "group norm grads odd", "op": "group_norm_grads", "n": 5, "m": 53 * 97, "c": 327, "groups": 3,
         "act": "gelu", "x": "f32", "y": "f32", "pitch": 5},
        # one new token far into a sequence: latency
        {"name": "rotary one token", "op": "rotary", "images": 1, "heads": 40, "d": 128, "p0": 64, "p1": 0, "p2": 0,
         "e0": 1, "e1": 1, "e2": 1, "far": 1_000_000, "layout": "halves", "shared": False, "type": "bf16",
         "inverse": False, "rest": 1024},
        # queries and keys of the 40x40 maps at batch 16, height and width, out of the rows of q, k and v
        {"name": "rotary 40x40 maps", "op": "rotary", "images": 16, "heads": 12, "d": 64, "p0": 16, "p1": 16, "p2": 0,
         "e0": 40, "e1": 40, "e2": 1, "far": 0, "layout": "halves", "shared": False, "type": "bf16", "inverse": False,
         "rest": 384},
        # gradients of queries and keys of video: 8 frames of 40x40, time, height and width
        {"name": "rotary grads video", "op": "rotary", "images": 4, "heads": 32, "d": 128, "p0": 16, "p1": 24, "p2": 24,
         "e0": 8, "e1": 40, "e2": 40, "far": 0, "layout": "pairs", "shared": True, "type": "bf16", "inverse": True,
         "rest": 0},
        # training on the coarsest maps at batch 16: every pixel of a map sees every other
        {"name": "attention 20x20 maps", "op": "attention", "batch": 16, "q": 400, "kv": 400, "heads": 9, "kv_heads": 9,
         "d": 64, "causal": False, "ragged": False, "keep": True},
        # serving: one query a sequence over long keys of several lengths, four heads a key head
        {"name": "attention one token", "op": "attention", "batch": 8, "q": 1, "kv": 8192, "heads": 32, "kv_heads": 8,
         "d": 128, "causal": False, "ragged": True, "keep": False},
        # a long batch of tokens
        {"name": "attention 8192 tokens", "op": "attention", "batch": 2, "q": 8192, "kv": 8192, "heads": 32,
         "kv_heads": 8, "d": 128, "causal": True, "ragged": False, "keep": True},
        # gradients on the 40x40 maps at batch 16, images of several sizes padded to the largest
        {"name": "attention grads 40x40 maps", "op": "attention_grads", "batch": 16, "q": 1600, "kv": 1600, "heads": 6,
         "kv_heads": 6, "d": 64, "causal": False, "ragged": True},
        # gradients of a long batch of tokens
        {"name": "attention grads 8192 tokens", "op": "attention_grads", "batch": 2, "q": 8192, "kv": 8192, "heads": 16,
         "kv_heads": 8, "d": 128, "causal": True, "ragged": False},
    ]


def _log(rng, lo, hi, odd=0.35):
    """A size between lo and hi, spread over its logarithm: odd ones and multiples of 8."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if v >= 8 and rng.random() > odd:
        v -= v % 8
    elif v > 2:
        v |= 1
    return min(max(v, lo), hi)


def draw(rng):
    op = rng.choice(("group_norm", "group_norm_grads", "rotary", "attention", "attention", "attention_grads"))
    if op in ("group_norm", "group_norm_grads"):
        while True:
            n, m, groups, each = _log(rng, 1, 32), _log(rng, 1, 25600), _log(rng, 1, 64), _log(rng, 1, 64)
            if n * m * groups * each <= MOST_ELEMENTS // 4 and groups * each >= 8 and m * each >= 8:
                break
        x = rng.choice(("bf16", "bf16", "f32"))
        case = {"op": op, "n": n, "m": m, "c": groups * each, "groups": groups,
                "act": rng.choice(("none", "relu", "gelu", "gelu_tanh", "silu")), "x": x,
                "y": rng.choice(("bf16", x)), "pitch": rng.choice((0, 0, 8, 192, 3))}
        return {**case, "keep": rng.random() < 0.5} if op == "group_norm" else case
    if op == "rotary":
        given, axes = rng.random() < 0.4, rng.choice((1, 2, 3))
        p = [_log(rng, 1, 64 // axes) if a < axes else 0 for a in range(3)]
        d = min(256, 2 * sum(p) + rng.choice((0, 0, 0, 2, 16)))
        while True:
            heads, images = _log(rng, 1, 64), _log(rng, 1, 64)
            e = [_log(rng, 1, 128) if a < axes else 1 for a in range(3)]
            if images * e[0] * e[1] * e[2] * heads * d <= MOST_ELEMENTS // 4:
                break
        return {"op": op, "images": images, "heads": heads, "d": d, "p0": p[0], "p1": p[1], "p2": p[2], "e0": e[0],
                "e1": e[1], "e2": e[2], "far": _log(rng, 16, 1_000_000) if given else 0,
                "layout": rng.choice(("halves", "pairs")), "shared": rng.random() < 0.5,
                "type": rng.choice(("bf16", "bf16", "f32")), "inverse": rng.random() < 0.5,
                "rest": rng.choice((0, 8, 64, 3))}
    while True:
        batch, q, kv_heads, group = _log(rng, 1, 16), _log(rng, 1, 8192), _log(rng, 1, 16), rng.choice((1, 1, 2, 3, 4, 8))
        kv = q if rng.random() < 0.6 else _log(rng, 1, 16384)
        d = rng.choice((8, 24, 32, 40, 64, 64, 72, 80, 96, 128, 128))
        heads = kv_heads * group
        # (the scores of a single key have no gradient)
        if batch * heads * q * kv * d <= (MOST_PAIRS if op == "attention" else MOST_PAIRS_BWD) \
                and batch * max(q, kv) * heads * d <= MOST_ELEMENTS // 4 and kv > (op == "attention_grads"):
            break
    causal = kv >= q and rng.random() < 0.4
    ragged = not causal and rng.random() < 0.4
    case = {"op": op, "batch": batch, "q": q, "kv": kv, "heads": heads, "kv_heads": kv_heads, "d": d, "causal": causal,
            "ragged": ragged}
    # (rows behind a sequence's end have no logarithm of a sum)
    return {**case, "keep": not ragged and rng.random() < 0.5} if op == "attention" else case


# ---------------------------------------------------------------------------------------- inputs
_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _normal(g, shape, std=1.0, dtype=torch.bfloat16):
    return torch.randn(shape, generator=g, device=DEV).mul_(std).to(dtype)


def _uniform(g, shape, lo, hi, dtype=torch.float32):
    return torch.rand(shape, generator=g, device=DEV).mul_(hi - lo).add_(lo).to(dtype)


def _rows(case):
    return case["images"] * case["e0"] * case["e1"] * case["e2"]


def _axes(case):
    return [case[f"p{a}"] for a in range(3) if case[f"p{a}"]], [case[f"e{a}"] for a in range(3) if case[f"p{a}"]]


def _lengths(case, of):
    """Rows of each sequence that count: all of them, or, in a padded batch, the first's all and fewer of the others."""
    full = case[of]
    if not case["ragged"] or full == 1:
        return [full] * case["batch"]
    return [max(1, full - (i * 37 % 16) * full // 24) for i in range(case["batch"])]


def prepare(case, seed):
    """What the program has before the call; where the framework runs, also the descriptors, output
    buffers and workspaces that a training or serving loop keeps."""
    g, s = _gen(seed), {"case": case}
    op = case["op"]
    if op in ("group_norm", "group_norm_grads"):
        n, m, c = case["n"], case["m"], case["c"]
        # channels of different means and spreads, as a convolution's have
        full = torch.randn((n * m, c + case["pitch"]), generator=g, device=DEV)
        full = full.mul_(_uniform(g, (c + case["pitch"],), 0.5, 2.0)).add_(_uniform(g, (c + case["pitch"],), -1.0, 1.0))
        s["x"] = full.to(_TYPES[case["x"]])[:, :c]
        s["gamma"] = _uniform(g, (c,), 0.5, 1.5)
        s["beta"] = _normal(g, (c,), 0.1, torch.float32)
        if op == "group_norm_grads":
            s["dy"] = _normal(g, (n * m, c), 0.01, _TYPES[case["y"]])
            s["mean"], s["rstd"] = _group_moments(s["x"], case)
    elif op == "rotary":
        width = case["heads"] * case["d"]
        s["x"] = _normal(g, (_rows(case), width + case["rest"]), dtype=_TYPES[case["type"]])[:, :width]
        s["positions"] = None
        if case["far"]:
            s["positions"] = torch.randint(0, case["far"], (_rows(case), len(_axes(case)[0])), generator=g, device=DEV,
                                           dtype=torch.int32)
    else:
        b, q, kv, h, kvh, d = (case[k] for k in ("batch", "q", "kv", "heads", "kv_heads", "d"))
        # scores of standard deviation 1.5: some keys count much more than others
        if q == kv:
            rows = _normal(g, (b * q, (h + 2 * kvh) * d))
            rows[:, :h * d].mul_(1.5)
            s["q"], s["k"], s["v"] = rows[:, :h * d], rows[:, h * d:(h + kvh) * d], rows[:, (h + kvh) * d:]
        else:
            s["q"] = _normal(g, (b * q, h * d), 1.5)
            rows = _normal(g, (b * kv, 2 * kvh * d))
            s["k"], s["v"] = rows[:, :kvh * d], rows[:, kvh * d:]
        s["q_lengths"] = s["kv_lengths"] = None
        if case["ragged"]:
            s["q_lengths"] = torch.tensor(_lengths(case, "q"), dtype=torch.int32, device=DEV)
            s["kv_lengths"] = torch.tensor(_lengths(case, "kv"), dtype=torch.int32, device=DEV)
        if op == "attention_grads":
            s["dy"] = _normal(g, (b * q, h * d), 0.1)
            out = _forward(s)
            s["y"], s["lse"] = out["y"], out["lse"].contiguous()
    if own:
        _plan(s)
    return s


def _plan(s):
    """The framework's descriptors, the buffers its results go to, and its workspaces."""
    from paper_2609_10632_amd import blocks
    from paper_2609_10632_amd import numbat as nb

    case, op = s["case"], s["case"]["op"]
    acts = {"none": nb.ACT_NONE, "relu": nb.ACT_RELU, "gelu": nb.ACT_GELU, "gelu_tanh": nb.ACT_GELU_TANH,
            "silu": nb.ACT_SILU}
    types = {"bf16": nb.BF16, "f32": nb.F32}
    new = lambda shape, dtype: torch.empty(shape, dtype=dtype, device=DEV)  # noqa: E731
    space = lambda code: blocks.workspace(nb.numbat_workspace_size(code, s["p"]))  # noqa: E731
    s["nb"] = nb
    if op in ("group_norm", "group_norm_grads"):
        n, m, c, groups = case["n"], case["m"], case["c"], case["groups"]
        s["p"] = nb.group_norm_problem(n, m, c, groups, act=acts[case["act"]], eps=GN_EPS, x_type=types[case["x"]],
                                       y_type=types[case["y"]], x_row_stride=c + case["pitch"])
        if op == "group_norm":
            s["y"] = new((n * m, c), _TYPES[case["y"]])
            s["mean"], s["rstd"] = (new((n, groups), torch.float32), new((n, groups), torch.float32)) \
                if case["keep"] else (None, None)
            s["ws"] = space(nb.OP_GROUP_NORM_FWD)
        else:
            s["dx"] = new((n * m, c), _TYPES[case["x"]])
            s["dgamma"], s["dbeta"] = new((c,), torch.float32), new((c,), torch.float32)
            s["ws"] = space(nb.OP_GROUP_NORM_BWD)
    elif op == "rotary":
        pairs, extents = _axes(case)
        width = case["heads"] * case["d"]
        s["p"] = nb.rotary_problem(_rows(case), case["heads"], case["d"], pairs, extents=None if case["far"] else extents,
                                   base=BASE, layout=nb.ROTARY_HALVES if case["layout"] == "halves" else nb.ROTARY_PAIRS,
                                   shared=case["shared"], inverse=case["inverse"], type=types[case["type"]],
                                   x_row_stride=width + case["rest"])
        s["y"] = new((_rows(case), width), _TYPES[case["type"]])
    else:
        b, q, kv, h, kvh, d = (case[k] for k in ("batch", "q", "kv", "heads", "kv_heads", "d"))
        s["p"] = nb.attention_problem(b, q, kv, h, kvh, d, causal=case["causal"], q_row_stride=s["q"].stride(0),
                                      k_row_stride=s["k"].stride(0), v_row_stride=s["v"].stride(0))
        if op == "attention":
            s["y"] = new((b * q, h * d), torch.bfloat16)
            s["lse"] = new((b, h, q), torch.float32) if case["keep"] else None
            s["ws"] = space(nb.OP_ATTENTION_FWD)
        else:  # gradients lie as what they are gradients of
            if q == kv:
                rows = new((b * q, (h + 2 * kvh) * d), torch.bfloat16)
                s["dq"], s["dk"], s["dv"] = rows[:, :h * d], rows[:, h * d:(h + kvh) * d], rows[:, (h + kvh) * d:]
            else:
                rows = new((b * kv, 2 * kvh * d), torch.bfloat16)
                s["dq"], s["dk"], s["dv"] = new((b * q, h * d), torch.bfloat16), rows[:, :kvh * d], rows[:, kvh * d:]
            s["ws"] = space(nb.OP_ATTENTION_BWD)


# ------------------------------------------------------------------------------------ plain forms
def _act(t, act):
    if act == "relu":
        return t.clamp_min(0.0)
    if act == "gelu":
        return t * (0.5 * (1.0 + torch.erf(t * 0.5 ** 0.5)))
    if act == "gelu_tanh":
        return 0.5 * t * (1.0 + torch.tanh((2.0 / math.pi) ** 0.5 * (t + 0.044715 * t * t * t)))
    if act == "silu":
        return t / (1.0 + torch.exp(-t))
    return t


def _act_slope(z, act):
    """The activation's derivative."""
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * 0.5 ** 0.5)) + z * torch.exp(-0.5 * z * z) * (2.0 * math.pi) ** -0.5
    if act == "gelu_tanh":
        a = (2.0 / math.pi) ** 0.5
        t = torch.tanh(a * (z + 0.044715 * z * z * z))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * a * (1.0 + 3 * 0.044715 * z * z)
    if act == "silu":
        q = 1.0 / (1.0 + torch.exp(-z))
        return q * (1.0 + z * (1.0 - q))
    return torch.ones_like(z)


def _group_moments(x, case):
    """Mean and reciprocal deviation [n][groups]."""
    x = x.float().reshape(case["n"], case["m"], case["groups"], -1)
    mean = x.mean((1, 3), keepdim=True)
    d = x - mean
    return mean.flatten(1), (1.0 / torch.sqrt((d * d).mean((1, 3)) + GN_EPS))


def _normed(s):
    """(x - mean) rstd as [n][m][c]."""
    case = s["case"]
    n, m, g = case["n"], case["m"], case["groups"]
    x = s["x"].float().reshape(n, m, g, -1)
    return ((x - s["mean"].view(n, 1, g, 1)) * s["rstd"].view(n, 1, g, 1)).view(n, m, -1)


def _plain_group_norm(s):
    case = s["case"]
    mean, rstd = _group_moments(s["x"], case)
    t = _normed({**s, "mean": mean, "rstd": rstd}) * s["gamma"] + s["beta"]
    y = _act(t, case["act"]).to(_TYPES[case["y"]]).view(case["n"] * case["m"], -1)
    return {"y": y, "mean": mean, "rstd": rstd} if case["keep"] else {"y": y}


def _plain_group_norm_grads(s):
    case = s["case"]
    n, m, g = case["n"], case["m"], case["groups"]
    xh = _normed(s)
    dt = s["dy"].float().view(n, m, -1) * _act_slope(xh * s["gamma"] + s["beta"], case["act"])
    out = {"dgamma": (dt * xh).sum((0, 1)), "dbeta": dt.sum((0, 1))}
    h, xh = (dt * s["gamma"]).view(n, m, g, -1), xh.view(n, m, g, -1)
    dx = h - h.mean((1, 3), keepdim=True) - xh * (h * xh).mean((1, 3), keepdim=True)
    dx = dx * s["rstd"].view(n, 1, g, 1)
    return {"dx": dx.view(n * m, -1).to(_TYPES[case["x"]]), **out}


def _angles(s):
    """The angle of every row's pairs, 64 bits."""
    case = s["case"]
    pairs, extents = _axes(case)
    if s["positions"] is not None:
        at = [s["positions"][:, a] for a in range(len(pairs))]
    else:
        r, at = torch.arange(_rows(case), device=DEV), []
        for e in reversed(extents):
            at.insert(0, r % e)
            r = torch.div(r, e, rounding_mode="floor")
    total, done, cols = sum(pairs), 0, []
    for p, pos in zip(pairs, at):
        i = torch.arange(p, device=DEV, dtype=torch.float64)
        power = (done + i) / total if case["shared"] else i / p
        cols.append(pos.double()[:, None] * torch.exp(-math.log(BASE) * power))
        done += p
    return torch.cat(cols, 1)


def _plain_rotary(s):
    case = s["case"]
    h, d, x = case["heads"], case["d"], s["x"].float()
    angle = _angles(s)
    p = angle.shape[1]
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    if case["inverse"]:
        sin = -sin
    x = x.reshape(-1, h, d)
    turned, rest = x[..., :2 * p], x[..., 2 * p:]
    if case["layout"] == "halves":
        a, b = turned[..., :p], turned[..., p:]
        turned = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    else:
        a, b = turned[..., 0::2], turned[..., 1::2]
        turned = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    return {"y": torch.cat((turned, rest), -1).to(_TYPES[case["type"]]).view(-1, h * d)}


def _heads(t, batch, heads, repeat=1):
    """[batch * rows][heads * d] as fp32 [batch * heads * repeat][rows][d]."""
    t = t.float().reshape(batch, -1, heads, t.shape[1] // heads).transpose(1, 2)
    return (t if repeat == 1 else t.repeat_interleave(repeat, 1)).flatten(0, 1)


def _unseen(s, first, count):
    """Which scores of (sequence, head) number first .. first + count - 1 are masked, or None."""
    case = s["case"]
    if case["causal"]:
        i, j = torch.arange(case["q"], device=DEV), torch.arange(case["kv"], device=DEV)
        return j > i[:, None] + (case["kv"] - case["q"])
    if s["kv_lengths"] is None:
        return None
    each = s["kv_lengths"].repeat_interleave(case["heads"])[first:first + count]
    return (torch.arange(case["kv"], device=DEV) >= each[:, None])[:, None]


def _pieces(s):
    case = s["case"]
    total = case["batch"] * case["heads"]
    step = max(1, min(total, SCORES // (case["q"] * case["kv"])))
    return [(i, min(step, total - i)) for i in range(0, total, step)]


def _padding(s, t, of, heads):
    """Zeros in the rows behind each sequence's end; t: [batch * heads][rows][d]."""
    if s[of] is None:
        return t
    each = s[of].repeat_interleave(heads)
    return t * (torch.arange(t.shape[1], device=DEV) < each[:, None])[..., None]


def _merge(t, batch):
    """[batch * heads][rows][d] as [batch * rows][heads * d]."""
    return t.view(batch, -1, *t.shape[1:]).transpose(1, 2).reshape(batch * t.shape[1], -1)


def _forward(s):
    case = s["case"]
    b, h, kvh = case["batch"], case["heads"], case["kv_heads"]
    q, k, v = _heads(s["q"], b, h), _heads(s["k"], b, kvh, h // kvh), _heads(s["v"], b, kvh, h // kvh)
    y, lse = torch.empty_like(q), torch.empty(q.shape[:2], device=DEV)
    for i, n in _pieces(s):
        t = torch.bmm(q[i:i + n], k[i:i + n].transpose(1, 2)) * case["d"] ** -0.5
        hidden = _unseen(s, i, n)
        if hidden is not None:
            t = t.masked_fill(hidden, -math.inf)
        most = t.amax(-1, keepdim=True)
        e = torch.exp(t - most)
        total = e.sum(-1, keepdim=True)
        y[i:i + n] = torch.bmm(e, v[i:i + n]) / total
        lse[i:i + n] = (most + torch.log(total)).squeeze(-1)
    y = _padding(s, y, "q_lengths", h)
    return {"y": _merge(y, b).to(torch.bfloat16), "lse": lse.view(b, h, -1)}


def _plain_attention(s):
    out = _forward(s)
    return out if s["case"]["keep"] else {"y": out["y"]}


def _plain_attention_grads(s):
    case = s["case"]
    b, h, kvh, scale = case["batch"], case["heads"], case["kv_heads"], case["d"] ** -0.5
    q, k, v = _heads(s["q"], b, h), _heads(s["k"], b, kvh, h // kvh), _heads(s["v"], b, kvh, h // kvh)
    dy = _padding(s, _heads(s["dy"], b, h), "q_lengths", h)
    delta = (dy * _heads(s["y"], b, h)).sum(-1, keepdim=True)
    lse = s["lse"].view(b * h, -1, 1)
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    for i, n in _pieces(s):
        at = slice(i, i + n)
        t = torch.bmm(q[at], k[at].transpose(1, 2)) * scale
        hidden = _unseen(s, i, n)
        if hidden is not None:
            t = t.masked_fill(hidden, -math.inf)
        p = torch.exp(t - lse[at])
        dv[at] = torch.bmm(p.transpose(1, 2), dy[at])
        ds = p * (torch.bmm(dy[at], v[at].transpose(1, 2)) - delta[at]) * scale
        dq[at] = torch.bmm(ds, k[at])
        dk[at] = torch.bmm(ds.transpose(1, 2), q[at])
    dk, dv = (t.view(b * kvh, h // kvh, *t.shape[1:]).sum(1) for t in (dk, dv))
    return {n: _merge(t, b).to(torch.bfloat16) for n, t in (("dq", dq), ("dk", dk), ("dv", dv))}


# --------------------------------------------------------------------------- the framework's calls
def _own_group_norm(s):
    s["nb"].numbat_group_norm_fwd(s["p"], s["x"], s["gamma"], s["beta"], s["y"], s["mean"], s["rstd"], s["ws"])
    return {"y": s["y"], "mean": s["mean"], "rstd": s["rstd"]} if s["mean"] is not None else {"y": s["y"]}


def _own_group_norm_grads(s):
    s["nb"].numbat_group_norm_bwd(s["p"], s["dy"], s["x"], s["mean"], s["rstd"], s["gamma"], s["beta"], s["dx"],
                                  s["dgamma"], s["dbeta"], False, s["ws"])
    return {"dx": s["dx"], "dgamma": s["dgamma"], "dbeta": s["dbeta"]}


def _own_rotary(s):
    s["nb"].numbat_rotary(s["p"], s["x"], s["positions"], s["y"])
    return {"y": s["y"]}


def _own_attention(s):
    s["nb"].numbat_attention_fwd(s["p"], s["q"], s["k"], s["v"], s["q_lengths"], s["kv_lengths"], s["y"], s["lse"],
                                 s["ws"])
    return {"y": s["y"], "lse": s["lse"]} if s["lse"] is not None else {"y": s["y"]}


def _own_attention_grads(s):
    s["nb"].numbat_attention_bwd(s["p"], s["dy"], s["q"], s["k"], s["v"], s["y"], s["lse"], s["q_lengths"],
                                 s["kv_lengths"], s["dq"], s["dk"], s["dv"], s["ws"])
    return {"dq": s["dq"], "dk": s["dk"], "dv": s["dv"]}


def run(state):
    """One pass: a norm, a rotation or an attention, or the gradients of one."""
    return globals()[("_own_" if own else "_plain_") + state["case"]["op"]](state)


# ------------------------------------------------------------------------------- floors and oracle
def _pairs(case):
    """(query, key) pairs that count, over all heads."""
    if case["causal"]:
        q, kv = case["q"], case["kv"]
        each = [q * (kv - q) + q * (q + 1) // 2] * case["batch"]
    else:
        each = [a * b for a, b in zip(_lengths(case, "q"), _lengths(case, "kv"))]
    return case["heads"] * sum(each)


def work(case):
    op = case["op"]
    if op in ("group_norm", "group_norm_grads"):
        xs, ys = (2 if case[t] == "bf16" else 4 for t in ("x", "y"))
        elements, c = case["n"] * case["m"] * case["c"], case["c"]
        if op == "group_norm":
            return {"bytes": elements * (xs + ys) + 8 * c + 8 * case["n"] * case["groups"] * case["keep"],
                    "flops": 10 * elements}
        return {"bytes": elements * (2 * xs + ys) + 16 * c + 8 * case["n"] * case["groups"], "flops": 20 * elements}
    if op == "rotary":
        size = 2 if case["type"] == "bf16" else 4
        elements = _rows(case) * case["heads"] * case["d"]
        return {"bytes": 2 * size * elements + (4 * _rows(case) * len(_axes(case)[0]) if case["far"] else 0),
                "flops": 3 * elements}
    q, kv = sum(_lengths(case, "q")), sum(_lengths(case, "kv"))
    h, kvh, d = case["heads"], case["kv_heads"], case["d"]
    if op == "attention":  # q, k and v read, y (and lse) written: the rows that count, and zeros behind them
        written = case["batch"] * case["q"]
        return {"bytes": 2 * d * (q * h + 2 * kv * kvh + written * h) + 4 * q * h * case["keep"],
                "flops": 4 * d * _pairs(case)}
    # q, k, v, y, dy and lse read; dq, dk and dv written
    return {"bytes": 2 * d * (3 * q * h + 2 * kv * kvh + case["batch"] * (case["q"] * h + 2 * case["kv"] * kvh))
            + 4 * q * h, "flops": 10 * d * _pairs(case)}


def _d(t):
    return t.to(torch.float64)


def exact(case, seed):
    """The same outputs from the definitions in 64 bits."""
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    op = case["op"]
    if op in ("group_norm", "group_norm_grads"):
        n, m, c, g = case["n"], case["m"], case["c"], case["groups"]
        # [n][groups][rows][channels of a group]
        split = lambda t: _d(t).reshape(n, m, g, c // g).permute(0, 2, 1, 3)  # noqa: E731
        join = lambda t: t.permute(0, 2, 1, 3).reshape(n * m, c)              # noqa: E731
        gamma, beta = _d(s["gamma"]).view(1, g, 1, -1), _d(s["beta"]).view(1, g, 1, -1)
        x = split(s["x"])
        if op == "group_norm":
            var, mean = torch.var_mean(x, (2, 3), correction=0)
            rstd = (var + GN_EPS).rsqrt()
            t = torch.addcmul(beta, x.sub_(mean[..., None, None]).mul_(rstd[..., None, None]), gamma)
            y = join(_exact_act(t, case["act"])[0])
            return {"y": y, "mean": mean, "rstd": rstd} if case["keep"] else {"y": y}
        rstd = _d(s["rstd"])[..., None, None]
        xh = x.sub_(_d(s["mean"])[..., None, None]).mul_(rstd)
        dt = split(s["dy"]) * _exact_act(torch.addcmul(beta, xh, gamma), case["act"])[1]
        dgamma, dbeta = (dt * xh).sum((0, 2)).flatten(), dt.sum((0, 2)).flatten()
        h = dt.mul_(gamma)
        inner, flat = (h * xh).mean((2, 3), keepdim=True), h.mean((2, 3), keepdim=True)
        return {"dx": join((h - flat).sub_(xh.mul_(inner)).mul_(rstd)), "dgamma": dgamma, "dbeta": dbeta}
    if op == "rotary":
        return {"y": _exact_rotary(s)}
    return _exact_attention(s) if op == "attention" else _exact_attention_grads(s)


def _exact_act(z, act):
    """The activation and its derivative in 64 bits."""
    if act == "relu":
        on = torch.heaviside(z, torch.zeros((), dtype=z.dtype, device=z.device))
        return z * on, on
    if act == "gelu":
        cdf = torch.special.ndtr(z)
        return z * cdf, cdf + z * torch.exp(z * z / -2.0) / math.sqrt(2.0 * math.pi)
    if act == "gelu_tanh":  # 1 + tanh(u) = 2 sigmoid(2u)
        a = math.sqrt(8.0 / math.pi)
        q = torch.special.expit(a * (z + 0.044715 * z ** 3))
        return z * q, q + z * q * (1.0 - q) * a * (1.0 + 0.134145 * z * z)
    if act == "silu":
        q = torch.special.expit(z)
        return z * q, q * (1.0 + z - z * q)
    return z, torch.ones_like(z)


def _exact_rotary(s):
    """Each pair as a complex number, times exp(i angle)."""
    case = s["case"]
    pairs, extents = _axes(case)
    h, d, total = case["heads"], case["d"], sum(pairs)
    x = _d(s["x"]).reshape(-1, h, d)
    out = x.clone()
    row = torch.arange(x.shape[0], device=DEV)
    j = 0
    for a, p in enumerate(pairs):
        if s["positions"] is not None:
            pos = s["positions"][:, a].double()
        else:
            pos = ((row // math.prod(extents[a + 1:])) % extents[a]).double()
        for i in range(p):
            angle = pos * BASE ** (-(j / total if case["shared"] else i / p))
            turn = torch.polar(torch.ones_like(angle), -angle if case["inverse"] else angle)[:, None]
            at = (j, j + total) if case["layout"] == "halves" else (2 * j, 2 * j + 1)
            z = torch.complex(x[..., at[0]], x[..., at[1]]) * turn
            out[..., at[0]], out[..., at[1]] = z.real, z.imag
            j += 1
    return out.view(-1, h * d)


def _each_head(s):
    """(sequence, head, its rows of q, k and v that count in 64 bits, the masked scores or None)"""
    case = s["case"]
    d, group = case["d"], case["heads"] // case["kv_heads"]
    for b, (nq, nk) in enumerate(zip(_lengths(case, "q"), _lengths(case, "kv"))):
        hidden = torch.ones((nq, nk), dtype=torch.bool, device=DEV).triu(nk - nq + 1) if case["causal"] else None
        for h in range(case["heads"]):
            rows, keys, mine = slice(b * case["q"], b * case["q"] + nq), slice(b * case["kv"], b * case["kv"] + nk), h // group
            cols, kcols = slice(h * d, h * d + d), slice(mine * d, mine * d + d)
            yield b, h, rows, keys, cols, kcols, _d(s["q"][rows, cols]), _d(s["k"][keys, kcols]), _d(s["v"][keys, kcols]), hidden


def _exact_attention(s):
    case = s["case"]
    y = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.zeros((case["batch"], case["heads"], case["q"]), dtype=torch.float64, device=DEV)
    for b, h, rows, _, cols, _, q, k, v, hidden in _each_head(s):
        t = torch.mm(q, k.t()).div_(math.sqrt(case["d"]))
        if hidden is not None:
            t.masked_fill_(hidden, -math.inf)
        total = torch.logsumexp(t, 1)
        lse[b, h, :len(total)] = total
        y[rows, cols] = torch.mm(t.sub_(total[:, None]).exp_(), v)
    return {"y": y, "lse": lse} if case["keep"] else {"y": y}


def _exact_attention_grads(s):
    root = math.sqrt(s["case"]["d"])
    dq, dk, dv = (torch.zeros(s[n].shape, dtype=torch.float64, device=DEV) for n in ("q", "k", "v"))
    for b, h, rows, keys, cols, kcols, q, k, v, hidden in _each_head(s):
        dy = _d(s["dy"][rows, cols])
        p = torch.mm(q, k.t()).div_(root)
        p.sub_(_d(s["lse"][b, h, :len(q)])[:, None]).exp_()
        if hidden is not None:
            p.masked_fill_(hidden, 0.0)
        dv[keys, kcols] += torch.mm(p.t(), dy)
        ds = torch.mm(dy, v.t()).sub_((dy * _d(s["y"][rows, cols])).sum(1, keepdim=True)).mul_(p).div_(root)
        dq[rows, cols] = torch.mm(ds, k)
        dk[keys, kcols] += torch.mm(ds.t(), q)
    return {"dq": dq, "dk": dk, "dv": dv}
