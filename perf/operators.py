"""Cases of the residual MLP block's operators: the linear layer with bias, activation and
residual in its epilogue and its gradients, layer norm and its gradients, and the AdamW step
over many tensors with states in 32 or 8 bits.

Rows are pixels of an NHWC map or tokens.  ``own`` chooses between the operators written out in
elementary torch operations (fp32 whatever the inputs' type, rounded once at the end) and the
framework's entry points.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
BLOCK = 256  # elements that share a scale in the 8-bit optimiser state
BETA1, BETA2, ADAM_EPS, STEP = 0.9, 0.95, 1e-8, 100
GROUPS = ((1e-3, 0.1), (1e-3, 0.0))  # (learning rate, weight decay): matrices, vectors
MAX_NORM = 1.0
LN_EPS = 1e-5

# no case costs more than the largest listed ones
MOST_MACS = 8192 * 4096 * 16384
MOST_ELEMENTS = 16384 * 8192
MOST_PARAMS = 134_250_496


def listed():
    return [
        # one token through a wide layer when serving: the weights' bytes and the call's latency
        {"name": "linear one token", "op": "linear", "m": 1, "k": 2048, "n": 8192, "act": "gelu_tanh", "res": False,
         "keep": False, "out": "bf16", "pitch": 0},
        # a batch of requests in decode, back to the stream's width with its residual
        {"name": "linear 24 tokens", "op": "linear", "m": 24, "k": 8192, "n": 4096, "act": "none", "res": True,
         "keep": False, "out": "bf16", "pitch": 0},
        # nothing a multiple of anything; fp32 results as a head's scores are
        {"name": "linear odd", "op": "linear", "m": 1531, "k": 1003, "n": 2049, "act": "relu", "res": False,
         "keep": False, "out": "f32", "pitch": 0},
        # the detector's 80x80 maps at batch 16, 192 channels of a 384-channel concatenation buffer,
        # widened four times in training (the pre-activation is kept)
        {"name": "linear 80x80 maps", "op": "linear", "m": 102400, "k": 192, "n": 768, "act": "silu", "res": False,
         "keep": True, "out": "bf16", "pitch": 192},
        # a long training batch of tokens through a wide layer
        {"name": "linear 8192 tokens", "op": "linear", "m": 8192, "k": 4096, "n": 16384, "act": "gelu", "res": False,
         "keep": True, "out": "bf16", "pitch": 0},
        # gradients of the narrowing layer on the 40x40 maps at batch 16
        {"name": "linear grads 40x40 maps", "op": "linear_grads", "m": 25600, "k": 1536, "n": 384, "act": "silu"},
        # gradients of the narrowing layer on the long batch of tokens
        {"name": "linear grads 8192 tokens", "op": "linear_grads", "m": 8192, "k": 16384, "n": 4096, "act": "gelu"},
        # a decode batch's norm: latency
        {"name": "norm 16 tokens", "op": "norm", "m": 16, "c": 4096, "x": "bf16", "keep": False},
        # gradients of the norm on the 80x80 maps at batch 16: many short rows
        {"name": "norm grads 80x80 maps", "op": "norm_grads", "m": 102400, "c": 192, "x": "bf16", "res": True},
        # a wide norm in training over an fp32 stream: few long rows
        {"name": "norm grads 16384 tokens", "op": "norm_grads", "m": 16384, "c": 8192, "x": "f32", "res": True},
        # the detector's optimiser step: 243 tensors, 25.9 million parameters, clipped
        {"name": "adamw 243 tensors", "op": "adamw", "tensors": 243, "params": 25_900_000, "bits": 32, "clip": True,
         "grad": "f32"},
        # the wide block's two matrices with their vectors, state in 8 bits
        {"name": "adamw 8 bits", "op": "adamw", "tensors": 6, "params": MOST_PARAMS, "bits": 8, "clip": False,
         "grad": "bf16"},
    ]


def _log(rng, lo, hi, odd=0.35):
    """A size between lo and hi, spread over its logarithm: odd ones and multiples of 8."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if v >= 8 and rng.random() > odd:
        v -= v % 8
    elif v > 2:
        v |= 1
    v = min(max(v, lo), hi)
    return v + 8 if v == 3072 else v


def draw(rng):
    op = rng.choice(("linear", "linear", "linear_grads", "norm", "norm_grads", "adamw"))
    if op in ("linear", "linear_grads"):
        while True:
            m, n, k = _log(rng, 1, 102400), _log(rng, 64, 16384), _log(rng, 64, 16384)
            if m * n * k <= MOST_MACS and m * max(n, k) <= MOST_ELEMENTS:
                break
        act = rng.choice(("none", "relu", "gelu", "gelu_tanh", "silu"))
        if op == "linear_grads":
            return {"op": op, "m": m, "k": k, "n": n, "act": act}
        return {"op": op, "m": m, "k": k, "n": n, "act": act, "res": rng.random() < 0.5, "keep": rng.random() < 0.5,
                "out": rng.choice(("bf16", "bf16", "f32")), "pitch": rng.choice((0, 0, 24, 192))}
    if op in ("norm", "norm_grads"):
        while True:
            m, c = _log(rng, 1, 102400), _log(rng, 64, 16384)
            if m * c <= MOST_ELEMENTS:
                break
        x = rng.choice(("bf16", "f32"))
        if op == "norm":
            return {"op": op, "m": m, "c": c, "x": x, "keep": rng.random() < 0.5}
        return {"op": op, "m": m, "c": c, "x": x, "res": rng.random() < 0.5}
    bits = rng.choice((32, 8))
    params = _log(rng, 20_000, MOST_PARAMS)
    # (a clipped step's coefficient comes from a sum over everything: in the last bit it depends on
    # the order of that sum, and the 8-bit codes would differ with it)
    return {"op": op, "tensors": _log(rng, 1, 300), "params": params, "bits": bits,
            "clip": bits == 32 and rng.random() < 0.5, "grad": rng.choice(("f32", "bf16"))}


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


def _sizes(case):
    """Elements of each tensor: a few matrices hold most of the parameters, the rest are vectors."""
    count, total = case["tensors"], case["params"]
    weight = [1.0 if i % 3 == 0 else 0.001 + 0.0001 * (i % 7) for i in range(count)]
    weight = [w * (1.0 + (i * 37 % 11) / 4.0) for i, w in enumerate(weight)]
    each = [max(1, int(total * w / sum(weight))) for w in weight]
    each[0] = max(1, each[0] + total - sum(each))
    return each


def _layout(case):
    """(elements, first element, group) of every tensor in one flat buffer; starts are whole blocks."""
    rows, at = [], 0
    for i, n in enumerate(_sizes(case)):
        rows.append((n, at, 0 if i % 3 == 0 else 1))
        at += -(-n // BLOCK) * BLOCK
    return rows, at


def prepare(case, seed):
    """What the program has before the call; where the framework runs, also the descriptors, output
    buffers and workspaces that a training or serving loop keeps."""
    g, s = _gen(seed), {"case": case}
    op = case["op"]
    if op in ("linear", "linear_grads"):
        m, n, k = case["m"], case["n"], case["k"]
        bound = k ** -0.5
        pitch = k + case.get("pitch", 0)
        s["x"] = _normal(g, (m, pitch))[:, :k]
        s["w"] = _uniform(g, (n, k), -bound, bound, torch.bfloat16)
        if op == "linear":
            s["bias"] = _uniform(g, (n,), -bound, bound)
            s["res"] = _normal(g, (m, n), dtype=_TYPES[case["out"]]) if case["res"] else None
        else:
            s["dy"] = _normal(g, (m, n), 0.01)
            s["z"] = _normal(g, (m, k))
    elif op in ("norm", "norm_grads"):
        m, c = case["m"], case["c"]
        # rows of different means and spreads, as a residual stream has
        s["x"] = (torch.randn((m, c), generator=g, device=DEV) * _uniform(g, (m, 1), 0.5, 2.0)
                  + _uniform(g, (m, 1), -1.0, 1.0)).to(_TYPES[case["x"]])
        s["gamma"] = _uniform(g, (c,), 0.5, 1.5)
        s["beta"] = _normal(g, (c,), 0.1, torch.float32)
        if op == "norm_grads":
            s["dy"] = _normal(g, (m, c), 0.01)
            s["res"] = _normal(g, (m, c), 0.01, _TYPES[case["x"]]) if case["res"] else None
            s["mean"], s["rstd"] = _moments(s["x"].float())
    else:
        rows, total = _layout(case)
        s["rows"], s["total"] = rows, total
        live = torch.zeros(total, dtype=torch.bool, device=DEV)
        for n, at, _ in rows:
            live[at:at + n] = True
        s["w"] = _normal(g, (total,), 0.05, torch.float32).mul_(live)
        s["grad"] = _normal(g, (total,), 0.01, torch.float32).mul_(live).to(_TYPES[case["grad"]])
        if case["bits"] == 32:
            s["m"] = _normal(g, (total,), 0.003, torch.float32).mul_(live)
            s["v"] = _normal(g, (total,), 0.01, torch.float32).square_().mul_(live)
        else:
            blocks = total // BLOCK
            codes = torch.randint(-127, 128, (total,), generator=g, device=DEV, dtype=torch.int16)
            s["m"] = (codes * live).to(torch.int8)
            s["m_unit"] = _uniform(g, (blocks,), 0.5, 1.0).mul_(0.01 / 127 ** 2)
            codes = torch.randint(1, 256, (total,), generator=g, device=DEV, dtype=torch.int16)
            s["v"] = (codes * live).to(torch.uint8)
            s["v_unit"] = _uniform(g, (blocks,), 0.5, 1.0).mul_(0.03 / 255 ** 2)
        s["group_of"] = torch.tensor([r[2] for r in rows], device=DEV)
        s["blocks_of"] = torch.tensor([-(-r[0] // BLOCK) for r in rows], device=DEV)
        s["lr"] = torch.tensor([x[0] for x in GROUPS], device=DEV)
        s["decay"] = torch.tensor([x[1] for x in GROUPS], device=DEV)
        s["copy"] = torch.empty(total, dtype=torch.bfloat16, device=DEV)
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
    s["nb"] = nb
    if op == "linear":
        m, n, k = case["m"], case["n"], case["k"]
        s["p"] = nb.linear_problem(m, n, k, act=acts[case["act"]], y_type=types[case["out"]],
                                   x_row_stride=k + case["pitch"])
        s["y"] = new((m, n), _TYPES[case["out"]])
        s["zout"] = new((m, n), torch.bfloat16) if case["keep"] else None
        s["ws"] = blocks.workspace(nb.numbat_workspace_size(nb.OP_LINEAR_FWD, s["p"]))
    elif op == "linear_grads":
        m, n, k = case["m"], case["n"], case["k"]
        s["p"] = nb.linear_problem(m, n, k, act=acts[case["act"]])
        s["dx"], s["dw"], s["db"] = new((m, k), torch.bfloat16), new((n, k), torch.float32), new((n,), torch.float32)
        s["ws"] = blocks.workspace(max(nb.numbat_workspace_size(o, s["p"])
                                       for o in (nb.OP_LINEAR_BWD_DATA, nb.OP_LINEAR_BWD_WEIGHT)))
    elif op in ("norm", "norm_grads"):
        m, c = case["m"], case["c"]
        s["p"] = nb.layer_norm_problem(m, c, eps=LN_EPS, x_type=types[case["x"]])
        if op == "norm":
            s["y"] = new((m, c), torch.bfloat16)
            s["mean"], s["rstd"] = (new((m,), torch.float32), new((m,), torch.float32)) if case["keep"] else (None, None)
        else:
            s["dx"] = new((m, c), _TYPES[case["x"]])
            s["dgamma"], s["dbeta"] = new((c,), torch.float32), new((c,), torch.float32)
            s["ws"] = blocks.workspace(nb.numbat_workspace_size(nb.OP_LAYER_NORM_BWD, s["p"]))
    else:
        ten = []
        for n, at, group in s["rows"]:
            e = {"w": s["w"][at:at + n], "grad": s["grad"][at:at + n], "m": s["m"][at:at + n], "v": s["v"][at:at + n],
                 "w_copy": s["copy"][at:at + n], "group": group}
            if case["bits"] == 8:
                at //= BLOCK
                e["m_unit"], e["v_unit"] = s["m_unit"][at:], s["v_unit"][at:]
            ten.append(e)
        table = torch.frombuffer(bytearray(nb.adamw_table(ten)), dtype=torch.uint8).to(DEV)
        s["table"], s["count"] = table, len(ten)
        s["copy"].zero_()
        s["norm"] = new((1,), torch.float32) if case["clip"] else None
        s["ws"] = blocks.workspace(nb.numbat_workspace_size(nb.OP_ADAMW, None))
        if case["bits"] == 8:
            s["m_value"], s["v_value"] = new((s["total"],), torch.float32), new((s["total"],), torch.float32)


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


def _moments(x):
    mean = x.mean(1)
    d = x - mean[:, None]
    return mean, 1.0 / torch.sqrt((d * d).mean(1) + LN_EPS)


def _plain_linear(s):
    case = s["case"]
    t = s["x"].float() @ s["w"].float().t() + s["bias"]
    y = _act(t, case["act"])
    if s["res"] is not None:
        y = y + s["res"].float()
    out = {"y": y.to(_TYPES[case["out"]])}
    if case["keep"]:
        out["z"] = t.to(torch.bfloat16)
    return out


def _plain_linear_grads(s):
    dy = s["dy"].float()
    dx = (dy @ s["w"].float()) * _act_slope(s["z"].float(), s["case"]["act"])
    return {"dx": dx.to(torch.bfloat16), "dw": dy.t() @ s["x"].float(), "db": dy.sum(0)}


def _plain_norm(s):
    x = s["x"].float()
    mean, rstd = _moments(x)
    y = ((x - mean[:, None]) * rstd[:, None] * s["gamma"] + s["beta"]).to(torch.bfloat16)
    return {"y": y, "mean": mean, "rstd": rstd} if s["case"]["keep"] else {"y": y}


def _plain_norm_grads(s):
    x, dy, rstd = s["x"].float(), s["dy"].float(), s["rstd"][:, None]
    xh = (x - s["mean"][:, None]) * rstd
    h = dy * s["gamma"]
    dx = rstd * (h - h.mean(1, keepdim=True) - xh * (h * xh).mean(1, keepdim=True))
    if s["res"] is not None:
        dx = dx + s["res"].float()
    return {"dx": dx.to(s["x"].dtype), "dgamma": (dy * xh).sum(0), "dbeta": dy.sum(0)}


def _unit(largest, codes):
    """A block's unit, zero where it would not be a normal number, and its reciprocal."""
    u = largest * (1.0 / codes ** 2)
    u = torch.where(u < 2.0 ** -126, torch.zeros_like(u), u)
    return u, torch.where(u > 0, 1.0 / u, torch.zeros_like(u))


def _plain_adamw(s):
    case, eight = s["case"], s["case"]["bits"] == 8
    grad = s["grad"].float()
    out = {}
    if case["clip"]:
        norm = torch.sqrt((grad * grad).sum())
        grad = grad * torch.clamp(MAX_NORM / (norm + 1e-6), max=1.0)
        out["norm"] = norm.reshape(1)
    if eight:
        q = s["m"].float().view(-1, BLOCK)
        m = (s["m_unit"][:, None] * (q * q.abs())).view(-1)
        q = s["v"].float().view(-1, BLOCK)
        r = (s["v_unit"][:, None] * (q * q)).view(-1)
        v = r * r
    else:
        m, v = s["m"], s["v"]
    m = m * BETA1 + grad * (1.0 - BETA1)
    v = v * BETA2 + (grad * grad) * (1.0 - BETA2)
    r = torch.sqrt(v)
    # each block of a tensor's elements takes the settings of the tensor's group
    group = torch.repeat_interleave(s["group_of"], s["blocks_of"], output_size=s["total"] // BLOCK)
    lr, decay = s["lr"][group][:, None], s["decay"][group][:, None]
    hat = m / (r / math.sqrt(1.0 - BETA2 ** STEP) + ADAM_EPS)
    w = s["w"].view(-1, BLOCK) * (1.0 - lr * decay)
    w = (w - (lr / (1.0 - BETA1 ** STEP)) * hat.view(-1, BLOCK)).view(-1)
    s["w"].copy_(w)
    s["copy"].copy_(w)
    if eight:
        mb, rb = m.view(-1, BLOCK), r.view(-1, BLOCK)
        u, inv = _unit(mb.abs().amax(1), 127.0)
        q = torch.sqrt(mb.abs() * inv[:, None]).round().clamp_max(127.0) * torch.sign(mb)
        s["m"].copy_(q.view(-1))
        s["m_unit"].copy_(u)
        out["m"] = (u[:, None] * (q * q.abs())).view(-1)
        u, inv = _unit(rb.amax(1), 255.0)
        q = torch.sqrt(rb * inv[:, None]).round().clamp(max=255.0)
        q = torch.where(rb > 0, q.clamp_min(1.0), q)
        s["v"].copy_(q.view(-1))
        s["v_unit"].copy_(u)
        r = u[:, None] * (q * q)
        out["v"] = (r * r).view(-1)
    else:
        s["m"].copy_(m)
        s["v"].copy_(v)
        out["m"], out["v"] = s["m"], s["v"]
    return {**out, "w": s["w"], "copy": s["copy"]}


# --------------------------------------------------------------------------- the framework's calls
def _own_linear(s):
    s["nb"].numbat_linear_fwd(s["p"], s["x"], s["w"], s["bias"], s["res"], s["zout"], s["y"], s["ws"])
    return {"y": s["y"], "z": s["zout"]} if s["zout"] is not None else {"y": s["y"]}


def _own_linear_grads(s):
    s["nb"].numbat_linear_bwd_data(s["p"], s["dy"], s["w"], s["z"], s["dx"], False, s["ws"])
    s["nb"].numbat_linear_bwd_weight(s["p"], s["x"], s["dy"], s["dw"], s["db"], False, s["ws"])
    return {"dx": s["dx"], "dw": s["dw"], "db": s["db"]}


def _own_norm(s):
    s["nb"].numbat_layer_norm_fwd(s["p"], s["x"], s["gamma"], s["beta"], s["y"], s["mean"], s["rstd"])
    return {"y": s["y"], "mean": s["mean"], "rstd": s["rstd"]} if s["mean"] is not None else {"y": s["y"]}


def _own_norm_grads(s):
    s["nb"].numbat_layer_norm_bwd(s["p"], s["dy"], s["x"], s["mean"], s["rstd"], s["gamma"], s["res"], s["dx"],
                                  s["dgamma"], s["dbeta"], False, s["ws"])
    return {"dx": s["dx"], "dgamma": s["dgamma"], "dbeta": s["dbeta"]}


def _own_adamw(s):
    nb, bits = s["nb"], s["case"]["bits"]
    nb.numbat_adamw_step(s["table"], s["count"], GROUPS, bits, BETA1, BETA2, ADAM_EPS, STEP,
                         MAX_NORM if s["norm"] is not None else 0.0, s["norm"], s["ws"])
    out = {"w": s["w"], "copy": s["copy"], "m": s["m"], "v": s["v"]}
    if bits == 8:
        nb.numbat_adamw_state_values(s["total"], s["m"], s["m_unit"], s["v"], s["v_unit"], s["m_value"], s["v_value"])
        out["m"], out["v"] = s["m_value"], s["v_value"]
    if s["norm"] is not None:
        out["norm"] = s["norm"]
    return out


def run(state):
    """One pass: a layer's forward, its gradients, or one optimiser step (weights and state in place)."""
    return globals()[("_own_" if own else "_plain_") + state["case"]["op"]](state)


# ------------------------------------------------------------------------------- floors and oracle
def work(case):
    op = case["op"]
    if op in ("linear", "linear_grads"):
        m, n, k = case["m"], case["n"], case["k"]
        if op == "linear_grads":
            # dy, x and w read; z read unless there is no activation; dx, dw, db written
            return {"bytes": 2 * (m * n + m * k + n * k) + 2 * m * k * (case["act"] != "none") + 2 * m * k
                    + 4 * n * k + 4 * n, "flops": 4 * m * n * k}
        size = 2 if case["out"] == "bf16" else 4
        return {"bytes": 2 * (m * k + n * k) + 4 * n + m * n * (size * (1 + case["res"]) + 2 * case["keep"]),
                "flops": 2 * m * n * k}
    if op in ("norm", "norm_grads"):
        m, c, size = case["m"], case["c"], 2 if case["x"] == "bf16" else 4
        if op == "norm":
            return {"bytes": m * c * (size + 2) + 8 * c + 8 * m * case["keep"], "flops": 8 * m * c}
        return {"bytes": m * c * (2 + size * (2 + case["res"])) + 12 * c + 8 * m, "flops": 14 * m * c}
    n = sum(_sizes(case))
    grad = 4 if case["grad"] == "f32" else 2
    # weights read and written, the copy written, gradients read; 32-bit moments read and written, or
    # 8-bit codes and their blocks' units read and written and the values they stand for written
    state = 16 if case["bits"] == 32 else 4 + 8 + 16 / BLOCK
    return {"bytes": n * (10 + grad + state), "flops": 20 * n}


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
    if op == "linear":
        t = torch.addmm(_d(s["bias"]), _d(s["x"]), _d(s["w"]).t())
        y = _exact_act(t, case["act"])[0] + (0.0 if s["res"] is None else _d(s["res"]))
        return {"y": y, "z": t} if case["keep"] else {"y": y}
    if op == "linear_grads":
        dy = _d(s["dy"])
        dx = torch.mm(dy, _d(s["w"])).mul_(_exact_act(_d(s["z"]), case["act"])[1])
        return {"dx": dx, "dw": torch.mm(dy.t(), _d(s["x"])), "db": torch.mv(dy.t(), dy.new_ones(dy.shape[0]))}
    if op == "norm":
        x = _d(s["x"])
        var, mean = torch.var_mean(x, 1, correction=0)
        rstd = (var + LN_EPS).rsqrt()
        y = torch.addcmul(_d(s["beta"]), x.sub_(mean[:, None]).mul_(rstd[:, None]), _d(s["gamma"]))
        return {"y": y, "mean": mean, "rstd": rstd} if case["keep"] else {"y": y}
    if op == "norm_grads":
        dy, rstd = _d(s["dy"]), _d(s["rstd"])[:, None]
        xh = _d(s["x"]).sub_(_d(s["mean"])[:, None]).mul_(rstd)
        dgamma, dbeta = torch.einsum("mc,mc->c", dy, xh), dy.sum(0)
        h = dy.mul_(_d(s["gamma"]))
        c = h.shape[1]
        inner = (h * xh).sum(1, keepdim=True).div_(c)
        dx = (h - h.sum(1, keepdim=True).div_(c)).sub_(xh.mul_(inner)).mul_(rstd)
        return {"dx": dx if s["res"] is None else dx.add_(_d(s["res"])), "dgamma": dgamma, "dbeta": dbeta}
    g, w = _d(s["grad"]), _d(s["w"])
    out = {}
    if case["clip"]:
        norm = torch.linalg.vector_norm(g)
        out["norm"] = norm.reshape(1)
        g = g * min(1.0, MAX_NORM / (float(norm) + 1e-6))
    if case["bits"] == 8:
        per = lambda u: _d(u).repeat_interleave(BLOCK)  # noqa: E731
        q, r = _d(s["m"]), _d(s["v"])
        m, v = q * q.abs() * per(s["m_unit"]), (r * r * per(s["v_unit"])) ** 2
    else:
        m, v = _d(s["m"]), _d(s["v"])
    m = torch.lerp(g, m, BETA1)
    v = torch.lerp(g * g, v, BETA2)
    for n, at, group in s["rows"]:
        lr, decay = (float(torch.tensor(x, dtype=torch.float32)) for x in GROUPS[group])
        here = slice(at, at + n)
        hat = m[here] / (1.0 - BETA1 ** STEP)
        w[here] -= lr * (decay * w[here] + hat / ((v[here] / (1.0 - BETA2 ** STEP)).sqrt() + ADAM_EPS))
    if case["bits"] == 8:  # what is rounded to a code has no value of its own here
        return {**out, "m": None, "v": None, "w": w, "copy": w}
    return {**out, "m": m, "v": v, "w": w, "copy": w}


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
