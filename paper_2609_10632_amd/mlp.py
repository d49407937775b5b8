"""The residual MLP block driven through the C ABI: y = x + W2 act(W1 norm(x) + b1) + b2 over the
rows of a matrix (the pixels of an NHWC map, or tokens), its backward and its AdamW step.

Device memory comes from PyTorch and every computation of the block is a call into the library:

  forward    layer_norm_fwd, linear_fwd (bias and activation in its epilogue, the pre-activation z
             kept), linear_fwd (bias and residual in its epilogue): 3 calls
  backward   linear_bwd_data (act'(z) in its epilogue) and linear_bwd_weight of each layer, then
             layer_norm_bwd, which adds the gradient that goes round the block: 5 calls
  step       adamw_step over the six parameter tensors, with the bf16 copies that the products read
             written on the way: 1 call

As a command it trains a block to follow another of the same shape on synthetic rows:

  python -m paper_2609_10632_amd.mlp --rows 6400 --width 192 --hidden 768 --steps 50 --state-bits 8
"""
from __future__ import annotations

import argparse

import torch

from . import numbat as nb
from .blocks import DEV, workspace

ACTS = {"none": nb.ACT_NONE, "relu": nb.ACT_RELU, "gelu": nb.ACT_GELU, "gelu_tanh": nb.ACT_GELU_TANH,
        "silu": nb.ACT_SILU}
STATE_BLOCK = 256  # elements that share a unit in the 8-bit optimiser state


class MlpBlock:
    """A block of `width` features, widened to `hidden`, and the buffers of steps of up to `rows` rows.

    Parameters (fp32, views of one flat buffer): ``w1`` [hidden][width], ``b1``, ``w2``
    [width][hidden], ``b2``, ``gamma``, ``beta``; gradients of the same names in ``grads``.  The
    products read the bf16 ``copies`` of ``w1`` and ``w2``, which step() writes: who writes parameters by
    hand (a checkpoint's) writes those too."""

    def __init__(self, rows, width, hidden, act="gelu", eps=1e-5, state_bits=32, seed=0, device=DEV):
        self.rows, self.width, self.hidden, self.eps, self.device = rows, width, hidden, eps, device
        self.act, self.state_bits, self.steps = ACTS[act], state_bits, 0
        shapes = {"w1": (hidden, width), "b1": (hidden,), "w2": (width, hidden), "b2": (width,), "gamma": (width,),
                  "beta": (width,)}
        at, spans = 0, {}
        for name, shape in shapes.items():  # every tensor starts a whole block of the 8-bit state
            n = shape[0] * (shape[1] if len(shape) == 2 else 1)
            spans[name] = (at, n)
            at += -(-n // STATE_BLOCK) * STATE_BLOCK
        new = lambda n, dtype: torch.zeros(n, dtype=dtype, device=device)  # noqa: E731
        cut = lambda flat: {k: flat[a:a + n].view(shapes[k]) for k, (a, n) in spans.items()}  # noqa: E731
        self.params, self.grads = cut(new(at, torch.float32)), cut(new(at, torch.float32))
        self.copies = cut(new(at, torch.bfloat16))
        moment = (torch.float32, torch.float32) if state_bits == 32 else (torch.int8, torch.uint8)
        self.m, self.v = cut(new(at, moment[0])), cut(new(at, moment[1]))
        units = at // STATE_BLOCK if state_bits == 8 else 0
        self.m_unit, self.v_unit = new(units, torch.float32), new(units, torch.float32)

        g = torch.Generator().manual_seed(seed)
        for name, fan in (("w1", width), ("w2", hidden), ("b1", width), ("b2", hidden)):
            p = self.params[name]
            p.copy_((torch.rand(p.shape, generator=g) * 2 - 1) * fan ** -0.5)
        self.params["gamma"].fill_(1.0)
        for name, p in self.params.items():
            self.copies[name].copy_(p)
        table = []
        for name, (a, _) in spans.items():  # matrices decay (group 0), vectors do not (group 1)
            e = {"w": self.params[name], "grad": self.grads[name], "m": self.m[name], "v": self.v[name],
                 "w_copy": self.copies[name], "group": 0 if name in ("w1", "w2") else 1}
            if state_bits == 8:
                e["m_unit"], e["v_unit"] = self.m_unit[a // STATE_BLOCK:], self.v_unit[a // STATE_BLOCK:]
            table.append(e)
        self.count = len(table)
        self.table = torch.frombuffer(bytearray(nb.adamw_table(table)), dtype=torch.uint8).to(device)

        bf = lambda *s: torch.empty(s, dtype=torch.bfloat16, device=device)  # noqa: E731
        self.normed, self.wide, self.z, self.y = bf(rows, width), bf(rows, hidden), bf(rows, hidden), bf(rows, width)
        self.dwide, self.dnormed, self.dx = bf(rows, hidden), bf(rows, width), bf(rows, width)
        self.mean, self.rstd = new(rows, torch.float32), new(rows, torch.float32)
        self.norm = new(1, torch.float32)
        self.kept = None  # rows of the forward whose activations, statistics and weights are at hand
        up, down, down_grad, ln = self._problems(rows, width, width)
        size = nb.numbat_workspace_size
        # all calls of the block are on one stream, one after another: they share a workspace
        self.ws_bytes = max(size(nb.OP_LINEAR_FWD, up), size(nb.OP_LINEAR_FWD, down), size(nb.OP_LINEAR_BWD_DATA, up),
                            size(nb.OP_LINEAR_BWD_DATA, down_grad), size(nb.OP_LINEAR_BWD_WEIGHT, up),
                            size(nb.OP_LINEAR_BWD_WEIGHT, down), size(nb.OP_LAYER_NORM_BWD, ln),
                            size(nb.OP_ADAMW, None))
        self.ws = workspace(self.ws_bytes, device)

    def _problems(self, rows, x_stride, g_stride):
        """The two layers', the second one's as its data gradient takes it, and the norm's."""
        up = nb.linear_problem(rows, self.hidden, self.width, act=self.act)
        down = nb.linear_problem(rows, self.width, self.hidden, r_row_stride=x_stride, y_row_stride=0)
        down_grad = nb.linear_problem(rows, self.width, self.hidden, act=self.act, y_row_stride=g_stride)
        ln = nb.layer_norm_problem(rows, self.width, eps=self.eps, x_row_stride=x_stride, r_row_stride=g_stride)
        return up, down, down_grad, ln

    def _workspace(self, *needs):
        """The block's workspace; a call of fewer rows may split a reduction where the full one does not."""
        need = max(nb.numbat_workspace_size(op, p) for op, p in needs)
        if need > self.ws_bytes:
            self.ws, self.ws_bytes = workspace(need, self.device), need
        return self.ws

    def _check(self, t, what):
        if t.dim() != 2 or t.shape[1] != self.width or t.shape[0] > self.rows or t.dtype != torch.bfloat16 \
                or t.stride(1) != 1 or t.stride(0) < self.width:
            raise ValueError(f"{what}: expected bf16 rows of {self.width}, at most {self.rows}")
        return t.shape[0], t.stride(0)

    def forward(self, x, keep=True):
        """x: bf16 [rows][width], rows as far apart as its stride says (``map[..., a:b].flatten(0, 2)``
        of an NHWC map).  keep: for backward(); without, as in serving, neither z nor the norm's
        statistics are written, and backward() refuses what an earlier forward has kept, as other
        activations are overwritten.  Returns a view of the block's output buffer, which x may
        be only without keep."""
        rows, stride = self._check(x, "x")
        if rows and x.untyped_storage().data_ptr() == self.y.untyped_storage().data_ptr():
            if keep or x.data_ptr() != self.y.data_ptr():
                raise ValueError("x: lies in the block's own output, which this forward overwrites")
        self.kept = None
        up, down, _, ln = self._problems(rows, stride, self.width)
        ws = self._workspace((nb.OP_LINEAR_FWD, up), (nb.OP_LINEAR_FWD, down))
        c = self.copies
        nb.numbat_layer_norm_fwd(ln, x, self.params["gamma"], self.params["beta"], self.normed,
                                 self.mean if keep else None, self.rstd if keep else None)
        nb.numbat_linear_fwd(up, self.normed, c["w1"], self.params["b1"], None, self.z if keep else None, self.wide, ws)
        nb.numbat_linear_fwd(down, self.wide, c["w2"], self.params["b2"], x, None, self.y, ws)
        self.kept = rows if keep else None
        return self.y[:rows]

    def backward(self, x, g, accumulate=False):
        """The gradients of sum(g y): parameters' into ``grads`` (accumulate: added), x's into the
        returned buffer.  The last forward has to be forward(x, keep=True), with no step() since."""
        rows, stride = self._check(x, "x")
        g_rows, g_stride = self._check(g, "g")
        if g_rows != rows:
            raise ValueError("g: one row for each of x")
        if self.kept != rows:
            raise RuntimeError(f"backward of {rows} rows: the last forward kept {self.kept or 'nothing'}, or a step followed it")
        up, _, down, ln = self._problems(rows, stride, g_stride)
        up.act = nb.ACT_NONE  # (the norm's output went into it as it is)
        ws = self._workspace(*[(o, p) for o in (nb.OP_LINEAR_BWD_DATA, nb.OP_LINEAR_BWD_WEIGHT) for p in (up, down)],
                             (nb.OP_LAYER_NORM_BWD, ln))
        c, d = self.copies, self.grads
        nb.numbat_linear_bwd_data(down, g, c["w2"], self.z, self.dwide, False, ws)
        nb.numbat_linear_bwd_weight(down, self.wide, g, d["w2"], d["b2"], accumulate, ws)
        nb.numbat_linear_bwd_data(up, self.dwide, c["w1"], None, self.dnormed, False, ws)
        nb.numbat_linear_bwd_weight(up, self.normed, self.dwide, d["w1"], d["b1"], accumulate, ws)
        nb.numbat_layer_norm_bwd(ln, self.dnormed, x, self.mean, self.rstd, self.params["gamma"], g, self.dx,
                                 d["gamma"], d["beta"], accumulate, ws)
        return self.dx[:rows]

    def step(self, lr, weight_decay=0.1, betas=(0.9, 0.95), eps=1e-8, max_norm=1.0):
        """One AdamW step from ``grads``; returns the device float that receives the gradients'
        norm, or None with max_norm = 0, which forms none."""
        nb.numbat_adamw_step(self.table, self.count, ((lr, weight_decay), (lr, 0.0)), self.state_bits, betas[0],
                             betas[1], eps, self.steps + 1, max_norm, self.norm if max_norm > 0 else None, self.ws)
        self.steps += 1
        self.kept = None
        return self.norm if max_norm > 0 else None


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--rows", type=int, default=6400)
    ap.add_argument("--width", type=int, default=192)
    ap.add_argument("--hidden", type=int, default=768)
    ap.add_argument("--act", choices=sorted(ACTS), default="gelu")
    ap.add_argument("--steps", type=int, default=50)
    ap.add_argument("--lr", type=float, default=2e-3)
    ap.add_argument("--state-bits", type=int, choices=(8, 32), default=32)
    a = ap.parse_args(argv)
    block = MlpBlock(a.rows, a.width, a.hidden, a.act, state_bits=a.state_bits, seed=1)
    goal = MlpBlock(a.rows, a.width, a.hidden, a.act, seed=2)
    gen = torch.Generator(device=DEV)
    gen.manual_seed(0)
    first = last = None
    for i in range(a.steps):
        x = torch.randn((a.rows, a.width), generator=gen, device=DEV).bfloat16()
        off = block.forward(x).float() - goal.forward(x, keep=False).float()
        block.backward(x, (off * (2.0 / a.rows)).bfloat16())
        norm = block.step(a.lr, weight_decay=0.0)
        last = float((off * off).sum() / a.rows)
        first = last if first is None else first
        if i % 10 == 0 or i == a.steps - 1:
            print(f"step {i}: squared error per row {last:.5f}, gradient norm {float(norm):.5f}", flush=True)
    return first, last


if __name__ == "__main__":
    main()
