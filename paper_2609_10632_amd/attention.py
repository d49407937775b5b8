"""The residual attention block driven through the C ABI, over the rows of maps (the pixels of NHWC images)
or of token sequences:

  y = x + Wo attention(rotate(q), rotate(k), v) + bo,   [q k v] = Wqkv act(group_norm(x)) + bqkv

Device memory comes from PyTorch and every computation of the block is a call into the library:

  forward    group_norm_fwd, linear_fwd (bias), rotary (q and k turned in place), attention_fwd, linear_fwd
             (bias and residual in its epilogue): 5 calls
  backward   linear_bwd_data and linear_bwd_weight of each layer, attention_bwd between them, rotary turned back in
             place on the gradients, then group_norm_bwd, which adds the gradient that goes round the block: 7 calls
  step       adamw_step over the six parameter tensors, with the bf16 copies that the products read written
             on the way: 1 call

q, k and v lie side by side in one matrix, and so do their gradients.  As a command it trains a block to
follow another of the same shape on synthetic maps:

  python -m paper_2609_10632_amd.attention --images 4 --side 20 --width 192 --heads 6 --steps 50
"""
from __future__ import annotations

import argparse
import functools
import math

import torch

from . import numbat as nb
from .blocks import DEV, workspace
from .mlp import ACTS, STATE_BLOCK


def _on_its_device(call):
    """A call of a block whose device is not the current one: the library launches on the current device."""
    @functools.wraps(call)
    def run(self, *a, **k):
        if self.place.type != "cuda" or self.place.index == torch.cuda.current_device():
            return call(self, *a, **k)
        with torch.cuda.device(self.place):
            return call(self, *a, **k)
    return run


class AttentionBlock:
    """A block of `width` features in `heads` heads (`kv_heads` of k and v, each shared by as many of q) and the
    buffers of batches of up to `images` maps of up to prod(extents) rows.

    extents: the axes of a map, the last the fastest: (height, width), (frames, height, width), or (tokens,).
    pairs: the pairs of features of each head that turn with each axis' position (an even share of half a head
    unless given; () for none).  causal: a row attends to itself and the rows before it; the norm's mean and deviation
    are over all rows all the same, so that through them a row's output depends on the rows behind it (a model that
    generates rows one by one needs a norm of each row, as layer_norm_fwd is).

    Parameters (fp32, views of one flat buffer): ``wqkv`` [(heads + 2 kv_heads) d][width], ``bqkv``, ``wo``
    [width][heads d], ``bo``, ``gamma``, ``beta``; gradients of the same names in ``grads``.  The products read the bf16
    ``copies`` of ``wqkv`` and ``wo``, which step() writes: who writes parameters by hand (a checkpoint's) writes those
    too."""

    def __init__(self, images, extents, width, heads, kv_heads=None, groups=32, pairs=None, act="none", causal=False,
                 base=10000.0, eps=1e-5, state_bits=32, seed=0, device=DEV):
        kv_heads = heads if kv_heads is None else kv_heads
        extents = tuple(extents)
        if min(width, heads, kv_heads, groups) < 1 or width % heads or heads % kv_heads or width % groups or (width // heads) % 8:
            raise ValueError("width: whole heads of a multiple of 8 features and whole groups; kv_heads divides heads")
        if width // heads > 128:
            raise ValueError(f"width: heads of {width // heads} features, at most 128")
        if min(extents, default=0) < 1:
            raise ValueError(f"extents: {extents}, at least one axis of at least one row")
        self.images, self.extents, self.width, self.heads, self.kv_heads = images, extents, width, heads, kv_heads
        self.d, self.groups, self.causal, self.base, self.eps = width // heads, groups, causal, base, eps
        if pairs is None:
            each = self.d // 2 // len(self.extents)
            pairs = (self.d // 2 - each * (len(self.extents) - 1),) + (each,) * (len(self.extents) - 1)
        self.pairs = tuple(pairs)
        if self.pairs and len(self.pairs) != len(self.extents):
            raise ValueError("pairs: a number for each axis, or none at all")
        if self.pairs and (len(self.pairs) > 4 or min(self.pairs) < 1 or 2 * sum(self.pairs) > self.d):
            raise ValueError(f"pairs: {self.pairs}, at least 1 for each of at most 4 axes and {self.d // 2} in all")
        self.act, self.state_bits, self.steps, self.device = ACTS[act], state_bits, 0, device
        self.qkv_width = (heads + 2 * kv_heads) * self.d
        shapes = {"wqkv": (self.qkv_width, width), "bqkv": (self.qkv_width,), "wo": (width, heads * self.d), "bo": (width,),
                  "gamma": (width,), "beta": (width,)}
        at, spans = 0, {}
        for name, shape in shapes.items():  # every tensor starts a whole block of the 8-bit state
            spans[name] = (at, math.prod(shape))
            at += -(-math.prod(shape) // STATE_BLOCK) * STATE_BLOCK
        new = lambda n, dtype: torch.zeros(n, dtype=dtype, device=device)  # noqa: E731
        cut = lambda flat: {k: flat[a:a + n].view(shapes[k]) for k, (a, n) in spans.items()}  # noqa: E731
        self.params, self.grads = cut(new(at, torch.float32)), cut(new(at, torch.float32))
        self.copies = cut(new(at, torch.bfloat16))
        moment = (torch.float32, torch.float32) if state_bits == 32 else (torch.int8, torch.uint8)
        self.m, self.v = cut(new(at, moment[0])), cut(new(at, moment[1]))
        units = at // STATE_BLOCK if state_bits == 8 else 0
        self.m_unit, self.v_unit = new(units, torch.float32), new(units, torch.float32)
        g = torch.Generator().manual_seed(seed)
        for name in ("wqkv", "bqkv", "wo", "bo"):
            p = self.params[name]
            p.copy_((torch.rand(p.shape, generator=g) * 2 - 1) * width ** -0.5)
        self.params["gamma"].fill_(1.0)
        for name, p in self.params.items():
            self.copies[name].copy_(p)
        table = []
        for name, (a, _) in spans.items():  # matrices decay (group 0), vectors do not (group 1)
            e = {"w": self.params[name], "grad": self.grads[name], "m": self.m[name], "v": self.v[name],
                 "w_copy": self.copies[name], "group": 0 if name in ("wqkv", "wo") else 1}
            if state_bits == 8:
                e["m_unit"], e["v_unit"] = self.m_unit[a // STATE_BLOCK:], self.v_unit[a // STATE_BLOCK:]
            table.append(e)
        self.count = len(table)
        self.table = torch.frombuffer(bytearray(nb.adamw_table(table)), dtype=torch.uint8).to(device)

        rows = images * math.prod(self.extents)
        bf = lambda n: torch.empty((rows, n), dtype=torch.bfloat16, device=device)  # noqa: E731
        self.normed, self.qkv, self.mixed, self.y = bf(width), bf(self.qkv_width), bf(heads * self.d), bf(width)
        self.dnormed, self.dqkv, self.dmixed, self.dx = bf(width), bf(self.qkv_width), bf(heads * self.d), bf(width)
        self.place = self.y.device
        self.mean, self.rstd = new((images, groups), torch.float32), new((images, groups), torch.float32)
        self.lse = new(rows * heads, torch.float32)
        self.lengths = new(images, torch.int32)  # of the forward that is kept, as its backward takes them
        self.norm = new(1, torch.float32)
        # where results go that later calls of a forward, or of a backward, still read over their operands
        self.written = {t.untyped_storage().data_ptr() for t in (self.y, self.normed, self.qkv, self.mixed)}
        self.written_back = {t.untyped_storage().data_ptr() for t in (self.dnormed, self.dqkv, self.dmixed)}
        self.kept = None  # (rows, extents, whether with lengths) of the forward whose activations, statistics and weights are at hand
        # all calls of the block are on one stream, one after another: they share a workspace (one that was too
        # small for a later batch is kept, as a captured graph may use it)
        self.ws, self.ws_bytes, self.outgrown = None, 0, []
        self._workspace(nb.numbat_workspace_size(nb.OP_ADAMW, None))

    def _workspace(self, need):
        if need > self.ws_bytes:
            self.outgrown.append(self.ws)
            self.ws, self.ws_bytes = workspace(need, self.place), need
        return self.ws

    def _problems(self, images, extents, x_stride, g_stride):
        """The norm's, the two layers' (the second as each direction takes it), the rotation's and the attention's."""
        n = math.prod(extents)
        rows, width, d = images * n, self.width, self.d
        norm = nb.group_norm_problem(images, n, width, self.groups, act=self.act, eps=self.eps, x_row_stride=x_stride,
                                     r_row_stride=g_stride)
        qkv = nb.linear_problem(rows, self.qkv_width, width)
        out = nb.linear_problem(rows, width, self.heads * d, r_row_stride=x_stride)
        out_grad = nb.linear_problem(rows, width, self.heads * d, y_row_stride=g_stride)
        turn = [nb.rotary_problem(rows, self.heads + self.kv_heads, d, self.pairs, extents=extents, base=self.base,
                                  inverse=back, x_row_stride=self.qkv_width, y_row_stride=self.qkv_width)
                for back in (False, True)] if self.pairs else None
        att = nb.attention_problem(images, n, n, self.heads, self.kv_heads, d, causal=self.causal,
                                   q_row_stride=self.qkv_width, k_row_stride=self.qkv_width, v_row_stride=self.qkv_width)
        return norm, qkv, out, out_grad, turn, att

    def _cut(self, qkv, rows):
        a, b = self.heads * self.d, (self.heads + self.kv_heads) * self.d
        return qkv[:rows, :a], qkv[:rows, a:b], qkv[:rows, b:]

    def _check(self, t, what, rows, written):
        """`written`: buffers that it may not lie in."""
        if t.dim() != 2 or t.shape != (rows, self.width) or t.dtype != torch.bfloat16 or t.stride(1) != 1 \
                or (rows > 1 and t.stride(0) < self.width) or t.device != self.place:
            raise ValueError(f"{what}: expected bf16 rows of {self.width}, {rows} of them, on the block's device")
        if rows and t.untyped_storage().data_ptr() in written:
            raise ValueError(f"{what}: lies in a buffer of the block that is written before it is read for the last time")
        return t.stride(0) if rows > 1 else self.width

    def _check_lengths(self, lengths, images):
        if lengths is not None and (lengths.dtype != torch.int32 or lengths.shape != (images,) or not lengths.is_contiguous()
                                    or lengths.device != self.place):
            raise ValueError(f"lengths: expected int32 [{images}] on the block's device")

    @_on_its_device
    def forward(self, x, extents=None, lengths=None, keep=True):
        """x: bf16 [images prod(extents)][width], rows as far apart as its stride says.  extents: of this batch's
        maps (the block's unless given; at most as many rows).  lengths: int32 [images] on the device, the rows of each
        map that take part in attention (a padded batch of sequences), or None for all; a row behind them attends to
        nothing.  They are the first rows of the map as it is laid out here, and their positions those of these extents:
        maps padded at the bottom, not at the side.  The norm's statistics are over all rows, the padding's too, whose
        values have to be finite and belong to the result.  keep: for backward(); without, as in serving, the statistics
        are not written, and backward() refuses what an earlier forward has kept.  Returns a view of the block's
        output buffer, in which x may not lie; nor in one of its activations', or with keep of their gradients'."""
        extents = self.extents if extents is None else tuple(extents)
        n = math.prod(extents)
        if len(extents) != len(self.extents) or min(extents) < 1 or x.dim() != 2 or x.shape[0] % n or x.shape[0] > self.y.shape[0] \
                or x.shape[0] // n > self.images:
            raise ValueError(f"x: whole maps of {extents}, at most {self.images} and {self.y.shape[0]} rows")
        rows, images = x.shape[0], x.shape[0] // n
        stride = self._check(x, "x", rows, self.written | self.written_back if keep else self.written)
        self._check_lengths(lengths, images)
        self.kept = None
        norm, qkv, out, _, turn, att = self._problems(images, extents, stride, self.width)
        size = nb.numbat_workspace_size
        ws = self._workspace(max(size(nb.OP_GROUP_NORM_FWD, norm), size(nb.OP_LINEAR_FWD, qkv), size(nb.OP_LINEAR_FWD, out),
                                 size(nb.OP_ATTENTION_FWD, att)))
        c = self.copies
        nb.numbat_group_norm_fwd(norm, x, self.params["gamma"], self.params["beta"], self.normed,
                                 self.mean if keep else None, self.rstd if keep else None, ws)
        nb.numbat_linear_fwd(qkv, self.normed, c["wqkv"], self.params["bqkv"], None, None, self.qkv, ws)
        if turn:
            nb.numbat_rotary(turn[0], self.qkv, None, self.qkv)
        q, k, v = self._cut(self.qkv, rows)
        if keep and lengths is not None:
            lengths = self.lengths[:images].copy_(lengths)
        nb.numbat_attention_fwd(att, q, k, v, lengths, lengths, self.mixed, self.lse if keep else None, ws)
        nb.numbat_linear_fwd(out, self.mixed, c["wo"], self.params["bo"], x, None, self.y, ws)
        self.kept = (rows, extents, lengths is not None) if keep else None
        return self.y[:rows]

    @_on_its_device
    def backward(self, x, g, extents=None, lengths=None, accumulate=False):
        """The gradients of sum(g y): parameters' into ``grads`` (accumulate: added), x's into the returned
        buffer.  The last forward has to be of the same x and extents with keep, with no step() since, and with
        lengths if they are given here; what they were then is what counts.  x or g may lie in the returned buffer (a
        backward of x there is the last of its forward), not in the gradients of the block's activations."""
        extents = self.extents if extents is None else tuple(extents)
        if self.kept != (x.shape[0], extents, lengths is not None):
            raise RuntimeError(f"backward of {x.shape[0]} rows in {extents}{' with' if lengths is not None else ' without'} "
                               f"lengths: the last forward kept {self.kept or 'nothing'}, or a step followed it")
        rows, images = x.shape[0], x.shape[0] // math.prod(extents)
        stride = self._check(x, "x", rows, self.written | self.written_back)
        g_stride = self._check(g, "g", rows, self.written_back)
        self._check_lengths(lengths, images)
        if lengths is not None:
            lengths = self.lengths[:images]
        norm, qkv, out, out_grad, turn, att = self._problems(images, extents, stride, g_stride)
        size = nb.numbat_workspace_size
        ws = self._workspace(max(size(nb.OP_LINEAR_BWD_DATA, out_grad), size(nb.OP_LINEAR_BWD_WEIGHT, out_grad),
                                 size(nb.OP_ATTENTION_BWD, att), size(nb.OP_LINEAR_BWD_DATA, qkv),
                                 size(nb.OP_LINEAR_BWD_WEIGHT, qkv), size(nb.OP_GROUP_NORM_BWD, norm)))
        c, d = self.copies, self.grads
        nb.numbat_linear_bwd_data(out_grad, g, c["wo"], None, self.dmixed, False, ws)
        nb.numbat_linear_bwd_weight(out_grad, self.mixed, g, d["wo"], d["bo"], accumulate, ws)
        q, k, v = self._cut(self.qkv, rows)
        dq, dk, dv = self._cut(self.dqkv, rows)
        nb.numbat_attention_bwd(att, self.dmixed, q, k, v, self.mixed, self.lse, lengths, lengths, dq, dk, dv, ws)
        if turn:
            nb.numbat_rotary(turn[1], self.dqkv, None, self.dqkv)
        nb.numbat_linear_bwd_data(qkv, self.dqkv, c["wqkv"], None, self.dnormed, False, ws)
        nb.numbat_linear_bwd_weight(qkv, self.normed, self.dqkv, d["wqkv"], d["bqkv"], accumulate, ws)
        nb.numbat_group_norm_bwd(norm, self.dnormed, x, self.mean, self.rstd, self.params["gamma"], self.params["beta"],
                                 self.dx, d["gamma"], d["beta"], accumulate, ws, residual_grad=g)
        if x.untyped_storage().data_ptr() == self.dx.untyped_storage().data_ptr():
            self.kept = None  # (x has become its gradient)
        return self.dx[:rows]

    @_on_its_device
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
    ap.add_argument("--images", type=int, default=4)
    ap.add_argument("--side", type=int, default=20)
    ap.add_argument("--width", type=int, default=192)
    ap.add_argument("--heads", type=int, default=6)
    ap.add_argument("--kv-heads", type=int, default=None)
    ap.add_argument("--groups", type=int, default=32)
    ap.add_argument("--act", choices=sorted(ACTS), default="none")
    ap.add_argument("--steps", type=int, default=50)
    ap.add_argument("--lr", type=float, default=2e-3)
    ap.add_argument("--state-bits", type=int, choices=(8, 32), default=32)
    a = ap.parse_args(argv)
    make = lambda seed: AttentionBlock(a.images, (a.side, a.side), a.width, a.heads, a.kv_heads, a.groups, act=a.act,  # noqa: E731
                                       state_bits=a.state_bits, seed=seed)
    block, goal = make(1), make(2)
    gen = torch.Generator(device=DEV)
    gen.manual_seed(0)
    rows = a.images * a.side * a.side
    first = last = None
    for i in range(a.steps):
        x = torch.randn((rows, a.width), generator=gen, device=DEV).bfloat16()
        off = block.forward(x).float() - goal.forward(x, keep=False).float()
        block.backward(x, (off * (2.0 / rows)).bfloat16())
        norm = block.step(a.lr, weight_decay=0.0)
        last = float((off * off).sum() / rows)
        first = last if first is None else first
        if i % 10 == 0 or i == a.steps - 1:
            print(f"step {i}: squared error per row {last:.5f}, gradient norm {float(norm):.5f}", flush=True)
    return first, last


if __name__ == "__main__":
    main()
