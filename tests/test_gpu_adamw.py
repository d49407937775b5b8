"""The AdamW step (numbat_adamw_step) against its formula: 32-bit state in 64 bits, 8-bit state code
for code against IEEE fp32 on the CPU, the norm's clip, groups, odd and misaligned tensors, the
copy, blocks of zeros, tiny and huge values, many steps.

Bounds: an update is a dozen fp32 operations on values of its own size: 16 2^-24 of each term."""
import math

import pytest

from mlp_ref import B, D, U, close

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
if torch.cuda.is_available():
    from paper_2609_10632_amd import blocks
    from paper_2609_10632_amd import numbat as nb

GROUPS = [(1e-3, 0.1), (3e-3, 0.0)]
B1, B2, EPS = 0.9, 0.95, 1e-8
BLOCK = 256
SIZES = [1, 3, 255, 256, 257, 1000, 4095, 4096, 4097, 70000]


class Tensors:
    """Tensors of the given sizes, each starting `shift` elements past a 16-byte boundary."""

    def __init__(self, sizes, bits, grad=torch.float32, seed=0, shift=0, scale=0.01, copy=True, zeros=False):
        g = torch.Generator().manual_seed(seed)
        self.bits, self.sizes, self.t = bits, sizes, []

        def place(v):
            room = torch.zeros(v.numel() + 64, dtype=v.dtype, device="cuda")
            room[shift:shift + v.numel()] = v.cuda()
            return room[shift:shift + v.numel()]

        for i, n in enumerate(sizes):
            e = {"w": place(torch.randn(n, generator=g) * 0.05), "group": i % 2,
                 "grad": place((torch.randn(n, generator=g) * scale).to(grad))}
            nb_ = -(-n // BLOCK)
            if bits == 32:
                e["m"] = place(torch.zeros(n) if zeros else torch.randn(n, generator=g) * 0.003)
                e["v"] = place(torch.zeros(n) if zeros else (torch.randn(n, generator=g) * 0.01) ** 2)
            else:
                k = 0 if zeros else 1
                e["m"] = place((torch.randint(-127, 128, (n,), generator=g) * k).to(torch.int8))
                e["v"] = place((torch.randint(1, 256, (n,), generator=g) * k).to(torch.uint8))
                e["m_unit"] = (torch.rand(nb_, generator=g) * 1e-6 * k).cuda()
                e["v_unit"] = (torch.rand(nb_, generator=g) * 5e-7 * k).cuda()
            if copy:
                e["w_copy"] = place(torch.zeros(n, dtype=torch.bfloat16))
            self.t.append(e)
        raw = nb.adamw_table(self.t)
        self.table = torch.frombuffer(bytearray(raw), dtype=torch.uint8).cuda()
        self.norm = torch.zeros(1, device="cuda")
        self.ws = blocks.workspace(nb.numbat_workspace_size(nb.OP_ADAMW, None))

    def step(self, t, max_norm=0.0, groups=GROUPS, stream=None):
        nb.numbat_adamw_step(self.table, len(self.t), groups, self.bits, B1, B2, EPS, t, max_norm,
                             self.norm if max_norm else None, self.ws, stream=stream)

    def host(self):
        return [{k: v.clone().cpu() if torch.is_tensor(v) else v for k, v in e.items()} for e in self.t]


def coefficient(entries, max_norm):
    total = math.sqrt(sum(float((e["grad"].to(D) ** 2).sum()) for e in entries))
    return total, (min(1.0, max_norm / (total + 1e-6)) if max_norm else 1.0)


def check32(ts, before, t, max_norm=0.0):
    total, c = coefficient(before, max_norm)
    for old, new in zip(before, ts.host()):
        lr, wd = GROUPS[old["group"]]
        g = old["grad"].to(D) * c
        m = B1 * old["m"].to(D) + (1 - B1) * g
        v = B2 * old["v"].to(D) + (1 - B2) * g * g
        move = lr / (1 - B1 ** t) * m / (torch.sqrt(v / (1 - B2 ** t)) + EPS)
        w = old["w"].to(D) * (1 - lr * wd) - move
        # where the terms of m cancel, its error stays of the terms' size, and so the step's
        em = 8 * U * (B1 * old["m"].to(D).abs() + (1 - B1) * g.abs())
        close(new["m"], m, em + 1e-40, "m")
        close(new["v"], v, 12 * U * v + 1e-40, "v")
        off = 16 * U * (move.abs() + old["w"].to(D).abs()) + lr / (1 - B1 ** t) * em / (torch.sqrt(v / (1 - B2 ** t)) + EPS)
        close(new["w"], w, off + 1e-40, "w")
        assert torch.equal(new["w_copy"], new["w"].bfloat16())
    if max_norm:
        close(ts.norm, torch.tensor([total], dtype=D), 2 * U * total, "norm")


@pytest.mark.parametrize("grad", (torch.float32, torch.bfloat16))
@pytest.mark.parametrize("shift", (0, 1, 2, 4))
def test_32_bit_state(grad, shift):
    ts = Tensors(SIZES, 32, grad, seed=shift, shift=shift)
    for t, max_norm in ((1, 0.0), (2, 0.5), (3, 100.0), (1000, 0.5)):
        before = ts.host()
        ts.step(t, max_norm)
        check32(ts, before, t, max_norm)


def root(x):
    """IEEE fp32 square root (torch's on the CPU is off by a bit now and then)."""
    return torch.sqrt(x.to(D)).float()


def codes(value, codes_max):
    """(unit, codes) of blocks of non-negative fp32 values [blocks, 256], in IEEE fp32."""
    u = value.amax(1) * torch.tensor(1.0 / codes_max ** 2, dtype=torch.float32)
    u = torch.where(u < 2.0 ** -126, torch.zeros_like(u), u)
    inv = torch.where(u > 0, 1.0 / u, torch.zeros_like(u))
    return u, root(value * inv[:, None]).round().clamp_max(codes_max)


def check8(ts, before, t, max_norm=0.0):
    """In fp32 on the CPU, whose +, * and / round as IEEE says: the codes and units are equal."""
    _, c = coefficient(before, max_norm)
    for old, new in zip(before, ts.host()):
        n = old["w"].numel()
        pad = lambda x: torch.nn.functional.pad(x, (0, -n % BLOCK)).view(-1, BLOCK)  # noqa: E731
        lr, wd = GROUPS[old["group"]]
        g = pad(old["grad"].float())
        if max_norm:
            g = g * torch.tensor(c, dtype=torch.float32)
        q = pad(old["m"].float())
        m = old["m_unit"][:, None] * (q * q.abs())
        q = pad(old["v"].float())
        r = old["v_unit"][:, None] * (q * q)
        m = m * B1 + g * (1 - B1)
        v = (r * r) * B2 + (g * g) * (1 - B2)
        r = root(v)
        um, qm = codes(m.abs(), 127.0)
        qm = qm * torch.sign(m)
        ur, qr = codes(r, 255.0)
        qr = torch.where(r > 0, qr.clamp_min(1), qr)
        flat = lambda x: x.reshape(-1)[:n]  # noqa: E731
        assert torch.equal(new["m_unit"], um) and torch.equal(new["v_unit"], ur), n
        assert torch.equal(new["m"], flat(qm).to(torch.int8)) and torch.equal(new["v"], flat(qr).to(torch.uint8)), n
        move = lr / (1 - B1 ** t) * flat(m).to(D) / (torch.sqrt(flat(v).to(D) / (1 - B2 ** t)) + EPS)
        w = old["w"].to(D) * (1 - lr * wd) - move
        close(new["w"], w, 16 * U * (move.abs() + old["w"].to(D).abs()) + 1e-40, "w")
        assert torch.equal(new["w_copy"], new["w"].bfloat16())


@pytest.mark.parametrize("grad", (torch.float32, torch.bfloat16))
@pytest.mark.parametrize("shift", (0, 1, 4))
def test_8_bit_state(grad, shift):
    ts = Tensors(SIZES, 8, grad, seed=shift, shift=shift)
    for t, max_norm in ((1, 0.0), (2, 0.5), (1000, 0.0)):
        before = ts.host()
        ts.step(t, max_norm)
        check8(ts, before, t, max_norm)


def test_8_bit_state_from_zeros_and_extremes():
    """First steps from empty state; gradients of zero, of one value, tiny and huge ones."""
    for scale in (0.0, 1e-30, 1e-20, 1e-3, 1e4, 1e15):
        ts = Tensors([700, 256, 3], 8, seed=1, scale=scale, zeros=True)
        if scale:
            ts.t[0]["grad"][300:] = 0.0
        for t in (1, 2, 3):
            before = ts.host()
            ts.step(t)
            check8(ts, before, t)
        for e in ts.host():
            assert bool(torch.isfinite(e["w"]).all())


def test_8_bit_moments_are_near_the_32_bit_ones():
    """The same gradients for 30 steps.  Rounding a moment to its code moves it by at most 1/127 (m) or
    1/255 (sqrt v) of its block's largest; what earlier steps moved shrinks by 0.9 or 0.95 a step, so
    the sums stay below a tenth of the largest, and the steps of lr within a fifth of lr."""
    n = 2048
    a, b = Tensors([n], 32, seed=3, zeros=True), Tensors([n], 8, seed=3, zeros=True)
    g = torch.Generator().manual_seed(9)
    for t in range(1, 31):
        grad = (torch.randn(n, generator=g) * 0.01).cuda()
        a.t[0]["grad"].copy_(grad)
        b.t[0]["grad"].copy_(grad)
        a.step(t)
        b.step(t)
    mv, vv = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    e = b.t[0]
    nb.numbat_adamw_state_values(n, e["m"], e["m_unit"], e["v"], e["v_unit"], mv, vv)
    close(mv, a.t[0]["m"].cpu().to(D), 0.1 * float(a.t[0]["m"].abs().max()), "m")
    close(vv.sqrt(), a.t[0]["v"].cpu().to(D).sqrt(), 0.1 * float(a.t[0]["v"].sqrt().max()), "sqrt v")
    close(e["w"], a.t[0]["w"].cpu().to(D), 0.2 * 30 * 1e-3, "w")


def test_state_values():
    for n in (1, 255, 256, 1000, 5000):
        ts = Tensors([n], 8, seed=n)
        e = ts.t[0]
        m, v = torch.full((n + 1,), 7.0, device="cuda"), torch.full((n + 1,), 7.0, device="cuda")
        nb.numbat_adamw_state_values(n, e["m"], e["m_unit"], e["v"], e["v_unit"], m, v)
        h = ts.host()[0]
        at = torch.arange(n) // BLOCK
        q, r = h["m"].float(), h["v"].float()
        r = h["v_unit"][at] * (r * r)
        assert torch.equal(m[:n].cpu(), h["m_unit"][at] * (q * q.abs())) and torch.equal(v[:n].cpu(), r * r)
        assert float(m[n]) == 7 and float(v[n]) == 7


def test_groups_empty_tensors_and_many():
    ts = Tensors([5, 0, 300, 0, 4096], 32, seed=2)
    ts.t[2]["group"] = 7  # outside the groups: left alone
    ts.table.copy_(torch.frombuffer(bytearray(nb.adamw_table(ts.t)), dtype=torch.uint8))
    before = ts.host()
    ts.step(1)
    after = ts.host()
    for k in ("w", "m", "v"):
        assert torch.equal(before[2][k], after[2][k])
        assert not torch.equal(before[4][k], after[4][k])
    ts = Tensors([1 + i % 700 for i in range(1024)], 32, seed=4)
    before = ts.host()
    ts.step(5, 0.3)
    check32(ts, before, 5, 0.3)


def test_a_gradient_that_is_not_finite_is_seen():
    for bits in (32, 8):
        ts = Tensors([600, 600], bits, seed=6)
        ts.t[0]["grad"][10] = float("nan")
        ts.step(1, 1.0)
        a, b = ts.host()
        assert bool(torch.isnan(a["w"][10])) and bool(torch.isfinite(a["w"][11:256]).all())
        assert bool(torch.isfinite(b["w"]).all()) and bool(torch.isnan(ts.norm).all())


def test_an_infinite_gradient_stays_in_its_element():
    """8-bit state: the unit of a block is that of its finite moments."""
    ts = Tensors([600], 8, seed=6)
    ts.t[0]["grad"][10] = float("inf")
    ts.step(1)
    ts.t[0]["grad"][10] = 0.01
    for t in (2, 3):
        before = ts.host()[0]["w"]
        ts.step(t)
        after = ts.host()[0]["w"]
        keep = torch.arange(600) != 10
        assert bool(torch.isfinite(after[keep]).all()) and float((after[keep] != before[keep]).float().mean()) > 0.9


def test_same_bits_on_a_stream_and_in_a_graph():
    for bits in (32, 8):
        one, two, three = (Tensors(SIZES, bits, seed=8) for _ in range(3))
        other = torch.cuda.Stream()
        other.wait_stream(torch.cuda.current_stream())
        three.step(4, 0.5)  # (first launches before the capture)
        three = Tensors(SIZES, bits, seed=8)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            three.step(4, 0.5)
        for _ in range(3):
            one.step(4, 0.5)
            two.step(4, 0.5, stream=other)
            g.replay()
            torch.cuda.synchronize()
            for a, b, c in zip(one.host(), two.host(), three.host()):
                for k in a:
                    if torch.is_tensor(a[k]):
                        assert torch.equal(a[k], b[k]) and torch.equal(a[k], c[k]), k
