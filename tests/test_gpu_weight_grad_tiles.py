"""iso_ckpt_weight_grad by each side of its tiles and each way of sharing them out (tests/wgrad_tile_cases.py), against
products in binary64 on the device.

Tolerances as in test_gpu_weight_grad.py: products are exact, T of them (three parts each for an fp32 dy) added in
binary32 in any order by instructions that may cut are off by at most 3 T 2^-23 of the sum of their magnitudes, accumulating
adds one rounding, the output its own."""
import pytest

import paper_2607_19331_amd as iso
from tests.gpu_helpers import say
from tests.grad_helpers import GUARD, code, ttype, unit
from tests.wgrad_tile_cases import CASES

pytestmark = pytest.mark.gpu

FORMS = [("bf16", False), ("bf16", True), ("f32", False), ("f32", True)]


class Layer:
    """A layer with random checkpoint bytes, a dy whose gaps and surroundings are NaN, and a guarded gradient."""

    def __init__(self, gen, t, o, i, gap, dtype, gtype, add):
        import torch
        ld = iso.iso_ckpt_ld(i)
        self.t, self.o, self.i, self.ld, self.gtype, self.add = t, o, i, o + gap, gtype, add
        self.q = torch.randint(-127, 128, (t, ld), generator=gen, device="cuda", dtype=torch.int8)
        self.e = torch.randint(116, 125, (t, ld // 32), generator=gen, device="cuda", dtype=torch.uint8)
        self.buf = torch.full((t * self.ld + 64,), float("nan"), dtype=ttype(dtype), device="cuda")
        self.dy = self.buf[:t * self.ld].view(t, self.ld)[:, :o]
        self.dy.copy_(torch.randn(t, o, generator=gen, device="cuda"))
        self.start = (torch.randn(o, i, generator=gen, device="cuda") * 5).to(ttype(gtype))
        self.out = torch.empty(o * i + 64, dtype=ttype(gtype), device="cuda")
        self.grad = self.out[:o * i].view(o, i)
        self.reset()

    def reset(self):
        self.out.fill_(GUARD)
        self.grad.copy_(self.start) if self.add else self.grad.fill_(float("nan"))

    def job(self):
        return iso.WeightGrad(iso.Ckpt(self.t, self.i, self.q, self.e), dy=self.buf, ld_dy=self.ld, grad=self.grad, rows=self.o)

    def values(self):
        """X in binary64, NaN where a group's byte is 255."""
        import torch
        k = torch.where(self.e == 255, float("nan"), torch.exp2(self.e.double() - 127.0))
        return (self.q.double() * k.repeat_interleave(32, dim=1))[:, :self.i].contiguous()

    def check(self, what):
        import torch
        assert bool((self.out[self.o * self.i:] == GUARD).all()), what
        x, dy = self.values(), self.dy.double()
        ref = torch.mm(dy.t().contiguous(), x)
        mass = torch.mm(dy.abs().t().contiguous(), x.abs())
        if self.add:
            ref += self.start.double()
            mass += self.start.double().abs()
        got, fine = self.grad.double(), torch.isfinite(ref)
        assert torch.equal(torch.isnan(got), torch.isnan(ref)), what
        assert torch.equal(got[torch.isinf(ref)], ref[torch.isinf(ref)]), what
        tol = 3 * self.t * 2.0 ** -23 * mass + 2.0 ** -24 * (ref.abs() + mass) + unit(self.gtype) * ref.abs()
        off = ((got - ref).abs() - tol)[fine]
        assert float(off.max()) <= 0, (what, float(off.max()))


def make(name, gtype, add):
    import torch
    dtype, layers = CASES[name][0], CASES[name][4]
    gen = torch.Generator(device="cuda").manual_seed(sum(map(ord, name)))
    return dtype, [Layer(gen, *l, dtype, gtype, add) for l in layers]


def call(layers, dtype, gtype, add, ws=None, stream=None):
    jobs = [l.job() for l in layers]
    if ws is None:
        ws = iso.weight_grad_workspace(jobs, code(dtype))
        ws.fill_(0xFF)                                     # NaN patterns: nothing may be read before it is written
    iso.iso_ckpt_weight_grad(jobs, code(dtype), code(gtype), accumulate=add, ws=ws, stream=stream)
    return ws


@pytest.mark.parametrize("gtype,add", FORMS)
@pytest.mark.parametrize("name", CASES)
def test_values(name, gtype, add):
    import torch
    say(f"weight grad tiles {name} -> {gtype} add={add}")
    dtype, layers = make(name, gtype, add)
    ws = call(layers, dtype, gtype, add)
    assert iso.iso_read_device_status(ws) == 0
    for l in layers:
        l.check((l.t, l.o, l.i))
    first = [l.grad.clone() for l in layers]
    for l in layers:
        l.reset()
    call(layers, dtype, gtype, add, ws)
    assert all(torch.equal(a, l.grad) for a, l in zip(first, layers))    # the same bits again


@pytest.mark.parametrize("name", ["whole_256", "both_256", "split_256_odd", "both_256_f32", "split_256_f32"])
def test_special_values(name):
    """NaN groups of X and infinities and NaN of dY reach their columns and rows, in the first, a middle and the last tile."""
    say(f"weight grad tiles {name}: special values")
    dtype, (l,) = make(name, "f32", False)
    groups = l.e.shape[1]
    for n, (t, g) in enumerate(((0, 0), (l.t // 2, groups // 2), (l.t - 1, groups - 1))):
        l.e[t, g], l.q[t, 32 * g:32 * g + 32] = 255, 0
        l.dy[l.t - 1 - t, (0, l.o // 2 + 1, l.o - 1)[n]] = (float("inf"), float("nan"), float("-inf"))[n]
    call([l], dtype, "f32", False)
    l.check(name)


@pytest.mark.parametrize("name", ["both_256", "split_256_f32"])
def test_graph(name):
    """Captured on a stream of its own: every replay works on what is then in the buffers."""
    import torch
    say(f"weight grad tiles {name}: graph")
    dtype, layers = make(name, "f32", False)
    l = layers[0]
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    ws = call(layers, dtype, "f32", False, stream=s)
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        call(layers, dtype, "f32", False, ws, s)
    for k in range(3):
        l.dy.copy_(torch.randn(l.t, l.o, device="cuda") * 2.0 ** k)
        l.reset()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        l.check(f"replay {k}")
