"""iso_ckpt_weight_grad against the binary64 oracle.

Products are exact in binary32 or split into exact parts, so the error is that of the sum: T products (three parts
each for an fp32 dy) added in binary32 in any order, by instructions that may cut instead of round, are off by at most
3 T 2^-23 of the sum of their magnitudes; accumulating adds one more rounding, the output its own."""
import numpy as np
import pytest

from oracle import gradients as gr

import paper_2607_19331_amd as iso
from tests.grad_helpers import Mat, close, code, ttype, unit
from tests.gpu_helpers import say

pytestmark = pytest.mark.gpu


def f64(a, dtype):
    import torch
    return torch.as_tensor(a).to(ttype(dtype)).double().numpy()


def to_dev(q, e):
    import torch
    return torch.as_tensor(q, device="cuda"), torch.as_tensor(e, device="cuda")


def pack(x):
    """The oracle's checkpoint, vectorised (the loop's result: tests/test_oracle_gradients.py pins it on small matrices)."""
    rows, cols = x.shape
    ld = -(-cols // 32) * 32
    v = np.zeros((rows, ld))
    v[:, :cols] = x
    v = v.reshape(rows, ld // 32, 32)
    top = np.abs(v).max(-1)
    k = np.full(top.shape, -126.0)
    mant, ex = np.frexp(top)
    k = np.where(top > 0, np.maximum(np.where(mant <= 127 / 128, ex - 7, ex - 6), -126), k)
    q = np.rint(v / 2.0 ** k[..., None]).astype(np.int8).reshape(rows, ld)
    return q, (k + 127).astype(np.uint8)


def activations(rng, t, n):
    return pack(rng.standard_normal((t, n)) * np.exp(rng.standard_normal(n)))


class Layer:
    def __init__(self, rng, t, o, i, dtype, gtype, gap, add, kept=None):
        self.t, self.o, self.i, self.gtype = t, o, i, gtype
        self.kept = kept or activations(rng, t, i)
        self.dev = to_dev(*self.kept) if kept is None else None
        self.dy = f64(rng.standard_normal((t, o)), dtype)
        self.m = Mat(t, o, dtype, gap, self.dy)
        self.start = f64(rng.standard_normal((o, i)) * 5, gtype) if add else None
        self.g = Mat(o, i, gtype, 0, self.start)

    def job(self, dev=None):
        return iso.WeightGrad(iso.Ckpt(self.t, self.i, *(dev or self.dev)), dy=self.m.view, ld_dy=self.m.ld, grad=self.g.view,
                              rows=self.o)

    def check(self):
        x = gr.ckpt_values(*self.kept, self.i)
        ref = gr.weight_grad(self.dy, x, self.start)
        mass = gr.weight_grad(np.abs(self.dy), np.abs(x))
        close(self.g.host(), ref, 3 * self.t * 2.0 ** -23 * mass + 2.0 ** -24 * (np.abs(ref) + mass) + unit(self.gtype) * np.abs(ref))


def run(layers, dtype, gtype, add, devs=None):
    jobs = [l.job(d) for l, d in zip(layers, devs or [None] * len(layers))]
    ws = iso.weight_grad_workspace(jobs, code(dtype))
    ws.fill_(0xFF)                                     # NaN patterns: nothing may be read before it is written
    iso.iso_ckpt_weight_grad(jobs, code(dtype), code(gtype), accumulate=add, ws=ws)
    assert iso.iso_read_device_status(ws) == 0


CASES = [(1, 1, 1, 0), (1, 64, 64, 0), (2, 130, 33, 0), (31, 17, 257, 3), (32, 64, 96, 0), (33, 256, 256, 8),
         (64, 300, 40, 0), (65, 128, 130, 1), (200, 517, 259, 3), (257, 96, 640, 0), (640, 256, 512, 0), (1000, 72, 72, 0),
         (3000, 8, 8, 0), (700, 1030, 300, 2)]


@pytest.mark.parametrize("dtype,gtype,add", [("bf16", "f32", False), ("bf16", "bf16", True), ("f32", "f32", True),
                                             ("f32", "bf16", False), ("bf16", "f32", True)])
@pytest.mark.parametrize("t,o,i,gap", CASES)
def test_one_layer(dtype, gtype, add, t, o, i, gap):
    say(f"weight grad {dtype}->{gtype} add={add} tokens={t} rows={o} cols={i} gap={gap}")
    layer = Layer(np.random.default_rng(t * 13 + o + i), t, o, i, dtype, gtype, gap, add)
    run([layer], dtype, gtype, add)
    layer.check()
    first = layer.g.host()
    layer.g = Mat(o, i, gtype, 0, layer.start)
    run([layer], dtype, gtype, add)
    assert np.array_equal(layer.g.host(), first)       # the same bits again


@pytest.mark.parametrize("dtype,gtype,add", [("bf16", "bf16", False), ("f32", "f32", True)])
def test_table(dtype, gtype, add):
    """More layers than one launch holds, of many sizes and strides, some sharing their checkpoint, some empty."""
    rng = np.random.default_rng(40)
    say(f"weight grad table {dtype}->{gtype} add={add}")
    layers, devs = [], []
    for n in range(6):
        t, i = int(rng.integers(1, 400)), int(rng.integers(1, 300))
        kept = activations(rng, t, i)
        dev = to_dev(*kept)
        for _ in range(3):
            layers.append(Layer(rng, t, int(rng.integers(1, 300)), i, dtype, gtype, int(rng.integers(0, 9)), add, kept))
            devs.append(dev)
    order = rng.permutation(len(layers))
    layers, devs = [layers[k] for k in order], [devs[k] for k in order]
    run(layers, dtype, gtype, add, devs)
    for l in layers:
        l.check()


@pytest.mark.parametrize("add", [False, True])
def test_no_tokens_and_empty_matrices(add):
    g = Mat(5, 40, "f32", 0, np.ones((5, 40)))
    jobs = [iso.WeightGrad(iso.Ckpt(0, 40, None, None), dy=None, grad=g.view, rows=5),
            iso.WeightGrad(iso.Ckpt(3, 0, None, None), dy=None, grad=None, rows=5, ld_dy=5),
            iso.WeightGrad(iso.Ckpt(3, 8, None, None), dy=None, grad=None, rows=0)]
    ws = iso.weight_grad_workspace(jobs, iso.BF16)
    iso.iso_ckpt_weight_grad(jobs, iso.BF16, iso.F32, accumulate=add, ws=ws)
    assert iso.iso_read_device_status(ws) == 0
    assert (g.host() == (1.0 if add else 0.0)).all()
    iso.iso_ckpt_weight_grad([], iso.BF16, iso.F32, accumulate=add, ws=ws)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_special_values(dtype):
    """A NaN group of x reaches its 32 columns of G, a NaN or infinity of dy its row, and nothing else changes: the values
    beyond a matrix's edges and past the last token, whatever they are, take no part."""
    rng = np.random.default_rng(41)
    t, o, i = 45, 70, 100
    l = Layer(rng, t, o, i, dtype, "f32", 2, False)
    l.m.buf.fill_(float("nan"))                        # between the rows and behind the last
    l.m.view.copy_(__import__("torch").as_tensor(l.dy))
    q, e = l.kept
    q, e = q.copy(), e.copy()
    e[7, 1], q[7, 32:64] = 255, 0
    l.m.view[9, 3] = float("inf")
    l.m.view[44, 69] = float("nan")
    run([l], dtype, "f32", False, [to_dev(q, e)])
    got = l.g.buf[:o * i].view(o, i).double().cpu().numpy()
    x = gr.ckpt_values(q, e, i)
    dy = l.dy.copy()
    dy[9, 3], dy[44, 69] = np.inf, np.nan
    assert np.isnan(got[:, 32:64]).all() and np.isnan(got[69]).all()
    rest = np.ones((o, i), bool)
    rest[:, 32:64], rest[69], rest[3] = False, False, False
    x0 = np.nan_to_num(x)
    ref = l.dy.T @ x0
    assert np.isfinite(got[rest]).all()
    assert np.abs(got - ref)[rest].max() <= 1e-3
    cols = np.r_[0:32, 64:100]
    live = x[9, cols] != 0
    assert np.array_equal(got[3, cols][live], np.sign(x[9, cols][live]) * np.inf)
    assert np.isnan(got[3, cols][~live]).all()


def test_split_of_a_binary32_gradient():
    """An fp32 dy keeps all its bits: with one token G = dy x exactly rounded, also near the largest value and far below one."""
    rng = np.random.default_rng(42)
    o, i = 96, 64
    l = Layer(rng, 1, o, i, "f32", "f32", 0, False)
    dy = (rng.standard_normal(o) * 2.0 ** rng.integers(-60, 60, o)).astype(np.float32)
    dy[:4] = [3.4e38, -3.4028235e38, 1.0 + 2.0 ** -23, -(2.0 - 2.0 ** -23)]
    x = np.ones((1, i))
    x[0, 32:] = 0.5
    q, e = gr.ckpt_pack(x)
    l.m.view.copy_(__import__("torch").as_tensor(dy[None]))
    run([l], "f32", "f32", False, [to_dev(q, e)])
    assert np.array_equal(l.g.host(), dy[:, None].astype(np.float64) * x)


def test_gradient_by_differences():
    """Central differences of L(W) = sum((X W^T) * dY) with few-bit values, for which both sides are exact."""
    rng = np.random.default_rng(43)
    t, o, i = 50, 9, 12
    x = rng.integers(-127, 128, (t, i)) / 64.0
    x[:, 0] = 127 / 64.0                               # one exponent for every group: x is kept exactly
    q, e = gr.ckpt_pack(x)
    assert np.array_equal(gr.ckpt_values(q, e, i), x)
    l = Layer(rng, t, o, i, "f32", "f32", 0, False)
    dy = rng.integers(-8, 9, (t, o)) / 8.0
    l.m.view.copy_(__import__("torch").as_tensor(dy))
    run([l], "f32", "f32", False, [to_dev(q, e)])
    got, w = l.g.host(), rng.integers(-4, 5, (o, i)) / 4.0
    for r in range(o):
        for c in range(i):
            step = np.zeros((o, i))
            step[r, c] = 0.5
            hi, lo = (float(((x @ (w + s * step).T) * dy).sum()) for s in (1, -1))
            assert hi - lo == got[r, c]


def test_stream_and_graph():
    import torch
    rng = np.random.default_rng(44)
    ls = [Layer(rng, 150, 200, 96, "bf16", "f32", 0, False), Layer(rng, 150, 40, 330, "bf16", "f32", 0, False)]
    jobs = [l.job() for l in ls]
    ws = iso.weight_grad_workspace(jobs, iso.BF16)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    call = lambda stream: iso.iso_ckpt_weight_grad(jobs, iso.BF16, iso.F32, ws=ws, stream=stream)  # noqa: E731
    call(s)
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        call(s)
    for k in range(4):
        for l in ls:
            l.dy = f64(rng.standard_normal((150, l.o)), "bf16")
            l.m.view.copy_(torch.as_tensor(l.dy))
            l.g.view.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for l in ls:
            l.check()
