"""8-bit activation checkpoints and the gated activation's gradients from them, against the binary64 oracle.

Packing is integer work on exact quotients: q and e equal the oracle's.  Unpacked values are exact.  The gate's
gradients: with A = |dh u| s (1 + |g| (1 - s)) (the magnitudes that the formula adds) fp32 is within
2^-20 A (the exponential, five products, two sums, a division: 16 roundings at most) + u |ref|, bf16 within 2^-16 A (the
hardware's exponential of -g: |g| 2^-23 for the product with log2 e, |g| <= 64 here) + u |ref|; dup likewise with
A = |dh g s|.  Results below 2^-120 may be flushed."""
import numpy as np
import pytest

from oracle import gradients as gr

import paper_2607_19331_amd as iso
from tests.grad_helpers import Mat, close, code, ttype, unit
from tests.gpu_helpers import say

pytestmark = pytest.mark.gpu


def buffers(rows, cols):
    """Checkpoint buffers within guarded allocations."""
    import torch
    ld = iso.iso_ckpt_ld(cols)
    q = torch.full((rows * ld + 64,), 85, dtype=torch.int8, device="cuda")
    e = torch.full((rows * ld // 32 + 64,), 85, dtype=torch.uint8, device="cuda")
    return q, e


def host(q, e, rows, cols):
    ld = iso.iso_ckpt_ld(cols)
    q, e = q.cpu().numpy(), e.cpu().numpy()
    assert (q[rows * ld:] == 85).all() and (e[rows * ld // 32:] == 85).all()
    return q[:rows * ld].reshape(rows, ld), e[:rows * ld // 32].reshape(rows, ld // 32)


def f64(a, dtype):
    import torch
    return torch.as_tensor(a).to(ttype(dtype)).double().numpy()


SHAPES = [(1, 1, 0), (1, 31, 0), (3, 32, 0), (2, 33, 1), (5, 64, 8), (7, 257, 3), (61, 1027, 1), (130, 96, 0), (4, 2048, 16),
          (2, 18944, 0)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_pack_and_unpack_a_table(dtype):
    """Every shape in one call: more tensors than one launch holds, aligned and unaligned strides, empty ones between."""
    rng = np.random.default_rng(21)
    say(f"ckpt table {dtype}: {SHAPES} twice and two empty tensors")
    jobs = []
    for rows, cols, gap in SHAPES + SHAPES:
        x = rng.standard_normal((rows, cols)) * np.exp(3 * rng.standard_normal((rows, cols)))
        x[rng.random((rows, cols)) < 0.1] = 0
        x = f64(x, dtype)
        m, b = Mat(rows, cols, dtype, gap, x), Mat(rows, cols, dtype, gap)
        jobs.append((rows, cols, x, m, b, *buffers(rows, cols)))
    empty = [iso.Ckpt(0, 16, None, None), iso.Ckpt(4, 0, None, None)]
    iso.iso_ckpt_pack(empty[:1] + [iso.Ckpt(r, c, q, e, x=m.view, ld_x=m.ld) for r, c, x, m, b, q, e in jobs] + empty[1:],
                      code(dtype))
    iso.iso_ckpt_unpack([iso.Ckpt(r, c, q, e, x=b.view, ld_x=b.ld) for r, c, x, m, b, q, e in jobs] + empty, code(dtype))
    for r, c, x, m, b, q, e in jobs:
        want_q, want_e = gr.ckpt_pack(x)
        got_q, got_e = host(q, e, r, c)
        assert np.array_equal(got_e, want_e), (r, c)
        assert np.array_equal(got_q, want_q), (r, c)
        assert np.array_equal(b.host(), gr.ckpt_values(want_q, want_e, c)), (r, c)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_pack_edges(dtype):
    """Ties, the boundary of an exponent, the smallest and largest finite values, zeros of both signs, NaN and infinities."""
    rng = np.random.default_rng(22)
    big = 3.3895313892515355e38 if dtype == "bf16" else float(np.finfo(np.float32).max)
    rows = [np.arange(-16, 16) + 0.5, np.r_[127.0, -126.5, np.arange(30) * 0.5], np.r_[128.0, np.arange(31) * 1.0],
            np.r_[big, -big / 2, np.ones(30)], np.full(32, 2.0 ** -133), np.r_[2.0 ** -126, np.full(31, 2.0 ** -127)],
            np.r_[-0.0, np.zeros(31)], np.r_[np.nan, np.ones(31)], np.r_[np.ones(31), -np.inf],
            np.r_[2.0 ** -119, 2.0 ** -126 * 1.5, np.full(30, 2.0 ** -126)], 127.0 * 2.0 ** rng.integers(-100, 100, 32)]
    if dtype == "f32":
        rows += [np.r_[np.nextafter(np.float32(127), np.float32(200)), np.ones(31)], np.full(32, 1e-45),
                 np.r_[np.nextafter(np.float32(127), np.float32(0)), np.ones(31)]]
    x = f64(np.array([np.r_[r, rng.permutation(r)[:7]] for r in rows], dtype=np.float64), dtype)
    m, (q, e) = Mat(*x.shape, dtype, 0, x), buffers(*x.shape)
    b = Mat(*x.shape, dtype)
    iso.iso_ckpt_pack([iso.Ckpt(*x.shape, q, e, x=m.view)], code(dtype))
    iso.iso_ckpt_unpack([iso.Ckpt(*x.shape, q, e, x=b.view)], code(dtype))
    want_q, want_e = gr.ckpt_pack(x)
    got_q, got_e = host(q, e, *x.shape)
    assert np.array_equal(got_e, want_e) and np.array_equal(got_q, want_q)
    close(b.host(), gr.ckpt_values(want_q, want_e, x.shape[1]), 0.0)


def gate_inputs(rng, rows, cols):
    g = gr.ckpt_pack(rng.standard_normal((rows, cols)) * np.where(rng.random(cols) < 0.1, 16, 2))
    u = gr.ckpt_pack(rng.standard_normal((rows, cols)) * 3)
    return g, u


def to_dev(q, e):
    import torch
    return torch.as_tensor(q, device="cuda"), torch.as_tensor(e, device="cuda")


def check_gate(dtype, g, u, dh, dgate, dup):
    cols = dh.shape[1]
    gv, uv = gr.ckpt_values(*g, cols), gr.ckpt_values(*u, cols)
    s = 1 / (1 + np.exp(-gv))
    want = gr.gate_grad(gv, uv, dh)
    mag = np.abs(dh * uv) * s * (1 + np.abs(gv) * (1 - s)), np.abs(dh * gv * s)
    share = 2.0 ** -16 if dtype == "bf16" else 2.0 ** -20
    for got, ref, a in zip((dgate, dup), want, mag):
        close(got, ref, share * a + unit(dtype) * np.abs(ref) + 2.0 ** -120)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gate_grad_table(dtype):
    rng = np.random.default_rng(23)
    say(f"gate grad table {dtype}: {SHAPES}")
    jobs = []
    for rows, cols, gap in SHAPES + SHAPES[:7]:
        g, u = gate_inputs(rng, rows, cols)
        dh = f64(rng.standard_normal((rows, cols)), dtype)
        jobs.append((rows, cols, g, u, dh, Mat(rows, cols, dtype, gap, dh), Mat(rows, cols, dtype, gap),
                     Mat(rows, cols, dtype, gap), to_dev(*g), to_dev(*u)))
    iso.iso_ckpt_gate_grad([iso.GateGrad(iso.Ckpt(r, c, *gd), iso.Ckpt(r, c, *ud), dh=m.view, dgate=a.view, dup=b.view,
                                         ld=m.ld) for r, c, g, u, dh, m, a, b, gd, ud in jobs], code(dtype))
    for r, c, g, u, dh, m, a, b, gd, ud in jobs:
        check_gate(dtype, g, u, dh, a.host(), b.host())
        assert np.array_equal(m.host(), dh)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gate_grad_over_its_input_and_extremes(dtype):
    """dgate written over dh; gates far into both tails; a NaN group gives NaN in its 32 columns and nowhere else."""
    rng = np.random.default_rng(24)
    rows, cols = 6, 160
    gate = rng.standard_normal((rows, cols))
    gate[0], gate[1], gate[2] = 60.0, -60.0, 0.0
    gate[3, 32:64] = -1e30
    gate[3, 64:96] = 1e30
    g, u = gr.ckpt_pack(gate), gr.ckpt_pack(rng.standard_normal((rows, cols)))
    g[1][4, 1], g[0][4, 32:64] = 255, 0
    dh = f64(rng.standard_normal((rows, cols)), dtype)
    m, b = Mat(rows, cols, dtype, 0, dh), Mat(rows, cols, dtype)
    iso.iso_ckpt_gate_grad([iso.GateGrad(iso.Ckpt(rows, cols, *to_dev(*g)), iso.Ckpt(rows, cols, *to_dev(*u)), dh=m.view,
                                         dgate=m.view, dup=b.view)], code(dtype))
    got = m.host(), b.host()
    nan = np.zeros((rows, cols), bool)
    nan[4, 32:64] = True
    for x in got:
        assert np.array_equal(np.isnan(x), nan)
    with np.errstate(over="ignore", invalid="ignore"):
        uv = gr.ckpt_values(*u, cols)
        assert not got[0][3, 32:64].any() and not got[1][3, 32:64].any()       # silu and its slope are zero far left
        assert np.array_equal(got[0][3, 64:96], f64(dh[3, 64:96] * uv[3, 64:96], "f32") if dtype == "f32" else
                              f64(f64(dh[3, 64:96] * uv[3, 64:96], "f32"), "bf16"))
    keep = [0, 1, 2, 5]
    check_gate(dtype, (g[0][keep], g[1][keep]), (u[0][keep], u[1][keep]), dh[keep], got[0][keep], got[1][keep])


def test_stream_and_graph():
    """Captured: every replay packs, unpacks and differentiates what is then in the buffers."""
    import torch
    rng = np.random.default_rng(25)
    rows, cols = 40, 200
    x, b = Mat(rows, cols, "bf16", 0, rng.standard_normal((rows, cols))), Mat(rows, cols, "bf16")
    da, du = Mat(rows, cols, "bf16"), Mat(rows, cols, "bf16")
    q, e = buffers(rows, cols)
    c = iso.Ckpt(rows, cols, q, e, x=x.view)
    back = iso.Ckpt(rows, cols, q, e, x=b.view)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()

    def all_three(stream):
        iso.iso_ckpt_pack([c], iso.BF16, stream=stream)
        iso.iso_ckpt_unpack([back], iso.BF16, stream=stream)
        iso.iso_ckpt_gate_grad([iso.GateGrad(c, c, dh=x.view, dgate=da.view, dup=du.view)], iso.BF16, stream=stream)

    all_three(s)
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        all_three(s)
    for k in range(4):
        x.view.copy_(torch.as_tensor(rng.standard_normal((rows, cols)) * 10.0 ** k))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = b.host(), da.host(), du.host()
        want_q, want_e = gr.ckpt_pack(x.host())
        assert np.array_equal(got[0], gr.ckpt_values(want_q, want_e, cols))
        all_three(None)
        torch.cuda.synchronize()
        for old, new in zip(got, (b, da, du)):
            assert np.array_equal(old, new.host())
