"""Rows whose logits are all large: a constant added to a row changes L by it, and neither its loss nor its gradient.

Bound.  A probability is exp of a difference that is formed from the logit as it is, a factor c = log2(e) / T (off by 2^-25) and L in
binary64; what rounding a row's reference takes, up to 2^6 in the exponent for logits of 10^9 T, counts with c's error: 2^-25 2^6.  With
the sum's own error that is E = 2^-24 (V / 256 + 64 + 32 + 6 |z / T - L|).  A loss adds t E, a share is off by 2^-24 (6 |y / T| + top + 16);
differences of z / T and L are exact to 2^-50 of their size in binary64.

Rows that are shared out, or longer than a workgroup's registers, have their gradient from the L that was written, as a call of
iso_distill_grad has: that L is binary32, off by up to 2^-24 |L|, which is in the exponent of every probability of the row and makes it
exp(2^-24 |L|) times as large or as small.  So long a row of one large number has no gradient to speak of, and is left out there."""
import numpy as np
import pytest

from oracle import gradients as gr

from tests.grad_helpers import close, unit
from tests.gpu_helpers import say
from tests.test_gpu_distill import E24, SLACK, Case

pytestmark = pytest.mark.gpu


def bounds(c, held):
    loss, lse, grad = c.want
    tl, tg = np.zeros(c.n), np.zeros(grad.shape)
    for r in range(c.n):
        live, t = gr.teacher_shares(c.ids[r], c.y[r], c.vocab, c.temp, c.pad)
        x = c.z[r] / c.temp
        e = E24 * (c.vocab / 256 + 96 + 6 * np.abs(x - lse[r])) + 2.0 ** -50 * np.abs(x[x > lse[r] - 1e3]).max()
        et = E24 * (6 * np.abs(c.y[r][live]).max() / c.temp + c.top + 16)
        tg[r] = c.temp * np.exp(x - lse[r]) * (e if held else (1 + e) * np.exp(E24 * abs(lse[r])) - 1)
        for i, s in zip(c.ids[r][live], t[live]):
            tg[r, i] += c.temp * s * et
            tl[r] += c.temp ** 2 * s * (et * (2 + abs(np.log(max(s, 1e-300)) - x[i] + lse[r])) + e[i])
    return SLACK * (tl + E24 * np.abs(loss)) + 2.0 ** -126, SLACK * (tg + (unit(c.dtype) + 4 * E24) * np.abs(grad)) + 2.0 ** -120


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab,n,held", [(300, 9, 2), (70001, 70, 2), (70001, 9, 0), (90001, 70, 1)])   # 1: in bf16
@pytest.mark.parametrize("temp", [1.0, 2.0])
def test_a_constant_added_to_a_row(dtype, vocab, n, held, temp):
    import torch
    held = held == 2 or (held == 1 and dtype == "bf16")
    say(f"distill large logits {dtype} {vocab} {temp}")
    shifts = [0.0, 7e4, -65504.0, 1e6, -3e6] + ([2e7, -1e8, 9e8, -1e9] if held else [3e5, -2e5, 4e4, -1e5])

    def edit(c):
        c.w[:] = 1.0
        c.z += np.array([shifts[r % 9] for r in range(n)])[:, None]
        if held:
            c.z[5::9], c.z[8::9] = 2e7, -1e9                  # all alike
    case = Case(dtype, n, vocab, 5, temp, 0, True, -1, edit=edit)
    case.ids[:, 0] = np.arange(n)                             # every list has an entry
    case.t[0][:, 0] = torch.arange(n)
    case.want = gr.distill(case.z, case.ids, case.y, temp, case.w, -1)
    case.call("both")
    assert case.status() == 0
    tl, tg = bounds(case, held)
    close(case.loss.host()[:, 0], case.want[0], tl)
    close(case.lse.host()[:, 0], case.want[1], case.bounds()[1])
    close(case.grad.host(), case.want[2], tg)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [300, 70001])
def test_rows_past_the_range_are_not_finite(dtype, vocab):
    """All logits a mask's lowest value: no number for the loss or a gradient that looks like one; none at weight 0."""
    say(f"distill past the range {dtype} {vocab}")
    lowest = -3.3895313892515355e38                           # of bf16

    def edit(c):
        c.w[:] = 1.0
        c.z[1], c.z[2], c.z[4], c.z[5] = lowest, -lowest, -1e30, 1e12
        c.z[3], c.w[3] = lowest, 0.0
        c.z[0, 20:], c.z[6, :30] = lowest, -1e30              # some of them: ordinary rows
    case = Case(dtype, 7, vocab, 4, 1.0, 0, True, None, edit=edit)
    case.ids[:], case.t[0][:] = 5, 5
    case.z[0, 5] = case.mat.host()[0, 5]
    case.want = gr.distill(case.z, case.ids, case.y, 1.0, case.w, None)
    for what in ("loss", "grad", "both"):
        case.grad.view.fill_(7.25)
        case.call(what)
        assert case.status() == 0
        loss, lse, grad = case.loss.host()[:, 0], case.lse.host()[:, 0], case.grad.host()
        far = [1, 2, 4, 5]
        assert not np.isfinite(loss[far]).any() and not np.isfinite(lse[far]).any() and loss[3] == 0
        assert np.isfinite(loss[[0, 6]]).all() and np.isfinite(lse[[0, 6]]).all()
        if what != "loss":
            assert not np.isfinite(grad[far]).any() and (grad[3] == 0).all() and np.isfinite(grad[[0, 6]]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,vocab,held", [(10, 5000, True), (70, 70001, True), (10, 70001, False), (70, 90001, False)])
def test_masked_columns_of_any_size(dtype, n, vocab, held):
    """A padded vocabulary: its last columns, and a range in the middle, hold a mask's value.  They have no part in a row, whatever it is."""
    say(f"distill masked columns {dtype} {n} {vocab}")
    fills = [-1e4, -65504.0, -1e9, -3e9, -1e10, -1e15, -1e30, -2.3e38, -3.3895313892515355e38, -np.inf]

    def edit(c):
        c.w[:] = 1.0
        c.ids = c.ids % 1000
        for r in range(n):
            c.z[r, vocab * 3 // 5:] = fills[r % 10]
            c.z[r, 1200:2400] = fills[(r + 3) % 10]
    case = Case(dtype, n, vocab, 5, 1.0, 0, True, None, edit=edit)
    for what in ("loss", "both", "grad"):
        case.grad.view.fill_(7.25)
        case.call(what)
        assert case.status() == 0
        with np.errstate(all="ignore"):
            tl, tg = bounds(case, held and what == "both")
        close(case.loss.host()[:, 0], case.want[0], tl)
        close(case.lse.host()[:, 0], case.want[1], SLACK * E24 * (vocab / 256 + 96 + 2 * np.abs(case.want[1])))
        if what != "loss":
            close(case.grad.host(), case.want[2], np.nan_to_num(tg))
