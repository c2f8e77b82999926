"""A teacher's logits at the ends of binary32: only minus infinity is no entry.  The bounds are those of tests/test_gpu_distill.py."""
import numpy as np
import pytest

from oracle import gradients as gr

from tests.gpu_helpers import say
from tests.test_gpu_distill import Case

pytestmark = pytest.mark.gpu

LOWEST, LARGEST = float(np.finfo(np.float32).min), float(np.finfo(np.float32).max)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [400, 70001])           # a launch for rows that are held, and rows that are shared out
@pytest.mark.parametrize("temp", [1.0, 0.25, 3.0])
def test_lowest_and_largest_logits_are_entries(dtype, vocab, temp):
    say(f"distill lowest {dtype} {vocab} {temp}")

    def edit(c):
        c.w[:] = 1.0
        c.ids = np.arange(8 * 6).reshape(8, 6) * 7
        c.y[0] = LOWEST                                      # all alike
        c.ids[1, 1:], c.y[1, 0] = -1, LOWEST                 # the only one
        c.y[2, 1:] = LOWEST                                  # next to an ordinary one: no share
        c.y[3] = LARGEST
        c.y[4, 0], c.y[4, 1:] = LARGEST, LOWEST
        c.y[5] = -3e38
        c.y[6, :3], c.y[6, 3:] = -np.inf, LOWEST
        c.ids[7], c.y[7] = 11, LOWEST                        # one id all through
    case = Case(dtype, 8, vocab, 6, temp, 0, True, -1, edit=edit)
    # shares are of differences of the logits, and one of e^-60 or less is none: the oracle has them from 0 down
    case.y = np.where(case.y == -np.inf, case.y, np.maximum(case.y - case.y.max(1, keepdims=True), -200.0))
    case.want = gr.distill(case.z, case.ids, case.y, temp, case.w, -1)
    for what in ("loss", "grad", "both"):
        case.grad.view.fill_(7.25)
        case.call(what)
        assert case.status() == 0
        assert (case.loss.host() != 0).all()
        case.check(what)
