"""iso_attend and iso_attend_grad where some offsets are no ranges: the other sequences come out as if those were not there, whatever
the workspace holds.  A sequence is left out if its offsets are no range of the rows, or if it begins before the end of an earlier one
whose offsets are ranges (offsets that ascend have none of these).  The bounds are those of tests/attn_helpers.py."""
import numpy as np
import pytest

import paper_2607_19331_amd as iso
from paper_2607_19331_amd import _lib
from tests.attn_helpers import Case
from tests.grad_helpers import code
from tests.gpu_helpers import say

pytestmark = pytest.mark.gpu


def kept(start_q, start_k, tokens_q, tokens_k):
    """Row ranges (of q, of k) of the sequences that are worked out."""
    out, end_q, end_k = [], 0, 0
    for s in range(len(start_q) - 1):
        q, k = start_q[s:s + 2], start_k[s:s + 2]
        if not (0 <= q[0] <= q[1] <= tokens_q and 0 <= k[0] <= k[1] <= tokens_k):
            continue
        if q[0] >= end_q and k[0] >= end_k:
            out.append((slice(q[0], q[1]), slice(k[0], k[1])))
        end_q, end_k = max(end_q, q[1]), max(end_k, k[1])
    return out


class Offsets(Case):
    """Rows for the largest offsets that are in range, five more behind them."""

    def __init__(self, dtype, start_q, start_k, heads, kv, dim, causal, seed=0):
        import torch
        tokens = [max(x for x in s if x < 10 ** 6) for s in (start_q, start_k)]
        super().__init__(dtype, [tokens[0]], [tokens[1]], heads, kv, dim, causal, before=0, seed=seed)
        self.ranges = kept(start_q, start_k, self.a.tokens_q, self.a.tokens_k)
        dev = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
        self.a.start_q, self.a.start_k, self.a.sequences = dev(start_q), dev(start_k), len(start_q) - 1

    def parts(self):
        group = self.heads // self.kv
        for rows, keys in self.ranges:
            for h in range(self.heads):
                yield (rows, keys, slice(h * self.dim, (h + 1) * self.dim), slice(h // group * self.dim, (h // group + 1) * self.dim), h)

    def left_alone(self, names):
        """Rows of no sequence are as they were; zero from now on, as the oracle has them."""
        import torch
        for name in names:
            m, which = getattr(self, name), 1 if name in ("dk", "dv") else 0
            free = np.ones(m.rows, dtype=bool)
            for r in self.ranges:
                free[r[which]] = False
            x = m.host()
            assert (x[free] == 7.25).all(), f"{name}: rows of no sequence were written"
            last = (self.at_k if which else self.at_q)[-1]
            m.view[torch.as_tensor(np.flatnonzero(free[:last]), device="cuda")] = 0.0

    def space(self, grad):
        """A workspace of NaN."""
        return iso.attend_workspace(self.a, code(self.dtype), grad=grad).fill_(0xFF)


FAR = 10 ** 6
OFFSETS = [
    ([0, 10, FAR, 20, 30], [0, 10, FAR, 20, 30]),
    ([0, 10, -5, 20, 30], [0, 10, -5, 20, 30]),
    ([0, 20, 10, 30, 45], [0, 20, 10, 30, 45]),                  # the third begins inside the first
    ([0, 300, 0, 300, 340], [0, 300, 0, 300, 340]),              # the first again
    ([0, 5, 9, 14], [0, 40, 3, 50]),                             # of the keys alone
    ([0, 1, FAR, 3, 4, 5], [0, 3000, 3001, 3002, 6000, 9000]),   # few rows: keys in pieces
    ([0, 2000, 1500, 2001, 4000], [0, 3, 700, 4, 8]),            # few keys: rows in pieces
    ([0, 3, FAR] + list(range(9, 196, 3)) + [-1] + list(range(201, 211, 3)), list(range(0, 211, 3))[:70]),
    (list(range(66)) + [5] + list(range(67, 71)), [300 * i if i != 3 else FAR for i in range(71)]),
    ([0, FAR, 1, FAR, 2], [0, FAR, 1, FAR, 2])]                  # none


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("at", range(len(OFFSETS)))
def test_other_sequences_are_worked_out(dtype, at):
    start_q, start_k = OFFSETS[at]
    n = min(len(start_q), len(start_k))
    start_q, start_k = start_q[:n], start_k[:n]
    say(f"attend offsets {dtype} {at}")
    case = Offsets(dtype, start_q, start_k, 2, 1, 16, True)
    ws = case.forward(case.space(False))
    assert iso.iso_read_device_status(ws) == _lib.ERR_INDEX
    case.left_alone(("out", "lse"))
    case.check_forward()
    ws = case.backward(case.space(True))
    assert iso.iso_read_device_status(ws) == _lib.ERR_INDEX
    case.left_alone(("dq", "dk", "dv"))
    case.check_backward()
