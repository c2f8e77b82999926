"""dK and dV of keys next to rows (and dQ of rows next to keys) that hold NaN and infinities and that they do not see: the same tiles and
panels, worked out row by row.  The bounds are those of tests/attn_helpers.py."""
import numpy as np
import pytest

from tests.attn_helpers import Case
from tests.gpu_helpers import say

pytestmark = pytest.mark.gpu


def spoilt(names, rows):
    def edit(case):
        for name in names:
            x, at = case.host[name], (case.at_q if name in ("q", "dout") else case.at_k)
            for i in rows:
                x[int(at[0]) + i, (5 * i) % x.shape[1]] = np.nan if name in ("q", "k") else [np.nan, np.inf, -np.inf][i % 3]
    return edit


# rows, window, causal, length: 1500 rows take pieces, 140 do not
PLACES = [(range(9), 0, True, 140), (range(9), 0, True, 1500), (range(60, 64), 20, False, 140), (range(700, 704), 40, False, 1500),
          ([0, 139], 20, True, 140)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("names", [("q",), ("dout",), ("q", "dout")], ids="-".join)
@pytest.mark.parametrize("rows,window,causal,length", PLACES)
def test_rows_that_a_key_does_not_see_do_not_reach_it(dtype, names, rows, window, causal, length):
    say(f"attend unseen rows {dtype} {names} {rows} {window} {length}")
    case = Case(dtype, [length], [length], 2, 1, 64, causal, window, edit=spoilt(names, rows))
    case.forward(), case.backward()
    case.check_backward()
    at = int(case.at_k[0])
    see = case.seen(length, length)[list(rows)].any(0)
    assert see.any() and not see.all()
    for m in (case.dk, case.dv):
        assert np.isfinite(m.host()[at:at + length][~see]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("names", [("k",), ("v",), ("k", "v")], ids="-".join)
@pytest.mark.parametrize("keys,window,causal,length", PLACES)
def test_keys_that_a_row_does_not_see_do_not_reach_it(dtype, names, keys, window, causal, length):
    say(f"attend unseen keys {dtype} {names} {keys} {window} {length}")
    keys = [length - 1 - i for i in keys]   # the last ones, which early rows do not see
    case = Case(dtype, [length], [length], 2, 1, 64, causal, window, edit=spoilt(names, keys))
    case.forward()
    case.check_forward()
    case.backward()
    at = int(case.at_q[0])
    see = case.seen(length, length)[:, keys].any(1)
    assert see.any() and not see.all()
    got = case.dq.host()[at:at + length]
    assert np.isfinite(got[~see]).all()
    clean = Case(dtype, [length], [length], 2, 1, 64, causal, window)
    clean.forward(), clean.backward()
    assert np.allclose(got[~see], clean.dq.host()[at:at + length][~see], rtol=2.0 ** -6, atol=2.0 ** -9)


def test_a_step_that_has_gone_to_nan_ends():
    """All of q, k, v and dout NaN: all results are, and a call takes a few times as long as it does otherwise (row by row over all keys it
    would be two hundred times; 40 is far from both)."""
    import torch

    import paper_2607_19331_amd as iso
    say("attend all NaN")
    tokens, heads, kv, dim = 4096, 28, 4, 128
    new = lambda *s: torch.randn(*s, device="cuda").to(torch.bfloat16)  # noqa: E731
    start = torch.tensor([0, tokens], dtype=torch.int32, device="cuda")
    x = {n: new(tokens, (heads if n in ("q", "out", "dout", "dq") else kv) * dim) for n in ("q", "k", "v", "out", "dout", "dq", "dk", "dv")}
    a = iso.Attn(start_q=start, start_k=start, sequences=1, tokens_q=tokens, tokens_k=tokens, heads=heads, heads_kv=kv, dim=dim, scale=dim ** -0.5,
                 lse=torch.zeros(tokens, heads, device="cuda"), causal=True, **x)
    ws = [iso.attend_workspace(a, iso.BF16, grad=g) for g in (False, True)]

    def took():
        best = []
        for call, w in zip((iso.iso_attend, iso.iso_attend_grad), ws):
            times = []
            for _ in range(4):
                b, e = (torch.cuda.Event(enable_timing=True) for _ in range(2))
                b.record(), call(a, iso.BF16, ws=w), e.record()
                torch.cuda.synchronize()
                times.append(b.elapsed_time(e))
            best.append(min(times))
        return best
    usual = took()
    for n in ("q", "k", "v", "dout"):
        x[n].fill_(float("nan"))
    bad = took()
    say(f"ms {usual} {bad}")
    for n in ("out", "dq", "dk", "dv"):
        assert bool(x[n].isnan().all())
    assert bool(a.lse.isnan().all())
    assert bad[0] < 40 * usual[0] and bad[1] < 40 * usual[1]
