"""iso_attend and iso_attend_grad against the binary64 oracle; the bounds are those of tests/attn_helpers.py."""
import numpy as np
import pytest

import paper_2607_19331_amd as iso
from paper_2607_19331_amd import _lib
from tests.attn_helpers import Case
from tests.grad_helpers import code
from tests.gpu_helpers import say

pytestmark = pytest.mark.gpu

SHAPES = [  # lens_q, lens_k, heads, kv, dim, causal, window, gap
    ([1], [1], 1, 1, 8, False, 0, 0),
    ([5, 0, 1, 37], [5, 0, 1, 37], 6, 2, 40, True, 0, 8),
    ([3, 10, 4], [0, 4, 0], 2, 2, 64, True, 0, 0),            # queries without keys: some, all
    ([0, 6], [9, 6], 4, 1, 64, True, 0, 0),                   # keys without queries
    ([65], [130], 4, 4, 64, False, 7, 0),
    ([129, 31], [129, 31], 7, 1, 128, True, 0, 16),
    ([1, 1, 1, 1], [300, 1, 77, 64], 8, 2, 128, True, 0, 0),  # one new token a sequence
    ([200], [200], 2, 1, 96, True, 33, 0),
    ([64, 128], [64, 128], 2, 2, 128, False, 0, 0),
    ([257], [120], 3, 3, 24, False, 0, 8),
    ([40], [40], 2, 1, 128, True, 1, 0),                      # every query sees itself alone
    ([17, 250], [333, 256], 14, 2, 128, True, 0, 0),
    ([1030], [1100], 1, 1, 64, True, 0, 0),
    ([2], [5000], 2, 1, 128, True, 0, 0),
    ([700], [9], 6, 1, 128, False, 0, 0)]                     # many queries, few keys


def run(case):
    ws = case.forward()
    assert iso.iso_read_device_status(ws) == 0
    case.check_forward()
    ws = case.backward()
    assert iso.iso_read_device_status(ws) == 0
    case.check_backward()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"q{sum(s[0])}k{sum(s[1])}h{s[2]}kv{s[3]}d{s[4]}c{int(s[5])}w{s[6]}")
def test_attend(dtype, shape):
    say(f"attend {dtype} {shape}")
    *rest, gap = shape
    run(Case(dtype, *rest, gap=gap))


def spoil(names, keep_rows):
    """Non-finite values in all rows from keep_rows of the one sequence on."""
    def edit(case):
        for name in names:
            x, at = case.host[name], (case.at_q if name in ("q", "dout") else case.at_k)
            for i, bad in zip(range(int(at[0]) + keep_rows, int(at[-1])), [np.nan, np.inf, -np.inf] * 1000):
                x[i, (i * 5) % x.shape[1]] = bad
    return edit


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("names", [("v",), ("k",), ("q",), ("dout",), ("q", "k", "v", "dout")], ids="-".join)
@pytest.mark.parametrize("length,keep", [(40, 33), (140, 70)])
def test_values_in_masked_places_reach_nothing(dtype, names, length, keep):
    """Rows `keep` ... of a causal sequence hold NaN and infinities: the rows before see none of them, and keys are reached by
    those of the rows that see them."""
    say(f"attend masked {dtype} {names} {length} {keep}")
    case = Case(dtype, [length], [length], 2, 1, 64, True, edit=spoil(names, keep))
    case.forward()
    out, lse = case.out.host(), case.lse.host()
    s = slice(int(case.at_q[0]), int(case.at_q[0]) + keep)
    assert np.isfinite(out[s]).all() and np.isfinite(lse[s]).all()
    if names == ("v",):
        case.check_forward()
    elif "k" in names or "q" in names:
        bad = ~np.isfinite(out[int(case.at_q[0]) + keep:int(case.at_q[-1])]).all(1)
        assert bad.any()
    good = Case(dtype, [length], [length], 2, 1, 64, True)
    good.forward()
    assert np.allclose(out[s], good.out.host()[s], rtol=2.0 ** -6, atol=2.0 ** -6)
    case.backward()
    got = case.dq.host()[s]
    assert np.isfinite(got).all()
    if names in (("v",), ("dout",)):
        case.check_backward()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_values_in_rows_of_other_sequences_reach_nothing(dtype):
    say(f"attend neighbours {dtype}")

    def edit(case):
        for name, at in (("q", case.at_q), ("dout", case.at_q), ("k", case.at_k), ("v", case.at_k)):
            case.host[name][at[1]:at[2]] = np.nan
    case = Case(dtype, [50, 30, 21], [50, 30, 21], 2, 2, 64, False, edit=edit)
    case.forward()
    out = case.out.host()
    case.backward()
    for m, at in ((case.out, case.at_q), (case.dq, case.at_q), (case.dk, case.at_k), (case.dv, case.at_k)):
        x = m.host()
        assert np.isnan(x[at[1]:at[2]]).all()
        assert np.isfinite(x[at[0]:at[1]]).all() and np.isfinite(x[at[2]:at[3]]).all()
    assert out.shape == case.host["q"].shape


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sigma,scale", [(30.0, 1.0), (1e-3, 1e-3)])
def test_wide_and_narrow_scores(dtype, sigma, scale):
    """Scores of thousands (one key takes a row) and of nothing (all keys alike)."""
    say(f"attend scores {dtype} {sigma}")

    def edit(case):
        for name in ("q", "k"):
            case.host[name] *= sigma
    run(Case(dtype, [90], [90], 2, 1, 64, True, edit=edit, scale=scale))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("bad", [[0, 40, 20, 90], [-3, 20, 40, 90], [0, 20, 40, 91]])
def test_offsets_that_are_no_ranges_are_reported(dtype, bad):
    """The sequences whose offsets are ranges are worked out, the others left out; nothing outside the rows is touched."""
    import torch
    say(f"attend offsets {dtype} {bad}")
    case = Case(dtype, [20, 20, 45], [20, 20, 45], 2, 1, 64, True, before=0)
    assert case.a.tokens_q == 90
    case.a.start_q = torch.tensor(bad, dtype=torch.int32, device="cuda")
    case.a.start_k = torch.tensor(bad, dtype=torch.int32, device="cuda")
    for call in (case.forward, case.backward):
        assert iso.iso_read_device_status(call()) == _lib.ERR_INDEX
    for m in (case.q, case.k, case.v, case.out, case.dq, case.dk, case.dv, case.lse):
        m.unchanged_guards()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_no_sequences_and_no_rows(dtype):
    import torch
    say(f"attend nothing {dtype}")
    start = torch.zeros(1, dtype=torch.int32, device="cuda")
    a = iso.Attn(q=None, k=None, v=None, start_q=start, start_k=start, sequences=0, tokens_q=0, tokens_k=0, heads=4, heads_kv=2,
                 dim=64, scale=1.0, out=None, lse=None)
    for grad, call in ((False, iso.iso_attend), (True, iso.iso_attend_grad)):
        ws = iso.attend_workspace(a, code(dtype), grad=grad)
        call(a, code(dtype), ws=ws)
        assert iso.iso_read_device_status(ws) == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens", [1, 300])
def test_rows_without_sequences_need_no_pointers(dtype, tokens):
    say(f"attend no sequences {dtype} {tokens}")
    a = iso.Attn(q=None, k=None, v=None, start_q=None, start_k=None, sequences=0, tokens_q=tokens, tokens_k=tokens, heads=4, heads_kv=2,
                 dim=64, scale=1.0, out=None, lse=None)
    for grad, call in ((False, iso.iso_attend), (True, iso.iso_attend_grad)):
        ws = iso.attend_workspace(a, code(dtype), grad=grad)
        call(a, code(dtype), ws=ws)
        assert iso.iso_read_device_status(ws) == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_captured_and_on_another_stream(dtype):
    """Forward and backward captured into one graph, replayed after new inputs and between eager calls on another stream."""
    import torch
    say(f"attend graph {dtype}")
    case = Case(dtype, [100, 30], [100, 30], 4, 2, 64, True)
    ws, ws2 = iso.attend_workspace(case.a, code(dtype)), iso.attend_workspace(case.a, code(dtype), grad=True)
    case.forward(ws), case.backward(ws2)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        case.forward(ws), case.backward(ws2)
    other = Case(dtype, [77], [80], 2, 1, 128, True, seed=3)
    side = torch.cuda.Stream()
    for _ in range(3):
        for m in (case.out, case.lse, case.dq, case.dk, case.dv):
            m.view.fill_(7.25)
        g.replay()
        side.wait_stream(torch.cuda.current_stream())
        w = other.forward(stream=side)
        w2 = other.backward(stream=side)
        torch.cuda.synchronize()
        assert iso.iso_read_device_status(ws) == 0 and iso.iso_read_device_status(ws2) == 0
        assert iso.iso_read_device_status(w) == 0 and iso.iso_read_device_status(w2) == 0
        case.check_forward(), case.check_backward()
        other.check_forward(), other.check_backward()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [([333, 90], [333, 90], 6, 2, 128, True), ([2], [3000], 4, 1, 64, True)])
def test_same_bits_every_time(dtype, shape):
    say(f"attend repeats {dtype} {shape}")
    case, first = Case(dtype, *shape), None
    for _ in range(3):
        case.forward(), case.backward()
        got = [m.host() for m in (case.out, case.lse, case.dq, case.dk, case.dv)]
        first = first or got
        assert all(np.array_equal(a, b) for a, b in zip(got, first))
