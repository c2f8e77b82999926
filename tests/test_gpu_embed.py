"""iso_embed_lookup and iso_embed_grad against the binary64 oracle.

Tolerances.  Lookup: the scale and the product are rounded to binary32 and the result to its type, so
|err| <= (2^-23 + u) |x| (u = 2^-8 bf16, 2^-24 fp32).  Gradient: m terms added in binary32 are off by at most
(m - 1) 2^-24 of the sum of their magnitudes, then scale, product and (accumulate) one more addition by 2^-24 each, and
u of the result; 1 + 2^-6 covers the products of these bounds."""
import numpy as np
import pytest

from oracle import gradients as gr

import paper_2607_19331_amd as iso
from paper_2607_19331_amd import _lib
from tests.grad_helpers import Mat, close, code, ttype, unit
from tests.gpu_helpers import say

pytestmark = pytest.mark.gpu

SLACK = 1 + 2.0 ** -6


def tokens(rng, n, vocab, pad_id, kind="mixed"):
    if kind == "one":
        ids = np.full(n, vocab // 2)
    elif kind == "zipf":
        ids = np.minimum((vocab + 1) ** rng.random(n) - 1, vocab - 1).astype(np.int64)
    else:
        ids = rng.integers(0, vocab, n)
    if pad_id is not None:
        ids[rng.random(n) < 0.2] = pad_id
    return ids.astype(np.int64)


def dev_ids(ids, wide):
    import torch
    return torch.as_tensor(ids, dtype=torch.int64 if wide else torch.int32, device="cuda")


def f64(a, dtype):
    import torch
    return torch.as_tensor(a).to(ttype(dtype)).double().numpy()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,vocab,dim,gap,wide,pad", [
    (1, 1, 1, 0, True, None), (1, 50, 64, 0, True, None), (3, 7, 5, 2, False, 6), (257, 100, 24, 8, True, -100),
    (40, 33, 1000, 0, False, None), (1030, 61, 136, 0, True, 60), (5, 11, 4099, 1, True, None)])
def test_lookup(dtype, n, vocab, dim, gap, wide, pad):
    rng = np.random.default_rng(n * 31 + dim)
    say(f"lookup {dtype} n={n} vocab={vocab} dim={dim} gap={gap} i{64 if wide else 32} pad={pad}")
    table = f64(rng.standard_normal((vocab, dim)), dtype)
    ids = tokens(rng, n, vocab, pad)
    w, x, t = Mat(vocab, dim, dtype, 0, table), Mat(n, dim, dtype, gap), dev_ids(ids, wide)
    e = iso.Embed(ids=t, tokens=n, vocab=vocab, dim=dim, x=x.view, ld_x=x.ld, table=w.view, scale=1.7, pad_id=pad)
    ws = iso.embed_workspace(e)
    iso.iso_embed_lookup(e, code(dtype), ws=ws)
    assert iso.iso_read_device_status(ws) == 0
    ref = gr.embed_lookup(table, ids, 1.7, pad)
    close(x.host(), ref, (2.0 ** -23 + unit(dtype)) * SLACK * np.abs(ref))


def test_lookup_special_values_and_bad_ids():
    """Infinities and NaN of a row come through, a padded row is zero whatever the table holds, an id outside the vocabulary
    gives zeros and a status, and the next call clears the status."""
    table = np.ones((4, 16))
    table[1], table[2, 3], table[3] = np.inf, np.nan, 1e30
    for wide in (True, False):
        ids = np.array([1, 2, 3, 0, 4, -1, 2])
        w, x = Mat(4, 16, "f32", 0, table), Mat(7, 16, "f32", 0)
        e = iso.Embed(ids=dev_ids(ids, wide), tokens=7, vocab=4, dim=16, x=x.view, table=w.view, scale=1e10, pad_id=3)
        ws = iso.embed_workspace(e)
        iso.iso_embed_lookup(e, iso.F32, ws=ws)
        assert iso.iso_read_device_status(ws) == _lib.ERR_INDEX
        got = x.host()
        assert np.isinf(got[0]).all() and np.isnan(got[1, 3]) and np.isfinite(got[1, :3]).all()
        assert not got[2].any() and not got[4].any() and not got[5].any()
        e.ids = dev_ids(np.array([0, 1, 2, 3, 0, 1, 2]), wide)
        iso.iso_embed_lookup(e, iso.F32, ws=ws)
        assert iso.iso_read_device_status(ws) == 0


GRAD = [  # n, vocab, dim, gap, wide, pad, kind
    (0, 5, 8, 0, True, None, "mixed"), (1, 1, 1, 0, True, None, "mixed"), (1, 300, 40, 0, False, None, "mixed"),
    (2, 3, 7, 3, True, 1, "mixed"), (33, 1, 16, 0, True, None, "one"), (64, 9, 24, 8, True, None, "one"),
    (65, 40, 2056, 0, False, 39, "zipf"), (311, 1031, 259, 5, False, 1020, "zipf"), (1500, 700, 48, 0, True, -100, "zipf"),
    (1025, 513, 64, 0, True, None, "one"), (3000, 5000, 96, 0, False, 17, "zipf"), (2500, 4, 12, 0, True, None, "mixed"),
    (66000, 1200, 8, 0, True, 3, "zipf")]


@pytest.mark.parametrize("n,vocab,dim,gap,wide,pad,kind", GRAD)
@pytest.mark.parametrize("dtype,gtype,add", [("f32", "f32", False), ("bf16", "bf16", False), ("bf16", "f32", True),
                                             ("f32", "bf16", True)])
def test_grad(dtype, gtype, add, n, vocab, dim, gap, wide, pad, kind):
    rng = np.random.default_rng(n * 7 + dim)
    say(f"embed grad {dtype}->{gtype} add={add} n={n} vocab={vocab} dim={dim} gap={gap} pad={pad} {kind}")
    ids = tokens(rng, n, vocab, pad, kind)
    dx = f64(rng.standard_normal((n, dim)), dtype)
    start = f64(rng.standard_normal((vocab, dim)) * 3, gtype) if add else None
    seen = dx.copy()
    if pad is not None:
        seen[ids == pad] = np.nan                       # padding's gradients are not looked at
    x, g, t = Mat(n, dim, dtype, gap, seen), Mat(vocab, dim, gtype, 0, start), dev_ids(ids, wide)
    e = iso.Embed(ids=t, tokens=n, vocab=vocab, dim=dim, x=x.view if n else None, ld_x=x.ld, grad=g.view, scale=0.37,
                  pad_id=pad)
    ws = iso.embed_workspace(e)
    ws.fill_(0xA5)
    iso.iso_embed_grad(e, code(dtype), code(gtype), accumulate=add, ws=ws)
    assert iso.iso_read_device_status(ws) == 0
    got = g.host()
    ref = gr.embed_grad(dx, ids, vocab, 0.37, pad, start)
    mass = gr.embed_grad(np.abs(dx), ids, vocab, 0.37, pad)
    m = np.bincount(ids[(ids >= 0) & (ids < vocab)], minlength=vocab)[:, None]
    close(got, ref, SLACK * ((m + 2) * 2.0 ** -24 * mass + (2.0 ** -24 + unit(gtype)) * np.abs(ref)))
    if add:
        untouched = ~np.isin(np.arange(vocab), ids[ids != (pad if pad is not None else -1)])
        assert np.array_equal(got[untouched], start[untouched])
    # the same call gives the same bits
    again = Mat(vocab, dim, gtype, 0, start)
    e.grad = again.view
    iso.iso_embed_grad(e, code(dtype), code(gtype), accumulate=add, ws=ws)
    assert np.array_equal(again.host(), got)


def test_grad_bad_ids_and_nonfinite_rows():
    """Ids outside the vocabulary add nothing and are reported; NaN and infinities of a row reach that id's gradient only."""
    n, vocab, dim = 200, 50, 32
    rng = np.random.default_rng(5)
    ids = rng.integers(0, vocab, n)
    ids[[3, 90]] = [vocab, -7]
    dx = f64(rng.standard_normal((n, dim)), "f32")
    dx[3] = np.nan
    dx[10], dx[11, 5] = np.inf, np.nan
    ids[10], ids[11] = 4, 5
    for wide in (True, False):
        x, g = Mat(n, dim, "f32", 0, dx), Mat(vocab, dim, "f32")
        e = iso.Embed(ids=dev_ids(ids, wide), tokens=n, vocab=vocab, dim=dim, x=x.view, grad=g.view)
        ws = iso.embed_workspace(e)
        iso.iso_embed_grad(e, iso.F32, iso.F32, ws=ws)
        assert iso.iso_read_device_status(ws) == _lib.ERR_INDEX
        got = g.host()
        assert np.isposinf(got[4]).all() and np.isnan(got[5, 5])
        rest = np.ones((vocab, dim), bool)
        rest[4], rest[5, 5] = False, False
        assert np.isfinite(got[rest]).all()


def test_grad_by_differences():
    """The gradient against central differences of L(W) = sum(lookup(W) * dX) through the library's own lookup; values with
    few bits make every product and sum exact, so the two agree exactly."""
    rng = np.random.default_rng(6)
    n, vocab, dim = 37, 11, 6
    ids = tokens(rng, n, vocab, 10)
    w = rng.integers(-8, 9, (vocab, dim)) / 8.0
    dx = rng.integers(-8, 9, (n, dim)) / 8.0
    t, x, xd = dev_ids(ids, True), Mat(n, dim, "f32"), Mat(n, dim, "f32", 0, dx)
    g = Mat(vocab, dim, "f32")
    e = iso.Embed(ids=t, tokens=n, vocab=vocab, dim=dim, x=xd.view, grad=g.view, scale=0.5, pad_id=10)
    ws = iso.embed_workspace(e)
    iso.iso_embed_grad(e, iso.F32, iso.F32, ws=ws)
    got = g.host()

    def loss(table):
        m = Mat(vocab, dim, "f32", 0, table)
        iso.iso_embed_lookup(iso.Embed(ids=t, tokens=n, vocab=vocab, dim=dim, x=x.view, table=m.view, scale=0.5, pad_id=10),
                             iso.F32, ws=ws)
        return float((x.host() * dx).sum())

    for v in range(vocab):
        for c in range(0, dim, 2):
            step = np.zeros((vocab, dim))
            step[v, c] = 0.25
            assert (loss(w + step) - loss(w - step)) / 0.5 == got[v, c]


def test_sorted_tokens_of_the_whole_range():
    """A vocabulary past 2^19 (the widest buckets) with ids at both ends."""
    vocab, dim = 1 << 20, 4
    ids = np.array([0, vocab - 1, 5, vocab - 1, 524287, 524288, 0, 2047, 2048] * 20)
    dx = np.arange(len(ids) * dim, dtype=np.float64).reshape(-1, dim) % 64
    g = Mat(vocab, dim, "f32")
    e = iso.Embed(ids=dev_ids(ids, True), tokens=len(ids), vocab=vocab, dim=dim, x=Mat(len(ids), dim, "f32", 0, dx).view,
                  grad=g.view)
    x = Mat(len(ids), dim, "f32", 0, dx)
    e.x = x.view
    ws = iso.embed_workspace(e)
    iso.iso_embed_grad(e, iso.F32, iso.F32, ws=ws)
    got = g.host()
    for v in np.unique(ids):
        assert np.array_equal(got[v], dx[ids == v].sum(0))
        got[v] = 0
    assert not got.any()


def test_stream_and_graph():
    """On a stream of its own, and captured: every replay gives the eager result for the ids then in the buffer."""
    import torch
    rng = np.random.default_rng(8)
    n, vocab, dim = 700, 900, 64
    g, w = Mat(vocab, dim, "bf16"), Mat(vocab, dim, "bf16", 0, rng.standard_normal((vocab, dim)))
    x, y = Mat(n, dim, "bf16", 0, rng.standard_normal((n, dim))), Mat(n, dim, "bf16")
    ids = dev_ids(tokens(rng, n, vocab, None, "zipf"), True)
    bwd = iso.Embed(ids=ids, tokens=n, vocab=vocab, dim=dim, x=x.view, grad=g.view)
    fwd = iso.Embed(ids=ids, tokens=n, vocab=vocab, dim=dim, x=y.view, table=w.view)
    ws = iso.embed_workspace(bwd)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()

    def both(stream):
        iso.iso_embed_lookup(fwd, iso.BF16, ws=ws, stream=stream)
        iso.iso_embed_grad(bwd, iso.BF16, iso.BF16, ws=ws, stream=stream)

    both(s)
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        both(s)
    for k in range(4):
        ids.copy_(dev_ids(tokens(rng, n, vocab, None, "zipf"), True))
        g.view.fill_(3.0)
        y.view.fill_(3.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = g.host(), y.host()
        both(None)
        torch.cuda.synchronize()
        assert np.array_equal(got[0], g.host()) and np.array_equal(got[1], y.host())


def test_lookup_of_many_tokens_with_bad_ids():
    """Past the number of tokens whose ids one workgroup looks at: status and rows as below it."""
    n, vocab, dim = 20001, 300, 24
    rng = np.random.default_rng(9)
    table = f64(rng.standard_normal((vocab, dim)), "bf16")
    w = Mat(vocab, dim, "bf16", 0, table)
    for bad in (True, False):
        ids = rng.integers(0, vocab, n)
        if bad:
            ids[[0, n - 1]] = [-3, vocab]
        x = Mat(n, dim, "bf16", 8)
        e = iso.Embed(ids=dev_ids(ids, True), tokens=n, vocab=vocab, dim=dim, x=x.view, ld_x=x.ld, table=w.view, pad_id=5)
        ws = iso.embed_workspace(e)
        ws.fill_(0xFF)
        iso.iso_embed_lookup(e, iso.BF16, ws=ws)
        assert iso.iso_read_device_status(ws) == (_lib.ERR_INDEX if bad else 0)
        good = (ids >= 0) & (ids < vocab) & (ids != 5)
        want = np.where(good[:, None], table[np.where(good, ids, 0)], 0.0)
        assert np.array_equal(x.host(), want)
