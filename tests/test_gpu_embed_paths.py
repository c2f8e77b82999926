"""The embedding's paths by size, against binary64 on the device: the sorted gradient of many tokens (small vocabularies, several
column blocks, odd widths and strides, bad ids, special values, a captured graph), the large gradient that few tokens
overwrite, and lookups whose output is streamed.  Tolerances as in test_gpu_embed.py."""
import math

import pytest

import paper_2607_19331_amd as iso
from paper_2607_19331_amd import _lib
from tests.gpu_helpers import say
from tests.grad_helpers import GUARD, code, ttype, unit

pytestmark = pytest.mark.gpu

SLACK = 1 + 2.0 ** -6
SCALE = 0.37


class Buf:
    """A rows x cols view (row stride cols + gap) of a device buffer whose other elements hold GUARD."""

    def __init__(self, rows, cols, dtype, gap=0):
        import torch
        self.n, self.ld = rows * (cols + gap), cols + gap
        self.buf = torch.full((self.n + 64,), GUARD, dtype=ttype(dtype), device="cuda")
        self.view = self.buf[:self.n].view(rows, self.ld)[:, :cols]

    def guards(self):
        gap = self.buf[:self.n].view(-1, self.ld)[:, self.view.shape[1]:]
        assert bool((gap == GUARD).all()) and bool((self.buf[self.n:] == GUARD).all())


def draw_ids(gen, n, vocab, pad, kind):
    import torch
    u = torch.rand(n, generator=gen, device="cuda", dtype=torch.float64)
    if kind == "zipf":
        ids = (torch.exp(u * math.log(vocab + 1)) - 1).long().clamp_(0, vocab - 1)
    else:
        ids = (u * vocab).long()
    if pad is not None:
        ids = torch.where(torch.rand(n, generator=gen, device="cuda") < 0.2, pad, ids)
    return ids


class Case:
    def __init__(self, seed, dtype, gtype, add, n, vocab, dim, gap, wide, pad, kind):
        import torch
        self.dtype, self.gtype, self.add, self.vocab, self.pad = dtype, gtype, add, vocab, pad
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        self.x, self.g = Buf(n, dim, dtype, gap), Buf(vocab, dim, gtype)
        self.start = (torch.randn(vocab, dim, generator=self.gen, device="cuda") * 3).to(ttype(gtype)) if add else None
        self.ids = torch.empty(n, dtype=torch.int64 if wide else torch.int32, device="cuda")
        self.e = iso.Embed(ids=self.ids, tokens=n, vocab=vocab, dim=dim, x=self.x.view, ld_x=self.x.ld, grad=self.g.view,
                           scale=SCALE, pad_id=pad)
        self.ws = iso.embed_workspace(self.e)
        self.ws.fill_(0xA5)
        self.renew(draw_ids(self.gen, n, vocab, pad, kind))

    def renew(self, ids):
        import torch
        self.ids.copy_(ids)
        self.x.view.copy_(torch.randn(self.x.view.shape, generator=self.gen, device="cuda"))
        if self.pad is not None:
            self.x.view[ids == self.pad] = float("nan")    # padding's gradients are not looked at
        self.reset()

    def reset(self):
        self.g.view.copy_(self.start) if self.add else self.g.view.fill_(float("nan"))

    def call(self, stream=None):
        iso.iso_embed_grad(self.e, code(self.dtype), code(self.gtype), accumulate=self.add, ws=self.ws, stream=stream)

    def status(self):
        return iso.iso_read_device_status(self.ws)

    def check(self):
        import torch
        ids = self.ids.long()
        live = (ids >= 0) & (ids < self.vocab)
        if self.pad is not None:
            live &= ids != self.pad
        ids, dx = ids[live], self.x.view[live].double() * SCALE
        mass = torch.zeros(self.vocab, dx.shape[1], dtype=torch.float64, device="cuda")
        ref = self.start.double() if self.add else mass.clone()
        ref.index_add_(0, ids, dx)
        mass.index_add_(0, ids, dx.abs())
        m = torch.bincount(ids, minlength=self.vocab).double()[:, None]
        got, fine = self.g.view.double(), torch.isfinite(ref)
        assert torch.equal(torch.isnan(got), torch.isnan(ref))
        assert torch.equal(got[torch.isinf(ref)], ref[torch.isinf(ref)])
        tol = SLACK * ((m + 2) * 2.0 ** -24 * mass + (2.0 ** -24 + unit(self.gtype)) * ref.abs())
        off = ((got - ref).abs() - tol)[fine]
        assert float(off.max()) <= 0, float(off.max())
        if self.add:
            untouched = m[:, 0] == 0
            assert torch.equal(self.g.view[untouched], self.start[untouched])
        self.g.guards()


MANY = [  # tokens, vocab, dim, gap, wide, pad, kind
    (4097, 1031, 259, 5, False, 1020, "zipf"), (4096, 1031, 259, 5, False, 1020, "zipf"), (9000, 4, 600, 0, True, None, "even"),
    (6000, 1, 7, 0, True, None, "even"), (5000, 15, 1030, 1, False, 3, "zipf"), (7000, 16, 64, 0, True, None, "even"),
    (20000, 300001, 520, 0, True, None, "zipf"), (33000, 152064, 40, 8, True, 152000, "even"),
    (5001, 1 << 20, 33, 0, False, None, "even"), (70001, 1200, 96, 0, True, 7, "zipf"), (4100, 511, 4099, 0, True, None, "even")]


@pytest.mark.parametrize("dtype,gtype,add", [("f32", "f32", False), ("bf16", "bf16", False), ("bf16", "f32", True),
                                             ("f32", "bf16", True)])
@pytest.mark.parametrize("n,vocab,dim,gap,wide,pad,kind", MANY)
def test_many_tokens(dtype, gtype, add, n, vocab, dim, gap, wide, pad, kind):
    import torch
    say(f"embed paths {dtype}->{gtype} add={add} n={n} vocab={vocab} dim={dim} gap={gap} pad={pad} {kind}")
    c = Case(n + dim, dtype, gtype, add, n, vocab, dim, gap, wide, pad, kind)
    c.call()
    assert c.status() == 0
    c.check()
    first = c.g.view.clone()
    c.reset()
    c.call()
    assert torch.equal(c.g.view, first)                    # the same bits again


@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("n,vocab", [(4000, 50), (6001, 50), (6001, 9), (30000, 40000)])
def test_bad_ids_and_special_rows(n, vocab, add):
    """Ids outside the vocabulary add nothing and are reported, at either end of the tokens; NaN and infinities of a row reach that
    id's gradient only; the next call clears the status."""
    say(f"embed paths: bad ids and special rows, n={n} vocab={vocab} add={add}")
    for wide in (True, False):
        c = Case(n, "bf16", "f32", add, n, vocab, 72, 0, wide, 5, "zipf")
        c.ids[0], c.ids[n // 2], c.ids[n - 1] = -1, vocab, vocab + 70000
        c.x.view[[0, n // 2, n - 1]] = float("nan")
        c.ids[[11, 12, 13]] = c.ids.new_tensor([2, 3, 4])
        c.x.view[11], c.x.view[12, 9], c.x.view[13, 70] = float("inf"), float("nan"), float("-inf")
        c.call()
        assert c.status() == _lib.ERR_INDEX
        c.check()
        c.renew(draw_ids(c.gen, n, vocab, 5, "zipf"))
        c.call()
        assert c.status() == 0
        c.check()


@pytest.mark.parametrize("n,vocab,add", [(9000, 3000, False), (9000, 3000, True), (5000, 12, False), (3000, 300000, False)])
def test_graph(n, vocab, add):
    """Captured: every replay works on the ids and rows then in the buffers, with eager calls in between."""
    import torch
    say(f"embed paths: graph, n={n} vocab={vocab} add={add}")
    c = Case(n, "bf16", "f32", add, n, vocab, 136, 0, True, None, "zipf")
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    c.call(s)
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        c.call(s)
    for kind in ("zipf", "even", "zipf"):
        c.renew(draw_ids(c.gen, n, vocab, None, kind))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        c.check()
        got = c.g.view.clone()
        c.reset()
        c.call()
        torch.cuda.synchronize()
        assert torch.equal(got, c.g.view)


@pytest.mark.parametrize("gtype,vocab,dim", [("bf16", 131071, 259), ("f32", 131071, 131), ("f32", 65537, 257), ("bf16", 131073, 264)])
@pytest.mark.parametrize("n", [0, 1, 300, 4096])
def test_few_tokens_overwrite_a_large_gradient(gtype, vocab, dim, n):
    """64 MiB and more, also of sizes that no whole number of vectors holds: cleared, and written where tokens are."""
    say(f"embed paths: {n} tokens over {vocab} x {dim} {gtype}")
    assert vocab * dim * (2 if gtype == "bf16" else 4) >= 64 << 20
    c = Case(n + dim, "bf16", gtype, False, n, vocab, dim, 1, True, 77, "even")
    if n > 1:
        c.ids[n - 1], c.ids[0] = vocab - 1, 0
        c.x.view[[0, n - 1]] = 1.5
    c.call()
    assert c.status() == 0
    c.check()


@pytest.mark.parametrize("dtype,n,vocab,dim,gap", [("bf16", 5000, 3000, 3584, 0), ("bf16", 20001, 700, 1029, 3),
                                                   ("f32", 4097, 999, 2301, 1), ("f32", 16384, 50, 520, 8),
                                                   ("bf16", 16385, 50, 1040, 0)])
def test_streamed_lookup(dtype, n, vocab, dim, gap):
    """Outputs past 32 MiB, on both sides of the number of tokens whose ids one workgroup looks at."""
    import torch
    say(f"embed paths: lookup {dtype} n={n} vocab={vocab} dim={dim} gap={gap}")
    assert n * dim * (2 if dtype == "bf16" else 4) > 32 << 20
    gen = torch.Generator(device="cuda").manual_seed(n)
    table = torch.randn(vocab, dim, generator=gen, device="cuda").to(ttype(dtype))
    x = Buf(n, dim, dtype, gap)
    for bad in (True, False):
        ids = draw_ids(gen, n, vocab, 9, "zipf")
        if bad:
            ids[0], ids[n - 1] = vocab, -1
        e = iso.Embed(ids=ids, tokens=n, vocab=vocab, dim=dim, x=x.view, ld_x=x.ld, table=table, scale=SCALE, pad_id=9)
        ws = iso.embed_workspace(e)
        ws.fill_(0xFF)
        iso.iso_embed_lookup(e, code(dtype), ws=ws)
        assert iso.iso_read_device_status(ws) == (_lib.ERR_INDEX if bad else 0)
        good = (ids >= 0) & (ids < vocab) & (ids != 9)
        ref = table[torch.where(good, ids, 0)].double() * SCALE * good[:, None]
        off = (x.view.double() - ref).abs() - (2.0 ** -23 + unit(dtype)) * SLACK * ref.abs()
        assert float(off.max()) <= 0
        x.guards()


@pytest.mark.parametrize("dtype,n,dim", [("bf16", 6144, 2048), ("bf16", 6145, 2048), ("bf16", 6145, 2049), ("f32", 16384, 1025),
                                         ("f32", 16385, 1025), ("f32", 6145, 1024), ("bf16", 6145, 1), ("bf16", 16384, 9)])
def test_who_looks_at_the_ids(dtype, n, dim):
    """On both sides of each bound: rows, status with the one bad id at either end, status cleared by the next call."""
    import torch
    say(f"embed paths: bad id in a lookup {dtype} n={n} dim={dim}")
    gen = torch.Generator(device="cuda").manual_seed(n + dim)
    table = torch.randn(301, dim, generator=gen, device="cuda").to(ttype(dtype))
    x = Buf(n, dim, dtype, 1)
    ws = iso.embed_workspace(iso.Embed(ids=1, tokens=n, vocab=301, dim=dim, x=None, id_type=iso.I64))
    ws.fill_(0xFF)
    for at in (0, None, n - 1, n // 2, None):
        ids = draw_ids(gen, n, 301, None, "even")
        if at is not None:
            ids[at] = 301
        iso.iso_embed_lookup(iso.Embed(ids=ids, tokens=n, vocab=301, dim=dim, x=x.view, ld_x=x.ld, table=table), code(dtype), ws=ws)
        assert iso.iso_read_device_status(ws) == (0 if at is None else _lib.ERR_INDEX)
        want = table[ids.clamp(max=300)] * (ids < 301)[:, None]
        assert torch.equal(x.view, want)
        x.guards()
