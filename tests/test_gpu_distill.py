"""iso_distill_loss and iso_distill_grad against the binary64 oracle.

Bounds.  z / T is off by 2^-23 of its size, L by E = 2^-24 (V / 256 + 64 + 6 max|z / T|): a chain adds at most V / 256 terms and
the sums of 64 others, and an exponential is off by 2^-23 and by what its argument is.  A teacher's share has a relative error of
2^-24 (6 max|y / T| + top + 16) likewise.  A loss adds t (log t - z / T + L) over the entries, a gradient takes one share
from one probability; the result's own rounding is u.  What lies under the smallest normal number may be taken as zero."""
import numpy as np
import pytest

from oracle import gradients as gr

import paper_2607_19331_amd as iso
from paper_2607_19331_amd import _lib
from tests.grad_helpers import Mat, close, code, ttype, unit
from tests.gpu_helpers import say

pytestmark = pytest.mark.gpu

E24 = 2.0 ** -24
SLACK = 1 + 2.0 ** -6


class Case:
    def __init__(self, dtype, n, vocab, top, temp=1.0, gap=0, wide=True, pad=None, weights=True, seed=0, in_place=False, edit=None):
        import torch
        rng = np.random.default_rng(seed + 31 * n + vocab)
        self.dtype, self.n, self.vocab, self.top, self.temp, self.pad = dtype, n, vocab, top, temp, pad
        self.z = rng.standard_normal((n, vocab)) * 2.0
        self.ids = rng.integers(0, vocab, (n, top))              # ids repeat in small vocabularies
        self.y = rng.standard_normal((n, top)) * 3.0 + 5.0
        if pad is not None:
            self.ids[rng.random((n, top)) < 0.3] = pad
        self.w = np.where(rng.random(n) < 0.2, 0.0, rng.random(n)) if weights else None
        for r in range(n):                                       # the student has learnt something
            live = (self.ids[r] >= 0) & (self.ids[r] < vocab)
            self.z[r, self.ids[r][live]] = self.y[r][live] + rng.standard_normal(live.sum())
        if edit is not None:
            edit(self)
        f = lambda a, t: torch.as_tensor(a).to(t)  # noqa: E731
        self.z = f(self.z, ttype(dtype)).double().numpy()
        self.y = f(self.y, torch.float32).double().numpy()
        self.w = None if self.w is None else f(self.w, torch.float32).double().numpy()
        self.mat, self.loss, self.lse = Mat(n, vocab, dtype, gap, self.z), Mat(n, 1, "f32"), Mat(n, 1, "f32")
        self.grad = self.mat if in_place else Mat(n, vocab, dtype, gap)
        self.t = [f(self.ids, torch.int64 if wide else torch.int32).cuda(), f(self.y, torch.float32).cuda(),
                  None if self.w is None else f(self.w, torch.float32).cuda()]
        self.d = iso.Distill(logits=self.mat.view, tokens=n, vocab=vocab, ld=self.mat.ld, ids=self.t[0], teacher=self.t[1], top=top,
                             loss=self.loss.view, lse=self.lse.view, weight=self.t[2], temperature=temp, pad_id=pad)
        self.ws = iso.distill_workspace(self.d)
        with np.errstate(all="ignore"):
            self.want = gr.distill(self.z, self.ids, self.y, temp, self.w, pad)

    def call(self, what, stream=None):
        """loss alone, the gradient alone (after the loss), or both in one call."""
        self.d.grad, self.d.ld_grad = (None, None) if what == "loss" else (self.grad.view, self.grad.ld)
        f = iso.iso_distill_grad if what == "grad" else iso.iso_distill_loss
        f(self.d, code(self.dtype), ws=self.ws, stream=stream)

    def status(self):
        return iso.iso_read_device_status(self.ws)

    def bounds(self):
        loss, lse, grad = self.want
        with np.errstate(all="ignore"):
            top = np.abs(np.where(np.isfinite(self.z), self.z, 0.0)).max(1) / self.temp
            e = E24 * (self.vocab / 256 + 64 + 6 * top)
            tl, tg = np.zeros(self.n), np.zeros(grad.shape)
            for r in range(self.n):
                live, t = gr.teacher_shares(self.ids[r], self.y[r], self.vocab, self.temp, self.pad)
                w = 1.0 if self.w is None else self.w[r]
                if not live.any() or w == 0:
                    continue
                et = E24 * (6 * np.abs(self.y[r][live]).max() / self.temp + self.top + 16)
                x = self.z[r] / self.temp
                p = np.exp(x - lse[r])
                tg[r] = w * self.temp * p * (e[r] + E24 * (6 * (np.abs(x) + abs(lse[r])) + 16))
                for i, s in zip(self.ids[r][live], t[live]):
                    tg[r, i] += w * self.temp * s * et
                    inner = np.abs(np.log(max(s, 1e-300)) - x[i] + lse[r])
                    tl[r] += w * self.temp ** 2 * s * (et * (1 + inner) + et + e[r] + 2 * E24 * (np.abs(x[i]) + abs(lse[r])))
            tl, tg = np.where(np.isfinite(tl), tl, 0.0), np.where(np.isfinite(tg), tg, 0.0)
        u = unit(self.dtype)
        fin = lambda a: np.where(np.isfinite(a), np.abs(a), 0.0)  # noqa: E731
        return (SLACK * (tl + E24 * fin(loss)) + 2.0 ** -126, SLACK * (e + E24 * fin(lse)),
                SLACK * (tg + (u + 4 * E24) * fin(grad)) + 2.0 ** -120)

    def check(self, what):
        tl, te, tg = self.bounds()
        loss, lse, grad = self.want
        if what != "grad":
            close(self.loss.host()[:, 0], loss, tl)
        close(self.lse.host()[:, 0], lse, te)
        if what != "loss":
            close(self.grad.host(), grad, tg)
        if self.grad is not self.mat:
            assert np.array_equal(self.mat.host(), self.z, equal_nan=True)


SHAPES = [  # tokens, vocab, top, temperature, gap, wide ids, pad
    (1, 1, 1, 1.0, 0, True, None), (1, 7, 3, 1.0, 0, False, None), (3, 50, 256, 2.0, 3, True, -1), (7, 1031, 5, 1.0, 1, False, -1),
    (1, 40001, 20, 0.7, 0, True, None), (2, 151936, 64, 1.0, 0, True, -1), (3, 152064, 32, 2.0, 8, True, 152063),
    (65, 2049, 17, 1.0, 0, True, 2000), (300, 333, 40, 3.0, 5, False, -7), (1100, 96, 8, 1.0, 0, True, -1),
    (3, 170001, 12, 1.0, 1, True, -1), (2, 90000, 9, 1.0, 0, False, None), (40, 20500, 100, 1.0, 2, True, -1)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"n{s[0]}v{s[1]}k{s[2]}")
def test_distill(dtype, shape):
    say(f"distill {dtype} {shape}")
    n, vocab, top, temp, gap, wide, pad = shape
    case = Case(dtype, n, vocab, top, temp, gap, wide, pad, weights=n > 2)
    for what in ("loss", "grad", "both"):
        if what != "grad":
            case.loss.view.fill_(7.25), case.lse.view.fill_(7.25)
        case.grad.view.fill_(7.25)
        case.call(what)
        assert case.status() == 0
        case.check(what)


@pytest.mark.parametrize("dtype,n,vocab", [("f32", 130, 82001), ("bf16", 129, 163841), ("bf16", 66, 131073), ("bf16", 5, 100003),
                                           ("f32", 66, 66001), ("f32", 129, 65600)])
@pytest.mark.parametrize("in_place", [False, True])
def test_long_rows(dtype, n, vocab, in_place):
    """Rows that fit into a workgroup's registers and rows that do not, shared out and whole."""
    say(f"distill long rows {dtype} {n} {vocab} {in_place}")
    c = Case(dtype, n, vocab, 12, 2.0, pad=-1, in_place=in_place)
    c.call("loss")
    assert c.status() == 0
    c.check("loss")
    c.call("both")
    assert c.status() == 0
    c.check("both")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,vocab", [(2, 700), (4, 70001), (1, 152064), (600, 515)])
@pytest.mark.parametrize("how", ["both", "grad"])
def test_gradient_over_the_logits(dtype, n, vocab, how):
    say(f"distill in place {dtype} {n} {vocab} {how}")
    case = Case(dtype, n, vocab, 30, 1.5, 3, True, -1, in_place=True)
    if how == "grad":
        case.call("loss")
    case.call(how)
    assert case.status() == 0
    case.check(how)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_that_add_nothing_and_odd_lists(dtype):
    """Without entries, of weight 0 with NaN logits, entries of -inf, one id all through, banned logits (-inf)."""
    say(f"distill odd lists {dtype}")

    def edit(c):
        c.w[:] = 1.0
        c.ids[0] = -1
        c.y[1] = -np.inf
        c.w[2], c.z[2] = 0.0, np.nan
        c.y[3, 2:] = -np.inf
        c.ids[4] = 77
        c.z[5, :40], c.ids[5] = -np.inf, np.arange(50, 56)
        c.z[6, :40], c.ids[6] = -np.inf, np.arange(6)            # the teacher asks for what is banned: an infinite loss
        c.ids[7], c.w[7] = -1, 0.0
    case = Case(dtype, 8, 400, 6, 1.0, 1, True, -1, edit=edit)
    for what in ("loss", "grad", "both"):
        case.grad.view.fill_(7.25)
        case.call(what)
        assert case.status() == 0
        loss, lse, grad = case.loss.host()[:, 0], case.lse.host()[:, 0], case.grad.host()
        assert (loss[[0, 1, 2, 7]] == 0).all()
        assert loss[6] == np.inf and np.isnan(lse[2])
        tl, te, tg = case.bounds()
        if what != "loss":
            assert (grad[[0, 1, 2, 7]] == 0).all()
            rest = [3, 4, 5, 6]
            close(grad[rest], case.want[2][rest], tg[rest])
        close(loss[[3, 4, 5]], case.want[0][[3, 4, 5]], tl[[3, 4, 5]])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,vocab", [(3, 100), (900, 100), (2, 60000)])
@pytest.mark.parametrize("bad", ["high", "low"])
def test_ids_outside_the_vocabulary_are_reported(dtype, n, vocab, bad):
    say(f"distill bad ids {dtype} {n} {vocab} {bad}")

    def edit(c):
        c.ids[n - 1, 3] = vocab if bad == "high" else -2
    case = Case(dtype, n, vocab, 11, 1.0, 0, True, -1, edit=edit)
    case.call("loss")
    assert case.status() == _lib.ERR_INDEX
    case.check("loss")
    case.call("grad")
    assert case.status() == _lib.ERR_INDEX
    case.check("grad")
    case.call("both")
    assert case.status() == _lib.ERR_INDEX
    case.check("both")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,vocab", [(2, 30000), (700, 200)])
def test_captured_and_on_another_stream(dtype, n, vocab):
    import torch
    say(f"distill graph {dtype} {n} {vocab}")
    case, other = Case(dtype, n, vocab, 13, 2.0, 0, True, -1), Case(dtype, n + 1, vocab, 13, 2.0, 0, True, -1)
    for what in ("loss", "grad", "both"):
        case.call(what)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        case.call("loss"), case.call("grad"), case.call("both")
    side = torch.cuda.Stream()
    for _ in range(3):
        for m in (case.loss, case.lse, case.grad):
            m.view.fill_(7.25)
        g.replay()
        side.wait_stream(torch.cuda.current_stream())
        other.call("both", stream=side)
        torch.cuda.synchronize()
        assert case.status() == 0 and other.status() == 0
        case.check("both"), other.check("both")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_no_tokens_and_same_bits(dtype):
    say(f"distill none, repeats {dtype}")
    case = Case(dtype, 3, 5000, 9, 1.0, 0, True, -1)
    first = None
    for _ in range(3):
        case.call("both")
        got = [m.host() for m in (case.loss, case.lse, case.grad)]
        first = first or got
        assert all(np.array_equal(a, b) for a, b in zip(got, first))
    case.d.tokens = 0
    case.call("loss")
    assert case.status() == 0
    case.call("grad")
    assert case.status() == 0
