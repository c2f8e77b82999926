"""Workspace sizes of the gradient operators through the library, tables of several launches included.  No GPU is used: the
pointers are never dereferenced."""
import ctypes
import random

import pytest

import paper_2607_19331_amd as iso
from paper_2607_19331_amd import _lib


def job(t, o, i, ld=None, q=None, dy=None, grad=None):
    return iso.WeightGrad(iso.Ckpt(t, i, q, q), dy=dy, grad=grad, rows=o, ld_dy=ld)


def size(jobs, dt):
    return _lib.load().iso_workspace_size_weight_grad(iso._weight_grads(jobs), len(jobs), dt)


@pytest.mark.parametrize("dt", [iso.F32, iso.BF16])
@pytest.mark.parametrize("n", [0, 1, 16, 17, 40])
def test_tables_of_several_launches(dt, n):
    """The need of a table is that of its largest launch."""
    rng = random.Random(n)
    for shared in (False, True):
        jobs = []
        for j in range(n):
            t, i = rng.choice([0, 1, 33, 4097]), rng.randint(0, 3000)
            q = (j + 1) << 32
            if shared and jobs and rng.random() < 0.5:
                c = rng.choice(jobs).ckpt
                t, i, q = c.rows, c.cols, c.q
            o = rng.randint(0, 3000)
            jobs.append(job(t, o, i, o + rng.randint(0, 8), q))
        need = size(jobs, dt)
        assert need >= 256 and need % 256 == 0
        launches = [size(jobs[k:k + 16], dt) for k in range(0, n, 16)]
        assert need == max([256] + launches)


@pytest.mark.parametrize("dt", [iso.F32, iso.BF16])
def test_largest_sizes(dt):
    big = [job(1 << 10, 1 << 24, 1 << 10), job(1 << 29, 1, 8), job(0, 1 << 24, 1 << 10), job(1 << 10, 1 << 10, 1 << 24)]
    parts = 3 if dt == iso.F32 else 1
    assert size(big, dt) >= 2 * (1 << 29) * 32 + 2 * parts * (1 << 29) * 8
    assert size(big * 4, dt) >= 4 * size(big[1:2], dt) - 4 * (64 << 20)
    for bad in (job(1, (1 << 24) + 1, 1), job(1 << 31, 1, 1), job((1 << 29) + 1, 1, 8), job(1, 1, (1 << 24) + 1), job(1, 1 << 18, 1 << 17), job(1, 5, 5, 4)):
        assert size([bad], dt) == 0


def test_embedding_sizes():
    L = _lib.load()

    def need(n, vocab, dim):
        return L.iso_workspace_size_embed(ctypes.byref(iso._embed(iso.Embed(ids=1, tokens=n, vocab=vocab, dim=dim, x=None,
                                                                            id_type=iso.I64))))
    for vocab, dim in ((1, 1), (300, 5), (1 << 20, 1 << 18)):
        sizes = [need(n, vocab, dim) for n in (0, 1, 4096, 4097, 5000, 65536, 65537, 1 << 20, (1 << 31) - 1)]
        assert sizes == sorted(sizes) and sizes[0] == sizes[2] == 256
        assert sizes[3] >= 4097 * (8 + 4 + 16) + 4 * dim * (4097 // 16)
    assert need(1 << 31, 5, 5) == 0 and need(1, (1 << 20) + 1, 5) == 0


@pytest.mark.parametrize("dt", [iso.F32, iso.BF16])
@pytest.mark.parametrize("o,i", [(2048, 2048), (1024, 1024), (517, 1027), (1, 1), (4100, 300)])
def test_longest_batch_holds_the_shorter_ones(dt, o, i):
    """A workspace made for the longest batch is enough for every other: the need does not fall as tokens grow."""
    tokens = sorted([*range(0, 9000, 31), 4992, 5024, 7104, 7392])
    sizes = [size([job(t, o, i)], dt) for t in tokens]
    assert sizes == sorted(sizes)


@pytest.mark.parametrize("dt", [iso.F32, iso.BF16])
def test_need_grows_with_the_table(dt):
    """Nor as one layer of a table gets tokens (from none on) or a layer joins the launch, and unknown pointers count most."""
    rng = random.Random(dt)
    for _ in range(60):
        shapes = [(rng.choice([0, 0, 5, 300, 3000, 8192]), rng.randint(1, 4000), rng.randint(1, 4000)) for _ in range(rng.randint(1, 16))]
        need = size([job(*s) for s in shapes], dt)
        k = rng.randrange(len(shapes))
        t, o, i = shapes[k]
        for more in (t + 1, t + 31, t + 32, 2 * t + 100):
            assert size([job(*s) for s in shapes[:k] + [(more, o, i)] + shapes[k + 1:]], dt) >= need
        if len(shapes) < 16:
            assert size([job(*s) for s in shapes + [(rng.choice([0, 700]), 900, 800)]], dt) >= need
        assert need >= max(size([job(*s)], dt) for s in shapes)
        assert need >= size([job(*s, q=1 << 32) for s in shapes], dt)
