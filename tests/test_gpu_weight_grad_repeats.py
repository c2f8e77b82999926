"""Tables of iso_ckpt_weight_grad in which several layers name the same gradient: tied weights, a layer used twice, micro-batches
of one layer.  The table stands for its layers one after another.  Values have few bits, so every sum is exact."""
import pytest

import paper_2607_19331_amd as iso
from tests.gpu_helpers import say
from tests.grad_helpers import code, ttype

pytestmark = pytest.mark.gpu


def layer(gen, t, o, i, dtype):
    """A job's inputs with small integers, and their exact product."""
    import torch
    q = torch.randint(-3, 4, (t, iso.iso_ckpt_ld(i)), generator=gen, device="cuda", dtype=torch.int8)
    e = torch.full((t, q.shape[1] // 32), 127, device="cuda", dtype=torch.uint8)
    dy = torch.randint(-2, 3, (t, o), generator=gen, device="cuda").to(ttype(dtype))
    return (t, i, q, e, dy), torch.mm(dy.double().t().contiguous(), q[:, :i].double().contiguous())


def job(inputs, grad):
    t, i, q, e, dy = inputs
    return iso.WeightGrad(iso.Ckpt(t, i, q, e), dy=dy, grad=grad, rows=dy.shape[1])


def call(jobs, dtype, add):
    ws = iso.weight_grad_workspace(jobs, code(dtype))
    iso.iso_ckpt_weight_grad(jobs, code(dtype), iso.F32, accumulate=add, ws=ws)
    assert iso.iso_read_device_status(ws) == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("at", [(0, 1), (0, 1, 2, 3), (3, 15), (15, 16), (2, 17, 18, 30)])
def test_the_same_gradient(dtype, at):
    """Repeats next to each other, within a launch's 16 layers and across them."""
    import torch
    say(f"weight grad repeats {dtype} at {at}")
    gen = torch.Generator(device="cuda").manual_seed(1)
    n, o, i = 32, 70, 90
    made = [layer(gen, 40 + 5 * j, o, i, dtype) for j in range(n)]
    for add in (True, False):
        grads = [torch.full((o, i), 3.0, device="cuda") for _ in range(n)]
        for j in at:
            grads[j] = grads[at[0]]
        call([job(m[0], g) for m, g in zip(made, grads)], dtype, add)
        for j in range(n):
            if j in at:
                want = 3.0 + sum(made[k][1] for k in at) if add else made[at[-1]][1]
            else:
                want = made[j][1] + (3.0 if add else 0.0)
            assert torch.equal(grads[j].double(), want), j


def test_micro_batches_of_a_large_layer():
    """Whole and split tiles of the large kernel that are added to by every layer of the table."""
    import torch
    say("weight grad repeats: three micro-batches of 4090 x 4100")
    gen = torch.Generator(device="cuda").manual_seed(2)
    made = [layer(gen, t, 4090, 4100, "bf16") for t in (1000, 64, 700)]
    g = torch.ones(4090, 4100, device="cuda")
    call([job(m[0], g) for m in made], "bf16", True)
    assert torch.equal(g.double(), 1.0 + made[0][1] + made[1][1] + made[2][1])


def test_gradients_that_overlap_in_part():
    import torch
    gen = torch.Generator(device="cuda").manual_seed(3)
    made = [layer(gen, 60, 32, 64, "bf16") for _ in range(2)]
    for add in (True, False):
        buf = torch.full((48, 64), 2.0, device="cuda")
        call([job(made[0][0], buf[:32]), job(made[1][0], buf[16:])], "bf16", add)
        want = torch.full((48, 64), 2.0, dtype=torch.float64, device="cuda")
        for m, rows in zip(made, (slice(0, 32), slice(16, 48))):
            want[rows] = want[rows] + m[1] if add else m[1]
        assert torch.equal(buf.double(), want)
