"""The gradient operators past 32-bit offsets: tables, activations and gradients of more than 4 GiB, whose few values that
differ from zero lie at both ends and past the 2^31-th element.  Values have few bits, so every result is exact."""
import numpy as np
import pytest

import paper_2607_19331_amd as iso
from tests.gpu_helpers import say

pytestmark = pytest.mark.gpu


def zeros(*shape, dtype):
    import torch
    return torch.zeros(*shape, dtype=dtype, device="cuda")


def test_embedding_table_of_5_gib():
    import torch
    vocab, dim = 1 << 20, 2400                             # 2.5e9 elements
    say(f"large embedding {vocab} x {dim}")
    w = zeros(vocab, dim, dtype=torch.bfloat16)
    rows = [0, 1 << 19, (1 << 31) // dim + 1, vocab - 1]
    for k, r in enumerate(rows):
        w[r] = torch.arange(dim, device="cuda") % 61 + k
    ids = torch.tensor([rows[3], rows[0], 7, rows[2], rows[1], rows[3]], device="cuda")
    x = zeros(6, dim, dtype=torch.bfloat16)
    e = iso.Embed(ids=ids, tokens=6, vocab=vocab, dim=dim, x=x, table=w, scale=0.5)
    ws = iso.embed_workspace(e)
    iso.iso_embed_lookup(e, iso.BF16, ws=ws)
    assert iso.iso_read_device_status(ws) == 0
    assert torch.equal(x, w[ids] * 0.5)
    e.grad, e.scale = w, 2.0                               # added in place over the table itself
    want = w[ids].float()
    want[[0, 5]] += 2.0 * (x[0].float() + x[5].float())
    for t in (1, 2, 3, 4):
        want[t] += 2.0 * x[t].float()
    before = w.float().abs().sum(dtype=torch.float64)
    iso.iso_embed_grad(e, iso.BF16, iso.BF16, accumulate=True, ws=ws)
    assert iso.iso_read_device_status(ws) == 0
    assert torch.equal(w[ids], want.bfloat16())
    added = (2.0 * x.float().abs()).sum(dtype=torch.float64)
    after = w.float().abs().sum(dtype=torch.float64)
    rounded = (want.bfloat16().double() - want.double())[[0, 1, 2, 3, 4]].sum()
    assert float(after - before - added - rounded) == 0.0   # and nothing else changed
    many = torch.full((5000,), vocab - 1, device="cuda")
    many[::2] = 3
    dx = zeros(5000, dim, dtype=torch.bfloat16)
    dx[:, 5] = 1.0
    g = iso.Embed(ids=many, tokens=5000, vocab=vocab, dim=dim, x=dx, grad=w)
    ws = iso.embed_workspace(g)
    w.fill_(9.0)
    iso.iso_embed_grad(g, iso.BF16, iso.BF16, ws=ws)       # the whole gradient, zeros included
    assert float(w[3, 5]) == float(w[vocab - 1, 5]) == 2496.0   # 2500 in bf16
    w[3, 5] = w[vocab - 1, 5] = 0.0
    assert not bool(w.any())


def test_checkpoint_of_9_gib():
    import torch
    rows, cols = 1 << 20, 4640                             # 4.9e9 elements
    say(f"large checkpoint {rows} x {cols}")
    x = zeros(rows, cols, dtype=torch.bfloat16)
    at = [0, (1 << 31) // cols, (1 << 32) // cols, rows - 1]
    for k, r in enumerate(at):
        x[r] = (torch.arange(cols, device="cuda") % 127 - 63) * 2.0 ** k
    q, e = iso.ckpt_buffers(rows, cols)
    q.fill_(77)
    iso.iso_ckpt_pack([iso.Ckpt(rows, cols, q, e, x=x)], iso.BF16)
    back = torch.full_like(x, 5.0)
    iso.iso_ckpt_unpack([iso.Ckpt(rows, cols, q, e, x=back)], iso.BF16)
    assert torch.equal(back, x)
    keep = [iso.Ckpt(rows, cols, q, e)] * 2
    back.fill_(1.0)
    dup = torch.full_like(x, 5.0)
    iso.iso_ckpt_gate_grad([iso.GateGrad(*keep, dh=back, dgate=back, dup=dup)], iso.BF16)
    g = x[at].float()
    s = torch.sigmoid(g)
    assert torch.allclose(dup[at].float(), g * s, rtol=2.0 ** -7, atol=2.0 ** -100)
    rest = torch.ones(rows, dtype=torch.bool, device="cuda")
    rest[at] = False
    assert int(dup.ne(0).any(1)[rest].sum()) == 0


@pytest.mark.parametrize("out", [18944, 18945])
def test_weight_gradient_of_many_tokens(out):
    """dy of 4.5 GiB, read in place and (odd stride) through its copy; tokens at both ends and around 2^31 and 2^32 bytes."""
    import torch
    tokens, cols = 120000, 72
    say(f"large weight gradient {tokens} tokens, {out} x {cols}")
    dy = zeros(tokens, out, dtype=torch.bfloat16)
    x = zeros(tokens, cols, dtype=torch.bfloat16)
    at = [0, 31, 56679, 56680, 113359, 113360, tokens - 1]
    for k, t in enumerate(at):
        dy[t] = (torch.arange(out, device="cuda") + 3 * k) % 17 - 8
        x[t] = (torch.arange(cols, device="cuda") + k) % 13 - 6
    q, e = iso.ckpt_buffers(tokens, cols)
    iso.iso_ckpt_pack([iso.Ckpt(tokens, cols, q, e, x=x)], iso.BF16)
    g = torch.full((out, cols), float("nan"), device="cuda")
    job = [iso.WeightGrad(iso.Ckpt(tokens, cols, q, e), dy=dy, grad=g, rows=out)]
    ws = iso.weight_grad_workspace(job, iso.BF16)
    iso.iso_ckpt_weight_grad(job, iso.BF16, iso.F32, ws=ws)
    assert iso.iso_read_device_status(ws) == 0
    want = dy[at].cpu().double().numpy().T @ x[at].cpu().double().numpy()
    assert np.array_equal(g.cpu().double().numpy(), want)
