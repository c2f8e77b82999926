"""One training step of a small language model with ISO-AdamW: every gradient that the optimizer step takes comes from the
library's gradient operators, and the activations wait for the backward pass in 8 bits.

    python examples/train_step.py [--steps N] [--dtype f32|bf16]

The model is an embedding, one gated MLP block with a residual, and an unembedding:

    x = s E[ids],  g = x Wg^T,  u = x Wu^T,  h = silu(g) u,  z = x + h Wd^T,  logits = z Wh^T.

Its task is to continue a cyclic sequence.  The dense products with the weights are torch's; the lookup, the checkpoints, the
gate's backward pass, the weight gradients, the embedding's gradient and the step on the frames are the library's.
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2607_19331_amd as iso  # noqa: E402

VOCAB, DIM, HIDDEN, PAD = 512, 64, 192, 511


class Weight:
    """One matrix W = U Sigma V^T with the frames, moments, gradient and weight that an ISO-AdamW step works on."""

    def __init__(self, rows, cols, dtype, gen):
        w = torch.randn(rows, cols, generator=gen, dtype=torch.float64) / math.sqrt(cols)
        u, s, vt = torch.linalg.svd(w, full_matrices=False)
        col = lambda a: a.t().contiguous().view(-1).cuda()  # noqa: E731  column-major
        zero = lambda n: torch.zeros(n * len(s), dtype=torch.float64, device="cuda")  # noqa: E731
        self.w = w.to(dtype).cuda()
        self.grad = torch.zeros_like(self.w)
        self.frame = iso.Frame(u=col(u), v=col(vt.t()), sigma=s.cuda(), m_u=zero(rows), v_u=zero(rows), m_v=zero(cols),
                               v_v=zero(cols), grad=self.grad, w_out=self.w, rows=rows, cols=cols, rank=len(s))


class Kept:
    """Activations in 8 bits between the two passes."""

    def __init__(self, x, code):
        rows, cols = x.shape
        self.ckpt = iso.Ckpt(rows, cols, *iso.ckpt_buffers(rows, cols), x=x, ld_x=x.stride(0))
        iso.iso_ckpt_pack([self.ckpt], code)
        self.ckpt.x = None                                  # the full-size activations may go


class Model:
    def __init__(self, dtype, seed=0):
        gen = torch.Generator().manual_seed(seed)
        self.dtype, self.code = dtype, iso.BF16 if dtype == torch.bfloat16 else iso.F32
        self.embed, self.head = (Weight(VOCAB, DIM, dtype, gen) for _ in range(2))
        self.gate, self.up = (Weight(HIDDEN, DIM, dtype, gen) for _ in range(2))
        self.down = Weight(DIM, HIDDEN, dtype, gen)
        self.weights = [self.embed, self.head, self.gate, self.up, self.down]
        self.scale = math.sqrt(DIM)
        self.ws = {}

    def workspace(self, name, make, tokens=0):
        """Kept until a longer batch comes: what a call needs does not fall as tokens grow."""
        if name not in self.ws or self.ws[name][0] < tokens:
            self.ws[name] = tokens, make()
        return self.ws[name][1]

    def gradients(self, ids, targets):
        """Loss of the tokens that are no padding; leaves the gradients in the weights' buffers."""
        n = ids.numel()
        table = iso.Embed(ids=ids, tokens=n, vocab=VOCAB, dim=DIM, x=torch.empty(n, DIM, dtype=self.dtype, device="cuda"),
                          table=self.embed.w, grad=self.embed.grad, scale=self.scale, pad_id=PAD)
        ws = self.workspace("embed", lambda: iso.embed_workspace(table), n)
        iso.iso_embed_lookup(table, self.code, ws=ws)
        x = table.x
        kept_x = Kept(x, self.code)
        g, u = x @ self.gate.w.t(), x @ self.up.w.t()
        h = (torch.nn.functional.silu(g.float()) * u.float()).to(self.dtype)
        kept_g, kept_u, kept_h = Kept(g, self.code), Kept(u, self.code), Kept(h, self.code)
        z = x + h @ self.down.w.t()
        kept_z = Kept(z, self.code)
        logits = (z @ self.head.w.t()).float()

        live = ids != PAD
        logp = torch.log_softmax(logits, -1)
        loss = -(logp.gather(1, targets[:, None])[:, 0] * live).sum() / live.sum()
        dlogits = torch.exp(logp)
        dlogits.scatter_add_(1, targets[:, None], torch.full((n, 1), -1.0, device="cuda"))
        dlogits = (dlogits * (live / live.sum())[:, None]).to(self.dtype)

        dz = dlogits @ self.head.w
        dh = dz @ self.down.w
        dg, du = torch.empty_like(dh), torch.empty_like(dh)
        iso.iso_ckpt_gate_grad([iso.GateGrad(kept_g.ckpt, kept_u.ckpt, dh=dh, dgate=dg, dup=du)], self.code)
        table.x = dz + dg @ self.gate.w + du @ self.up.w
        jobs = [iso.WeightGrad(kept.ckpt, dy=dy, grad=w.grad, rows=w.w.shape[0])
                for kept, dy, w in ((kept_z, dlogits, self.head), (kept_h, dz, self.down), (kept_x, dg, self.gate),
                                    (kept_x, du, self.up))]
        jobs_ws = self.workspace("jobs", lambda: iso.weight_grad_workspace(jobs, self.code), n)
        iso.iso_ckpt_weight_grad(jobs, self.code, self.code, ws=jobs_ws)
        iso.iso_embed_grad(table, self.code, self.code, ws=ws)
        return loss

    def step(self, t, lr=0.02):
        frames = [w.frame for w in self.weights]
        ws = self.workspace("step", lambda: iso.optimizer_workspace(frames))
        iso.iso_optimizer_step(frames, self.code, lr=lr, step=t, ws=ws)
        if iso.iso_read_device_status(ws) != 0:
            raise RuntimeError("the optimizer step reported an error")


def batch(seed, rows=16, length=32):
    """Cyclic sequences of random start and stride, the last quarter of every other row padded; and their continuations."""
    gen = torch.Generator().manual_seed(seed)
    start = torch.randint(0, 64, (rows, 1), generator=gen)
    ids = (start + 3 * torch.arange(length + 1)) % 64
    ids, targets = ids[:, :-1].clone(), ids[:, 1:].clone()
    ids[::2, length * 3 // 4:] = PAD
    return ids.reshape(-1).cuda(), targets.reshape(-1).cuda()


def train(steps, dtype):
    model, losses = Model(dtype), []
    for t in range(1, steps + 1):
        losses.append(float(model.gradients(*batch(t))))
        model.step(t)
    return losses


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=40)
    ap.add_argument("--dtype", choices=("f32", "bf16"), default="bf16")
    a = ap.parse_args()
    for t, loss in enumerate(train(a.steps, torch.bfloat16 if a.dtype == "bf16" else torch.float32), 1):
        print(f"step {t:3d}  loss {loss:.4f}")
