"""The gradient operators together, as examples/train_step.py runs them: the gradients of a step against automatic
differentiation in binary64, and a few steps of training.

The activations that the backward pass reads are off by their 8 bits: at most 1/254 of the largest of 32 neighbours each,
which for normal values (the largest of 32 is about twice their width) is 2^-8 of their norm or less.  A gradient is a
product of two such factors at most, and the fp32 rest is far more exact, so each gradient is within 2^-6 of its norm."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("train_step", os.path.join(ROOT, "examples", "train_step.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_gradients_of_a_step():
    import torch
    ex = example()
    model = ex.Model(torch.float32, seed=3)
    ids, targets = ex.batch(7)
    loss = model.gradients(ids, targets)
    names = ("embed", "head", "gate", "up", "down")
    w = {n: getattr(model, n).w.double().cpu().requires_grad_() for n in names}
    i, t = ids.cpu(), targets.cpu()
    live = i != ex.PAD
    x = w["embed"][i] * model.scale * live[:, None]
    z = x + (torch.nn.functional.silu(x @ w["gate"].t()) * (x @ w["up"].t())) @ w["down"].t()
    logp = torch.log_softmax(z @ w["head"].t(), -1)
    ref = -(logp.gather(1, t[:, None])[:, 0] * live).sum() / live.sum()
    ref.backward()
    ref = float(ref.detach())
    assert abs(float(loss) - ref) <= 1e-4 * ref
    for n in names:
        got, want = getattr(model, n).grad.double().cpu(), w[n].grad
        assert float((got - want).norm()) <= 2.0 ** -6 * float(want.norm()), n
    assert not model.embed.grad[ex.PAD].any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_training_learns(dtype):
    import torch
    losses = example().train(25, torch.bfloat16 if dtype == "bf16" else torch.float32)
    assert losses[0] > 5.0 and losses[-1] < 0.5 * losses[0], losses
