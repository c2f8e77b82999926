"""examples/train_step.py with batches of changing sizes: one model, whose workspaces stay between the steps, gives the gradients
that a model made for the batch gives, bit for bit."""
import pytest

from tests.test_gpu_train_example import example

pytestmark = pytest.mark.gpu


def test_batches_of_changing_sizes():
    import torch
    ex = example()
    kept = ex.Model(torch.bfloat16, seed=4)
    for rows in (3, 160, 16, 200, 1):                      # 32 tokens a row
        ids, targets = ex.batch(rows, rows=rows)
        own = ex.Model(torch.bfloat16, seed=4)
        assert float(kept.gradients(ids, targets)) == float(own.gradients(ids, targets))
        for a, b in zip(kept.weights, own.weights):
            assert torch.equal(a.grad, b.grad), rows
