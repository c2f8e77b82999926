"""The binary64 oracle of the gradient operators against hand-worked values, brute force and central differences."""
import numpy as np
import pytest

from oracle import gradients as gr


def test_embedding_by_hand():
    table = np.arange(12.0).reshape(4, 3)
    ids = [2, 0, 2, 3, 1]
    x = gr.embed_lookup(table, ids, 0.5, pad_id=3)
    assert x.tolist() == [[3, 3.5, 4], [0, 0.5, 1], [3, 3.5, 4], [0, 0, 0], [1.5, 2, 2.5]]
    dx = np.array([[1.0, 0, 0], [0, 1, 0], [2, 0, 0], [np.nan, 9, 9], [0, 0, 4]])
    g = gr.embed_grad(dx, ids, 4, 0.5, pad_id=3)
    assert g.tolist() == [[0, 0.5, 0], [0, 0, 2], [1.5, 0, 0], [0, 0, 0]]
    assert gr.embed_grad(dx, [2, 0, -1, 4, 1], 4, 1.0)[2].tolist() == [1, 0, 0]


def test_embedding_gradient_is_the_lookups_adjoint():
    rng = np.random.default_rng(1)
    ids = rng.integers(0, 9, 40)
    dx = rng.standard_normal((40, 5))
    g = gr.embed_grad(dx, ids, 9, 1.7, pad_id=4)
    for v in range(9):
        for c in range(5):
            step = np.zeros((9, 5))
            step[v, c] = 1e-3
            hi, lo = (float((gr.embed_lookup(s * step, ids, 1.7, pad_id=4) * dx).sum()) for s in (1, -1))
            assert abs((hi - lo) / 2e-3 - g[v, c]) < 1e-9


def test_checkpoint_by_hand():
    x = np.zeros((1, 64))
    x[0, :4] = [127.0, -63.5, 0.5, 1.5]           # k = 0: halves go to even
    x[0, 32:35] = [127.00001, 3.0, 1.0]           # just past 127: k = 1
    q, e = gr.ckpt_pack(x)
    assert e.tolist() == [[127, 128]]
    assert q[0, :4].tolist() == [127, -64, 0, 2]
    assert q[0, 32:35].tolist() == [64, 2, 0]
    q, e = gr.ckpt_pack(np.array([[0.0, 1e-45, np.inf]]))
    assert e.tolist() == [[255]] and not q.any()
    assert np.isnan(gr.ckpt_values(q, e, 3)).all()
    assert gr.ckpt_pack(np.zeros((2, 5)))[1].tolist() == [[1], [1]]


@pytest.mark.parametrize("cols", [1, 31, 32, 33, 100])
def test_checkpoint_error_bound_and_exactness(cols):
    rng = np.random.default_rng(cols)
    x = rng.standard_normal((7, cols)) * np.exp(4 * rng.standard_normal((7, cols)))
    q, e = gr.ckpt_pack(x)
    back = gr.ckpt_values(q, e, cols)
    for g in range(e.shape[1]):
        part = slice(32 * g, min(32 * g + 32, cols))
        top = np.abs(x[:, part]).max(1, keepdims=True)
        assert (np.abs(back[:, part] - x[:, part]) <= top / 127).all()
    again = gr.ckpt_values(*gr.ckpt_pack(back), cols)
    assert np.array_equal(again, back)             # what came back packs to itself
    f = back.astype(np.float32)
    assert np.array_equal(f.astype(np.float64), back)
    assert not (f.view(np.uint32) & 0xFFFF).any()  # and is a bf16 value


def test_gate_gradient_by_central_differences():
    rng = np.random.default_rng(3)
    g, u, dh = (rng.standard_normal(200) * 3 for _ in range(3))
    dg, du = gr.gate_grad(g, u, dh)
    h = 1e-6
    assert np.allclose(dg, dh * (gr.gate_forward(g + h, u) - gr.gate_forward(g - h, u)) / (2 * h), rtol=1e-6, atol=1e-8)
    assert np.allclose(du, dh * (gr.gate_forward(g, u + h) - gr.gate_forward(g, u - h)) / (2 * h), rtol=1e-6, atol=1e-8)


def test_weight_gradient_by_differences():
    rng = np.random.default_rng(4)
    x, dy, w = rng.standard_normal((6, 4)), rng.standard_normal((6, 3)), rng.standard_normal((3, 4))
    g = gr.weight_grad(dy, x)
    for o in range(3):
        for i in range(4):
            step = np.zeros_like(w)
            step[o, i] = 1e-4
            hi, lo = (float(((x @ (w + s * step).T) * dy).sum()) for s in (1, -1))
            assert abs((hi - lo) / 2e-4 - g[o, i]) < 1e-8
