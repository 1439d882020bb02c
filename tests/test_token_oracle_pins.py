"""Pins of the oracle of norms, embeddings, clipping and adjusted logits: closed forms, and differences for the gradients."""
import numpy as np

from oracle import token_oracle as to


def test_norm_closed_forms():
    h, y = to.rms_norm([[3.0, 4.0]], None, [1.0, 2.0], 0.0)
    assert np.allclose(y, np.array([[3.0, 8.0]]) / np.sqrt(12.5)) and np.array_equal(h, [[3.0, 4.0]])
    h, y = to.rms_norm([[1.0, 2.0]], [[-1.0, 2.0]], None, 1.0)
    assert np.array_equal(h, [[0.0, 4.0]]) and np.allclose(y, [[0.0, 4.0 / 3.0]])
    assert np.array_equal(to.rms_norm(np.zeros((1, 4)), None, None, 1e-6)[1], np.zeros((1, 4)))


def test_norm_gradient_by_differences():
    rng = np.random.default_rng(1)
    x, res, w, dy, d_h = rng.standard_normal((3, 5)), rng.standard_normal((3, 5)), rng.standard_normal(5), rng.standard_normal((3, 5)), rng.standard_normal((3, 5))

    def loss(x, w):
        h, y = to.rms_norm(x, res, w, 0.1)
        return (y * dy).sum() + (h * d_h).sum()
    dx, dw, _, _ = to.rms_norm_backward(dy, x + res, w, 0.1, d_h)
    t = 1e-6
    for i in np.ndindex(3, 5):
        e = np.zeros((3, 5))
        e[i] = t
        assert abs((loss(x + e, w) - loss(x - e, w)) / (2 * t) - dx[i]) < 1e-8 * (1 + abs(dx[i]))
    for j in range(5):
        e = np.zeros(5)
        e[j] = t
        assert abs((loss(x, w + e) - loss(x, w - e)) / (2 * t) - dw[j]) < 1e-8 * (1 + abs(dw[j]))


def test_embedding_and_its_gradient():
    table, ids = np.arange(8.0).reshape(4, 2), np.array([3, -1, 0, 3, 4])
    assert np.array_equal(to.embedding(table, ids, 2.0), [[12, 14], [0, 0], [0, 2], [12, 14], [0, 0]])
    rng = np.random.default_rng(2)
    d = rng.standard_normal((5, 2))
    grad, mag, n = to.embedding_backward(d, ids, 4, 2.0)
    assert np.allclose((to.embedding(table, ids, 2.0) * d).sum(), (table * grad).sum())        # linear: its adjoint
    assert np.array_equal(n, [1, 0, 0, 2]) and np.allclose(mag[3], 2 * (np.abs(d[0]) + np.abs(d[3])))


def test_clip():
    norm, out = to.grad_clip([np.array([3.0]), np.array([[4.0]])], 1.0)
    assert norm == 5.0 and np.allclose(out[0], 0.6) and np.allclose(out[1], 0.8)
    norm, out = to.grad_clip([np.array([3.0]), np.array([4.0])], 5.0)
    assert norm == 5.0 and out[0][0] == 3.0
    assert to.grad_clip([np.array([np.inf, 1.0])], 1.0)[1][0][1] == 1.0


def test_logits():
    z = np.array([[2.0, -2.0, 0.5, 1.0, -np.inf]])
    out, _ = to.logits_adjust(z, history=[[0, 1, 1, 3, 7, -1]], n_prompt=[1], repetition=[2.0], presence=[0.25], frequency=[0.5],
                              bias_id=[[2, 0, 2, 9]], bias=[[5.0, 1.0, -1.0, 3.0]], allowed=[[0b10111]])
    assert np.array_equal(out, [[2.0, -5.25, -0.5, -np.inf, -np.inf]])
    assert np.array_equal(to.logits_adjust(z)[0], z)
