"""The fp64 definitions of the operators around the linear layers against differences (CPU)."""
import numpy as np
import pytest

from oracle import model_oracle as orc


def along(f, eps=1e-6):
    return (f(eps) - f(-eps)) / (2 * eps)


@pytest.mark.parametrize("layer", [True, False])
def test_norm_gradients(layer):
    r = np.random.default_rng(0)
    x, dy, u = (r.normal(size=(5, 12)) + 0.5 for _ in range(3))
    w, b, uw, ub = (r.normal(size=12) for _ in range(4))

    def f(e):
        return (orc.norm(x + e * u, w + e * uw, b + e * ub, layer, 1e-3)[0] * dy).sum()
    _, mean, rstd = orc.norm(x, w, b, layer, 1e-3)
    dx, dw, db = orc.norm_backward(x, w, layer, mean, rstd, dy)
    assert abs(along(f) - (dx * u).sum() - (dw * uw).sum() - (db * ub).sum()) < 1e-7


def test_norm_closed_forms():
    x = np.array([[1.0, 3.0], [2.0, 2.0]])
    y, mean, rstd = orc.norm(x, None, None, True, 0.0 + 1e-300)
    assert np.allclose(y[0], [-1, 1]) and np.allclose(mean, [2, 2]) and rstd[0] == 1
    y, _, rstd = orc.norm(x, None, None, False, 0.0)
    assert np.allclose((y ** 2).mean(1), 1) and np.allclose(rstd[1], 0.5)


def test_embedding_gradient():
    r = np.random.default_rng(1)
    table, u, dy = r.normal(size=(7, 4)), r.normal(size=(7, 4)), r.normal(size=(6, 4))
    ids = [3, 0, -1, 3, 6, 0]

    def f(e):
        return (orc.embedding(table + e * u, ids, 1.7) * dy).sum()
    d, size = orc.embedding_backward(dy, ids, 1.7, 7)
    assert abs(along(f) - (d * u).sum()) < 1e-8
    assert np.all(d[[1, 2, 4, 5]] == 0) and np.all(size >= np.abs(d))


@pytest.mark.parametrize("shape", [(6, 6), (5, 11), (11, 5)])
def test_newton_schulz_is_a_polynomial_in_the_singular_values(shape):
    r = np.random.default_rng(2)
    u = r.normal(size=shape)
    k = [(3.4445, -4.7750, 2.0315), (2.0, -1.5, 0.5), (1.5, -0.5, 0.0)]
    left, s, right = np.linalg.svd(u, full_matrices=False)
    s = s / np.linalg.norm(s)
    for a, b, c in k:
        s = a * s + b * s ** 3 + c * s ** 5
    assert np.allclose(orc.newton_schulz(u, k), (left * s) @ right, atol=1e-12)
    assert not orc.newton_schulz(np.zeros(shape), k).any()
    x = orc.newton_schulz(u, [(1.5, -0.5, 0.0)] * 40)
    assert np.allclose(x @ x.T if shape[0] <= shape[1] else x.T @ x, np.eye(min(shape)))


def test_muon_step_closed_form():
    w, m, x = orc.muon_step(np.array([[2.0]]), np.array([[-3.0]]), np.zeros((1, 1)), 0.1, 0.9, True,
                            [(1.0, 0.0, 0.0)], 2.0, 0.5)
    assert np.allclose([w, m, x], [[[2.0 - 0.1 * (-2.0 + 1.0)]], [[-0.3]], [[-1.0]]])
