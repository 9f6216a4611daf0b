"""The float64 orthogonalised update against its singular value form."""
import numpy as np
import pytest

from oracle import ortho_oracle as oo


@pytest.mark.parametrize("shape", [(1, 1), (4, 4), (3, 7), (9, 5)], ids=str)
def test_acts_on_singular_values_alone(shape):
    rng = np.random.default_rng(5)
    G = rng.standard_normal(shape)
    U, s, V = np.linalg.svd(G, full_matrices=False)
    s = s / (np.linalg.norm(G) + 1e-7)
    a, b, c = oo.COEFFS
    for _ in range(5):
        s = a * s + b * s ** 3 + c * s ** 5
    assert np.allclose(oo.orthogonalize(G), (U * s) @ V, atol=1e-12)


def test_cubic_iteration_orthogonalises():
    G = np.random.default_rng(6).standard_normal((2, 5, 8))
    X = oo.orthogonalize(G, steps=60, coeffs=(1.5, -0.5, 0.0), eps=0.0)
    assert np.allclose(X @ X.swapaxes(1, 2), np.eye(5), atol=1e-10)


def test_no_steps_and_zero():
    G = np.array([[3.0, 0.0], [0.0, 4.0]])
    assert np.allclose(oo.orthogonalize(G, steps=0, eps=0.0), G / 5)
    assert np.all(oo.orthogonalize(np.zeros((3, 2, 2)), eps=0.0) == 0)
    assert 400 < oo.gain() < 500      # 3.4445^5 = 484.9, at zero
