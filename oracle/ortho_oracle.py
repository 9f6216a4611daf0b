"""Float64 definition of the orthogonalised update (numpy; shares no code
with the HIP path)."""
import numpy as np

COEFFS = (3.4445, -4.7750, 2.0315)


def orthogonalize(G, steps=5, coeffs=COEFFS, eps=1e-7):
    """[N, m, n] or [m, n]."""
    X = np.asarray(G, dtype=np.float64)
    a, b, c = coeffs
    norm = np.sqrt(np.sum(X * X, axis=(-2, -1), keepdims=True))
    X = np.divide(X, norm + eps, out=np.zeros_like(X), where=np.broadcast_to(norm > 0, X.shape))
    for _ in range(steps):
        if X.shape[-2] <= X.shape[-1]:
            A = X @ np.swapaxes(X, -1, -2)
            X = a * X + (b * A + c * A @ A) @ X
        else:
            A = np.swapaxes(X, -1, -2) @ X
            X = a * X + X @ (b * A + c * A @ A)
    return X


def gain(steps=5, coeffs=COEFFS):
    """The largest slope over [0, 1] of the map of singular values: how much an
    error of the start is magnified at most where singular vectors stay."""
    a, b, c = coeffs
    s = np.linspace(0, 1, 200001)
    slope = np.ones_like(s)
    for _ in range(steps):
        slope *= a + 3 * b * s ** 2 + 5 * c * s ** 4
        s = s * (a + b * s ** 2 + c * s ** 4)
    return float(np.max(np.abs(slope)))
