"""The float64 gated scan against hand values, the block-bidiagonal solve
with diagonal blocks, and central differences."""
import numpy as np
import pytest

import oracle
from oracle import scan_oracle as so


def test_forward_by_hand():
    a = np.array([[[0.5], [2.0], [0.0]]])
    u = np.array([[[1.0], [3.0], [4.0]]])
    x, last = so.scan_forward(a, u, x0=np.array([[8.0]]))
    assert x.ravel().tolist() == [5.0, 13.0, 4.0] and last.ravel().tolist() == [4.0]
    x, last = so.scan_forward(a, u, x0=np.array([[8.0]]), lengths=[2])
    assert x.ravel().tolist() == [5.0, 13.0, 0.0] and last.ravel().tolist() == [13.0]
    x, last = so.scan_forward(a, u, x0=np.array([[8.0]]), lengths=[0])
    assert x.ravel().tolist() == [0.0, 0.0, 0.0] and last.ravel().tolist() == [8.0]
    x, _ = so.scan_forward(np.zeros((1, 1, 1)), np.full((1, 1, 1), 6.0), np.full((1, 1), 2.0),
                           gate=so.SIGMOID)
    assert x.ravel().tolist() == [4.0]      # half of each


def test_is_the_block_solve_with_diagonal_blocks():
    rng = np.random.default_rng(1)
    a, u = rng.standard_normal((2, 9, 3)), rng.standard_normal((2, 9, 3))
    J = a[..., None] * np.eye(3)
    assert np.allclose(so.scan_forward(a, u)[0], oracle.seq_solve(J, u, False), rtol=1e-12)
    lam = so.scan_backward(a, u, u, u)[3]
    assert np.allclose(lam, oracle.seq_solve(J, u, True), rtol=1e-12)


@pytest.mark.parametrize("gate", [so.DIRECT, so.SIGMOID])
@pytest.mark.parametrize("lengths", [None, [4, 0, 2]])
def test_backward_against_central_differences(gate, lengths):
    rng = np.random.default_rng(2)
    B, L, w = 3, 4, 2
    v = {k: rng.standard_normal((B, L, w)) for k in "aug"}
    v["x0"], v["g_last"] = rng.standard_normal((B, w)), rng.standard_normal((B, w))

    def loss(v):
        x, last = so.scan_forward(v["a"], v["u"], v["x0"], lengths, gate)
        return np.sum(x * v["g"]) + np.sum(last * v["g_last"])

    x, _ = so.scan_forward(v["a"], v["u"], v["x0"], lengths, gate)
    da, du, dx0, _ = so.scan_backward(v["a"], v["u"], x, v["g"], v["g_last"], v["x0"], lengths,
                                      gate)
    for k, got in (("a", da), ("u", du), ("x0", dx0)):
        for i in np.ndindex(got.shape):
            d = {}
            for sgn in (1, -1):
                p = {n: t.copy() for n, t in v.items()}
                p[k][i] += sgn * 1e-5
                d[sgn] = loss(p)
            assert abs((d[1] - d[-1]) / 2e-5 - got[i]) < 1e-8 * max(1, abs(got[i]))
