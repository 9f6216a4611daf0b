"""The float64 residual norm against hand values and central differences."""
import numpy as np
import pytest

from oracle import norm_oracle as no


def test_forward_by_hand():
    x, y = np.array([[[1.0, 2.0]]]), np.array([[[3.0, -4.0]]])
    two = np.array([2.0, 2.0])
    out, h, rp, rq = no.norm_forward(x, y, None, two, np.array([0.5, 1.0]), two, eps=0.0)
    r = 1 / np.sqrt(12.5)
    assert np.allclose(out, [[[1 + 3 * r, 2 - 8 * r]]])
    assert np.allclose(h, 2 * out / np.sqrt(np.mean(out ** 2)))
    assert np.allclose(rp, r) and rq.shape == (1, 1)
    # no norm behind, no norm in front
    out, h, rp, rq = no.norm_forward(x, y, np.array([[2.0, -2.0]]), gate=no.LINEAR)
    assert np.allclose(out, [[[7.0, 10.0]]]) and h is None and rp is None and rq is None


def test_gates():
    z = np.array([-3.0, 0.0, 2.0])
    for gate in (no.SIGMOID, no.SILU, no.LINEAR):
        v, s = no.gate_values(gate, z)
        d = (no.gate_values(gate, z + 1e-6)[0] - no.gate_values(gate, z - 1e-6)[0]) / 2e-6
        assert np.allclose(s, d, atol=1e-9)
    assert no.gate_values(no.SIGMOID, z)[0][1] == 0.5 and no.gate_values(no.SILU, z)[0][1] == 0.0


@pytest.mark.parametrize("gate", [no.NONE, no.SIGMOID, no.SILU, no.LINEAR])
@pytest.mark.parametrize("per_seq", [False, True])
@pytest.mark.parametrize("left_out", [(), ("w_post",), ("scale",), ("w_pre", "dh"), ("dx_out",)])
def test_backward_against_central_differences(gate, per_seq, left_out):
    if per_seq and gate == no.NONE:
        return
    rng = np.random.default_rng(3)
    B, L, w = 2, 3, 4
    v = {k: rng.standard_normal((B, L, w)) for k in ("x", "y", "z", "dx_out", "dh")}
    v.update({k: 1 + 0.3 * rng.standard_normal(w) for k in ("w_post", "scale", "w_pre")})
    if per_seq:
        v["z"] = v["z"][:, 0]
    if gate == no.NONE:
        v["z"] = None
    for k in left_out:
        v[k] = None

    def loss(v):
        out, h, _, _ = no.norm_forward(v["x"], v["y"], v["z"], v["w_post"], v["scale"],
                                       v["w_pre"], gate, 1e-3)
        return sum(np.sum(p * q) for p, q in ((out, v["dx_out"]), (h, v["dh"])) if q is not None)

    got = no.norm_backward(v["x"], v["y"], v["z"], v["w_post"], v["scale"], v["w_pre"], gate,
                           1e-3, v["dx_out"], v["dh"])
    for k, g in zip(("x", "y", "z", "w_post", "scale", "w_pre"), got):
        if v[k] is None:
            assert g is None
            continue
        for i in np.ndindex(g.shape):
            d = {}
            for s in (1, -1):
                p = {n: None if t is None else t.copy() for n, t in v.items()}
                p[k][i] += s * 1e-5
                d[s] = loss(p)
            assert abs((d[1] - d[-1]) / 2e-5 - g[i]) < 1e-7 * max(1, abs(g[i])), k
