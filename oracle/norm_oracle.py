"""Float64 definition of the residual norm and its backward pass (numpy;
shares no code with the HIP path)."""
import numpy as np

from .scan_oracle import sigmoid

NONE, SIGMOID, SILU, LINEAR = 0, 1, 2, 3


def gate_values(gate, z):
    """act(z) and its slope."""
    if gate == NONE:
        return 1.0, None
    if gate == LINEAR:
        return z, np.ones_like(z)
    s, c = sigmoid(z), sigmoid(-z)
    return (s, s * c) if gate == SIGMOID else (z * s, s * (1 + z * c))


def _wide(z):
    return None if z is None else z[:, None] if z.ndim == 2 else z


def norm_forward(x, y=None, z=None, w_post=None, scale=None, w_pre=None, gate=NONE, eps=1e-6):
    """x_out, h, rstd_post, rstd_pre (None where a piece is left out)."""
    rp = rq = h = None
    out = x
    if y is not None:
        v = gate_values(gate, _wide(z))[0]
        if w_post is not None:
            rp = 1 / np.sqrt(np.mean(y * y, axis=-1) + eps)
            y = y * rp[..., None] * w_post
        out = x + (1.0 if scale is None else scale) * v * y
    if w_pre is not None:
        rq = 1 / np.sqrt(np.mean(out * out, axis=-1) + eps)
        h = out * rq[..., None] * w_pre
    return out, h, rp, rq


def norm_backward(x, y, z, w_post, scale, w_pre, gate, eps, dx_out, dh):
    """dx, dy, dz, dw_post, dscale, dw_pre for dx_out and dh (None: zero)."""
    out, _, rp, rq = norm_forward(x, y, z, w_post, scale, w_pre, gate, eps)
    d = np.zeros_like(x) if dx_out is None else dx_out.copy()
    dpre = None
    if w_pre is not None:
        m, e = out * rq[..., None], dh * w_pre
        d += rq[..., None] * (e - m * np.mean(e * m, axis=-1, keepdims=True))
        dpre = np.sum(dh * m, axis=(0, 1))
    if y is None:
        return d, None, None, None, None, dpre
    v, slope = gate_values(gate, _wide(z))
    sc = 1.0 if scale is None else scale
    wp = 1.0 if w_post is None else w_post
    n = y if w_post is None else y * rp[..., None]
    dscale = None if scale is None else np.sum(d * v * n * wp, axis=(0, 1))
    dpost = None if w_post is None else np.sum(d * v * n * sc, axis=(0, 1))
    dz = None
    if gate != NONE:
        dz = d * sc * wp * n * slope
        if z.ndim == 2:
            dz = dz.sum(axis=1)
    dy = d * sc * wp * v
    if w_post is not None:
        dy = rp[..., None] * (dy - n * np.mean(dy * n, axis=-1, keepdims=True))
    return d, dy, dz, dpost, dscale, dpre
