"""Float64 definition of the gated linear recurrence and its backward pass,
row after row (numpy; shares no code with the HIP path)."""
import numpy as np

DIRECT, SIGMOID = 0, 1


def sigmoid(a):
    """1 / (1 + exp(-a)) without overflow."""
    a = np.asarray(a, dtype=np.float64)
    t = np.exp(-np.abs(a))
    return np.where(a >= 0, 1.0, t) / (1.0 + t)


def gates(a, gate):
    """Multiplier s and the factor of u."""
    a = np.asarray(a, dtype=np.float64)
    return (sigmoid(a), sigmoid(-a)) if gate == SIGMOID else (a, np.ones_like(a))


def clamp_lengths(lengths, B, L):
    return np.full(B, L) if lengths is None else np.clip(np.asarray(lengths), 0, L)


def scan_forward(a, u, x0=None, lengths=None, gate=DIRECT):
    """x [B, L, w] (zero from lengths[b] on) and the state after the last row."""
    B, L, w = np.shape(a)
    n = clamp_lengths(lengths, B, L)
    s, q = gates(a, gate)
    x = np.zeros((B, L, w))
    last = np.zeros((B, w)) if x0 is None else np.array(x0, dtype=np.float64)
    for b in range(B):
        for l in range(n[b]):
            last[b] = s[b, l] * last[b] + q[b, l] * np.asarray(u[b, l], dtype=np.float64)
            x[b, l] = last[b]
    return x, last


def scan_backward(a, u, x, g, g_last=None, x0=None, lengths=None, gate=DIRECT):
    """da, du, dx0 from the stored states x, and the adjoints."""
    B, L, w = np.shape(a)
    n = clamp_lengths(lengths, B, L)
    s, q = gates(a, gate)
    da, du, lam = np.zeros((B, L, w)), np.zeros((B, L, w)), np.zeros((B, L, w))
    back = np.zeros((B, w)) if g_last is None else np.array(g_last, dtype=np.float64)
    for b in range(B):
        for l in reversed(range(n[b])):
            lam[b, l] = np.asarray(g[b, l], dtype=np.float64) + back[b]
            back[b] = s[b, l] * lam[b, l]
            if l > 0:
                xp = np.asarray(x[b, l - 1], dtype=np.float64)
            else:
                xp = np.zeros(w) if x0 is None else np.asarray(x0[b], dtype=np.float64)
            if gate == SIGMOID:
                xp = (xp - np.asarray(u[b, l], dtype=np.float64)) * s[b, l] * q[b, l]
            da[b, l] = lam[b, l] * xp
            du[b, l] = lam[b, l] * q[b, l]
    return da, du, back, lam
