"""The operators of recurrent language models reject invalid arguments before
any HIP call (so these run without a GPU)."""
import ctypes

import pytest

from paper_2309_16318_amd import deeppcr

E = deeppcr.EINVAL
# Fake, non-overlapping "device" addresses: validation must reject before use.
P = [ctypes.c_void_p(0x10000000 * (i + 1)) for i in range(16)]
BIG = 1 << 40


def off(p, n):
    return ctypes.c_void_p(p.value + n)


def _fwd(a=P[0], lda=40, u=P[1], ldu=40, x0=P[2], ln=P[3], x=P[4], last=P[5], B=2, L=8, w=40,
         gate=1, dtype=1, ws=P[6], nws=BIG):
    return deeppcr.lib().deeppcr_gated_scan_forward(a, lda, u, ldu, x0, ln, x, last, B, L, w, gate,
                                                    dtype, ws, nws, None)


def _bwd(a=P[0], lda=40, u=P[1], ldu=40, x=P[2], x0=P[3], ln=P[4], g=P[5], ldg=40, gl=P[6],
         da=P[7], du=P[8], dx0=P[9], B=2, L=8, w=40, gate=1, dtype=1, ws=P[10], nws=BIG):
    return deeppcr.lib().deeppcr_gated_scan_backward(a, lda, u, ldu, x, x0, ln, g, ldg, gl, da, du,
                                                     dx0, B, L, w, gate, dtype, ws, nws, None)


def _step(a=P[0], lda=40, u=P[1], ldu=40, s=P[2], so=P[3], x=P[4], B=2, w=40, gate=1, dtype=1):
    return deeppcr.lib().deeppcr_gated_scan_step(a, lda, u, ldu, s, so, x, B, w, gate, dtype, None)


def test_gated_scan_sizes():
    f = deeppcr.gated_scan_workspace_bytes
    assert f(1, 1, 1) > 0 and f(8, 65536, 1024) > 0
    for bad in ((0, 1, 1), (1, 0, 1), (1, 1, 0), (-1, 4, 4), (1 << 20, 4, 1 << 11),
                ((1 << 19) + 1, 4, 1 << 10), (1, (1 << 30) + 1, 4)):
        assert f(*bad) == 0
    # many channels run through a sequence tile after tile and need no board
    assert f(256, 4096, 8192) == f(1, 1, 1) < f(1, 4096, 8192)


@pytest.mark.parametrize("call,required,arrays", [
    (_fwd, "a u x ws", "a u x0 ln x last ws"),
    (_bwd, "a u x g da du ws", "a u x x0 ln g gl da du dx0 ws"),
    (_step, "a u s so", "a u s so x"),
])
def test_gated_scan_rejects_invalid_arguments(call, required, arrays):
    import inspect
    default = {k: v.default for k, v in inspect.signature(call).parameters.items()}
    for k in required.split():
        assert call(**{k: None}) == E, k
    for k in arrays.split():
        # sequences with a row stride start at any element, the rest at 16 bytes
        for n in (1, 3) if "ld" + k in default else (4, 8):
            assert call(**{k: off(default[k], n)}) == E, k
    for bad in (dict(B=0), dict(B=-1), dict(w=0), dict(gate=2), dict(gate=-1), dict(dtype=3),
                dict(dtype=-1), dict(lda=39), dict(ldu=39), dict(lda=-40),
                dict(B=1 << 20, w=1 << 11, lda=1 << 11, ldu=1 << 11, ldg=1 << 11)):
        if call is not _bwd:
            bad.pop("ldg", None)
        assert call(**bad) == E, bad
    if call is not _step:
        assert call(L=0) == E
        assert call(nws=deeppcr.gated_scan_workspace_bytes(2, 8, 40) - 1) == deeppcr.EWORKSPACE


def test_gated_scan_rejects_overlaps():
    for out in ("x", "last", "ws"):
        for other in (P[0], P[1], off(P[2], 16), P[3], off(P[0], 2 * 8 * 40 * 2 - 16)):
            assert _fwd(**{out: other}) == E, (out, other)
    assert _fwd(last=off(P[4], 16)) == E                # x_last over x
    assert _fwd(ws=P[5]) == E                           # workspace over x_last
    # a strided input reaches to its last row's end
    assert _fwd(lda=400, x=off(P[0], (15 * 400 + 40) * 2 - 16)) == E
    for out in ("da", "du", "dx0", "ws"):
        for other in (P[0], P[1], P[2], P[3], P[4], P[5], off(P[6], 16)):
            assert _bwd(**{out: other}) == E, (out, other)
    assert _bwd(da=P[8]) == E and _bwd(dx0=P[8]) == E and _bwd(ldg=39) == E
    assert _step(so=off(P[2], 16)) == E and _step(x=P[0]) == E and _step(x=P[3]) == E
    assert _step(so=P[1]) == E


def test_binding_rejects_what_is_not_a_gpu_sequence():
    torch = pytest.importorskip("torch")
    a = torch.zeros(2, 3, 4)
    with pytest.raises(ValueError):
        deeppcr.deeppcr_gated_scan_forward(a, a)                    # on the CPU
    with pytest.raises(ValueError):
        deeppcr.deeppcr_gated_scan_forward(a.double(), a.double())  # no such type
    with pytest.raises(ValueError):
        deeppcr.deeppcr_gated_scan_step(a[:, 0], a[:, 0], a[:, 0])


def _nfwd(x=P[0], y=P[1], ldy=40, z=P[2], ldz=40, post=P[3], sc=P[4], pre=P[5], xo=P[6], h=P[7],
          rp=P[8], rq=P[9], B=2, L=8, w=40, gate=2, per=0, eps=1e-6, dtype=1):
    return deeppcr.lib().deeppcr_residual_norm_forward(x, y, ldy, z, ldz, post, sc, pre, xo, h, rp,
                                                       rq, B, L, w, gate, per, eps, dtype, None)


def _nbwd(x=P[0], y=P[1], ldy=40, z=P[2], ldz=40, post=P[3], sc=P[4], pre=P[5], rp=P[6], rq=P[7],
          dxo=P[8], dh=P[9], dx=P[10], dy=P[11], dz=P[12], dpost=P[13], dsc=P[14], dpre=P[15],
          B=2, L=8, w=40, gate=2, per=0, dtype=1, ws=off(P[15], 1 << 27), nws=BIG):
    return deeppcr.lib().deeppcr_residual_norm_backward(
        x, y, ldy, z, ldz, post, sc, pre, rp, rq, dxo, dh, dx, dy, dz, dpost, dsc, dpre, B, L, w,
        gate, per, dtype, ws, nws, None)


def test_residual_norm_sizes():
    f = deeppcr.residual_norm_workspace_bytes
    assert f(2, 8, 40) > 0 and f(2, 8, 40, True) > 0 and f(1, 1, deeppcr.MAX_NORM_WIDTH) > 0
    for bad in ((0, 1, 1), (1, 0, 1), (1, 1, 0), (1, 1, 8193), ((1 << 23) + 1, 1, 8, True)):
        assert f(*bad) == 0
    assert deeppcr.lib().deeppcr_residual_norm_workspace_bytes(1, 1, 8, 2) == 0


def test_residual_norm_rejects_invalid_arguments():
    for call, arrays, strided in (
            (_nfwd, "x post sc pre xo h rp rq", "y z"),
            (_nbwd, "x post sc pre rp rq dxo dh dx dy dz dpost dsc dpre ws", "y z")):
        import inspect
        default = {k: v.default for k, v in inspect.signature(call).parameters.items()}
        for k in arrays.split():
            assert call(**{k: off(default[k], 8)}) == E, k
        for k in strided.split():
            assert call(**{k: off(default[k], 1)}) == E, k
        for bad in (dict(x=None), dict(B=0), dict(L=0), dict(w=0), dict(w=8193), dict(gate=4),
                    dict(gate=-1), dict(gate=0), dict(z=None), dict(z=None, gate=0, per=1),
                    dict(per=2), dict(dtype=3), dict(ldy=39), dict(ldz=39), dict(y=None),
                    dict(pre=None), dict(per=1, B=(1 << 23) + 1)):
            assert call(**bad) == E, bad
    assert _nfwd(xo=None) == E and _nfwd(h=None) == E
    assert _nfwd(post=None) == E                # its statistics are asked for
    for eps in (-1.0, float("nan"), float("inf")):
        assert _nfwd(eps=eps) == E
    assert _nfwd(y=None, z=None, gate=0, post=None, sc=None, xo=None, rp=None, pre=None, h=None,
                 rq=None) == E                  # nothing to do
    for k in ("rp", "rq", "dx", "dy", "dz", "ws", "dh"):
        assert _nbwd(**{k: None}) == E, k
    assert _nbwd(dxo=None, dh=None, pre=None, dpre=None) == E     # no gradient comes in
    assert _nbwd(sc=None) == E and _nbwd(post=None) == E          # gradient of a missing weight
    need = deeppcr.residual_norm_workspace_bytes(2, 8, 40)
    assert _nbwd(nws=need - 1) == deeppcr.EWORKSPACE


def test_residual_norm_rejects_overlaps():
    for out in ("h", "rp", "rq"):
        for other in (P[0], P[1], P[2], P[3], P[4], P[5], P[6]):
            assert _nfwd(**{out: other}) == E, out
    assert _nfwd(xo=off(P[0], 16)) == E and _nfwd(xo=P[1]) == E
    for out in ("dx", "dy", "dz", "dpost", "dsc", "dpre", "ws"):
        for i in range(10):
            assert _nbwd(**{out: P[i]}) == E, (out, i)
    assert _nbwd(dx=P[11]) == E and _nbwd(ws=P[13]) == E


def _ortho(G=P[0], X=P[1], N=3, m=20, n=30, steps=5, a=3.4445, b=-4.7750, c=2.0315, eps=1e-7,
           dtype=0, ws=P[2], nws=BIG):
    return deeppcr.lib().deeppcr_orthogonalize(G, X, N, m, n, steps, a, b, c, eps, dtype, ws, nws,
                                               None)


def test_orthogonalize_rejects_invalid_arguments():
    f = deeppcr.orthogonalize_workspace_bytes
    assert f(1, 1, 1) > 0 and f(2, 8192, 8192) > 0
    for bad in ((0, 1, 1), (1, 0, 1), (1, 1, 0), (1, 8193, 8), (1, 8, 8193), (-1, 2, 2)):
        assert f(*bad) == 0
    for k, p in (("G", P[0]), ("X", P[1]), ("ws", P[2])):
        assert _ortho(**{k: None}) == E and _ortho(**{k: off(p, 8)}) == E
    for bad in (dict(N=0), dict(m=0), dict(n=8193), dict(steps=-1), dict(dtype=3),
                dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf"))):
        assert _ortho(**bad) == E, bad
    assert _ortho(X=off(P[0], 16)) == E and _ortho(ws=P[0]) == E and _ortho(ws=P[1]) == E
    assert _ortho(nws=f(3, 20, 30) - 1) == deeppcr.EWORKSPACE


def test_orthogonalize_rejects_polynomials_that_run_away():
    W = deeppcr.EWORKSPACE        # a valid call with a short workspace
    assert _ortho(nws=1) == W
    for ok in ((1.5, -0.5, 0.0), (1.875, -1.25, 0.375), (3.4445, -4.7750, 2.0315),
               (0.0625, 0, 0), (-1, 0, 0), (1, 0, 0)):
        assert _ortho(a=ok[0], b=ok[1], c=ok[2], steps=8, nws=1) == W, ok
    for bad in ((0, 0, 0), (0.06, 1, 0), (100.0, 0, 0), (3.4445, 4.7750, 2.0315), (2.0, 0, 0), (1.5, -0.5, 30.0),
                (float("nan"), 0, 0), (1, float("inf"), 0)):
        assert _ortho(a=bad[0], b=bad[1], c=bad[2], steps=8, nws=1) == E, bad
    assert _ortho(a=2.0, b=0, c=0, steps=2, nws=1) == W


def test_gated_scan_channels_end_below_the_threads_of_a_launch():
    """With 8 threads to a channel 2^29 channels would be a launch of 2^32 threads."""
    f = deeppcr.gated_scan_workspace_bytes
    for B, w in ((1 << 19, 1 << 10), (1 << 29, 1), (1, 1 << 29)):
        assert f(B, 113, w) == 0
        for call in (_fwd, _step):
            assert call(B=B, w=w, lda=w, ldu=w) == E
        assert _bwd(B=B, w=w, lda=w, ldu=w, ldg=w) == E
    assert f((1 << 29) - 1, 113, 1) > 0 and f((1 << 19) - 1, 1, 1 << 10) > 0


def test_in_place_means_one_argument():
    """An output may be the argument that the text names, not another one that is
    the same memory and laid out, or read, otherwise."""
    for n in (0, 1):   # the workspace is looked at first: only a large one gets to the overlaps
        want = E if n else deeppcr.EWORKSPACE
        nws = BIG if n else 0
        # dx0 over g_last that is x0 too: x0 is read while dx0 is written
        assert _bwd(x0=P[6], gl=P[6], dx0=P[6], nws=nws) == want
        # x_last over x0 that is the gates too
        assert _fwd(a=P[2], dtype=0, last=P[2], nws=nws) == want
    # the stream in place, and the block's output the same memory in other rows
    assert _nfwd(y=P[0], ldy=80, xo=P[0]) == E
    assert _nfwd(z=P[0], ldz=48, xo=P[0]) == E
    assert _nfwd(z=P[0], per=1, xo=P[0]) == E
    assert _step(a=P[2], lda=80, dtype=0, so=P[2]) == E
