"""ctypes binding of libdeeppcr.so (include/deeppcr.h).

Argument marshalling only: torch tensors provide device memory and the
current HIP stream; every step of the computation runs in the library's
kernels.  With ``stream`` a call works, and allocates, on that stream instead;
its inputs have to be ready there (``stream.wait_stream``).  No call is
recorded for automatic differentiation: results have no graph, whatever their
inputs require, and the gradients are the ``_backward`` calls'.  There is no
CPU fallback: if the library is missing, every call raises.
"""
from __future__ import annotations

import ctypes
import functools
import os
from dataclasses import dataclass

OK, EINVAL, ENOCONV, ENONFINITE, EHIP, EWORKSPACE = range(6)
TANH_MLP, TANH_RESIDUAL, SIGMOID_MLP, SIGMOID_RESIDUAL, RELU_MLP, RELU_RESIDUAL = range(6)
OP_PCR, OP_FWD, OP_BWD = 0, 1, 2
ACT_TANH, ACT_SIGMOID, ACT_RELU = 0, 1, 2
F32, BF16, F16 = range(3)
GATE_DIRECT = GATE_NONE = 0
GATE_SIGMOID, GATE_SILU, GATE_LINEAR = 1, 2, 3
(KCLASS_PCR_LEVEL, KCLASS_LAYER, KCLASS_UPDATE, KCLASS_WGRAD, KCLASS_OTHER, KCLASS_SEQUENTIAL,
 KCLASS_PCR_TAIL, KCLASS_SCAN, KCLASS_NORM, KCLASS_ORTHO) = range(10)
KCLASS_NAMES = ("pcr_level", "layer", "update", "wgrad", "other", "sequential", "pcr_tail",
                "scan", "norm", "ortho")
MAX_WIDTH = 1024
MAX_BLOCK_WIDTH = 128  # collapsed-skip ResNet and the chunked solve
MAX_NORM_WIDTH = 8192
MAX_ORTHO_SIDE = 8192

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libdeeppcr.so")

# Every symbol declared in include/deeppcr.h, with its ctypes signature.
_c = ctypes
SIGNATURES = {
    "deeppcr_workspace_bytes": (_c.c_size_t, [_c.c_int, _c.c_int, _c.c_int, _c.c_int]),
    "deeppcr_status_string": (_c.c_char_p, [_c.c_int]),
    "deeppcr_last_error": (_c.c_char_p, []),
    "pcr_solve_block_bidiag": (_c.c_int, [_c.c_void_p, _c.c_void_p, _c.c_void_p, _c.c_int,
                                          _c.c_int, _c.c_int, _c.c_int, _c.c_void_p,
                                          _c.c_size_t, _c.c_void_p]),
    "pcr_solve_block_bidiag_noalloc": (_c.c_int, [_c.c_void_p, _c.c_void_p, _c.c_void_p,
                                                  _c.c_int, _c.c_int, _c.c_int, _c.c_int,
                                                  _c.c_void_p]),
    "deeppcr_noalloc_scratch_bytes": (_c.c_size_t, []),
    "deeppcr_chunked_workspace_bytes": (_c.c_size_t, [_c.c_int] * 4),
    "pcr_solve_block_bidiag_chunked": (_c.c_int, [_c.c_void_p] * 3 + [_c.c_int] * 5 +
                                       [_c.c_void_p, _c.c_size_t, _c.c_void_p]),
    "deeppcr_mlp_forward": (_c.c_int, [_c.c_void_p, _c.c_void_p, _c.c_void_p, _c.c_void_p,
                                       _c.c_int, _c.c_int, _c.c_int, _c.c_int, _c.c_float,
                                       _c.c_float, _c.c_int, _c.c_void_p, _c.c_void_p,
                                       _c.c_size_t, _c.POINTER(_c.c_int),
                                       _c.POINTER(_c.c_float), _c.c_void_p]),
    "deeppcr_newton_step": (_c.c_int, [_c.c_void_p] * 3 + [_c.c_int] * 3 +
                            [_c.c_float, _c.c_void_p, _c.c_size_t] +
                            [_c.POINTER(_c.c_float)] * 3 + [_c.c_void_p]),
    "deeppcr_release_thread_state": (None, []),
    "deeppcr_mlp_forward_residual": (_c.c_int, [_c.c_void_p, _c.c_void_p, _c.c_void_p,
                                                _c.c_void_p, _c.c_int, _c.c_int, _c.c_int,
                                                _c.c_int, _c.c_float, _c.c_float, _c.c_float,
                                                _c.c_int, _c.c_void_p, _c.c_void_p, _c.c_size_t,
                                                _c.POINTER(_c.c_int), _c.POINTER(_c.c_float),
                                                _c.c_void_p]),
    "deeppcr_mlp_backward": (_c.c_int, [_c.c_void_p] * 9 + [_c.c_int, _c.c_int, _c.c_int,
                                                           _c.c_int, _c.c_float, _c.c_void_p,
                                                           _c.c_size_t, _c.c_void_p]),
    "deeppcr_resnet_workspace_bytes": (_c.c_size_t, [_c.c_int] * 5),
    "deeppcr_resnet_forward": (_c.c_int, [_c.c_void_p] * 4 + [_c.c_int] * 5 +
                               [_c.c_float, _c.c_int, _c.c_void_p, _c.c_void_p, _c.c_size_t,
                                _c.POINTER(_c.c_int), _c.POINTER(_c.c_float), _c.c_void_p]),
    "deeppcr_resnet_backward": (_c.c_int, [_c.c_void_p] * 8 + [_c.c_int] * 5 +
                                [_c.c_void_p, _c.c_size_t, _c.c_void_p]),
    "deeppcr_resnet_seq_forward": (_c.c_int, [_c.c_void_p] * 4 + [_c.c_int] * 6 + [_c.c_void_p]),
    "deeppcr_resnet_seq_backward": (_c.c_int, [_c.c_void_p] * 6 + [_c.c_int] * 6 +
                                    [_c.c_void_p]),
    "deeppcr_seq_forward": (_c.c_int, [_c.c_void_p] * 4 + [_c.c_int] * 4 + [_c.c_float, _c.c_int,
                                                                          _c.c_void_p]),
    "deeppcr_seq_backward": (_c.c_int, [_c.c_void_p] * 7 + [_c.c_int] * 4 + [_c.c_float, _c.c_int,
                                                                           _c.c_void_p]),
    "deeppcr_gated_scan_workspace_bytes": (_c.c_size_t, [_c.c_int] * 3),
    "deeppcr_gated_scan_forward": (_c.c_int, [_c.c_void_p, _c.c_longlong] * 2 +
                                   [_c.c_void_p] * 4 + [_c.c_int] * 5 +
                                   [_c.c_void_p, _c.c_size_t, _c.c_void_p]),
    "deeppcr_gated_scan_backward": (_c.c_int, [_c.c_void_p, _c.c_longlong] * 2 +
                                    [_c.c_void_p] * 4 + [_c.c_longlong] + [_c.c_void_p] * 4 +
                                    [_c.c_int] * 5 + [_c.c_void_p, _c.c_size_t, _c.c_void_p]),
    "deeppcr_gated_scan_step": (_c.c_int, [_c.c_void_p, _c.c_longlong] * 2 + [_c.c_void_p] * 3 +
                                [_c.c_int] * 4 + [_c.c_void_p]),
    "deeppcr_residual_norm_workspace_bytes": (_c.c_size_t, [_c.c_int] * 4),
    "deeppcr_residual_norm_forward": (_c.c_int, [_c.c_void_p] +
                                      [_c.c_void_p, _c.c_longlong] * 2 + [_c.c_void_p] * 7 +
                                      [_c.c_int] * 5 + [_c.c_float, _c.c_int, _c.c_void_p]),
    "deeppcr_residual_norm_backward": (_c.c_int, [_c.c_void_p] +
                                       [_c.c_void_p, _c.c_longlong] * 2 + [_c.c_void_p] * 13 +
                                       [_c.c_int] * 6 +
                                       [_c.c_void_p, _c.c_size_t, _c.c_void_p]),
    "deeppcr_orthogonalize_workspace_bytes": (_c.c_size_t, [_c.c_int] * 3),
    "deeppcr_orthogonalize": (_c.c_int, [_c.c_void_p] * 2 + [_c.c_int] * 4 + [_c.c_float] * 4 +
                              [_c.c_int, _c.c_void_p, _c.c_size_t, _c.c_void_p]),
    "deeppcr_profile_enable": (_c.c_int, [_c.c_int]),
    "deeppcr_profile_select": (_c.c_int, [_c.c_uint]),
    "deeppcr_profile_reset": (None, []),
    "deeppcr_profile_read": (_c.c_int, [_c.c_int, _c.POINTER(_c.c_longlong),
                                        _c.POINTER(_c.c_double), _c.POINTER(_c.c_double),
                                        _c.POINTER(_c.c_double)]),
}

_lib = None


class DeepPCRError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        msg = f"{where}: {status_string(status)} (status {status})"
        if status == EHIP:
            msg += f": {lib().deeppcr_last_error().decode()}"
        super().__init__(msg)


def lib() -> ctypes.CDLL:
    """The loaded library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2309_16318_amd.build`")
        l = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in SIGNATURES.items():
            f = getattr(l, name)
            f.restype = res
            f.argtypes = args
        _lib = l
    return _lib


def status_string(status: int) -> str:
    return lib().deeppcr_status_string(status).decode()


def workspace_bytes(op: int, B: int, L: int, w: int) -> int:
    return int(lib().deeppcr_workspace_bytes(op, B, L, w))


# ------------------------------------------------------------------ helpers
def _torch():
    import torch
    return torch


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _check(t, shape, name):
    torch = _torch()
    if t.dtype != torch.float32 or not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous float32 GPU tensor")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")


def _stream():
    return ctypes.c_void_p(_torch().cuda.current_stream().cuda_stream)


def _tensors(v):
    """The tensors of a call's arguments or of what it returns."""
    if isinstance(v, _torch().Tensor):
        yield v
    elif isinstance(v, (tuple, list)):
        for x in v:
            yield from _tensors(x)
    elif hasattr(v, "__dataclass_fields__"):
        yield from _tensors(tuple(vars(v).values()))


def _on(stream, call, *args):
    """`call` with `stream` as the current stream, so that outputs and workspaces
    which the binding makes come from that stream's memory: what the caller's own
    stream has freed may still be read by work on it.  Memory that crosses between
    the two streams is not given out again before both are past it."""
    cuda = _torch().cuda
    given = list(_tensors(args))
    for t in given:
        if t.is_cuda and t.device != stream.device:
            raise ValueError(f"the stream is on {stream.device}, the tensors on {t.device}")
    before = cuda.current_stream(stream.device)
    with cuda.stream(stream):
        result = call(*args)
    for t in given:
        if t.is_cuda:
            t.record_stream(stream)
    for t in _tensors(result):
        t.record_stream(before)
    return result


def _workspace(op, B, L, w, workspace, device):
    torch = _torch()
    n = workspace_bytes(op, B, L, w)
    if workspace is None:
        workspace = torch.empty(n, dtype=torch.uint8, device=device)
    return workspace, workspace.numel() * workspace.element_size()


# ------------------------------------------------------------- entry points
def pcr_solve_block_bidiag(J, r, x=None, transpose: int = 0, workspace=None, stream=None):
    """x with M x = r (transpose=0) or M^T x = r (transpose=1); J [B, L, w, w], r [B, L, w]."""
    if stream is not None:
        return _on(stream, pcr_solve_block_bidiag, J, r, x, transpose, workspace)
    torch = _torch()
    B, L, w = r.shape
    _check(J, (B, L, w, w), "J")
    _check(r, (B, L, w), "r")
    if x is None:
        x = torch.empty_like(r)
    _check(x, (B, L, w), "x")
    ws, nbytes = _workspace(OP_PCR, B, L, w, workspace, r.device)
    st = lib().pcr_solve_block_bidiag(_ptr(J), _ptr(r), _ptr(x), B, L, w, int(transpose),
                                      _ptr(ws), nbytes, _stream())
    if st != OK:
        raise DeepPCRError(st, "pcr_solve_block_bidiag")
    return x


def pcr_solve_block_bidiag_noalloc(J, r, x, transpose: int = 0, stream=None):
    """The same solve into the caller's x without a workspace: the library
    uses its own fixed scratch array and allocates nothing."""
    if stream is not None:
        return _on(stream, pcr_solve_block_bidiag_noalloc, J, r, x, transpose)
    B, L, w = r.shape
    _check(J, (B, L, w, w), "J")
    _check(r, (B, L, w), "r")
    _check(x, (B, L, w), "x")
    st = lib().pcr_solve_block_bidiag_noalloc(_ptr(J), _ptr(r), _ptr(x), B, L, w, int(transpose),
                                              _stream())
    if st != OK:
        raise DeepPCRError(st, "pcr_solve_block_bidiag_noalloc")
    return x


def pcr_solve_block_bidiag_chunked(J, r, G: int, x=None, transpose: int = 0, workspace=None,
                                   stream=None):
    """The same solve computed over G row chunks (chunk-local PCR keeping each
    chunk's coupling, a pass over the chunk ends, then the apply)."""
    if stream is not None:
        return _on(stream, pcr_solve_block_bidiag_chunked, J, r, G, x, transpose, workspace)
    torch = _torch()
    B, L, w = r.shape
    _check(J, (B, L, w, w), "J")
    _check(r, (B, L, w), "r")
    if x is None:
        x = torch.empty_like(r)
    _check(x, (B, L, w), "x")
    n = int(lib().deeppcr_chunked_workspace_bytes(B, L, w, int(G)))
    if workspace is None:
        workspace = torch.empty(max(n, 1), dtype=torch.uint8, device=r.device)
    nbytes = workspace.numel() * workspace.element_size()
    st = lib().pcr_solve_block_bidiag_chunked(_ptr(J), _ptr(r), _ptr(x), B, L, w, int(transpose),
                                              int(G), _ptr(workspace), nbytes, _stream())
    if st != OK:
        raise DeepPCRError(st, "pcr_solve_block_bidiag_chunked")
    return x


@dataclass
class ForwardResult:
    Z: object
    iters: int
    last_update: float
    status: int


def deeppcr_mlp_forward(W, bias, z0, Z=None, layer: int = TANH_MLP, alpha: float = 1.0,
                        tol: float = 1e-5, max_iter: int = 20, Z_init=None, workspace=None,
                        stream=None) -> ForwardResult:
    """Newton + PCR forward pass; raises on EINVAL/EHIP/EWORKSPACE and returns
    ENOCONV / ENONFINITE in ``status``."""
    if stream is not None:
        return _on(stream, deeppcr_mlp_forward,
                   W, bias, z0, Z, layer, alpha, tol, max_iter, Z_init, workspace)
    torch = _torch()
    L, w, _ = W.shape
    B = z0.shape[0]
    _check(W, (L, w, w), "W")
    _check(bias, (L, w), "bias")
    _check(z0, (B, w), "z0")
    if Z is None:
        Z = torch.empty((B, L, w), dtype=torch.float32, device=z0.device)
    _check(Z, (B, L, w), "Z")
    if Z_init is not None:
        _check(Z_init, (B, L, w), "Z_init")
    ws, nbytes = _workspace(OP_FWD, B, L, w, workspace, z0.device)
    iters = ctypes.c_int(0)
    last = ctypes.c_float(0.0)
    st = lib().deeppcr_mlp_forward(_ptr(W), _ptr(bias), _ptr(z0), _ptr(Z), B, L, w, int(layer),
                                   float(alpha), float(tol), int(max_iter), _ptr(Z_init),
                                   _ptr(ws), nbytes, ctypes.byref(iters), ctypes.byref(last),
                                   _stream())
    if st not in (OK, ENOCONV, ENONFINITE):
        raise DeepPCRError(st, "deeppcr_mlp_forward")
    return ForwardResult(Z, iters.value, last.value, st)


@dataclass
class NewtonStepResult:
    residual: float
    max_update: float
    max_abs: float
    status: int


def deeppcr_newton_step(J, F, Z, tol: float = 1e-5, workspace=None,
                        stream=None) -> NewtonStepResult:
    """One Newton + PCR iteration for caller-evaluated step values F and
    Jacobians J at the iterate Z (updated in place); ``status`` is OK once
    the update meets ``tol``, ENOCONV before, ENONFINITE on a NaN/Inf."""
    if stream is not None:
        return _on(stream, deeppcr_newton_step, J, F, Z, tol, workspace)
    B, L, w = Z.shape
    _check(J, (B, L, w, w), "J")
    _check(F, (B, L, w), "F")
    _check(Z, (B, L, w), "Z")
    ws, nbytes = _workspace(OP_PCR, B, L, w, workspace, Z.device)
    res, mx, mz = ctypes.c_float(0.0), ctypes.c_float(0.0), ctypes.c_float(0.0)
    st = lib().deeppcr_newton_step(_ptr(J), _ptr(F), _ptr(Z), B, L, w, float(tol), _ptr(ws),
                                   nbytes, ctypes.byref(res), ctypes.byref(mx), ctypes.byref(mz),
                                   _stream())
    if st not in (OK, ENOCONV, ENONFINITE):
        raise DeepPCRError(st, "deeppcr_newton_step")
    return NewtonStepResult(res.value, mx.value, mz.value, st)


@dataclass
class ResidualForwardResult:
    Z: object
    iters: int
    residual: float
    status: int


def deeppcr_mlp_forward_residual(W, bias, z0, Z=None, layer: int = TANH_MLP, alpha: float = 1.0,
                                 atol: float = 1e-4, rtol: float = 1e-4, max_iter: int = 15,
                                 Z_init=None, workspace=None,
                                 stream=None) -> ResidualForwardResult:
    """Newton + PCR forward pass stopped by the residual rule (defaults: the
    paper's forward-pass solver settings); raises on EINVAL/EHIP/EWORKSPACE
    and returns ENOCONV / ENONFINITE in ``status``."""
    if stream is not None:
        return _on(stream, deeppcr_mlp_forward_residual,
                   W, bias, z0, Z, layer, alpha, atol, rtol, max_iter, Z_init, workspace)
    torch = _torch()
    L, w, _ = W.shape
    B = z0.shape[0]
    _check(W, (L, w, w), "W")
    _check(bias, (L, w), "bias")
    _check(z0, (B, w), "z0")
    if Z is None:
        Z = torch.empty((B, L, w), dtype=torch.float32, device=z0.device)
    _check(Z, (B, L, w), "Z")
    if Z_init is not None:
        _check(Z_init, (B, L, w), "Z_init")
    ws, nbytes = _workspace(OP_FWD, B, L, w, workspace, z0.device)
    iters = ctypes.c_int(0)
    res = ctypes.c_float(0.0)
    st = lib().deeppcr_mlp_forward_residual(_ptr(W), _ptr(bias), _ptr(z0), _ptr(Z), B, L, w,
                                            int(layer), float(alpha), float(atol), float(rtol),
                                            int(max_iter), _ptr(Z_init), _ptr(ws), nbytes,
                                            ctypes.byref(iters), ctypes.byref(res),
                                            _stream())
    if st not in (OK, ENOCONV, ENONFINITE):
        raise DeepPCRError(st, "deeppcr_mlp_forward_residual")
    return ResidualForwardResult(Z, iters.value, res.value, st)


def deeppcr_mlp_backward(W, bias, z0, Z, G, layer: int = TANH_MLP, alpha: float = 1.0,
                         Lambda=None, dz0=None, dW=None, db=None, workspace=None, stream=None):
    """Transposed-PCR backward pass; returns (Lambda, dz0, dW, db)."""
    if stream is not None:
        return _on(stream, deeppcr_mlp_backward,
                   W, bias, z0, Z, G, layer, alpha, Lambda, dz0, dW, db, workspace)
    torch = _torch()
    L, w, _ = W.shape
    B = z0.shape[0]
    for t, shp, n in ((W, (L, w, w), "W"), (bias, (L, w), "bias"), (z0, (B, w), "z0"),
                      (Z, (B, L, w), "Z"), (G, (B, w), "G")):
        _check(t, shp, n)
    dev = z0.device
    Lambda = torch.empty((B, L, w), dtype=torch.float32, device=dev) if Lambda is None else Lambda
    dz0 = torch.empty((B, w), dtype=torch.float32, device=dev) if dz0 is None else dz0
    dW = torch.empty((L, w, w), dtype=torch.float32, device=dev) if dW is None else dW
    db = torch.empty((L, w), dtype=torch.float32, device=dev) if db is None else db
    for t, shp, n in ((Lambda, (B, L, w), "Lambda"), (dz0, (B, w), "dz0"), (dW, (L, w, w), "dW"),
                      (db, (L, w), "db")):
        _check(t, shp, n)
    ws, nbytes = _workspace(OP_BWD, B, L, w, workspace, dev)
    st = lib().deeppcr_mlp_backward(_ptr(W), _ptr(bias), _ptr(z0), _ptr(Z), _ptr(G),
                                    _ptr(Lambda), _ptr(dz0), _ptr(dW), _ptr(db), B, L, w,
                                    int(layer), float(alpha), _ptr(ws), nbytes, _stream())
    if st != OK:
        raise DeepPCRError(st, "deeppcr_mlp_backward")
    return Lambda, dz0, dW, db


def resnet_workspace_bytes(op: int, B: int, L: int, w: int, skip: int) -> int:
    return int(lib().deeppcr_resnet_workspace_bytes(op, B, L, w, skip))


def deeppcr_resnet_forward(W, bias, z0, skip: int, act: int = ACT_RELU, Z=None,
                           tol: float = 1e-5, max_iter: int = 20, Z_init=None, workspace=None,
                           stream=None) -> ForwardResult:
    """Newton + PCR forward pass of the collapsed-skip ResNet; raises on
    EINVAL/EHIP/EWORKSPACE and returns ENOCONV / ENONFINITE in ``status``."""
    if stream is not None:
        return _on(stream, deeppcr_resnet_forward,
                   W, bias, z0, skip, act, Z, tol, max_iter, Z_init, workspace)
    torch = _torch()
    L, w, _ = W.shape
    B = z0.shape[0]
    _check(W, (L, w, w), "W")
    _check(bias, (L, w), "bias")
    _check(z0, (B, w), "z0")
    if Z is None:
        Z = torch.empty((B, L, w), dtype=torch.float32, device=z0.device)
    _check(Z, (B, L, w), "Z")
    if Z_init is not None:
        _check(Z_init, (B, L, w), "Z_init")
    n = resnet_workspace_bytes(OP_FWD, B, L, w, skip)
    if workspace is None:
        workspace = torch.empty(max(n, 1), dtype=torch.uint8, device=z0.device)
    nbytes = workspace.numel() * workspace.element_size()
    iters = ctypes.c_int(0)
    last = ctypes.c_float(0.0)
    st = lib().deeppcr_resnet_forward(_ptr(W), _ptr(bias), _ptr(z0), _ptr(Z), B, L, w, int(skip),
                                      int(act), float(tol), int(max_iter), _ptr(Z_init),
                                      _ptr(workspace), nbytes, ctypes.byref(iters),
                                      ctypes.byref(last), _stream())
    if st not in (OK, ENOCONV, ENONFINITE):
        raise DeepPCRError(st, "deeppcr_resnet_forward")
    return ForwardResult(Z, iters.value, last.value, st)


def deeppcr_resnet_backward(W, z0, Z, G, skip: int, act: int = ACT_RELU, Lambda=None, dz0=None,
                            dW=None, db=None, workspace=None, stream=None):
    """Backward pass of the collapsed-skip ResNet; returns (Lambda, dz0, dW, db)."""
    if stream is not None:
        return _on(stream, deeppcr_resnet_backward,
                   W, z0, Z, G, skip, act, Lambda, dz0, dW, db, workspace)
    torch = _torch()
    L, w, _ = W.shape
    B = z0.shape[0]
    for t, shp, n in ((W, (L, w, w), "W"), (z0, (B, w), "z0"), (Z, (B, L, w), "Z"),
                      (G, (B, w), "G")):
        _check(t, shp, n)
    dev = z0.device
    Lambda = torch.empty((B, L, w), dtype=torch.float32, device=dev) if Lambda is None else Lambda
    dz0 = torch.empty((B, w), dtype=torch.float32, device=dev) if dz0 is None else dz0
    dW = torch.empty((L, w, w), dtype=torch.float32, device=dev) if dW is None else dW
    db = torch.empty((L, w), dtype=torch.float32, device=dev) if db is None else db
    for t, shp, n in ((Lambda, (B, L, w), "Lambda"), (dz0, (B, w), "dz0"), (dW, (L, w, w), "dW"),
                      (db, (L, w), "db")):
        _check(t, shp, n)
    n = resnet_workspace_bytes(OP_BWD, B, L, w, skip)
    if workspace is None:
        workspace = torch.empty(max(n, 1), dtype=torch.uint8, device=dev)
    nbytes = workspace.numel() * workspace.element_size()
    st = lib().deeppcr_resnet_backward(_ptr(W), _ptr(z0), _ptr(Z), _ptr(G), _ptr(Lambda),
                                       _ptr(dz0), _ptr(dW), _ptr(db), B, L, w, int(skip),
                                       int(act), _ptr(workspace), nbytes, _stream())
    if st != OK:
        raise DeepPCRError(st, "deeppcr_resnet_backward")
    return Lambda, dz0, dW, db


def deeppcr_resnet_seq_forward(W, bias, z0, skip: int, act: int = ACT_RELU, Z=None,
                               launch_per_layer: bool = False, stream=None):
    """Sequential GPU pass of the collapsed-skip ResNet; returns Z."""
    if stream is not None:
        return _on(stream, deeppcr_resnet_seq_forward, W, bias, z0, skip, act, Z, launch_per_layer)
    torch = _torch()
    L, w, _ = W.shape
    B = z0.shape[0]
    Z = torch.empty((B, L, w), dtype=torch.float32, device=z0.device) if Z is None else Z
    _check(Z, (B, L, w), "Z")
    st = lib().deeppcr_resnet_seq_forward(_ptr(W), _ptr(bias), _ptr(z0), _ptr(Z), B, L, w,
                                          int(skip), int(act), int(bool(launch_per_layer)),
                                          _stream())
    if st != OK:
        raise DeepPCRError(st, "deeppcr_resnet_seq_forward")
    return Z


def deeppcr_resnet_seq_backward(W, z0, Z, G, skip: int, act: int = ACT_RELU, Lambda=None,
                                dz0=None, launch_per_layer: bool = False, stream=None):
    """Sequential GPU adjoints of the collapsed-skip ResNet; returns (Lambda, dz0)."""
    if stream is not None:
        return _on(stream, deeppcr_resnet_seq_backward,
                   W, z0, Z, G, skip, act, Lambda, dz0, launch_per_layer)
    torch = _torch()
    L, w, _ = W.shape
    B = z0.shape[0]
    dev = z0.device
    Lambda = torch.empty((B, L, w), dtype=torch.float32, device=dev) if Lambda is None else Lambda
    dz0 = torch.empty((B, w), dtype=torch.float32, device=dev) if dz0 is None else dz0
    st = lib().deeppcr_resnet_seq_backward(_ptr(W), _ptr(z0), _ptr(Z), _ptr(G), _ptr(Lambda),
                                           _ptr(dz0), B, L, w, int(skip), int(act),
                                           int(bool(launch_per_layer)), _stream())
    if st != OK:
        raise DeepPCRError(st, "deeppcr_resnet_seq_backward")
    return Lambda, dz0


def deeppcr_seq_forward(W, bias, z0, Z=None, layer: int = TANH_MLP, alpha: float = 1.0,
                        launch_per_layer: bool = False, stream=None):
    """Sequential layer-by-layer forward pass on the GPU (the comparison baseline)."""
    if stream is not None:
        return _on(stream, deeppcr_seq_forward, W, bias, z0, Z, layer, alpha, launch_per_layer)
    torch = _torch()
    L, w, _ = W.shape
    B = z0.shape[0]
    for t, shp, n in ((W, (L, w, w), "W"), (bias, (L, w), "bias"), (z0, (B, w), "z0")):
        _check(t, shp, n)
    if Z is None:
        Z = torch.empty((B, L, w), dtype=torch.float32, device=z0.device)
    _check(Z, (B, L, w), "Z")
    st = lib().deeppcr_seq_forward(_ptr(W), _ptr(bias), _ptr(z0), _ptr(Z), B, L, w, int(layer),
                                   float(alpha), int(bool(launch_per_layer)), _stream())
    if st != OK:
        raise DeepPCRError(st, "deeppcr_seq_forward")
    return Z


def deeppcr_seq_backward(W, bias, z0, Z, G, layer: int = TANH_MLP, alpha: float = 1.0,
                         Lambda=None, dz0=None, launch_per_layer: bool = False, stream=None):
    """Sequential adjoint pass on the GPU; returns (Lambda, dz0)."""
    if stream is not None:
        return _on(stream, deeppcr_seq_backward,
                   W, bias, z0, Z, G, layer, alpha, Lambda, dz0, launch_per_layer)
    torch = _torch()
    L, w, _ = W.shape
    B = z0.shape[0]
    for t, shp, n in ((W, (L, w, w), "W"), (bias, (L, w), "bias"), (z0, (B, w), "z0"),
                      (Z, (B, L, w), "Z"), (G, (B, w), "G")):
        _check(t, shp, n)
    dev = z0.device
    Lambda = torch.empty((B, L, w), dtype=torch.float32, device=dev) if Lambda is None else Lambda
    dz0 = torch.empty((B, w), dtype=torch.float32, device=dev) if dz0 is None else dz0
    _check(Lambda, (B, L, w), "Lambda")
    _check(dz0, (B, w), "dz0")
    st = lib().deeppcr_seq_backward(_ptr(W), _ptr(bias), _ptr(z0), _ptr(Z), _ptr(G), _ptr(Lambda),
                                    _ptr(dz0), B, L, w, int(layer), float(alpha),
                                    int(bool(launch_per_layer)), _stream())
    if st != OK:
        raise DeepPCRError(st, "deeppcr_seq_backward")
    return Lambda, dz0


# ------------------------------------------------ recurrent language models
# A step of one token is a few microseconds on the GPU: what these calls do on
# the host is kept short (library functions and sizes looked up once, addresses
# passed as integers).
@functools.lru_cache(maxsize=None)
def _codes():
    torch = _torch()
    return {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}


@functools.lru_cache(maxsize=None)
def _entry(name):
    return getattr(lib(), name)


@functools.lru_cache(maxsize=None)
def _raw_stream():
    """The handle of a device's current stream, without a Python object for the
    stream where torch has that (2.5 us less per call)."""
    torch = _torch()
    get = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return get or (lambda index: torch.cuda.current_stream(index).cuda_stream)


def _dtype_code(t, name):
    code = _codes().get(t.dtype)
    if code is None:
        raise ValueError(f"{name} must be float32, bfloat16 or float16, not {t.dtype}")
    return code


def _addr(t):
    return None if t is None else t.data_ptr()


def _rows(t, shape, name, like):
    """Checks a sequence [.., w] of like's type on like's device whose rows lie
    a fixed stride apart (a slice of a wider tensor's last axis, say);
    returns that stride."""
    if t.dtype != like.dtype or t.device != like.device or not t.is_cuda:
        raise ValueError(f"{name} must be a {like.dtype} GPU tensor on {like.device}")
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    w = shape[-1]
    if t.is_contiguous():
        return w
    ld, n = None, 1
    for size, stride in zip(reversed(shape[:-1]), reversed(t.stride()[:-1])):
        if size > 1:
            if ld is None:
                ld = stride
            elif stride != ld * n:
                raise ValueError(f"the rows of {name} must lie a fixed stride apart")
        n *= size
    ld = w if ld is None else ld
    if (w > 1 and t.stride(-1) != 1) or ld < w:
        raise ValueError(f"the rows of {name} must be contiguous and apart")
    return ld


def _typed(t, shape, name, dtype, device):
    """Checks a contiguous tensor of the given type; None passes."""
    if t is None:
        return
    if t.dtype != dtype or t.device != device or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor on {device}")
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")


def _out(t, shape, name, dtype, device):
    """An output: checked if the caller gave it, else made."""
    if t is None:
        return _torch().empty(shape, dtype=dtype, device=device)
    _typed(t, shape, name, dtype, device)
    return t


def _launch(name, device, args):
    """Calls entry point `name` with `args` and the current stream of `device`, on
    `device`."""
    cuda = _torch().cuda
    if cuda.current_device() != device.index:
        with cuda.device(device):
            return _launch(name, device, args)
    st = _entry(name)(*args, _raw_stream()(device.index))
    if st != OK:
        raise DeepPCRError(st, name)


def _space(workspace, nbytes, device):
    if workspace is None:
        return _torch().empty(max(nbytes, 1), dtype=_torch().uint8, device=device), nbytes
    if workspace.device != device or not workspace.is_contiguous():
        raise ValueError(f"workspace must be a contiguous tensor on {device}")
    return workspace, workspace.numel() * workspace.element_size()


@functools.lru_cache(maxsize=1024)
def gated_scan_workspace_bytes(B: int, L: int, w: int) -> int:
    return int(lib().deeppcr_gated_scan_workspace_bytes(B, L, w))


def deeppcr_gated_scan_forward(a, u, x0=None, lengths=None, gate: int = GATE_DIRECT, x=None,
                               x_last=None, workspace=None, stream=None):
    """x_l = s_l x_{l-1} + r_l over [B, L, w] (direct: s = a, r = u; sigmoid:
    s = sigmoid(a), r = (1 - s) u) from x0; returns (x, x_last)."""
    if stream is not None:
        return _on(stream, deeppcr_gated_scan_forward,
                   a, u, x0, lengths, gate, x, x_last, workspace)
    torch = _torch()
    dt = _dtype_code(a, "a")
    B, L, w = a.shape
    dev = a.device
    lda, ldu = _rows(a, (B, L, w), "a", a), _rows(u, (B, L, w), "u", a)
    _typed(x0, (B, w), "x0", torch.float32, dev)
    _typed(lengths, (B,), "lengths", torch.int32, dev)
    x = _out(x, (B, L, w), "x", a.dtype, dev)
    x_last = _out(x_last, (B, w), "x_last", torch.float32, dev)
    ws, nbytes = _space(workspace, gated_scan_workspace_bytes(B, L, w), dev)
    _launch("deeppcr_gated_scan_forward", dev,
            (_addr(a), lda, _addr(u), ldu, _addr(x0), _addr(lengths), _addr(x), _addr(x_last), B, L, w,
             int(gate), dt, _addr(ws), nbytes))
    return x, x_last


def deeppcr_gated_scan_backward(a, u, x, g, g_last=None, x0=None, lengths=None,
                                gate: int = GATE_DIRECT, da=None, du=None, dx0=None,
                                workspace=None, stream=None):
    """Backward pass of the gated scan from its output x (rounded to its type, as da
    then is twice), for g = dLoss/dx and g_last = dLoss/dx_last; returns
    (da, du, dx0).  u may be None for the direct gate."""
    if stream is not None:
        return _on(stream, deeppcr_gated_scan_backward,
                   a, u, x, g, g_last, x0, lengths, gate, da, du, dx0, workspace)
    torch = _torch()
    dt = _dtype_code(a, "a")
    B, L, w = a.shape
    dev = a.device
    lda, ldg = _rows(a, (B, L, w), "a", a), _rows(g, (B, L, w), "g", a)
    ldu = 0 if u is None else _rows(u, (B, L, w), "u", a)
    _typed(x, (B, L, w), "x", a.dtype, dev)
    for t, n in ((x0, "x0"), (g_last, "g_last")):
        _typed(t, (B, w), n, torch.float32, dev)
    _typed(lengths, (B,), "lengths", torch.int32, dev)
    da = _out(da, (B, L, w), "da", a.dtype, dev)
    du = _out(du, (B, L, w), "du", a.dtype, dev)
    dx0 = _out(dx0, (B, w), "dx0", torch.float32, dev)
    ws, nbytes = _space(workspace, gated_scan_workspace_bytes(B, L, w), dev)
    _launch("deeppcr_gated_scan_backward", dev,
            (_addr(a), lda, _addr(u), ldu, _addr(x), _addr(x0), _addr(lengths), _addr(g), ldg,
             _addr(g_last), _addr(da), _addr(du), _addr(dx0), B, L, w, int(gate), dt, _addr(ws),
             nbytes))
    return da, du, dx0


def deeppcr_gated_scan_step(a, u, state, gate: int = GATE_DIRECT, x=None, state_out=None,
                            stream=None):
    """One row [B, w] of the gated scan on running float32 states; writes the
    new states to state_out (default: state, in place) and returns x, the
    states in a's type."""
    if stream is not None:
        return _on(stream, deeppcr_gated_scan_step, a, u, state, gate, x, state_out)
    torch = _torch()
    dt = _dtype_code(a, "a")
    B, w = a.shape
    dev = a.device
    lda, ldu = _rows(a, (B, w), "a", a), _rows(u, (B, w), "u", a)
    x = _out(x, (B, w), "x", a.dtype, dev)
    _typed(state, (B, w), "state", torch.float32, dev)
    if state_out is None:
        state_out = state
    else:
        _typed(state_out, (B, w), "state_out", torch.float32, dev)
    _launch("deeppcr_gated_scan_step", dev,
            (_addr(a), lda, _addr(u), ldu, _addr(state), _addr(state_out), _addr(x), B, w, int(gate),
             dt))
    return x


@dataclass
class NormResult:
    x_out: object
    h: object
    rstd_post: object
    rstd_pre: object


@dataclass
class NormGrads:
    dx: object
    dy: object
    dz: object
    dw_post: object
    dscale: object
    dw_pre: object


@functools.lru_cache(maxsize=1024)
def residual_norm_workspace_bytes(B: int, L: int, w: int, z_per_seq: bool = False) -> int:
    return int(lib().deeppcr_residual_norm_workspace_bytes(B, L, w, int(bool(z_per_seq))))


def _norm_inputs(x, y, z, w_post, scale, w_pre):
    """Checks the pieces; returns (dtype code, B, L, w, ldy, ldz, z_per_seq)."""
    torch = _torch()
    dt = _dtype_code(x, "x")
    B, L, w = x.shape
    _typed(x, (B, L, w), "x", x.dtype, x.device)
    if not x.is_cuda:
        raise ValueError("x must be a GPU tensor")
    ldy = 0 if y is None else _rows(y, (B, L, w), "y", x)
    per_seq = z is not None and z.dim() == 2
    ldz = 0 if z is None else _rows(z, (B, w) if per_seq else (B, L, w), "z", x)
    for t, n in ((w_post, "w_post"), (scale, "scale"), (w_pre, "w_pre")):
        _typed(t, (w,), n, torch.float32, x.device)
    return dt, B, L, w, ldy, ldz, int(per_seq)


def deeppcr_residual_norm_forward(x, y=None, z=None, w_post=None, scale=None, w_pre=None,
                                  gate: int = GATE_NONE, eps: float = 1e-6, x_out=None, h=None,
                                  stream=None) -> NormResult:
    """x_out = x + scale act(z) norm(y; w_post), h = norm(x_out; w_pre) over
    [B, L, w]; each piece that is None is left out (without y: h = norm(x)).
    z [B, L, w], or [B, w] for one gate per sequence."""
    if stream is not None:
        return _on(stream, deeppcr_residual_norm_forward,
                   x, y, z, w_post, scale, w_pre, gate, eps, x_out, h)
    torch = _torch()
    dt, B, L, w, ldy, ldz, per_seq = _norm_inputs(x, y, z, w_post, scale, w_pre)
    dev = x.device
    if x_out is not None or y is not None:
        x_out = _out(x_out, (B, L, w), "x_out", x.dtype, dev)
    if h is not None or w_pre is not None:
        h = _out(h, (B, L, w), "h", x.dtype, dev)
    rpost = rpre = None
    if w_post is not None:
        rpost = _out(None, (B, L), "rstd_post", torch.float32, dev)
    if w_pre is not None:
        rpre = _out(None, (B, L), "rstd_pre", torch.float32, dev)
    _launch("deeppcr_residual_norm_forward", dev,
            (_addr(x), _addr(y), ldy, _addr(z), ldz, _addr(w_post), _addr(scale), _addr(w_pre),
             _addr(x_out), _addr(h), _addr(rpost), _addr(rpre), B, L, w, int(gate), per_seq,
             float(eps), dt))
    return NormResult(x_out if y is not None else x, h, rpost, rpre)


def deeppcr_residual_norm_backward(x, y=None, rstd_post=None, rstd_pre=None, dx_out=None, dh=None,
                                   z=None, w_post=None, scale=None, w_pre=None,
                                   gate: int = GATE_NONE, dx=None, dy=None, dz=None,
                                   workspace=None, stream=None) -> NormGrads:
    """Gradients of the residual norm from its inputs, its statistics and
    dx_out, dh; those of pieces that are None are None."""
    if stream is not None:
        return _on(stream, deeppcr_residual_norm_backward,
                   x, y, rstd_post, rstd_pre, dx_out, dh, z, w_post, scale, w_pre, gate, dx, dy,
                   dz, workspace)
    torch = _torch()
    dt, B, L, w, ldy, ldz, per_seq = _norm_inputs(x, y, z, w_post, scale, w_pre)
    dev = x.device
    for t, n in ((rstd_post, "rstd_post"), (rstd_pre, "rstd_pre")):
        _typed(t, (B, L), n, torch.float32, dev)

    def out(given, like, name, dtype=x.dtype):
        return None if like is None else _out(given, like.shape, name, dtype, dev)

    for t, n in ((dx_out, "dx_out"), (dh, "dh")):
        _typed(t, (B, L, w), n, x.dtype, dev)
    dx, dy, dz = out(dx, x, "dx"), out(dy, y, "dy"), out(dz, z, "dz")
    dpost, dscale, dpre = (out(None, p, "", torch.float32) for p in (w_post, scale, w_pre))
    ws, nbytes = _space(workspace, residual_norm_workspace_bytes(B, L, w, per_seq), dev)
    _launch("deeppcr_residual_norm_backward", dev,
            (_addr(x), _addr(y), ldy, _addr(z), ldz, _addr(w_post), _addr(scale), _addr(w_pre),
             _addr(rstd_post), _addr(rstd_pre), _addr(dx_out), _addr(dh), _addr(dx), _addr(dy),
             _addr(dz), _addr(dpost), _addr(dscale), _addr(dpre), B, L, w, int(gate), per_seq, dt,
             _addr(ws), nbytes))
    return NormGrads(dx, dy, dz, dpost, dscale, dpre)


@functools.lru_cache(maxsize=1024)
def orthogonalize_workspace_bytes(N: int, m: int, n: int) -> int:
    return int(lib().deeppcr_orthogonalize_workspace_bytes(N, m, n))


def deeppcr_orthogonalize(G, X=None, steps: int = 5, coeffs=(3.4445, -4.7750, 2.0315),
                          eps: float = 1e-7, workspace=None, stream=None):
    """The orthogonalised update of a stack of gradients G [N, m, n] (or one,
    [m, n]): Newton-Schulz steps of the polynomial `coeffs` on G / (|G| + eps);
    X may be G."""
    if stream is not None:
        return _on(stream, deeppcr_orthogonalize, G, X, steps, coeffs, eps, workspace)
    torch = _torch()
    dt = _dtype_code(G, "G")
    if not G.is_cuda or G.dim() not in (2, 3):
        raise ValueError("G must be a GPU tensor [N, m, n] or [m, n]")
    N, (m, n) = (1 if G.dim() == 2 else G.shape[0]), G.shape[-2:]
    _typed(G, G.shape, "G", G.dtype, G.device)
    X = _out(X, G.shape, "X", G.dtype, G.device)
    ws, nbytes = _space(workspace, orthogonalize_workspace_bytes(N, m, n), G.device)
    ca, cb, cc = (float(c) for c in coeffs)
    _launch("deeppcr_orthogonalize", G.device,
            (_addr(G), _addr(X), N, m, n, int(steps), ca, cb, cc, float(eps), dt, _addr(ws),
             nbytes))
    return X


def release_thread_state() -> None:
    """Frees the calling thread's pinned read-back buffer and profiler events."""
    lib().deeppcr_release_thread_state()


# ---------------------------------------------------------- instrumentation
def profile_enable(on: bool = True) -> None:
    lib().deeppcr_profile_enable(1 if on else 0)


def profile_select(kclasses) -> None:
    """Times only the given kernel classes (KCLASS_* values) while enabled."""
    mask = 0
    for c in kclasses:
        mask |= 1 << int(c)
    lib().deeppcr_profile_select(mask)


def profile_reset() -> None:
    lib().deeppcr_profile_reset()


def profile_read(kclass: int) -> dict:
    n = ctypes.c_longlong(0)
    ms = ctypes.c_double(0)
    by = ctypes.c_double(0)
    fl = ctypes.c_double(0)
    st = lib().deeppcr_profile_read(kclass, ctypes.byref(n), ctypes.byref(ms), ctypes.byref(by),
                                    ctypes.byref(fl))
    if st != OK:
        raise DeepPCRError(st, "deeppcr_profile_read")
    return {"launches": n.value, "ms": ms.value, "bytes": by.value, "flops": fl.value}
