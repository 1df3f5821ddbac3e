"""ctypes binding of libsolar.so: same names as the C entry points of
include/solar.h, argument marshalling only.  torch supplies device memory and the
stream; every step of the computation runs in the library's HIP kernels.  There
is no fallback: if the library is missing, importing this module raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libsolar.so")

SOLAR_OK = 0
SOLAR_ERR_NOT_CONVERGED = 5
SOLAR_ERR_SCRATCH_LIMIT = 6
SOLAR_DEBUG_EIG_MAX_ITER = 0
SOLAR_DEBUG_FORCE_GUARDED_PASS = 1
SOLAR_STATIC_SCRATCH_BYTES = 48 * 1024 * 1024
SOLAR_F32 = 0
SOLAR_BF16 = 1
SOLAR_ATTN_SEQ_SOFTMAX = 0
SOLAR_ATTN_EIGEN_SOFTMAX = 1
SOLAR_ATTN_LINEAR = 2
SOLAR_ROTARY_HALF = 0
SOLAR_ROTARY_INTERLEAVED = 1
SOLAR_ROTARY_UNSCALED = 0
SOLAR_ROTARY_LINEAR = 1
SOLAR_ROTARY_BASE = 2
SOLAR_ROTARY_BY_PARTS = 3

if not os.path.exists(LIB_PATH):
    raise ImportError(
        f"{LIB_PATH} is missing: build it with `python -m paper_2603_02561_amd.build` "
        "(hipcc, gfx950). There is no CPU fallback.")

_lib = ctypes.CDLL(LIB_PATH)
_vp, _ci, _cf, _sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_size_t
_lib.solar_status_string.argtypes = [_ci]
_lib.solar_status_string.restype = ctypes.c_char_p
_lib.solar_workspace_bytes.argtypes = [_ci, _ci, _ci, _ci, _ci, _ci]
_lib.solar_workspace_bytes.restype = _sz
_lib.solar_gram.argtypes = [_vp, _vp, _ci, _ci, _ci, _ci, _vp, _vp, _sz, _vp]
_lib.solar_gram.restype = _ci
_lib.solar_svd_factorize.argtypes = [_vp, _vp, _ci, _ci, _ci, _ci, _ci, _vp, _vp, _vp, _vp, _vp,
                                     _sz, _vp]
_lib.solar_svd_factorize.restype = _ci
_lib.solar_svd_factorize_static.argtypes = [_vp, _vp, _ci, _ci, _ci, _ci, _ci, _vp, _vp, _vp, _vp, _vp]
_lib.solar_svd_factorize_static.restype = _ci
_lib.solar_svd_attention.argtypes = [_vp, _vp, _vp, _vp, _vp, _ci, _ci, _ci, _ci, _ci, _cf, _ci,
                                     _ci, _vp, _vp, _sz, _vp]
_lib.solar_svd_attention.restype = _ci
_lib.solar_svd_attention_from_x.argtypes = [_vp, _vp, _vp, _vp, _vp, _ci, _ci, _ci, _ci, _ci, _cf, _ci, _vp, _vp,
                                            _sz, _vp]
_lib.solar_svd_attention_from_x.restype = _ci
_lib.solar_dense_attention_ref.argtypes = [_vp, _vp, _vp, _ci, _ci, _ci, _ci, _cf, _ci, _vp, _vp,
                                           _sz, _vp]
_lib.solar_dense_attention_ref.restype = _ci
_lib.solar_rsvd_workspace_bytes.argtypes = [_ci, _ci, _ci, _ci]
_lib.solar_rsvd_workspace_bytes.restype = _sz
_lib.solar_svd_factorize_rsvd.argtypes = [_vp, _vp, _ci, _ci, _ci, _ci, _ci, _vp, _ci, _vp, _vp, _vp,
                                          _vp, _vp, _sz, _vp]
_lib.solar_svd_factorize_rsvd.restype = _ci
_lib.solar_linear_attention.argtypes = [_vp, _vp, _vp, _ci, _ci, _ci, _ci, _cf, _ci, _vp, _vp, _sz, _vp]
_lib.solar_linear_attention.restype = _ci
_lib.solar_apply_weights.argtypes = [_vp, _vp, _ci, _ci, _ci, _ci, _vp, _vp]
_lib.solar_apply_weights.restype = _ci
_lib.solar_svd_backward.argtypes = [_vp, _vp, _vp, _vp, _vp, _ci, _ci, _ci, _ci, _cf, _vp, _vp, _sz, _vp]
_lib.solar_svd_backward.restype = _ci
_cd, _i64 = ctypes.c_double, ctypes.c_int64
_lib.solar_rotary_frequencies.argtypes = [_ci, _cd, _ci, _cd, _ci, _cd, _cd, _vp]
_lib.solar_rotary_frequencies.restype = _ci
_lib.solar_rotary.argtypes = [_vp, _vp, _vp, _vp, _vp, _ci, _ci, _ci, _ci, _ci, _ci, _ci, _ci, _cf, _ci, _vp, _vp, _vp, _vp]
_lib.solar_rotary.restype = _ci
_lib.solar_decay_workspace_bytes.argtypes = [_ci, _ci, _ci, _ci, _ci, _ci, _ci]
_lib.solar_decay_workspace_bytes.restype = _sz
_lib.solar_decay_attention.argtypes = [_vp, _vp, _vp, _vp, _vp, _vp, _ci, _ci, _ci, _ci, _ci, _cf, _ci, _vp, _vp, _vp, _vp,
                                       _sz, _vp]
_lib.solar_decay_attention.restype = _ci
_lib.solar_decay_attention_backward.argtypes = [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _ci, _ci, _ci, _ci, _ci, _cf, _ci,
                                                _vp, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]
_lib.solar_decay_attention_backward.restype = _ci
_lib.solar_layer_norm.argtypes = [_vp, _vp, _vp, _ci, _ci, _ci, _cf, _ci, _ci, _vp, _vp, _vp, _vp]
_lib.solar_layer_norm.restype = _ci
_lib.solar_layer_norm_workspace_bytes.argtypes = [_ci, _ci, _ci]
_lib.solar_layer_norm_workspace_bytes.restype = _sz
_lib.solar_layer_norm_backward.argtypes = [_vp, _vp, _vp, _vp, _vp, _ci, _ci, _ci, _ci, _ci, _vp, _vp, _vp, _vp, _sz, _vp]
_lib.solar_layer_norm_backward.restype = _ci
_lib.solar_info_status.argtypes = [_vp, _ci]
_lib.solar_info_status.restype = _ci
_lib.solar_debug_option.argtypes = [_ci, _ci]
_lib.solar_debug_option.restype = _ci
_lib.solar_phase_timing_begin.argtypes = []
_lib.solar_phase_timing_begin.restype = None
_lib.solar_phase_timing_end.argtypes = [ctypes.POINTER(ctypes.c_float)]
_lib.solar_phase_timing_end.restype = _ci


class SolarError(RuntimeError):
    def __init__(self, code: int):
        self.code = code
        super().__init__(f"solar status {code}: {solar_status_string(code)}")


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream() -> ctypes.c_void_p:
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return SOLAR_F32
    if t.dtype == torch.bfloat16:
        return SOLAR_BF16
    raise TypeError(f"X and Q must be float32 or bfloat16, got {t.dtype}")


def _check(*tensors):
    for t in tensors:
        if t is not None and (not t.is_cuda or not t.is_contiguous()):
            raise ValueError("tensors must be contiguous CUDA tensors")


def solar_status_string(code: int) -> str:
    return _lib.solar_status_string(int(code)).decode()


def solar_workspace_bytes(B: int, N: int, d: int, r: int, M: int, dtype_code: int) -> int:
    return int(_lib.solar_workspace_bytes(B, N, d, r, M, dtype_code))


def solar_info_status(info) -> int:
    """Status over a factorization's per-user info (waits for the device and copies it to the host)."""
    host = info.detach().to("cpu", torch.int32).contiguous()
    return int(_lib.solar_info_status(ctypes.c_void_p(host.data_ptr()), host.numel()))


def solar_debug_option(key: int, value: int) -> int:
    return int(_lib.solar_debug_option(int(key), int(value)))


def solar_phase_timing_begin() -> None:
    _lib.solar_phase_timing_begin()


def solar_phase_timing_end():
    """Returns (calls, [gram_ms, eig_ms, project_ms]) summed over the timed calls."""
    buf = (ctypes.c_float * 3)()
    n = _lib.solar_phase_timing_end(buf)
    return int(n), [float(buf[i]) for i in range(3)]


def solar_gram(X, lengths, G, workspace, raise_on_error: bool = True) -> int:
    _check(X, lengths, G, workspace)
    B, N, d = X.shape
    rc = _lib.solar_gram(_ptr(X), _ptr(lengths), B, N, d, _dtype_code(X), _ptr(G), _ptr(workspace),
                         workspace.numel() * workspace.element_size(), _stream())
    if rc != SOLAR_OK and raise_on_error:
        raise SolarError(rc)
    return rc


def solar_svd_factorize(X, lengths, r: int, S, V, P, info, workspace,
                        raise_on_error: bool = True) -> int:
    _check(X, lengths, S, V, P, info, workspace)
    B, N, d = X.shape
    rc = _lib.solar_svd_factorize(_ptr(X), _ptr(lengths), B, N, d, int(r), _dtype_code(X), _ptr(S),
                                  _ptr(V), _ptr(P), _ptr(info), _ptr(workspace),
                                  workspace.numel() * workspace.element_size(), _stream())
    if rc != SOLAR_OK and raise_on_error:
        raise SolarError(rc)
    return rc


def solar_svd_factorize_static(X, lengths, r: int, S, V, P, info, raise_on_error: bool = True) -> int:
    """solar_svd_factorize with the library's built-in scratch array instead of a workspace."""
    _check(X, lengths, S, V, P, info)
    B, N, d = X.shape
    rc = _lib.solar_svd_factorize_static(_ptr(X), _ptr(lengths), B, N, d, int(r), _dtype_code(X), _ptr(S),
                                         _ptr(V), _ptr(P), _ptr(info), _stream())
    if rc != SOLAR_OK and raise_on_error:
        raise SolarError(rc)
    return rc


def solar_rsvd_workspace_bytes(B: int, N: int, d: int, r: int) -> int:
    return int(_lib.solar_rsvd_workspace_bytes(B, N, d, r))


def solar_svd_factorize_rsvd(X, lengths, r: int, Omega, n_iter: int, S, V, P, info, workspace,
                             raise_on_error: bool = True) -> int:
    _check(X, lengths, Omega, S, V, P, info, workspace)
    B, N, d = X.shape
    rc = _lib.solar_svd_factorize_rsvd(_ptr(X), _ptr(lengths), B, N, d, int(r), _dtype_code(X),
                                       _ptr(Omega), int(n_iter), _ptr(S), _ptr(V), _ptr(P), _ptr(info),
                                       _ptr(workspace), workspace.numel() * workspace.element_size(),
                                       _stream())
    if rc != SOLAR_OK and raise_on_error:
        raise SolarError(rc)
    return rc


def solar_svd_attention(Q, S, V, P, lengths, N: int, scale: float, mode: int, O, workspace=None,
                        raise_on_error: bool = True) -> int:
    _check(Q, S, V, P, lengths, O, workspace)
    B, M, d = Q.shape
    r = V.shape[2]
    wsb = 0 if workspace is None else workspace.numel() * workspace.element_size()
    rc = _lib.solar_svd_attention(_ptr(Q), _ptr(S), _ptr(V), _ptr(P), _ptr(lengths), B, int(N), d,
                                  r, M, float(scale), int(mode), _dtype_code(Q), _ptr(O),
                                  _ptr(workspace), wsb, _stream())
    if rc != SOLAR_OK and raise_on_error:
        raise SolarError(rc)
    return rc


def solar_svd_attention_from_x(Q, X, S, V, lengths, scale: float, O, raise_on_error: bool = True) -> int:
    _check(Q, X, S, V, lengths, O)
    B, M, d = Q.shape
    N = X.shape[1]
    r = V.shape[2]
    rc = _lib.solar_svd_attention_from_x(_ptr(Q), _ptr(X), _ptr(S), _ptr(V), _ptr(lengths), B, N, d, r, M,
                                         float(scale), _dtype_code(Q), _ptr(O), None, 0, _stream())
    if rc != SOLAR_OK and raise_on_error:
        raise SolarError(rc)
    return rc


def solar_dense_attention_ref(Q, X, lengths, scale: float, O, workspace=None,
                              raise_on_error: bool = True) -> int:
    _check(Q, X, lengths, O, workspace)
    B, M, d = Q.shape
    N = X.shape[1]
    wsb = 0 if workspace is None else workspace.numel() * workspace.element_size()
    rc = _lib.solar_dense_attention_ref(_ptr(Q), _ptr(X), _ptr(lengths), B, N, d, M, float(scale),
                                        _dtype_code(Q), _ptr(O), _ptr(workspace), wsb, _stream())
    if rc != SOLAR_OK and raise_on_error:
        raise SolarError(rc)
    return rc


def solar_svd_backward(S, V, P, S_bar, V_bar, gap_rel: float, dX, workspace,
                       raise_on_error: bool = True) -> int:
    _check(S, V, P, S_bar, V_bar, dX, workspace)
    B, N, r = P.shape
    d = V.shape[1]
    rc = _lib.solar_svd_backward(_ptr(S), _ptr(V), _ptr(P), _ptr(S_bar), _ptr(V_bar), B, N, d, r,
                                 float(gap_rel), _ptr(dX), _ptr(workspace),
                                 workspace.numel() * workspace.element_size(), _stream())
    if rc != SOLAR_OK and raise_on_error:
        raise SolarError(rc)
    return rc


def solar_linear_attention(Q, X, lengths, scale: float, O, workspace, raise_on_error: bool = True) -> int:
    _check(Q, X, lengths, O, workspace)
    B, M, d = Q.shape
    N = X.shape[1]
    rc = _lib.solar_linear_attention(_ptr(Q), _ptr(X), _ptr(lengths), B, N, d, M, float(scale),
                                     _dtype_code(Q), _ptr(O), _ptr(workspace),
                                     workspace.numel() * workspace.element_size(), _stream())
    if rc != SOLAR_OK and raise_on_error:
        raise SolarError(rc)
    return rc


def solar_apply_weights(In, W, Out, raise_on_error: bool = True) -> int:
    _check(In, W, Out)
    d = In.shape[-1]
    rows = In.numel() // d
    rc = _lib.solar_apply_weights(_ptr(In), _ptr(W), rows, d, _dtype_code(In), _dtype_code(Out), _ptr(Out),
                                  _stream())
    if rc != SOLAR_OK and raise_on_error:
        raise SolarError(rc)
    return rc


# ---------------------------------------------------------------------------------------
# Sequence operators.  Tensors of heads [B,N,heads,D] may be views with any strides that include/solar.h allows (a slice of
# a packed projection, [B,heads,N,D] transposed); the calls go to the tensors' device and its current stream.

# the current stream's handle without the Stream object around it, which takes as long to make as a launch
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _run(fn, tensors, args, raise_on_error: bool) -> int:
    """fn(*args, stream) on the device that all tensors are on."""
    dev = -1
    for t in tensors:
        if t is not None:
            i = t.get_device()
            if i < 0:
                raise ValueError("tensors must be CUDA tensors")
            if dev < 0:
                dev = i
            elif i != dev:
                raise ValueError("tensors must be on one device")
    stream = torch.cuda.current_stream(dev).cuda_stream if _raw_stream is None else _raw_stream(dev)
    if dev == torch.cuda.current_device():
        rc = fn(*args, stream)
    else:
        with torch.cuda.device(dev):
            rc = fn(*args, stream)
    if rc != SOLAR_OK and raise_on_error:
        raise SolarError(rc)
    return rc


def _like(name: str, t: Optional[torch.Tensor], dtype, shape):
    """data_ptr of a contiguous tensor of this type and shape, None for None."""
    if t is None:
        return None
    if t.dtype != dtype or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {shape}, got {t.dtype} {tuple(t.shape)}")
    return t.data_ptr()


def _heads(dtype, **tensors):
    """The strides of tensors of heads, given as (tensor, shape), as the library takes them: None where all are contiguous."""
    plain = True
    for name, (t, shape) in tensors.items():
        if t.dtype != dtype or t.shape != shape:
            raise ValueError(f"{name} must be a {dtype} tensor of shape {tuple(shape)}, got {t.dtype} {tuple(t.shape)}")
        if not t.is_contiguous():
            plain = False
            if t.stride(3) != 1 and shape[3] > 1:
                raise ValueError(f"the columns of {name} must be contiguous")
    if plain:
        return None
    return (_i64 * (3 * len(tensors)))(*[x for t, _ in tensors.values() for x in t.stride()[:3]])


def _scratch(workspace: Optional[torch.Tensor]):
    if workspace is None:
        return None, 0
    if not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size()


def solar_rotary_frequencies(rot: int, base: float = 10000.0, scaling: int = SOLAR_ROTARY_UNSCALED, factor: float = 1.0,
                             original_length: int = 0, turns_low: float = 1.0, turns_high: float = 32.0) -> torch.Tensor:
    """[rot/2] double on the host; copy it to the device once."""
    freq = torch.empty(max(int(rot) // 2, 1), dtype=torch.float64)
    rc = _lib.solar_rotary_frequencies(int(rot), float(base), int(scaling), float(factor), int(original_length),
                                       float(turns_low), float(turns_high), freq.data_ptr())
    if rc != SOLAR_OK:
        raise SolarError(rc)
    return freq


def solar_rotary(Q, K, freq, Qout, Kout, positions=None, lengths=None, layout: int = SOLAR_ROTARY_HALF,
                 inverse: bool = False, amplitude: float = 1.0, raise_on_error: bool = True) -> int:
    """Rotates the first 2 * len(freq) columns of every head of Q [B,N,H,D] and K [B,N,Hkv,D] (K and Kout may be None)."""
    code = _dtype_code(Q)
    B, N, H, D = Q.shape
    if (K is None) != (Kout is None):
        raise ValueError("K and Kout go together")
    k, ko = (Q, Qout) if K is None else (K, Kout)
    Hkv = k.shape[2]
    st = _heads(Q.dtype, Q=(Q, Q.shape), K=(k, (B, N, Hkv, D)), Qout=(Qout, Q.shape), Kout=(ko, (B, N, Hkv, D)))
    args = (Q.data_ptr(), None if K is None else K.data_ptr(), _like("lengths", lengths, torch.int32, (B,)),
            _like("positions", positions, torch.int32, (B, N)), _like("freq", freq, torch.float64, (freq.numel(),)), B, N, H,
            Hkv, D, 2 * freq.numel(), int(layout), int(inverse), float(amplitude), code, st,
            Qout.data_ptr(), None if Kout is None else Kout.data_ptr())
    return _run(_lib.solar_rotary, (Q, K, freq, Qout, Kout, positions, lengths), args, raise_on_error)


def solar_decay_workspace_bytes(B: int, N: int, H: int, Hkv: int, D: int, dtype_code: int, backward: bool) -> int:
    return int(_lib.solar_decay_workspace_bytes(B, N, H, Hkv, D, dtype_code, int(backward)))


def solar_decay_attention(Q, K, V, log_decay, lengths, scale: float, O, state_in, state_out, workspace=None,
                          raise_on_error: bool = True) -> int:
    """O and state_out from Q [B,N,H,D], K and V [B,N,Hkv,D]; Q and O may be None (the state alone)."""
    code = _dtype_code(K)
    B, N, Hkv, D = K.shape
    H = log_decay.numel()
    shared = K.shape
    if O is None:
        st = _heads(K.dtype, Q=(K, shared), K=(K, shared), V=(V, shared), O=(K, shared))
    else:
        st = _heads(K.dtype, Q=(Q, (B, N, H, D)), K=(K, shared), V=(V, shared), O=(O, (B, N, H, D)))
    ws, wsb = _scratch(workspace)
    args = (None if O is None else Q.data_ptr(), K.data_ptr(), V.data_ptr(),
            _like("log_decay", log_decay, torch.float32, (H,)), _like("lengths", lengths, torch.int32, (B,)),
            _like("state_in", state_in, torch.float32, (B, H, D, D)), B, N, H, Hkv, D, float(scale), code,
            st, None if O is None else O.data_ptr(),
            _like("state_out", state_out, torch.float32, (B, H, D, D)), ws, wsb)
    return _run(_lib.solar_decay_attention,
                (Q if O is not None else None, K, V, log_decay, lengths, O, state_in, state_out, workspace), args,
                raise_on_error)


def solar_decay_attention_backward(Q, K, V, dO, log_decay, lengths, scale: float, state_in, dstate_out, dQ, dK, dV,
                                   dstate_in, dlog_decay, workspace, raise_on_error: bool = True) -> int:
    """Gradients of solar_decay_attention; state_in, dstate_out, dstate_in and dlog_decay may be None."""
    code = _dtype_code(Q)
    B, N, H, D = Q.shape
    Hkv = K.shape[2]
    shape, shared, dt = (B, N, H, D), (B, N, Hkv, D), Q.dtype
    st = _heads(dt, Q=(Q, shape), K=(K, shared), V=(V, shared), dO=(dO, shape), dQ=(dQ, shape), dK=(dK, shared),
                dV=(dV, shared))
    ws, wsb = _scratch(workspace)
    states = (B, H, D, D)
    args = (Q.data_ptr(), K.data_ptr(), V.data_ptr(), dO.data_ptr(), _like("log_decay", log_decay, torch.float32, (H,)),
            _like("lengths", lengths, torch.int32, (B,)), _like("state_in", state_in, torch.float32, states),
            _like("dstate_out", dstate_out, torch.float32, states), B, N, H, Hkv, D, float(scale), code, st, dQ.data_ptr(),
            dK.data_ptr(), dV.data_ptr(), _like("dstate_in", dstate_in, torch.float32, states),
            _like("dlog_decay", dlog_decay, torch.float32, (H,)), ws, wsb)
    return _run(_lib.solar_decay_attention_backward,
                (Q, K, V, dO, log_decay, lengths, state_in, dstate_out, dQ, dK, dV, dstate_in, dlog_decay, workspace), args,
                raise_on_error)


def _norm_sizes(In, weight, bias):
    """(rows, groups, d): the weight [d] or [groups, d] says what is normalised, or the last dimension without one."""
    p = weight if weight is not None else bias
    if p is None:
        groups, d = 1, In.shape[-1]
    else:
        groups, d = (1, p.shape[0]) if p.dim() == 1 else (p.shape[0], p.shape[1])
    if In.dim() == 0 or groups * d == 0 or In.numel() % (groups * d) or (In.shape[-1] not in (d, groups * d)) or (
            groups > 1 and In.shape[-1] == d and (In.dim() < 2 or In.shape[-2] != groups)):
        raise ValueError(f"a weight of {groups} x {d} does not fit an input of shape {tuple(In.shape)}")
    return In.numel() // (groups * d), groups, d


def _param(name: str, t, groups: int, d: int):
    return None if t is None else _like(name, t, torch.float32, (d,) if t.dim() == 1 and groups == 1 else (groups, d))


def solar_layer_norm(In, weight, bias, eps: float, Out, mean=None, rstd=None, raise_on_error: bool = True) -> int:
    """Layer norm of In [..., groups, d], [..., groups * d] or [..., d] with weight and bias [groups, d] or [d]."""
    _check(In, Out, mean, rstd)
    rows, groups, d = _norm_sizes(In, weight, bias)
    if Out.shape != In.shape:
        raise ValueError("Out must have the shape of In")
    for name, t in (("mean", mean), ("rstd", rstd)):
        if t is not None and (t.dtype != torch.float32 or t.numel() != rows * groups):
            raise ValueError(f"{name} must hold {rows * groups} float32 values")
    args = (In.data_ptr(), _param("weight", weight, groups, d), _param("bias", bias, groups, d), rows, groups, d, float(eps),
            _dtype_code(In), _dtype_code(Out), Out.data_ptr(), None if mean is None else mean.data_ptr(),
            None if rstd is None else rstd.data_ptr())
    return _run(_lib.solar_layer_norm, (In, weight, bias, Out, mean, rstd), args, raise_on_error)


def solar_layer_norm_workspace_bytes(rows: int, groups: int, d: int) -> int:
    return int(_lib.solar_layer_norm_workspace_bytes(rows, groups, d))


def solar_layer_norm_backward(In, weight, mean, rstd, dOut, dIn, dweight, dbias, workspace=None,
                              raise_on_error: bool = True) -> int:
    """Gradients of solar_layer_norm; dweight and dbias may be None."""
    _check(In, mean, rstd, dOut, dIn, dweight, dbias, workspace)
    rows, groups, d = _norm_sizes(In, weight if weight is not None else dweight, dbias)
    if dOut.shape != In.shape or dIn.shape != In.shape or dIn.dtype != In.dtype:
        raise ValueError("dOut and dIn must have the shape of In, and dIn its type")
    for name, t in (("mean", mean), ("rstd", rstd)):
        if t.dtype != torch.float32 or t.numel() != rows * groups:
            raise ValueError(f"{name} must hold {rows * groups} float32 values")
    ws, wsb = _scratch(workspace)
    args = (In.data_ptr(), _param("weight", weight, groups, d), mean.data_ptr(), rstd.data_ptr(), dOut.data_ptr(), rows,
            groups, d, _dtype_code(In), _dtype_code(dOut), dIn.data_ptr(), _param("dweight", dweight, groups, d),
            _param("dbias", dbias, groups, d), ws, wsb)
    return _run(_lib.solar_layer_norm_backward, (In, weight, mean, rstd, dOut, dIn, dweight, dbias, workspace), args,
                raise_on_error)


# ---------------------------------------------------------------------------------------
# Convenience for tests and the benchmark: device buffers for one workload.

class DeviceBatch:
    """Device-resident inputs, outputs and workspace of one batch (allocation only)."""

    def __init__(self, X_host, Q_host, lengths_host, r: int, bf16: bool, device="cuda:0"):
        dev = torch.device(device)
        X = torch.from_numpy(X_host)
        Q = torch.from_numpy(Q_host)
        if bf16:
            # the host values are already bf16-representable, so this conversion is exact
            X = X.to(torch.bfloat16)
            Q = Q.to(torch.bfloat16)
        self.X = X.to(dev).contiguous()
        self.Q = Q.to(dev).contiguous()
        self.lengths = None if lengths_host is None else torch.from_numpy(lengths_host).to(dev)
        B, N, d = X_host.shape
        M = Q_host.shape[1]
        self.B, self.N, self.d, self.r, self.M = B, N, d, r, M
        self.S = torch.empty((B, r), dtype=torch.float32, device=dev)
        self.V = torch.empty((B, d, r), dtype=torch.float32, device=dev)
        self.P = torch.empty((B, N, r), dtype=torch.float32, device=dev)
        self.O = torch.empty((B, M, d), dtype=torch.float32, device=dev)
        self.info = torch.zeros((B,), dtype=torch.int32, device=dev)
        nbytes = solar_workspace_bytes(B, N, d, r, M, SOLAR_BF16 if bf16 else SOLAR_F32)
        self.workspace = torch.empty((max(nbytes, 256),), dtype=torch.uint8, device=dev)

    def factorize(self):
        return solar_svd_factorize(self.X, self.lengths, self.r, self.S, self.V, self.P, self.info,
                                   self.workspace)

    def factorize_rsvd(self, Omega, n_iter: int):
        """Algorithm 1 as printed (passes over X); Omega is a [B,d,r] float device tensor."""
        if getattr(self, "rsvd_workspace", None) is None:
            nbytes = solar_rsvd_workspace_bytes(self.B, self.N, self.d, self.r)
            self.rsvd_workspace = torch.empty((max(nbytes, 256),), dtype=torch.uint8,
                                              device=self.X.device)
        return solar_svd_factorize_rsvd(self.X, self.lengths, self.r, Omega, n_iter, self.S, self.V,
                                        self.P, self.info, self.rsvd_workspace)

    def attention(self, scale: float, mode: int = SOLAR_ATTN_SEQ_SOFTMAX, O=None):
        return solar_svd_attention(self.Q, self.S, self.V, self.P, self.lengths, self.N, scale,
                                   mode, self.O if O is None else O, self.workspace)

    def backward(self, S_bar, V_bar, gap_rel: float = 0.0, dX=None):
        """Gradient through the factorization held in S, V, P; S_bar [B,r] and V_bar [B,d,r] are
        float device tensors.  Returns dX [B,N,d] float."""
        if dX is None:
            dX = torch.empty((self.B, self.N, self.d), dtype=torch.float32, device=self.X.device)
        solar_svd_backward(self.S, self.V, self.P, S_bar, V_bar, gap_rel, dX, self.workspace)
        return dX

    def attention_from_x(self, scale: float, O=None):
        """Mode 0 with P = X V formed inside the attention kernel (bf16 inputs, r a multiple of 4)."""
        return solar_svd_attention_from_x(self.Q, self.X, self.S, self.V, self.lengths, scale,
                                          self.O if O is None else O)

    def factorize_no_p(self):
        return solar_svd_factorize(self.X, self.lengths, self.r, self.S, self.V, None, self.info,
                                   self.workspace)

    def linear(self, scale: float, O=None):
        return solar_linear_attention(self.Q, self.X, self.lengths, scale, self.O if O is None else O,
                                      self.workspace)

    def dense(self, scale: float, O=None):
        return solar_dense_attention_ref(self.Q, self.X, self.lengths, scale,
                                         self.O if O is None else O, self.workspace)


class SequenceMixer:
    """A mixing layer over sequences in their order, from the sequence operators: rotary positions on queries and keys, linear
    attention with a decay for each head, layer norm of every head's output.  Holds the buffers of one batch of B users with up
    to N rows, the states that single tokens go on from, and with `training` the gradients.  Rows at or past a length hold anything
    in the inputs and come out zero.  Whole sequences start from states of zeros at position 0; rotations
    have amplitude 1.

    log_decay [H] float, freq [rot/2] double, weight and bias [H,D] float: device tensors."""

    def __init__(self, B: int, N: int, H: int, Hkv: int, D: int, dtype, log_decay, freq, weight, bias, eps: float = 1e-5,
                 layout: int = SOLAR_ROTARY_HALF, training: bool = False):
        dev = log_decay.device

        def empty(*shape, dtype=torch.float32):
            return torch.empty(shape, dtype=dtype, device=dev)

        self.B, self.N, self.H, self.Hkv, self.D = B, N, H, Hkv, D
        self.log_decay, self.freq, self.weight, self.bias, self.eps, self.layout = log_decay, freq, weight, bias, eps, layout
        self.scale = D ** -0.5
        self.Q, self.K = empty(B, N, H, D, dtype=dtype), empty(B, N, Hkv, D, dtype=dtype)
        self.O, self.Y = empty(B, N, H, D, dtype=dtype), empty(B, N, H, D, dtype=dtype)
        self.mean, self.rstd = empty(B * N, H), empty(B * N, H)
        self.state = torch.zeros((B, H, D, D), dtype=torch.float32, device=dev)
        self.positions = torch.zeros((B, 1), dtype=torch.int32, device=dev)
        code = SOLAR_BF16 if dtype == torch.bfloat16 else SOLAR_F32
        # neither direction's need is a bound of the other's: they cut a sequence into parts of their own
        nbytes = solar_decay_workspace_bytes(B, N, H, Hkv, D, code, False)
        if training:
            nbytes = max(nbytes, solar_decay_workspace_bytes(B, N, H, Hkv, D, code, True),
                         solar_layer_norm_workspace_bytes(B * N, H, D))
            self.dO = empty(B, N, H, D, dtype=dtype)
            self.dQ, self.dK, self.dV = (empty(B, N, h, D, dtype=dtype) for h in (H, Hkv, Hkv))
            self.dweight, self.dbias, self.dlog_decay = empty(H, D), empty(H, D), empty(H)
        self.workspace = empty(max(nbytes, 256), dtype=torch.uint8)

    def forward(self, Q, K, V, lengths=None):
        """Y [B,N,H,D] for whole sequences, whose last states and lengths steps go on from."""
        self._V, self._lengths = V, lengths
        solar_rotary(Q, K, self.freq, self.Q, self.K, lengths=lengths, layout=self.layout)
        solar_decay_attention(self.Q, self.K, V, self.log_decay, lengths, self.scale, self.O, None, self.state,
                              self.workspace)
        solar_layer_norm(self.O, self.weight, self.bias, self.eps, self.Y, self.mean, self.rstd)
        if lengths is None:
            self.positions.fill_(self.N)
        else:
            self.Y.masked_fill_(self._past(), 0.0)
            self.positions.copy_(lengths.clamp(0, self.N)[:, None])     # as the operators take them
        return self.Y

    def _past(self):
        """[B,N,1,1] truth values of the rows at or past the last forward call's lengths.  The norm knows none: a row of zeros gets
        its bias, and adds its gradient to the bias's."""
        return (torch.arange(self.N, device=self._lengths.device) >= self._lengths[:, None])[:, :, None, None]

    def step(self, Q, K, V):
        """Y [B,1,H,D] for the next token of every user: Q [B,1,H,D], K and V [B,1,Hkv,D], K and Q rotated in place."""
        solar_rotary(Q, K, self.freq, Q, K, positions=self.positions, layout=self.layout)
        Y = torch.empty_like(Q)
        solar_decay_attention(Q, K, V, self.log_decay, None, self.scale, Y, self.state, self.state)
        solar_layer_norm(Y, self.weight, self.bias, self.eps, Y)
        self.positions += 1
        return Y

    def backward(self, dY):
        """Gradients of the last forward call: (dQ, dK, dV); dweight, dbias and dlog_decay are left in attributes.  What dY holds in
        rows at or past the lengths does not matter."""
        if self._lengths is not None:
            dY = dY.masked_fill(self._past(), 0.0)
        solar_layer_norm_backward(self.O, self.weight, self.mean, self.rstd, dY, self.dO, self.dweight, self.dbias,
                                  self.workspace)
        solar_decay_attention_backward(self.Q, self.K, self._V, self.dO, self.log_decay, self._lengths, self.scale, None, None,
                                       self.dQ, self.dK, self.dV, None, self.dlog_decay, self.workspace)
        solar_rotary(self.dQ, self.dK, self.freq, self.dQ, self.dK, lengths=self._lengths, layout=self.layout, inverse=True)
        return self.dQ, self.dK, self.dV
