"""Thin ctypes binding over libfavorsharp.so: argument marshalling only.

Function names mirror the C ABI (include/favorsharp.h).  PyTorch supplies device
memory and the current stream; every step of the computation runs in the HIP
kernels of the library.  There is no fallback: if the library has not been built
the import of `lib()` raises.
"""
from __future__ import annotations

import contextlib
import ctypes
import math
import os
import struct
from ctypes import c_char_p, c_double, c_float, c_int, c_int32, c_int64, c_size_t, c_void_p

from typing import NamedTuple

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libfavorsharp.so")

VARIANTS = {"posrf": 0, "gerf": 1, "saderf": 2, "aderf": 3, "sderf": 4}
FS_F32, FS_BF16 = 0, 1
THETA_HEADER = 8


class FsTensor(ctypes.Structure):
    _fields_ = [("ptr", c_void_p), ("dtype", c_int32), ("stride_b", c_int64), ("stride_h", c_int64),
                ("stride_l", c_int64)]


class FsRotary(ctypes.Structure):
    _fields_ = [("freqs", c_void_p), ("positions", c_void_p), ("stride_b", c_int64), ("stride_l", c_int64), ("rot_dim", c_int32),
                ("interleaved", c_int32), ("amplitude", c_float)]


class FsState(ctypes.Structure):
    _fields_ = [("T", c_void_p), ("z", c_void_p), ("shift", c_void_p), ("slots", c_int32)]


class FsFeatures(ctypes.Structure):
    _fields_ = [("ptr", c_void_p), ("bytes", c_size_t), ("heads", c_int32), ("d", c_int32), ("M", c_int32), ("sets", c_int32),
                ("dense_c2", c_int32), ("qk_scale", c_float)]


class FsRotaryAxes(ctypes.Structure):
    _fields_ = [("freqs", c_void_p), ("axis_of", c_void_p), ("positions", c_void_p), ("stride_a", c_int64), ("stride_b", c_int64),
                ("stride_l", c_int64), ("axes", c_int32), ("rot_dim", c_int32), ("interleaved", c_int32), ("amplitude", c_float)]


class FsDecayState(ctypes.Structure):
    _fields_ = [("S", c_void_p), ("slots", c_int32)]


class FavorSharpError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {lib().favorsharp_status_string(status).decode()} (status {status})")


_lib = None


def lib() -> ctypes.CDLL:
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2302_00787_amd.build` "
                              "(there is no CPU fallback)")
        L = ctypes.CDLL(LIB_PATH)
        P = ctypes.POINTER(FsTensor)
        L.favorsharp_theta_floats.restype = c_size_t
        L.favorsharp_theta_floats.argtypes = [c_int]
        L.favorsharp_status_string.restype = c_char_p
        L.favorsharp_status_string.argtypes = [c_int]
        L.favorsharp_version.restype = c_char_p
        L.favorsharp_version.argtypes = []
        L.favorsharp_orthogonal_omega.restype = c_int
        L.favorsharp_orthogonal_omega.argtypes = [c_void_p, c_void_p, c_int, c_int, c_int, c_void_p]
        L.favorsharp_fit_workspace_bytes.restype = c_size_t
        L.favorsharp_fit_workspace_bytes.argtypes = [c_int] * 6
        L.favorsharp_fit_params.restype = c_int
        L.favorsharp_fit_params.argtypes = [c_int, P, P, c_int, c_int, c_int, c_int, c_int, c_float, c_int, c_float,
                                            c_void_p, c_void_p, c_size_t, c_void_p]
        L.favorsharp_fit_device_workspace_bytes.restype = c_size_t
        L.favorsharp_fit_device_workspace_bytes.argtypes = [c_int] * 6
        L.favorsharp_fit_params_device.restype = c_int
        L.favorsharp_fit_params_device.argtypes = [c_int, P, P, c_int, c_int, c_int, c_int, c_int, c_float, c_int, c_float,
                                                   c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]
        L.favorsharp_features_workspace_bytes.restype = c_size_t
        L.favorsharp_features_workspace_bytes.argtypes = [c_int] * 3
        L.favorsharp_features.restype = c_int
        L.favorsharp_features.argtypes = [c_void_p, c_int, P, c_int, c_int, c_float, c_float, c_void_p, c_int,
                                          c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]
        L.favorsharp_attention_workspace_bytes.restype = c_size_t
        L.favorsharp_attention_workspace_bytes.argtypes = [c_int] * 10
        L.favorsharp_attention.restype = c_int
        L.favorsharp_attention.argtypes = [c_void_p, c_int, P, P, P, c_int, c_int, c_int, c_int, c_int, c_int, c_float,
                                           c_void_p, c_int, c_int, c_int, c_int, P, c_void_p, c_size_t, c_void_p]
        L.favorsharp_attention_timed.restype = c_int
        L.favorsharp_attention_timed.argtypes = L.favorsharp_attention.argtypes + [c_void_p, c_void_p]
        L.favorsharp_prepared_bytes.restype = c_size_t
        L.favorsharp_prepared_bytes.argtypes = [c_int] * 6
        L.favorsharp_attention_prepare.restype = c_int
        L.favorsharp_attention_prepare.argtypes = [c_void_p, c_int, c_void_p, c_int, c_int, c_int, c_int, c_int, c_float,
                                                   c_void_p, c_size_t, ctypes.POINTER(c_int), c_void_p]
        L.favorsharp_attention_prepared.restype = c_int
        L.favorsharp_attention_prepared.argtypes = [c_void_p, c_size_t, c_int] + L.favorsharp_attention.argtypes
        L.favorsharp_attention_noalloc.restype = c_int
        L.favorsharp_attention_noalloc.argtypes = L.favorsharp_attention.argtypes[:18] + [c_void_p]
        L.favorsharp_attention_flushed_rows.restype = c_int
        L.favorsharp_attention_flushed_rows.argtypes = [c_void_p, ctypes.POINTER(c_int), c_void_p]
        L.favorsharp_attention_backward_workspace_bytes.restype = c_size_t
        L.favorsharp_attention_backward_workspace_bytes.argtypes = [c_int] * 10
        L.favorsharp_attention_backward.restype = c_int
        L.favorsharp_attention_backward.argtypes = [c_void_p, c_int, P, P, P, P, c_int, c_int, c_int, c_int, c_int, c_int,
                                                    c_float, c_void_p, c_int, c_int, c_int, P, P, P, c_void_p, c_size_t,
                                                    c_void_p]
        L.favorsharp_attention_backward_prepared.restype = c_int
        L.favorsharp_attention_backward_prepared.argtypes = [c_void_p, c_size_t, c_int] + L.favorsharp_attention_backward.argtypes
        L.favorsharp_kernel_matvec_workspace_bytes.restype = c_size_t
        L.favorsharp_kernel_matvec_workspace_bytes.argtypes = [c_int] * 5
        L.favorsharp_kernel_matvec.restype = c_int
        L.favorsharp_kernel_matvec.argtypes = [c_void_p, P, P, c_int, c_int, c_int, c_float, c_float, c_void_p, c_int,
                                               c_void_p, c_int, c_void_p, c_void_p, c_size_t, c_void_p]
        R, S, F = ctypes.POINTER(FsRotary), ctypes.POINTER(FsState), ctypes.POINTER(FsFeatures)
        V = c_void_p                # of calls whose descriptors are packed together (_packed)
        ws = [c_void_p, c_size_t, c_void_p]
        for name, restype, argtypes in (
                ("rotary_frequencies", c_int, [c_int, c_double, c_int, c_double, c_int, c_double, c_double, c_void_p]),
                ("rotary", c_int, [R, P, c_int, P, c_int, c_int, c_int, c_int, c_int, P, P, c_void_p]),
                ("state_features_bytes", c_size_t, [c_int] * 5),
                ("state_prepare", c_int, [c_void_p, c_int, c_void_p, c_int, c_int, c_int, c_int, c_float, F, c_void_p]),
                ("state_append_workspace_bytes", c_size_t, [F, c_int, c_int, c_int, c_int]),
                ("state_append", c_int, [F, S, c_void_p, P, P, c_int, c_int, c_int, c_void_p, R, c_int, c_void_p] + ws),
                ("state_attention_workspace_bytes", c_size_t, [F, c_int, c_int, c_int, c_int, c_int]),
                ("state_attention", c_int, [F, S, c_void_p, P, c_int, c_int, c_int, c_int, c_void_p, R, P, c_void_p] + ws),
                ("state_step_workspace_bytes", c_size_t, [F, c_int, c_int]),
                ("state_step", c_int, [F, S, c_void_p, P, P, P, c_int, c_int, c_int, R, P, c_void_p] + ws),
                ("state_attention_backward_workspace_bytes", c_size_t, [F, c_int, c_int, c_int, c_int, c_int]),
                ("state_attention_backward", c_int, [F, S, c_void_p, P, P, c_int, c_int, c_int, c_int, c_void_p, R, P, S] + ws),
                ("state_append_backward_workspace_bytes", c_size_t, [F, c_int, c_int, c_int, c_int]),
                ("state_append_backward", c_int, [F, S, c_void_p, S, P, P, c_int, c_int, c_int, c_void_p, R, P, P] + ws),
                ("rotary_sections", c_int, [c_int, c_void_p, c_double, c_int, c_int, c_void_p, c_void_p]),
                ("rotary_axes", c_int, [V, V, c_int, V, c_int, c_int, c_int, c_int, c_int, V, V, c_void_p]),
                ("decay_attention_workspace_bytes", c_size_t, [c_int] * 6),
                ("decay_attention", c_int, [V, V, V] + [c_int] * 6 + [c_void_p, c_float, V, V, c_void_p, c_void_p, V, c_void_p] + ws),
                ("decay_attention_backward_workspace_bytes", c_size_t, [c_int] * 7),
                ("decay_attention_backward", c_int, [V, V, V, V] + [c_int] * 6 + [c_void_p, c_float, V, V, c_void_p, c_void_p, c_int, V, V, V, V] + ws),
                ("decay_step", c_int, [V, c_void_p, V, V, V] + [c_int] * 5 + [c_void_p, c_float, V, c_void_p, c_void_p])):
            fn = getattr(L, "favorsharp_" + name)
            fn.restype, fn.argtypes = restype, argtypes
        _lib = L
    return _lib


# ------------------------------------------------------------------ marshalling helpers
def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return FS_F32
    if t.dtype == torch.bfloat16:
        return FS_BF16
    raise TypeError(f"unsupported dtype {t.dtype}")


def _desc4(t: torch.Tensor) -> FsTensor:
    """[B, H, L, d] (or [L, d]) CUDA tensor -> fs_tensor."""
    if not t.is_cuda:
        raise ValueError("device tensor expected")
    if t.dim() == 2:
        sb = sh = 0
        sl, sd = t.stride()
    elif t.dim() == 4:
        sb, sh, sl, sd = t.stride()
    else:
        raise ValueError("expected a [B,H,L,d] or [L,d] tensor")
    if sd != 1 and t.shape[-1] > 1:
        raise ValueError("innermost stride must be 1")
    return FsTensor(t.data_ptr(), _dtype_code(t), sb, sh, sl)


def _stream() -> int:
    return torch.cuda.current_stream().cuda_stream


def _workspace(nbytes: int, device, workspace: torch.Tensor | None) -> torch.Tensor:
    if workspace is not None:
        if workspace.dtype != torch.uint8 or not workspace.is_cuda:
            raise ValueError("workspace must be a CUDA uint8 tensor")
        return workspace
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


def _check(status: int, where: str):
    if status != 0:
        raise FavorSharpError(status, where)


def theta_floats(d: int) -> int:
    return int(lib().favorsharp_theta_floats(d))


def pack_theta(A, B1, B2, C1, C2, logD, lbar=float("nan"), variant=4) -> np.ndarray:
    """Lay one parameter set out as the library expects it (float32 vector)."""
    A = np.asarray(A, dtype=np.float64)
    d = A.shape[0]
    C1, C2 = np.asarray(C1, dtype=np.float64), np.asarray(C2, dtype=np.float64)
    B1, B2 = np.asarray(B1, dtype=np.float64), np.asarray(B2, dtype=np.float64)
    flags = 0
    if np.array_equal(C1, -0.5 * np.eye(d)) and np.array_equal(C2, -0.5 * np.eye(d)):
        flags |= 1
    if np.array_equal(B1, B2):
        flags |= 2
    head = np.zeros(THETA_HEADER)
    head[0], head[1], head[2], head[3] = logD, lbar if lbar is not None else float("nan"), flags, variant
    return np.concatenate([head, A, B1.ravel(), B2.ravel(), C1.ravel(), C2.ravel()]).astype(np.float32)


def unpack_theta(vec: np.ndarray, d: int) -> dict:
    vec = np.asarray(vec, dtype=np.float32)
    o = THETA_HEADER
    dd = d * d
    return dict(logD=float(vec[0]), lbar=float(vec[1]), flags=int(vec[2]), variant=int(vec[3]),
                A=vec[o:o + d].copy(), B1=vec[o + d:o + d + dd].reshape(d, d).copy(),
                B2=vec[o + d + dd:o + d + 2 * dd].reshape(d, d).copy(),
                C1=vec[o + d + 2 * dd:o + d + 3 * dd].reshape(d, d).copy(),
                C2=vec[o + d + 3 * dd:o + d + 4 * dd].reshape(d, d).copy())


def to_device(a: np.ndarray, dtype: str) -> torch.Tensor:
    """Host array -> device tensor, float32 ("f32") or bfloat16 ("bf16": the values must already be representable,
    as the input generators leave them; their upper 16 bits are uploaded)."""
    if dtype == "bf16":
        from . import synth
        bits = synth.to_bf16_bits(a)
        return torch.from_numpy(bits.view(np.int16)).view(torch.bfloat16).cuda()
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda()


def to_host(t: torch.Tensor) -> np.ndarray:
    """Device tensor -> float64 host array."""
    return t.detach().float().cpu().numpy().astype(np.float64)


# ------------------------------------------------------------------ entry points
def fit_workspace_bytes(B, H, Lx, Ly, d, groups) -> int:
    return int(lib().favorsharp_fit_workspace_bytes(B, H, Lx, Ly, d, groups))


def fit_params(variant, X: torch.Tensor, Y: torch.Tensor, qk_scale: float, groups: int = 1, eig_ridge: float = 0.0,
               workspace: torch.Tensor | None = None) -> torch.Tensor:
    """favorsharp_fit_params: X [B,H,Lx,d], Y [B,H,Ly,d] -> theta [groups, theta_floats(d)] (float32, device)."""
    v = VARIANTS[variant] if isinstance(variant, str) else int(variant)
    if X.dim() == 2:
        X, Y = X[None, None], Y[None, None]
    B, H, Lx, d = X.shape
    Ly = Y.shape[2]
    theta = torch.empty((groups, theta_floats(d)), dtype=torch.float32, device=X.device)
    nbytes = fit_workspace_bytes(B, H, Lx, Ly, d, groups)
    ws = _workspace(nbytes, X.device, workspace)
    dx, dy = _desc4(X), _desc4(Y)
    st = lib().favorsharp_fit_params(v, ctypes.byref(dx), ctypes.byref(dy), B, H, Lx, Ly, d, qk_scale, groups,
                                     eig_ridge, theta.data_ptr(), ws.data_ptr(), ws.numel(), _stream())
    _check(st, "favorsharp_fit_params")
    return theta


def fit_device_workspace_bytes(B, H, Lx, Ly, d, groups) -> int:
    return int(lib().favorsharp_fit_device_workspace_bytes(B, H, Lx, Ly, d, groups))


def fit_params_device(variant, X: torch.Tensor, Y: torch.Tensor, qk_scale: float, groups: int = 1,
                      eig_ridge: float = 0.0, workspace: torch.Tensor | None = None):
    """favorsharp_fit_params_device: as fit_params, without a host round trip.  Returns (theta, status), both on the
    device; status [groups] int32 is valid once the stream has run the call (no synchronisation happens here)."""
    v = VARIANTS[variant] if isinstance(variant, str) else int(variant)
    if X.dim() == 2:
        X, Y = X[None, None], Y[None, None]
    B, H, Lx, d = X.shape
    Ly = Y.shape[2]
    theta = torch.empty((groups, theta_floats(d)), dtype=torch.float32, device=X.device)
    status = torch.empty((groups,), dtype=torch.int32, device=X.device)
    nbytes = fit_device_workspace_bytes(B, H, Lx, Ly, d, groups)
    ws = _workspace(nbytes, X.device, workspace)
    dx, dy = _desc4(X), _desc4(Y)
    st = lib().favorsharp_fit_params_device(v, ctypes.byref(dx), ctypes.byref(dy), B, H, Lx, Ly, d, qk_scale, groups,
                                            eig_ridge, theta.data_ptr(), status.data_ptr(), ws.data_ptr(), ws.numel(),
                                            _stream())
    _check(st, "favorsharp_fit_params_device")
    return theta, status


def features_workspace_bytes(n, d, M) -> int:
    return int(lib().favorsharp_features_workspace_bytes(n, d, M))


def features(theta: torch.Tensor, side: int, X: torch.Tensor, qk_scale: float, alpha: float, Omega: torch.Tensor,
             stabilise: bool = False, workspace: torch.Tensor | None = None):
    """favorsharp_features: X [n,d] -> out [n,M] float32 (and row_logscale [n] when stabilise)."""
    n, d = X.shape
    M = Omega.shape[-2]
    out = torch.empty((n, M), dtype=torch.float32, device=X.device)
    rls = torch.empty((n,), dtype=torch.float32, device=X.device) if stabilise else None
    ws = _workspace(features_workspace_bytes(n, d, M), X.device, workspace)
    dx = _desc4(X)
    st = lib().favorsharp_features(theta.data_ptr(), side, ctypes.byref(dx), n, d, qk_scale, alpha, Omega.data_ptr(), M,
                                   out.data_ptr(), rls.data_ptr() if stabilise else None, ws.data_ptr(), ws.numel(),
                                   _stream())
    _check(st, "favorsharp_features")
    return (out, rls) if stabilise else out


def attention_workspace_bytes(B, H, Lq, Lk, d, dv, M, causal, groups, omega_groups) -> int:
    return int(lib().favorsharp_attention_workspace_bytes(B, H, Lq, Lk, d, dv, M, int(causal), groups, omega_groups))


def attention(theta: torch.Tensor, Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, qk_scale: float,
              Omega: torch.Tensor, causal: bool = False, chunk: int = 0, out: torch.Tensor | None = None,
              out_dtype=None, workspace: torch.Tensor | None = None, events=None) -> torch.Tensor:
    """favorsharp_attention: Q [B,H,Lq,d], K [B,H,Lk,d], V [B,H,Lk,dv], theta [groups,*], Omega [og,M,d] -> Y."""
    B, H, Lq, d = Q.shape
    Lk, dv = K.shape[2], V.shape[3]
    groups = theta.shape[0] if theta.dim() == 2 else 1
    og, M = (Omega.shape[0], Omega.shape[1]) if Omega.dim() == 3 else (1, Omega.shape[0])
    if out is None:
        out = torch.empty((B, H, Lq, dv), dtype=out_dtype or Q.dtype, device=Q.device)
    nbytes = attention_workspace_bytes(B, H, Lq, Lk, d, dv, M, causal, groups, og)
    ws = _workspace(nbytes, Q.device, workspace)
    dq, dk, dvv, dy = _desc4(Q), _desc4(K), _desc4(V), _desc4(out)
    args = (theta.data_ptr(), groups, ctypes.byref(dq), ctypes.byref(dk), ctypes.byref(dvv),
            B, H, Lq, Lk, d, dv, qk_scale, Omega.data_ptr(), og, M, int(causal), chunk,
            ctypes.byref(dy), ws.data_ptr(), ws.numel(), _stream())
    if events is None:
        st = lib().favorsharp_attention(*args)
    else:       # (hipEvent_t begin, hipEvent_t end) as integers: favorsharp_attention_timed
        st = lib().favorsharp_attention_timed(*args, events[0], events[1])
    _check(st, "favorsharp_attention")
    return out


def prepared_bytes(B, H, d, M, groups, omega_groups) -> int:
    return int(lib().favorsharp_prepared_bytes(B, H, d, M, groups, omega_groups))


def attention_prepare(theta: torch.Tensor, Omega: torch.Tensor, B: int, H: int, qk_scale: float):
    """favorsharp_attention_prepare: the projection constants of (theta, Omega) -> (prepared buffer, dense_c2)."""
    groups = theta.shape[0] if theta.dim() == 2 else 1
    og, M, d = (Omega.shape[0], Omega.shape[1], Omega.shape[2]) if Omega.dim() == 3 else (1, Omega.shape[0], Omega.shape[1])
    buf = torch.empty(max(prepared_bytes(B, H, d, M, groups, og), 256), dtype=torch.uint8, device=theta.device)
    dense = c_int(0)
    st = lib().favorsharp_attention_prepare(theta.data_ptr(), groups, Omega.data_ptr(), og, B, H, d, M, qk_scale,
                                            buf.data_ptr(), buf.numel(), ctypes.byref(dense), _stream())
    _check(st, "favorsharp_attention_prepare")
    return buf, int(dense.value)


def attention_prepared(prepared, theta: torch.Tensor, Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, qk_scale: float,
                       Omega: torch.Tensor, causal: bool = False, chunk: int = 0, out: torch.Tensor | None = None,
                       out_dtype=None, workspace: torch.Tensor | None = None) -> torch.Tensor:
    """favorsharp_attention_prepared: `prepared` = what attention_prepare returned for the same theta, Omega, qk_scale."""
    buf, dense = prepared
    B, H, Lq, d = Q.shape
    Lk, dv = K.shape[2], V.shape[3]
    groups = theta.shape[0] if theta.dim() == 2 else 1
    og, M = (Omega.shape[0], Omega.shape[1]) if Omega.dim() == 3 else (1, Omega.shape[0])
    if out is None:
        out = torch.empty((B, H, Lq, dv), dtype=out_dtype or Q.dtype, device=Q.device)
    ws = _workspace(attention_workspace_bytes(B, H, Lq, Lk, d, dv, M, causal, groups, og), Q.device, workspace)
    dq, dk, dvv, dy = _desc4(Q), _desc4(K), _desc4(V), _desc4(out)
    st = lib().favorsharp_attention_prepared(buf.data_ptr(), buf.numel(), dense, theta.data_ptr(), groups, ctypes.byref(dq),
                                             ctypes.byref(dk), ctypes.byref(dvv), B, H, Lq, Lk, d, dv, qk_scale,
                                             Omega.data_ptr(), og, M, int(causal), chunk, ctypes.byref(dy), ws.data_ptr(),
                                             ws.numel(), _stream())
    _check(st, "favorsharp_attention_prepared")
    return out


NOALLOC_SCRATCH_BYTES = 64 << 20


def attention_noalloc(theta: torch.Tensor, Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, qk_scale: float,
                      Omega: torch.Tensor, out: torch.Tensor, causal: bool = False, chunk: int = 0) -> torch.Tensor:
    """favorsharp_attention_noalloc: as `attention`, on the library's own scratch array; `out` is required (nothing
    is allocated here either)."""
    B, H, Lq, d = Q.shape
    Lk, dv = K.shape[2], V.shape[3]
    groups = theta.shape[0] if theta.dim() == 2 else 1
    og, M = (Omega.shape[0], Omega.shape[1]) if Omega.dim() == 3 else (1, Omega.shape[0])
    dq, dk, dvv, dy = _desc4(Q), _desc4(K), _desc4(V), _desc4(out)
    st = lib().favorsharp_attention_noalloc(theta.data_ptr(), groups, ctypes.byref(dq), ctypes.byref(dk), ctypes.byref(dvv),
                                            B, H, Lq, Lk, d, dv, qk_scale, Omega.data_ptr(), og, M, int(causal), chunk,
                                            ctypes.byref(dy), _stream())
    _check(st, "favorsharp_attention_noalloc")
    return out


def attention_flushed_rows(workspace: torch.Tensor | None = None) -> int:
    """favorsharp_attention_flushed_rows: how many output rows of the last attention call on `workspace` (None: the
    scratch array of `attention_noalloc`) had a zero normaliser and were written as zeros.  Waits for the stream."""
    n = c_int(0)
    st = lib().favorsharp_attention_flushed_rows(None if workspace is None else workspace.data_ptr(), ctypes.byref(n),
                                                 _stream())
    _check(st, "favorsharp_attention_flushed_rows")
    return int(n.value)


def attention_backward_workspace_bytes(B, H, Lq, Lk, d, dv, M, causal, groups, omega_groups) -> int:
    return int(lib().favorsharp_attention_backward_workspace_bytes(B, H, Lq, Lk, d, dv, M, int(causal), groups,
                                                                    omega_groups))


def attention_backward(theta: torch.Tensor, Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, dY: torch.Tensor,
                       qk_scale: float, Omega: torch.Tensor, causal: bool = False, grad_dtype=None,
                       workspace: torch.Tensor | None = None, grads=None, prepared=None):
    """favorsharp_attention_backward: gradients of sum(Y * dY) -> (dQ, dK, dV), shaped like Q, K, V
    (`grads`: three preallocated tensors to write into, any row strides; `prepared`: what attention_prepare returned
    for the same theta, Omega, qk_scale: favorsharp_attention_backward_prepared)."""
    B, H, Lq, d = Q.shape
    Lk, dv = K.shape[2], V.shape[3]
    groups = theta.shape[0] if theta.dim() == 2 else 1
    og, M = (Omega.shape[0], Omega.shape[1]) if Omega.dim() == 3 else (1, Omega.shape[0])
    gd = grad_dtype or Q.dtype
    if grads is not None:
        gQ, gK, gV = grads
    else:
        gQ = torch.empty((B, H, Lq, d), dtype=gd, device=Q.device)
        gK = torch.empty((B, H, Lk, d), dtype=gd, device=Q.device)
        gV = torch.empty((B, H, Lk, dv), dtype=gd, device=Q.device)
    nbytes = attention_backward_workspace_bytes(B, H, Lq, Lk, d, dv, M, causal, groups, og)
    ws = _workspace(nbytes, Q.device, workspace)
    descs = [_desc4(t) for t in (Q, K, V, dY, gQ, gK, gV)]
    args = (theta.data_ptr(), groups, ctypes.byref(descs[0]), ctypes.byref(descs[1]), ctypes.byref(descs[2]),
            ctypes.byref(descs[3]), B, H, Lq, Lk, d, dv, qk_scale, Omega.data_ptr(), og, M, int(causal),
            ctypes.byref(descs[4]), ctypes.byref(descs[5]), ctypes.byref(descs[6]), ws.data_ptr(), ws.numel(), _stream())
    if prepared is None:
        _check(lib().favorsharp_attention_backward(*args), "favorsharp_attention_backward")
    else:
        buf, dense = prepared
        _check(lib().favorsharp_attention_backward_prepared(buf.data_ptr(), buf.numel(), dense, *args),
               "favorsharp_attention_backward_prepared")
    return gQ, gK, gV


def orthogonal_omega(gauss_dir: np.ndarray, gauss_len: np.ndarray) -> np.ndarray:
    """favorsharp_orthogonal_omega (host): [groups, M, d] or [M, d] Gaussian draws -> block-orthogonal omega, float32."""
    g = np.ascontiguousarray(gauss_dir, dtype=np.float32)
    n = np.ascontiguousarray(gauss_len, dtype=np.float32)
    if g.shape != n.shape or g.ndim not in (2, 3):
        raise ValueError("gauss_dir and gauss_len must have the same shape [groups, M, d] or [M, d]")
    groups = 1 if g.ndim == 2 else g.shape[0]
    M, d = g.shape[-2], g.shape[-1]
    out = np.empty_like(g)
    _check(lib().favorsharp_orthogonal_omega(g.ctypes.data_as(c_void_p), n.ctypes.data_as(c_void_p), groups, M, d,
                                             out.ctypes.data_as(c_void_p)), "favorsharp_orthogonal_omega")
    return out


def kernel_matvec_workspace_bytes(Nx, Ny, d, M, n) -> int:
    return int(lib().favorsharp_kernel_matvec_workspace_bytes(Nx, Ny, d, M, n))


def kernel_matvec(theta: torch.Tensor, X: torch.Tensor, Y: torch.Tensor, qk_scale: float, alpha: float,
                  Omega: torch.Tensor, C: torch.Tensor, workspace: torch.Tensor | None = None) -> torch.Tensor:
    """favorsharp_kernel_matvec: X [Nx,d], Y [Ny,d], C [Ny,n] float32 -> out [Nx,n] float32."""
    Nx, d = X.shape
    Ny, n = C.shape
    M = Omega.shape[-2]
    if C.dtype != torch.float32 or not C.is_contiguous():
        raise ValueError("C must be contiguous float32")
    out = torch.empty((Nx, n), dtype=torch.float32, device=X.device)
    ws = _workspace(kernel_matvec_workspace_bytes(Nx, Ny, d, M, n), X.device, workspace)
    dx, dy = _desc4(X), _desc4(Y)
    st = lib().favorsharp_kernel_matvec(theta.data_ptr(), ctypes.byref(dx), ctypes.byref(dy), Nx, Ny, d, qk_scale,
                                        alpha, Omega.data_ptr(), M, C.data_ptr(), n, out.data_ptr(), ws.data_ptr(),
                                        ws.numel(), _stream())
    _check(st, "favorsharp_kernel_matvec")
    return out


# ------------------------------------------------------------------ rotary positions and attention through kept states
AXES_ORDERS = {"blocks": 0, "cyclic": 1}
ROTARY_SCALINGS = {"plain": 0, "linear": 1, "base": 2, "blend": 3}
_SAME_DEVICE = contextlib.nullcontext()


class Rotary(NamedTuple):
    """fs_rotary.  freqs [rot_dim / 2] float64 (radians a position) on the device; positions [B, L] (or [L]: shared) int32, None:
    row l is at position l."""
    freqs: torch.Tensor
    positions: torch.Tensor | None = None
    interleaved: bool = False
    amplitude: float = 1.0


class RotaryAxes(NamedTuple):
    """fs_rotary_axes.  freqs [rot_dim / 2] float64 and axis_of [rot_dim / 2] int32 on the device; positions [axes, B, L] (or [axes, L]:
    shared) int32."""
    freqs: torch.Tensor
    axis_of: torch.Tensor
    positions: torch.Tensor
    interleaved: bool = False
    amplitude: float = 1.0


class Features(NamedTuple):
    """What state_prepare returns: the buffer of projection constants and the host's fs_features of it."""
    buffer: torch.Tensor
    desc: FsFeatures


class State(NamedTuple):
    """fs_state: T [slots, heads, M, dv], z [slots, heads, M], shift [slots, heads] (None in a pool of gradients), float32."""
    T: torch.Tensor
    z: torch.Tensor
    shift: torch.Tensor | None


# (a tensor is there, so the runtime is up: torch.cuda.current_device() asks for that first)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _on(device):
    """The library launches on the current device: that of the tensors has to be it."""
    return _SAME_DEVICE if device.index == _current_device() else torch.cuda.device(device)


# (current_stream() makes a Stream object, 2.7 of the 17 us of a small call)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)


def _new(shape, like: torch.Tensor) -> torch.Tensor:
    """_empty of a tensor's dtype on its device, at less cost."""
    return like.new_empty(shape) if shape[-1] % 8 == 0 else _empty(shape, like.dtype, like.device)


def _empty(shape, dtype, device) -> torch.Tensor:
    """A result, its rows at multiples of 16 bytes as the library wants them."""
    if shape[-1] % 8 == 0:
        return torch.empty(shape, dtype=dtype, device=device)
    return torch.empty((*shape[:-1], shape[-1] + 7 & ~7), dtype=dtype, device=device)[..., :shape[-1]]


def _room(nbytes: int, device, workspace: torch.Tensor | None):
    """Workspace of a call on states: (pointer, bytes, what holds it)."""
    if workspace is None and nbytes == 0:
        return None, 0, None
    ws = _workspace(nbytes, device, workspace)
    return ws.data_ptr(), ws.numel(), ws


def _one_device(*tensors) -> torch.device:
    device = tensors[0].device
    index = tensors[0].get_device()          # (compared as numbers: half the time)
    for t in tensors:
        if t is not None and t.get_device() != index:
            raise ValueError("tensors of one call must be on one device")
    if device.type != "cuda":
        raise ValueError("device tensor expected")
    return device


# Descriptors of a call in one piece of memory: 40 bytes for each fs_tensor, then what follows them.  (A ctypes structure for each takes
# twice as long, 0.5 us a tensor of a call whose launch takes 4.)
_TENSOR, _AXES, _POOL = "Qi4xqqq", "QQQqqqiiif", "Qi4x"
_CODES = {torch.float32: FS_F32, torch.bfloat16: FS_BF16}
_packs = {}


def _packed(tensors, more: str, values):
    """(what holds it, its address) of the descriptors of [B,H,L,d] tensors and of `values` behind them."""
    v = []
    for t in tensors:
        code = _CODES.get(t.dtype)
        if code is None:
            raise TypeError(f"unsupported dtype {t.dtype}")
        sb, sh, sl, sd = t.stride()
        if sd != 1 and t.shape[-1] > 1:
            raise ValueError("innermost stride must be 1")
        v += (t.data_ptr(), code, sb, sh, sl)
    key = (len(tensors), more)
    pack = _packs.get(key)
    if pack is None:
        form = struct.Struct("=" + _TENSOR * len(tensors) + more)
        pack = _packs[key] = (form.pack, (ctypes.c_char * form.size).from_buffer_copy)
    held = pack[1](pack[0](*v, *values))
    return held, ctypes.addressof(held)


def _shaped(name: str, t: torch.Tensor, shape):
    if t.shape != shape:          # (a torch.Size is a tuple)
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")


def _int32(name: str, t: torch.Tensor | None, shape):
    if t is None:
        return None
    if t.dtype != torch.int32 or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous int32")
    _shaped(name, t, shape)
    return t.data_ptr()


def _counter(name: str, t: torch.Tensor | None):
    if t is not None and (t.dtype != torch.int32 or t.numel() != 1):
        raise ValueError(f"{name} must be one int32")
    return None if t is None else t.data_ptr()


def _rotary_desc(rot: Rotary | None, B: int, L: int):
    """(fs_rotary or None, rot_dim)"""
    if rot is None:
        return None, 0
    if isinstance(rot, RotaryAxes):
        raise TypeError("positions with several axes are for rotary() alone: turn the rows first")
    if rot.freqs.dtype != torch.float64 or rot.freqs.dim() != 1 or not rot.freqs.is_contiguous():
        raise ValueError("freqs must be a contiguous float64 vector")
    p, sb, sl = rot.positions, 0, 0
    if p is not None:
        if p.dtype != torch.int32:
            raise ValueError("positions must be int32")
        _shaped("positions", p, (L,) if p.dim() == 1 else (B, L))
        sb, sl = (0, p.stride(0)) if p.dim() == 1 else p.stride()
    rot_dim = 2 * rot.freqs.shape[0]
    return ctypes.byref(FsRotary(rot.freqs.data_ptr(), None if p is None else p.data_ptr(), sb, sl, rot_dim, int(rot.interleaved),
                                 rot.amplitude)), rot_dim


def _rotary_axes(rot: RotaryAxes, B: int, L: int):
    """The members of fs_rotary_axes."""
    f, p = rot.freqs, rot.positions
    if f.dtype != torch.float64 or f.dim() != 1 or not f.is_contiguous():
        raise ValueError("freqs must be a contiguous float64 vector")
    axis_of = _int32("axis_of", rot.axis_of, f.shape)
    if p.dtype != torch.int32:
        raise ValueError("positions must be int32")
    if p.dim() == 2:
        _shaped("positions", p, (p.shape[0], L))
        (sa, sl), sb = p.stride(), 0
    else:
        _shaped("positions", p, (p.shape[0], B, L))
        sa, sb, sl = p.stride()
    return f.data_ptr(), axis_of, p.data_ptr(), sa, sb, sl, p.shape[0], 2 * f.shape[0], int(rot.interleaved), rot.amplitude


def _rotary_tensors(rot: Rotary | RotaryAxes | None):
    if isinstance(rot, RotaryAxes):
        return (rot.freqs, rot.axis_of, rot.positions)
    return () if rot is None else (rot.freqs, rot.positions)


def _state_desc(f: Features, state: State, dv: int, shift: bool = True):
    slots, heads, M = state.z.shape
    if heads != f.desc.heads or M != f.desc.M:
        raise ValueError("the state has other heads or features than the constants")
    _shaped("T", state.T, (slots, heads, M, dv))
    if shift:
        _shaped("shift", state.shift, (slots, heads))
    for t in state[:3 if shift else 2]:
        if t.dtype != torch.float32 or not t.is_contiguous():
            raise ValueError("states must be contiguous float32")
    return ctypes.byref(FsState(state.T.data_ptr(), state.z.data_ptr(), state.shift.data_ptr() if shift else None, slots))


def rotary_frequencies(rot_dim: int, base: float = 10000.0, scaling: str = "plain", factor: float = 1.0, original_length: int = 0,
                       low_turns: float = 1.0, high_turns: float = 32.0, device="cuda") -> torch.Tensor:
    """favorsharp_rotary_frequencies: [rot_dim / 2] float64, radians a position."""
    out = np.empty(max(rot_dim // 2, 1), dtype=np.float64)
    _check(lib().favorsharp_rotary_frequencies(rot_dim, base, ROTARY_SCALINGS[scaling], factor, original_length, low_turns, high_turns,
                                               out.ctypes.data_as(c_void_p)), "favorsharp_rotary_frequencies")
    return torch.from_numpy(out).to(device)


def rotary_sections(pairs, base: float = 10000.0, order: str = "blocks", whole: bool = False, device="cuda"):
    """favorsharp_rotary_sections: pairs[a] pairs of axis a -> (freqs float64, axis_of int32) of a RotaryAxes."""
    n = np.asarray(pairs, dtype=np.int32)
    freqs, axis_of = np.empty(max(int(n.sum()), 1), dtype=np.float64), np.empty(max(int(n.sum()), 1), dtype=np.int32)
    _check(lib().favorsharp_rotary_sections(n.size, n.ctypes.data_as(c_void_p), base, AXES_ORDERS[order], int(whole),
                                            freqs.ctypes.data_as(c_void_p), axis_of.ctypes.data_as(c_void_p)), "favorsharp_rotary_sections")
    return torch.from_numpy(freqs).to(device), torch.from_numpy(axis_of).to(device)


def rotary(X: torch.Tensor, rot: Rotary | RotaryAxes, X2: torch.Tensor | None = None, transposed: bool = False, out: torch.Tensor | None = None,
           out2: torch.Tensor | None = None):
    """favorsharp_rotary, or favorsharp_rotary_axes for a RotaryAxes: X [B,H,L,d] (and X2 [B,H2,L,d]) turned by their positions -> Y (or (Y, Y2)); transposed: the backward pass.
    out may be X itself, out2 X2."""
    B, H, L, d = X.shape
    if out is None:
        out = _empty((B, H, L, d), X.dtype, X.device)
    _shaped("out", out, X.shape)
    H2 = 0
    if X2 is not None:
        H2 = X2.shape[1]
        _shaped("X2", X2, (B, H2, L, d))
        if out2 is None:
            out2 = _empty((B, H2, L, d), X2.dtype, X.device)
        _shaped("out2", out2, X2.shape)
    device = _one_device(X, X2, out, out2, *_rotary_tensors(rot))
    if isinstance(rot, RotaryAxes):
        tensors = (X, out) if X2 is None else (X, out, X2, out2)
        held, at = _packed(tensors, _AXES, _rotary_axes(rot, B, L))
        second = (at + 80, at + 120) if H2 else (None, None)
        with _on(device):
            st = lib().favorsharp_rotary_axes(at + 40 * len(tensors), at, H, second[0], H2, B, L, d, int(transposed), at + 40, second[1],
                                              _raw_stream(device.index))
        _check(st, "favorsharp_rotary_axes")
        return out if X2 is None else (out, out2)
    r, _ = _rotary_desc(rot, B, L)
    two = (ctypes.byref(_desc4(X2)), ctypes.byref(_desc4(out2))) if H2 else (None, None)
    with _on(device):
        st = lib().favorsharp_rotary(r, ctypes.byref(_desc4(X)), H, two[0], H2, B, L, d, int(transposed), ctypes.byref(_desc4(out)), two[1],
                                     _raw_stream(device.index))
    _check(st, "favorsharp_rotary")
    return out if X2 is None else (out, out2)


def state_prepare(theta: torch.Tensor, Omega: torch.Tensor, qk_scale: float, heads: int | None = None) -> Features:
    """favorsharp_state_prepare: theta [groups,*], Omega [omega_groups,M,d] -> the constants of `heads` key heads (default: the larger
    number of sets).  Waits for the stream."""
    theta, Omega = (theta if theta.dim() == 2 else theta[None]), (Omega if Omega.dim() == 3 else Omega[None])
    og, M, d = Omega.shape
    heads = max(theta.shape[0], og) if heads is None else heads
    if theta.dtype != torch.float32 or Omega.dtype != torch.float32 or not theta.is_contiguous() or not Omega.is_contiguous():
        raise ValueError("theta and Omega must be contiguous float32")
    _shaped("theta", theta, (theta.shape[0], theta_floats(d)))
    device = _one_device(theta, Omega)
    nbytes = int(lib().favorsharp_state_features_bytes(heads, d, M, theta.shape[0], og))
    buf = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)
    desc = FsFeatures(buf.data_ptr(), buf.numel())
    with _on(device):
        st = lib().favorsharp_state_prepare(theta.data_ptr(), theta.shape[0], Omega.data_ptr(), og, heads, d, M, qk_scale, ctypes.byref(desc),
                                            _raw_stream(device.index))
    _check(st, "favorsharp_state_prepare")
    return Features(buf, desc)


def state_new(slots: int, heads: int, M: int, dv: int, device="cuda") -> State:
    """Empty states."""
    return State(torch.zeros((slots, heads, M, dv), dtype=torch.float32, device=device),
                 torch.zeros((slots, heads, M), dtype=torch.float32, device=device),
                 torch.full((slots, heads), -math.inf, dtype=torch.float32, device=device))


def state_append(f: Features, state: State, K: torch.Tensor, V: torch.Tensor, lengths: torch.Tensor | None = None,
                 slots: torch.Tensor | None = None, rotary: Rotary | None = None, fresh: bool = False,
                 left_out: torch.Tensor | None = None, workspace: torch.Tensor | None = None) -> State:
    """favorsharp_state_append: K [B,heads,L,d], V [B,heads,L,dv] onto the states of the slots (in place)."""
    B, heads, L, d = K.shape
    dv = V.shape[3]
    _shaped("K", K, (B, f.desc.heads, L, f.desc.d))
    _shaped("V", V, (B, heads, L, dv))
    device = _one_device(K, V, f.buffer, *state, lengths, slots, left_out, workspace, *_rotary_tensors(rotary))
    r, rot_dim = _rotary_desc(rotary, B, L)
    if slots is None and B > state.z.shape[0]:
        raise ValueError("more sequences than slots")
    fd = ctypes.byref(f.desc)
    ws, ws_bytes, held = _room(lib().favorsharp_state_append_workspace_bytes(fd, B, L, dv, rot_dim), device, workspace)
    with _on(device):
        st = lib().favorsharp_state_append(fd, _state_desc(f, state, dv), _int32("slots", slots, (B,)), ctypes.byref(_desc4(K)),
                                           ctypes.byref(_desc4(V)), B, L, dv, _int32("lengths", lengths, (B,)), r, int(fresh),
                                           _counter("left_out", left_out), ws, ws_bytes, _raw_stream(device.index))
    _check(st, "favorsharp_state_append")
    return state


def state_attention(f: Features, state: State, Q: torch.Tensor, lengths: torch.Tensor | None = None, slots: torch.Tensor | None = None,
                    rotary: Rotary | None = None, out: torch.Tensor | None = None, out_dtype=None, unread: torch.Tensor | None = None,
                    workspace: torch.Tensor | None = None) -> torch.Tensor:
    """favorsharp_state_attention: Q [B,H,L,d] against the states of the slots -> Y [B,H,L,dv]."""
    B, H, L, d = Q.shape
    dv = state.T.shape[3]
    _shaped("Q", Q, (B, H, L, f.desc.d))
    if out is None:
        out = _empty((B, H, L, dv), out_dtype or Q.dtype, Q.device)
    _shaped("out", out, (B, H, L, dv))
    device = _one_device(Q, out, f.buffer, *state, lengths, slots, unread, workspace, *_rotary_tensors(rotary))
    r, rot_dim = _rotary_desc(rotary, B, L)
    fd = ctypes.byref(f.desc)
    ws, ws_bytes, held = _room(lib().favorsharp_state_attention_workspace_bytes(fd, B, H, L, dv, rot_dim), device, workspace)
    with _on(device):
        st = lib().favorsharp_state_attention(fd, _state_desc(f, state, dv), _int32("slots", slots, (B,)), ctypes.byref(_desc4(Q)), B, H, L, dv,
                                              _int32("lengths", lengths, (B,)), r, ctypes.byref(_desc4(out)), _counter("unread", unread),
                                              ws, ws_bytes, _raw_stream(device.index))
    _check(st, "favorsharp_state_attention")
    return out


def state_step(f: Features, state: State, Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, slots: torch.Tensor | None = None,
               rotary: Rotary | None = None, out: torch.Tensor | None = None, out_dtype=None,
               unread: torch.Tensor | None = None, workspace: torch.Tensor | None = None) -> torch.Tensor:
    """favorsharp_state_step: K [B,heads,1,d], V [B,heads,1,dv] onto the states (in place), then Q [B,H,1,d] against them -> Y."""
    B, H, L, d = Q.shape
    dv = V.shape[3]
    _shaped("Q", Q, (B, H, 1, f.desc.d))
    _shaped("K", K, (B, f.desc.heads, 1, d))
    _shaped("V", V, (B, f.desc.heads, 1, dv))
    if out is None:
        out = _empty((B, H, 1, dv), out_dtype or Q.dtype, Q.device)
    _shaped("out", out, (B, H, 1, dv))
    device = _one_device(Q, K, V, out, f.buffer, *state, slots, unread, workspace, *_rotary_tensors(rotary))
    r, _ = _rotary_desc(rotary, B, 1)
    fd = ctypes.byref(f.desc)
    ws, ws_bytes, held = _room(lib().favorsharp_state_step_workspace_bytes(fd, B, H), device, workspace)
    with _on(device):
        st = lib().favorsharp_state_step(fd, _state_desc(f, state, dv), _int32("slots", slots, (B,)), ctypes.byref(_desc4(Q)),
                                         ctypes.byref(_desc4(K)), ctypes.byref(_desc4(V)), B, H, dv, r, ctypes.byref(_desc4(out)),
                                         _counter("unread", unread), ws, ws_bytes, _raw_stream(device.index))
    _check(st, "favorsharp_state_step")
    return out


def state_attention_backward(f: Features, state: State, Q: torch.Tensor, dY: torch.Tensor, lengths: torch.Tensor | None = None,
                             slots: torch.Tensor | None = None, rotary: Rotary | None = None, grad_dtype=None,
                             dQ: torch.Tensor | None = None, dstate: State | None = None, workspace: torch.Tensor | None = None):
    """favorsharp_state_attention_backward: gradients of sum(Y * dY) -> (dQ, dstate), dstate a State of the pool's shape without shift."""
    B, H, L, d = Q.shape
    dv = state.T.shape[3]
    _shaped("Q", Q, (B, H, L, f.desc.d))
    _shaped("dY", dY, (B, H, L, dv))
    if dQ is None:
        dQ = _empty((B, H, L, d), grad_dtype or Q.dtype, Q.device)
    if dstate is None:
        dstate = State(torch.empty_like(state.T), torch.empty_like(state.z), None)
    _shaped("dQ", dQ, Q.shape)
    device = _one_device(Q, dY, dQ, f.buffer, *state, *dstate, lengths, slots, workspace, *_rotary_tensors(rotary))
    r, rot_dim = _rotary_desc(rotary, B, L)
    fd = ctypes.byref(f.desc)
    ws, ws_bytes, held = _room(lib().favorsharp_state_attention_backward_workspace_bytes(fd, B, H, L, dv, rot_dim), device, workspace)
    with _on(device):
        st = lib().favorsharp_state_attention_backward(fd, _state_desc(f, state, dv), _int32("slots", slots, (B,)), ctypes.byref(_desc4(Q)),
                                                       ctypes.byref(_desc4(dY)), B, H, L, dv, _int32("lengths", lengths, (B,)), r,
                                                       ctypes.byref(_desc4(dQ)), _state_desc(f, dstate, dv, False), ws, ws_bytes,
                                                       _raw_stream(device.index))
    _check(st, "favorsharp_state_attention_backward")
    return dQ, dstate


def state_append_backward(f: Features, state: State, dstate: State, K: torch.Tensor, V: torch.Tensor, lengths: torch.Tensor | None = None,
                          slots: torch.Tensor | None = None, rotary: Rotary | None = None, grad_dtype=None, grads=None,
                          workspace: torch.Tensor | None = None):
    """favorsharp_state_append_backward: dstate (at `state`, the append's result) -> (dK, dV)."""
    B, heads, L, d = K.shape
    dv = V.shape[3]
    _shaped("K", K, (B, f.desc.heads, L, f.desc.d))
    _shaped("V", V, (B, heads, L, dv))
    if grads is None:
        grads = (_empty((B, heads, L, d), grad_dtype or K.dtype, K.device),
                 _empty((B, heads, L, dv), grad_dtype or V.dtype, K.device))
    dK, dV = grads
    _shaped("dK", dK, K.shape)
    _shaped("dV", dV, V.shape)
    device = _one_device(K, V, dK, dV, f.buffer, *state, *dstate, lengths, slots, workspace, *_rotary_tensors(rotary))
    r, rot_dim = _rotary_desc(rotary, B, L)
    fd = ctypes.byref(f.desc)
    ws, ws_bytes, held = _room(lib().favorsharp_state_append_backward_workspace_bytes(fd, B, L, dv, rot_dim), device, workspace)
    with _on(device):
        st = lib().favorsharp_state_append_backward(fd, _state_desc(f, state, dv), _int32("slots", slots, (B,)),
                                                    _state_desc(f, dstate, dv, False), ctypes.byref(_desc4(K)), ctypes.byref(_desc4(V)), B, L, dv,
                                                    _int32("lengths", lengths, (B,)), r, ctypes.byref(_desc4(dK)), ctypes.byref(_desc4(dV)),
                                                    ws, ws_bytes, _raw_stream(device.index))
    _check(st, "favorsharp_state_append_backward")
    return dK, dV


# ------------------------------------------------------------------ linear attention with a decay for each head
def _decay_checked(Q, K, V, log_decay, L, slots, pools, more=()):
    """Shapes of a call's tensors: (B, H, heads, d, dv, slots of the pools)."""
    B, H, n, d = Q.shape
    heads, dv = K.shape[1], V.shape[3]
    if K.shape != (B, heads, L, d) or V.shape != (B, heads, L, dv) or n != L:
        _shaped("Q", Q, (B, H, L, d))
        _shaped("K", K, (B, heads, L, d))
        _shaped("V", V, (B, heads, L, dv))
    for name, t, like in more:
        _shaped(name, t, (B, H, L, dv) if like is None else like.shape)
    if log_decay.dtype != torch.float32 or not log_decay.is_contiguous():
        raise ValueError("log_decay must be contiguous float32")
    _shaped("log_decay", log_decay, (heads,))
    size = 0
    for p in pools:
        if p is None:
            continue
        if p.dtype != torch.float32 or not p.is_contiguous():
            raise ValueError("states must be contiguous float32")
        size = size or p.shape[0]
        _shaped("state", p, (size, heads, d, dv))
        if slots is None and B > size:
            raise ValueError("more sequences than slots")
    return B, H, heads, d, dv, size


def decay_state_new(slots: int, heads: int, d: int, dv: int, device="cuda") -> torch.Tensor:
    """Empty states of decay_attention and decay_step: [slots, heads, d, dv] float32."""
    return torch.zeros((slots, heads, d, dv), dtype=torch.float32, device=device)


def decay_attention(Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, log_decay: torch.Tensor, scale: float = 1.0,
                    before: torch.Tensor | None = None, after: torch.Tensor | None = None, lengths: torch.Tensor | None = None,
                    slots: torch.Tensor | None = None, out: torch.Tensor | None = None, out_dtype=None, left_out: torch.Tensor | None = None,
                    workspace: torch.Tensor | None = None) -> torch.Tensor:
    """favorsharp_decay_attention: Q [B,H,L,d], K [B,heads,L,d], V [B,heads,L,dv], log_decay [heads] -> Y [B,H,L,dv].  before, after: pools
    [slots,heads,d,dv] (the same one: in place)."""
    L = Q.shape[2]
    B, H, heads, d, dv, size = _decay_checked(Q, K, V, log_decay, L, slots, (before, after))
    if out is None:
        out = _new((B, H, L, dv), Q) if out_dtype is None else _empty((B, H, L, dv), out_dtype, Q.device)
    else:
        _shaped("out", out, (B, H, L, dv))
    device = _one_device(Q, K, V, out, log_decay, before, after, lengths, slots, left_out, workspace)
    held, at = _packed((Q, K, V, out), _POOL + _POOL, (0 if before is None else before.data_ptr(), size, 0 if after is None else after.data_ptr(), size))
    L_ = lib()
    ws, ws_bytes, room = _room(L_.favorsharp_decay_attention_workspace_bytes(B, H, heads, L, d, dv), device, workspace)
    with _on(device):
        st = L_.favorsharp_decay_attention(at, at + 40, at + 80, B, H, heads, L, d, dv, log_decay.data_ptr(), scale,
                                           None if before is None else at + 160, None if after is None else at + 176,
                                           _int32("slots", slots, (B,)), _int32("lengths", lengths, (B,)), at + 120, _counter("left_out", left_out),
                                           ws, ws_bytes, _raw_stream(device.index))
    _check(st, "favorsharp_decay_attention")
    return out


def decay_attention_backward(Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, dY: torch.Tensor, log_decay: torch.Tensor, scale: float = 1.0,
                             before: torch.Tensor | None = None, dafter: torch.Tensor | None = None, lengths: torch.Tensor | None = None,
                             slots: torch.Tensor | None = None, exclusive: bool | None = None, grad_dtype=None, grads=None,
                             dbefore: torch.Tensor | None = None, workspace: torch.Tensor | None = None):
    """favorsharp_decay_attention_backward: gradients of sum(Y * dY) + sum(after * dafter) -> (dQ, dK, dV, dbefore), dbefore a pool if there
    is one of `before` (or is given), else None.  exclusive: the forward call had `after` (None: it did if there is dafter)."""
    L = Q.shape[2]
    if grads is None:
        grads = tuple(_empty(t.shape, grad_dtype or t.dtype, t.device) for t in (Q, K, V))
    if dbefore is None and before is not None:
        dbefore = torch.empty_like(before)
    B, H, heads, d, dv, size = _decay_checked(Q, K, V, log_decay, L, slots, (before, dafter, dbefore),
                                              (("dY", dY, None), ("dQ", grads[0], Q), ("dK", grads[1], K), ("dV", grads[2], V)))
    device = _one_device(Q, K, V, dY, *grads, log_decay, before, dafter, dbefore, lengths, slots, workspace)
    pools = (before, dafter, dbefore)
    held, at = _packed((Q, K, V, dY, *grads), 3 * _POOL, [x for p in pools for x in (0 if p is None else p.data_ptr(), size)])
    pool = [None if p is None else at + 280 + 16 * i for i, p in enumerate(pools)]
    exclusive = dafter is not None if exclusive is None else exclusive
    L_ = lib()
    ws, ws_bytes, room = _room(L_.favorsharp_decay_attention_backward_workspace_bytes(B, H, heads, L, d, dv, int(dbefore is not None)), device,
                               workspace)
    with _on(device):
        st = L_.favorsharp_decay_attention_backward(at, at + 40, at + 80, at + 120, B, H, heads, L, d, dv, log_decay.data_ptr(), scale, pool[0], pool[1],
                                                    _int32("slots", slots, (B,)), _int32("lengths", lengths, (B,)), int(exclusive), at + 160,
                                                    at + 200, at + 240, pool[2], ws, ws_bytes, _raw_stream(device.index))
    _check(st, "favorsharp_decay_attention_backward")
    return (*grads, dbefore)


def decay_step(state: torch.Tensor, Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, log_decay: torch.Tensor, scale: float = 1.0,
               slots: torch.Tensor | None = None, out: torch.Tensor | None = None, out_dtype=None,
               left_out: torch.Tensor | None = None) -> torch.Tensor:
    """favorsharp_decay_step: K [B,heads,1,d], V [B,heads,1,dv] into the states (in place), then Q [B,H,1,d] -> Y [B,H,1,dv]."""
    B, H, heads, d, dv, size = _decay_checked(Q, K, V, log_decay, 1, slots, (state,))
    if out is None:
        out = _new((B, H, 1, dv), Q) if out_dtype is None else _empty((B, H, 1, dv), out_dtype, Q.device)
    else:
        _shaped("out", out, (B, H, 1, dv))
    device = _one_device(Q, K, V, out, log_decay, state, slots, left_out)
    held, at = _packed((Q, K, V, out), _POOL, (state.data_ptr(), size))
    with _on(device):
        st = lib().favorsharp_decay_step(at + 160, _int32("slots", slots, (B,)), at, at + 40, at + 80, B, H, heads, d, dv, log_decay.data_ptr(), scale,
                                         at + 120, _counter("left_out", left_out), _raw_stream(device.index))
    _check(st, "favorsharp_decay_step")
    return out
