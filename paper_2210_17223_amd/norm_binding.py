"""Thin Python binding of include/moe_norm.h (argument marshalling only)."""
from __future__ import annotations

import ctypes as C

import torch

from .binding import DTYPE, _check, arg, lib, opt, raw_stream

F32 = torch.float32
KIND = {"rms": 0, "layer": 1}
_Z = {**DTYPE, "f16": 2}
_TORCH = {0: torch.float32, 1: torch.bfloat16, 2: torch.float16}


class NormShape(C.Structure):
    """Mirror of moe_norm_shape in include/moe_norm.h."""
    _fields_ = [("T", C.c_int32), ("d", C.c_int32), ("kind", C.c_int32), ("dtype", C.c_int32), ("res", C.c_int32),
                ("z", C.c_int32), ("gate_tokens", C.c_int32), ("eps", C.c_float), ("scale", C.c_float)]

    @classmethod
    def make(cls, T, d, kind="rms", dtype="bf16", res="f32", z="f32", eps=1e-5, scale=1.0, gate_tokens=0):
        return cls(T, d, KIND[kind], DTYPE[dtype], DTYPE[res], _Z[z], gate_tokens, eps, scale)

    @property
    def gates(self):
        """Rows of the gate matrix."""
        return -(-self.T // self.gate_tokens) if self.gate_tokens else 1

    @property
    def torch_dtype(self):
        return _TORCH[self.dtype]

    @property
    def res_torch_dtype(self):
        return _TORCH[self.res]

    @property
    def z_torch_dtype(self):
        return _TORCH[self.z]

    @property
    def dz_torch_dtype(self):
        """Type of z's gradient: fp32 where z is, else bf16."""
        return torch.float32 if self.z == 0 else torch.bfloat16


_ready = False


def _lib():
    global _ready
    L = lib()
    if not _ready:
        sp, vp = C.POINTER(NormShape), C.c_void_p
        L.moe_norm_workspace_bytes.restype = C.c_size_t
        L.moe_norm_workspace_bytes.argtypes = [sp]
        for name, pointers in (("before", 5), ("before_backward", 9), ("after", 10), ("after_backward", 17)):
            f = getattr(L, "moe_norm_" + name)
            f.restype = C.c_int
            f.argtypes = [sp] + [vp] * pointers
        _ready = True
    return L


def moe_norm_workspace_bytes(n: NormShape) -> int:
    return int(_lib().moe_norm_workspace_bytes(C.byref(n)))


def moe_norm_before(n: NormShape, x, w_next, b_next, next, stream=None) -> None:
    m = n.T * n.d
    _check(_lib().moe_norm_before(
        C.byref(n), arg(x, n.res_torch_dtype, m, "x"), arg(w_next, F32, n.d, "w_next"), opt(b_next, F32, n.d, "b_next"),
        arg(next, n.torch_dtype, m, "next"), raw_stream(stream, x)))


def moe_norm_before_backward(n: NormShape, x, w_next, dnext, dr, dx, dw_next, db_next, workspace,
                             stream=None) -> None:
    m, d, res = n.T * n.d, n.d, n.res_torch_dtype
    _check(_lib().moe_norm_before_backward(
        C.byref(n), arg(x, res, m, "x"), arg(w_next, F32, d, "w_next"), arg(dnext, n.torch_dtype, m, "dnext"),
        arg(dr, res, m, "dr"), arg(dx, res, m, "dx"), arg(dw_next, F32, d, "dw_next"), opt(db_next, F32, d, "db_next"),
        arg(workspace, torch.uint8, moe_norm_workspace_bytes(n), "workspace"), raw_stream(stream, x)))


def moe_norm_after(n: NormShape, x, z, w, b, gate, r, w_next, b_next, next, stream=None) -> None:
    m, d, res = n.T * n.d, n.d, n.res_torch_dtype
    _check(_lib().moe_norm_after(
        C.byref(n), arg(x, res, m, "x"), arg(z, n.z_torch_dtype, m, "z"), arg(w, F32, d, "w"), opt(b, F32, d, "b"),
        opt(gate, F32, n.gates * d, "gate"), arg(r, res, m, "r"), arg(w_next, F32, d, "w_next"),
        opt(b_next, F32, d, "b_next"), arg(next, n.torch_dtype, m, "next"), raw_stream(stream, x)))


def moe_norm_after_backward(n: NormShape, z, r, w, b, gate, w_next, dr, dnext, dx, dz, dw, db, dgate, dw_next,
                            db_next, workspace, stream=None) -> None:
    m, d, res, g = n.T * n.d, n.d, n.res_torch_dtype, n.gates * n.d
    _check(_lib().moe_norm_after_backward(
        C.byref(n), arg(z, n.z_torch_dtype, m, "z"), arg(r, res, m, "r"), arg(w, F32, d, "w"), opt(b, F32, d, "b"),
        opt(gate, F32, g, "gate"), arg(w_next, F32, d, "w_next"), arg(dr, res, m, "dr"),
        arg(dnext, n.torch_dtype, m, "dnext"), arg(dx, res, m, "dx"), arg(dz, n.dz_torch_dtype, m, "dz"),
        arg(dw, F32, d, "dw"), opt(db, F32, d, "db"), opt(dgate, F32, g, "dgate"), arg(dw_next, F32, d, "dw_next"),
        opt(db_next, F32, d, "db_next"), arg(workspace, torch.uint8, moe_norm_workspace_bytes(n), "workspace"),
        raw_stream(stream, z)))
