"""Thin Python binding of include/moe_q8.h (argument marshalling only)."""
from __future__ import annotations

import ctypes as C

import torch

from .binding import ACT, MoeError, Shape, _check, arg, lib, moe_max_rows, moe_workspace_bytes, opt, raw_stream
from .norm_binding import NormShape

F32, I8, I32, U8 = torch.float32, torch.int8, torch.int32, torch.uint8
_TYPE = {"f32": 0, "bf16": 1, "f16": 2}
_TORCH = {0: torch.float32, 1: torch.bfloat16, 2: torch.float16}
_NUMBER = {v: k for k, v in _TORCH.items()}


class Q8Shape(C.Structure):
    """Mirror of moe_q8_shape in include/moe_q8.h."""
    _fields_ = [(name, C.c_int32) for name in ("R", "E", "N", "K", "act", "res", "y")]

    @classmethod
    def make(cls, R, E, N, K, act="identity", res="f32", y="bf16"):
        return cls(R, E, N, K, ACT[act], _TYPE[res], _TYPE[y])

    @property
    def res_torch_dtype(self):
        return _TORCH[self.res]

    @property
    def y_torch_dtype(self):
        return _TORCH[self.y]


_ready = False


def _lib():
    global _ready
    L = lib()
    if not _ready:
        vp, i32, i64 = C.c_void_p, C.c_int32, C.c_int64
        L.moe_q8_rows.argtypes = L.moe_q8_values.argtypes = [i64, i32, i32] + [vp] * 4
        for name, shape, pointers in (("norm_before_q8", NormShape, 7), ("norm_after_q8", NormShape, 12), ("q8_linear", Q8Shape, 9),
                                      ("dispatch_q8", Shape, 11), ("gated_ffn_q8", Shape, 11)):
            getattr(L, "moe_" + name).argtypes = [C.POINTER(shape)] + [vp] * pointers
        for name in ("q8_rows", "q8_values", "norm_before_q8", "norm_after_q8", "q8_linear", "dispatch_q8", "gated_ffn_q8"):
            getattr(L, "moe_" + name).restype = C.c_int
        L.moe_q8_linear_kernel.argtypes = [C.POINTER(Q8Shape), C.c_char_p, C.c_size_t]
        L.moe_gated_q8_kernel.argtypes = [C.POINTER(Shape), i32, C.c_char_p, C.c_size_t]
        L.moe_q8_linear_kernel.restype = L.moe_gated_q8_kernel.restype = C.c_int
        L.moe_gated_q8_workspace_bytes.restype = C.c_size_t
        L.moe_gated_q8_workspace_bytes.argtypes = [C.POINTER(Shape)]
        _ready = True
    return L


def _rows_of(x, name):
    """Rows, row length and type number of a matrix (of more axes: the last one's rows)."""
    if x is None or x.dim() < 1 or x.dtype not in _NUMBER:
        raise MoeError(f"{name}: expected rows of float32, bfloat16 or float16")
    K = x.shape[-1]
    return x.numel() // max(K, 1), K, _NUMBER[x.dtype]


def moe_q8_rows(x, q, scale, stream=None) -> None:
    """x [..., K] in 8 bits: q [..., K] and a scale for every row."""
    R, K, type = _rows_of(x, "x")
    _check(_lib().moe_q8_rows(R, K, type, arg(x, x.dtype, R * K, "x"), arg(q, I8, R * K, "q"), arg(scale, F32, R, "scale"),
                              raw_stream(stream, x)))


def moe_q8_values(q, scale, x, stream=None) -> None:
    """The values that q [..., K] and its scales stand for, in x's type."""
    R, K, type = _rows_of(x, "x")
    _check(_lib().moe_q8_values(R, K, type, arg(q, I8, R * K, "q"), arg(scale, F32, R, "scale"), arg(x, x.dtype, R * K, "x"),
                                raw_stream(stream, x)))


def moe_norm_before_q8(n: NormShape, x, w_next, b_next, next, q, scale, stream=None) -> None:
    m = n.T * n.d
    _check(_lib().moe_norm_before_q8(
        C.byref(n), arg(x, n.res_torch_dtype, m, "x"), arg(w_next, F32, n.d, "w_next"), opt(b_next, F32, n.d, "b_next"),
        opt(next, n.torch_dtype, m, "next"), arg(q, I8, m, "q"), arg(scale, F32, n.T, "scale"), raw_stream(stream, x)))


def moe_norm_after_q8(n: NormShape, x, z, w, b, gate, r, w_next, b_next, next, q, scale, stream=None) -> None:
    m, d, res = n.T * n.d, n.d, n.res_torch_dtype
    _check(_lib().moe_norm_after_q8(
        C.byref(n), arg(x, res, m, "x"), arg(z, n.z_torch_dtype, m, "z"), arg(w, F32, d, "w"), opt(b, F32, d, "b"),
        opt(gate, F32, n.gates * d, "gate"), arg(r, res, m, "r"), arg(w_next, F32, d, "w_next"),
        opt(b_next, F32, d, "b_next"), opt(next, n.torch_dtype, m, "next"), arg(q, I8, m, "q"), arg(scale, F32, n.T, "scale"),
        raw_stream(stream, x)))


def moe_q8_linear(s: Q8Shape, x, x_scale, offsets, w, w_scale, bias, r, y, stream=None) -> None:
    _check(_lib().moe_q8_linear(
        C.byref(s), arg(x, I8, s.R * s.K, "x"), arg(x_scale, F32, s.R, "x_scale"), arg(offsets, I32, s.E + 1, "offsets"),
        arg(w, I8, s.E * s.N * s.K, "w"), arg(w_scale, F32, s.E * s.N, "w_scale"), opt(bias, F32, s.E * s.N, "bias"),
        opt(r, _TORCH.get(s.res), s.R * s.N, "r"), arg(y, _TORCH.get(s.y), s.R * s.N, "y"), raw_stream(stream, x)))


def moe_q8_linear_kernel(s: Q8Shape) -> str:
    """Name, tile and form of the kernel that moe_q8_linear launches."""
    buf = C.create_string_buffer(96)
    _check(_lib().moe_q8_linear_kernel(C.byref(s), buf, C.sizeof(buf)))
    return buf.value.decode()


def moe_gated_q8_kernel(s: Shape, which: int) -> str:
    """The same of moe_gated_ffn_q8's products (0: first projections, 1: second)."""
    buf = C.create_string_buffer(96)
    _check(_lib().moe_gated_q8_kernel(C.byref(s), int(which), buf, C.sizeof(buf)))
    return buf.value.decode()


def moe_dispatch_q8(s: Shape, x, x_scale, expert_idx, counts, offsets, slot_of, src_of, xe, xe_scale, workspace,
                    stream=None) -> None:
    rows, A = moe_max_rows(s), s.T * s.k
    _check(_lib().moe_dispatch_q8(
        C.byref(s), arg(x, I8, s.T * s.d_model, "x"), arg(x_scale, F32, s.T, "x_scale"), arg(expert_idx, I32, A, "expert_idx"),
        arg(counts, I32, s.E, "counts"), arg(offsets, I32, s.E + 1, "offsets"), arg(slot_of, I32, A, "slot_of"),
        arg(src_of, I32, rows, "src_of"), opt(xe, I8, rows * s.d_model, "xe"), opt(xe_scale, F32, rows, "xe_scale"),
        arg(workspace, U8, moe_workspace_bytes(s, 1), "workspace"), raw_stream(stream, x)))


def moe_gated_q8_workspace_bytes(s: Shape) -> int:
    return int(_lib().moe_gated_q8_workspace_bytes(C.byref(s)))


def moe_gated_ffn_q8(s: Shape, x, x_scale, src_of, offsets, q13, scale13, q2, scale2, ye, workspace, stream=None) -> None:
    rows, d, h, n = moe_max_rows(s), s.d_model, s.d_ff, s.E * s.d_model * s.d_ff
    held = rows if src_of is None else s.T
    _check(_lib().moe_gated_ffn_q8(
        C.byref(s), arg(x, I8, held * d, "x"), arg(x_scale, F32, held, "x_scale"), opt(src_of, I32, rows, "src_of"),
        arg(offsets, I32, s.E + 1, "offsets"), arg(q13, I8, 2 * n, "q13"), arg(scale13, F32, s.E * 2 * h, "scale13"),
        arg(q2, I8, n, "q2"), arg(scale2, F32, s.E * d, "scale2"), arg(ye, torch.float16, rows * d, "ye"),
        arg(workspace, U8, moe_gated_q8_workspace_bytes(s), "workspace"), raw_stream(stream, x)))
