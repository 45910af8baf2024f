"""Thin Python binding of include/moe_gated.h (argument marshalling only)."""
from __future__ import annotations

import ctypes as C

import torch

from .binding import Shape, _check, arg, lib, moe_max_rows, moe_packed_weight_bytes, opt, raw_stream

F16, F32, U8 = torch.float16, torch.float32, torch.uint8


class Q4Shape(C.Structure):
    """Mirror of moe_q4_shape in include/moe_gated.h."""
    _fields_ = [(name, C.c_int32) for name in ("R", "E", "N", "K", "group", "x")]

    @classmethod
    def make(cls, R, E, N, K, group, x="bf16"):
        return cls(R, E, N, K, group, {"bf16": 1, "f16": 2}[x])

    @property
    def x_torch_dtype(self):
        return torch.bfloat16 if self.x == 1 else F16


_ready = False


def _lib():
    global _ready
    L = lib()
    if not _ready:
        sp, vp = C.POINTER(Shape), C.c_void_p
        for name in ("packed", "workspace", "kept_workspace", "backward_workspace", "kept_backward_workspace"):
            f = getattr(L, f"moe_gated_{name}_bytes")
            f.restype = C.c_size_t
            f.argtypes = [sp]
        L.moe_gated_q4_workspace_bytes.restype = C.c_size_t
        L.moe_gated_q4_workspace_bytes.argtypes = [sp]
        L.moe_q4_linear.restype = C.c_int
        L.moe_q4_linear.argtypes = [C.POINTER(Q4Shape)] + [vp] * 7
        L.moe_gated_ffn_q4.restype = C.c_int
        L.moe_gated_ffn_q4.argtypes = [sp, C.c_int32] + [vp] * 11
        for name, pointers in (("pack_gated_weights", 5), ("gated_ffn", 9), ("gated_ffn_backward", 13)):
            f = getattr(L, "moe_" + name)
            f.restype = C.c_int
            f.argtypes = [sp] + [vp] * pointers
        L.moe_gated_gemm_kernel.restype = C.c_int
        L.moe_gated_gemm_kernel.argtypes = [sp, C.c_int32, C.c_char_p, C.c_size_t]
        _ready = True
    return L


def moe_gated_gemm_kernel(s: Shape, which: int) -> str:
    """Name, tile and form of the kernel of a gated block's GEMM (0: first projections, 1: second, 2: dH, 3: dxe, 4: dW2, 5: dW13)."""
    buf = C.create_string_buffer(96)
    _check(_lib().moe_gated_gemm_kernel(C.byref(s), int(which), buf, C.sizeof(buf)))
    return buf.value.decode()


def moe_gated_packed_bytes(s: Shape) -> int:
    return int(_lib().moe_gated_packed_bytes(C.byref(s)))


def moe_gated_workspace_bytes(s: Shape) -> int:
    return int(_lib().moe_gated_workspace_bytes(C.byref(s)))


def moe_gated_backward_workspace_bytes(s: Shape) -> int:
    return int(_lib().moe_gated_backward_workspace_bytes(C.byref(s)))


def moe_gated_kept_workspace_bytes(s: Shape) -> int:
    """Of a call that is given pre and hid."""
    return int(_lib().moe_gated_kept_workspace_bytes(C.byref(s)))


def moe_gated_kept_backward_workspace_bytes(s: Shape) -> int:
    """Of a call that is given pre and hid."""
    return int(_lib().moe_gated_kept_backward_workspace_bytes(C.byref(s)))


_sizes = {}


def _sizes_of(s: Shape):
    """Rows and bytes that depend on the shape's values alone: (rows, W13p, W2p, workspace).  The table is read once: another
    thread may clear it at any time."""
    key = bytes(s)
    sizes = _sizes.get(key)
    if sizes is None:
        if len(_sizes) >= 1024:
            _sizes.clear()
        sizes = _sizes[key] = (moe_max_rows(s), moe_gated_packed_bytes(s), moe_packed_weight_bytes(s), moe_gated_workspace_bytes(s))
    return sizes


def moe_pack_gated_weights(s: Shape, W13, W2, W13p, W2p, stream=None) -> None:
    n, dt = s.E * s.d_model * s.d_ff, s.torch_dtype
    _check(_lib().moe_pack_gated_weights(
        C.byref(s), arg(W13, dt, 2 * n, "W13"), arg(W2, dt, n, "W2"),
        arg(W13p, torch.uint8, moe_gated_packed_bytes(s), "W13p"),
        arg(W2p, torch.uint8, moe_packed_weight_bytes(s), "W2p"), raw_stream(stream, W13)))


def moe_gated_ffn(s: Shape, xe, offsets, W13p, W2p, ye, pre, hid, workspace, stream=None) -> None:
    (rows, n13, n2, nw), d, h = _sizes_of(s), s.d_model, s.d_ff
    _check(_lib().moe_gated_ffn(
        C.byref(s), arg(xe, s.torch_dtype, rows * d, "xe"), arg(offsets, torch.int32, s.E + 1, "offsets"),
        arg(W13p, U8, n13, "W13p"), arg(W2p, U8, n2, "W2p"), arg(ye, s.ye_dtype, rows * d, "ye"),
        opt(pre, F16, rows * 2 * h, "pre"), opt(hid, F16, rows * h, "hid"),
        arg(workspace, U8, nw if hid is None else moe_gated_kept_workspace_bytes(s), "workspace"),
        raw_stream(stream, xe)))


def moe_gated_ffn_backward(s: Shape, xe, offsets, W13, W2, W13p, pre, hid, dye, dxe, dW13, dW2, workspace,
                           stream=None) -> None:
    rows, n, h, b = moe_max_rows(s), s.E * s.d_model * s.d_ff, s.d_ff, torch.bfloat16
    nw = moe_gated_backward_workspace_bytes(s) if pre is None else moe_gated_kept_backward_workspace_bytes(s)
    _check(_lib().moe_gated_ffn_backward(
        C.byref(s), arg(xe, b, rows * s.d_model, "xe"), arg(offsets, torch.int32, s.E + 1, "offsets"),
        arg(W13, b, 2 * n, "W13"), arg(W2, b, n, "W2"), arg(W13p, torch.uint8, moe_gated_packed_bytes(s), "W13p"),
        opt(pre, torch.float16, rows * 2 * h, "pre"), opt(hid, torch.float16, rows * h, "hid"),
        arg(dye, b, rows * s.d_model, "dye"), arg(dxe, b, rows * s.d_model, "dxe"), arg(dW13, b, 2 * n, "dW13"),
        arg(dW2, b, n, "dW2"), arg(workspace, torch.uint8, nw, "workspace"),
        raw_stream(stream, xe)))


def moe_gated_q4_workspace_bytes(s: Shape) -> int:
    return int(_lib().moe_gated_q4_workspace_bytes(C.byref(s)))


def _codes(q, scale, zero, values, group, name):
    g = values // group
    return (arg(q, U8, values // 2, "q" + name), arg(scale, F16, g, "scale" + name), opt(zero, U8, g, "zero" + name))


def moe_q4_linear(s: Q4Shape, x, offsets, q, scale, zero, y, stream=None) -> None:
    _check(_lib().moe_q4_linear(
        C.byref(s), arg(x, s.x_torch_dtype, s.R * s.K, "x"), arg(offsets, torch.int32, s.E + 1, "offsets"),
        *_codes(q, scale, zero, s.E * s.N * s.K, s.group or 1, ""), arg(y, F32, s.R * s.N, "y"), raw_stream(stream, x)))


def moe_gated_ffn_q4(s: Shape, group: int, xe, offsets, q13, scale13, zero13, q2, scale2, zero2, ye, workspace,
                     stream=None) -> None:
    rows, n = moe_max_rows(s), s.E * s.d_model * s.d_ff
    _check(_lib().moe_gated_ffn_q4(
        C.byref(s), group, arg(xe, torch.bfloat16, rows * s.d_model, "xe"), arg(offsets, torch.int32, s.E + 1, "offsets"),
        *_codes(q13, scale13, zero13, 2 * n, group or 1, "13"), *_codes(q2, scale2, zero2, n, group or 1, "2"),
        arg(ye, F16, rows * s.d_model, "ye"), arg(workspace, U8, moe_gated_q4_workspace_bytes(s), "workspace"),
        raw_stream(stream, xe)))
