"""Thin Python binding of include/moe_gated.h (argument marshalling only)."""
from __future__ import annotations

import ctypes as C

import torch

from .binding import Shape, _check, arg, lib, moe_max_rows, moe_packed_weight_bytes, opt, raw_stream

_ready = False


def _lib():
    global _ready
    L = lib()
    if not _ready:
        sp, vp = C.POINTER(Shape), C.c_void_p
        for name in ("packed", "workspace", "backward_workspace"):
            f = getattr(L, f"moe_gated_{name}_bytes")
            f.restype = C.c_size_t
            f.argtypes = [sp]
        for name, pointers in (("pack_gated_weights", 5), ("gated_ffn", 9), ("gated_ffn_backward", 13)):
            f = getattr(L, "moe_" + name)
            f.restype = C.c_int
            f.argtypes = [sp] + [vp] * pointers
        _ready = True
    return L


def moe_gated_packed_bytes(s: Shape) -> int:
    return int(_lib().moe_gated_packed_bytes(C.byref(s)))


def moe_gated_workspace_bytes(s: Shape) -> int:
    return int(_lib().moe_gated_workspace_bytes(C.byref(s)))


def moe_gated_backward_workspace_bytes(s: Shape) -> int:
    return int(_lib().moe_gated_backward_workspace_bytes(C.byref(s)))


def moe_pack_gated_weights(s: Shape, W13, W2, W13p, W2p, stream=None) -> None:
    n, dt = s.E * s.d_model * s.d_ff, s.torch_dtype
    _check(_lib().moe_pack_gated_weights(
        C.byref(s), arg(W13, dt, 2 * n, "W13"), arg(W2, dt, n, "W2"),
        arg(W13p, torch.uint8, moe_gated_packed_bytes(s), "W13p"),
        arg(W2p, torch.uint8, moe_packed_weight_bytes(s), "W2p"), raw_stream(stream, W13)))


def moe_gated_ffn(s: Shape, xe, offsets, W13p, W2p, ye, pre, hid, workspace, stream=None) -> None:
    rows, h = moe_max_rows(s), s.d_ff
    _check(_lib().moe_gated_ffn(
        C.byref(s), arg(xe, s.torch_dtype, rows * s.d_model, "xe"), arg(offsets, torch.int32, s.E + 1, "offsets"),
        arg(W13p, torch.uint8, moe_gated_packed_bytes(s), "W13p"),
        arg(W2p, torch.uint8, moe_packed_weight_bytes(s), "W2p"), arg(ye, s.ye_dtype, rows * s.d_model, "ye"),
        opt(pre, torch.float16, rows * 2 * h, "pre"), opt(hid, torch.float16, rows * h, "hid"),
        arg(workspace, torch.uint8, moe_gated_workspace_bytes(s), "workspace"), raw_stream(stream, xe)))


def moe_gated_ffn_backward(s: Shape, xe, offsets, W13, W2, W13p, pre, hid, dye, dxe, dW13, dW2, workspace,
                           stream=None) -> None:
    rows, n, h, b = moe_max_rows(s), s.E * s.d_model * s.d_ff, s.d_ff, torch.bfloat16
    _check(_lib().moe_gated_ffn_backward(
        C.byref(s), arg(xe, b, rows * s.d_model, "xe"), arg(offsets, torch.int32, s.E + 1, "offsets"),
        arg(W13, b, 2 * n, "W13"), arg(W2, b, n, "W2"), arg(W13p, torch.uint8, moe_gated_packed_bytes(s), "W13p"),
        opt(pre, torch.float16, rows * 2 * h, "pre"), opt(hid, torch.float16, rows * h, "hid"),
        arg(dye, b, rows * s.d_model, "dye"), arg(dxe, b, rows * s.d_model, "dxe"), arg(dW13, b, 2 * n, "dW13"),
        arg(dW2, b, n, "dW2"), arg(workspace, torch.uint8, moe_gated_backward_workspace_bytes(s), "workspace"),
        raw_stream(stream, xe)))
