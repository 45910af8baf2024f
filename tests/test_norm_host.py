"""CPU-side checks of include/moe_norm.h: sizes, and refusals before anything is enqueued."""
import ctypes as C

import pytest
import torch

import paper_2210_17223_amd as moe
from paper_2210_17223_amd import norm_binding


def shape(**kw):
    return moe.NormShape.make(**{**dict(T=64, d=128), **kw})


def test_shape_properties():
    n = shape(T=10, kind="layer", res="bf16", z="f16", gate_tokens=3)
    assert n.gates == 4 and n.torch_dtype == torch.bfloat16 and n.res_torch_dtype == torch.bfloat16
    assert n.z_torch_dtype == torch.float16 and n.dz_torch_dtype == torch.bfloat16
    assert shape().gates == 1 and shape(z="f32").dz_torch_dtype == torch.float32


def test_workspace_holds_six_vectors_per_run_and_stays_small():
    assert moe.moe_norm_workspace_bytes(shape(T=1, d=8)) == 6 * 8 * 4
    for T, d in ((1, 16384), (7, 64), (4096, 2048), (1 << 20, 8192), ((1 << 31) - 1, 8)):
        b = moe.moe_norm_workspace_bytes(shape(T=T, d=d))
        assert 0 < b <= 6 * 4 * max(1 << 21, 256 * d)


@pytest.mark.parametrize("kw,frag", [
    (dict(T=0), ">= 1"), (dict(d=0), ">= 1"), (dict(gate_tokens=-1), "gate_tokens"), (dict(eps=-1.0), "eps"),
    (dict(eps=float("nan")), "eps"), (dict(d=100), "multiples of 8"), (dict(d=16392), "up to 16384"),
])
def test_bad_shapes_are_refused(kw, frag):
    n = shape(**kw)
    assert moe.moe_norm_workspace_bytes(n) == 0
    assert frag in moe.moe_last_error()


@pytest.mark.parametrize("field,value", [("kind", 2), ("kind", -1), ("dtype", 2), ("res", 2), ("z", 3), ("z", -1)])
def test_unknown_kinds_and_types_are_refused(field, value):
    n = shape()
    setattr(n, field, value)
    assert moe.moe_norm_workspace_bytes(n) == 0
    assert "norm" in moe.moe_last_error()


def test_null_and_misaligned_pointers_are_refused():
    L = norm_binding._lib()
    n, ok, z, odd = shape(), C.c_void_p(4096), C.c_void_p(0), C.c_void_p(4100)
    counts = {"before": 4, "before_backward": 8, "after": 9, "after_backward": 16}
    required = {"before": [0, 1, 3], "before_backward": [0, 1, 2, 3, 4, 5, 7],
                "after": [0, 1, 2, 5, 6, 8], "after_backward": [0, 1, 2, 5, 6, 7, 8, 9, 10, 13, 15]}
    for name, count in counts.items():
        f = getattr(L, "moe_norm_" + name)
        for i in range(count):
            args = [ok] * count
            args[i] = odd
            assert f(C.byref(n), *args, z) == 1 and "aligned" in moe.moe_last_error()
        for i in required[name]:
            args = [ok] * count
            args[i] = z
            assert f(C.byref(n), *args, z) == 1 and "is NULL" in moe.moe_last_error()
        assert f(None, *[ok] * count, z) == 1
