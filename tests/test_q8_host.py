"""Host side of the 8-bit operators: shapes and pointers that are refused before anything is enqueued (no GPU needed)."""
import ctypes as C

import pytest
import torch

import paper_2210_17223_amd as moe
from paper_2210_17223_amd import q8_binding

OK, ODD, NULL = C.c_void_p(4096), C.c_void_p(4100), C.c_void_p(0)


def linear(args=None, **kw):
    base = dict(R=4, E=2, N=64, K=128, act="silu", res="f32", y="bf16")
    fields = {k: v for k, v in kw.items() if k in ("act_number", "res_number", "y_number")}
    base.update({k: v for k, v in kw.items() if k not in fields})
    s = moe.Q8Shape.make(**base)
    for k, v in fields.items():
        setattr(s, k.split("_")[0], v)
    return q8_binding._lib().moe_q8_linear(C.byref(s), *(args or [OK] * 8), NULL)


@pytest.mark.parametrize("kw,status,frag", [
    (dict(R=0), 1, ">= 1"), (dict(E=0), 1, ">= 1"), (dict(N=0), 1, ">= 1"), (dict(K=0), 1, ">= 1"), (dict(R=-5), 1, ">= 1"),
    (dict(act_number=5), 1, "moe_act"), (dict(act_number=-1), 1, "moe_act"), (dict(res_number=3), 1, "res and y"),
    (dict(y_number=-1), 1, "res and y"), (dict(K=120), 2, "multiple of 16"), (dict(K=65552), 2, "65536"), (dict(E=65), 2, "at most 64"),
    (dict(N=1 << 21), 2, "2^21"), (dict(R=1 << 30), 2, "2^30"), (dict(R=(1 << 30) - 1, N=(1 << 21) - 1), 2, "tiles"),
])
def test_linear_refuses_bad_shapes(kw, status, frag):
    assert linear(**kw) == status and frag in moe.moe_last_error()


def test_linear_refuses_bad_pointers():
    assert q8_binding._lib().moe_q8_linear(None, *[OK] * 8, NULL) == 1
    for i, name in enumerate(("x", "x_scale", "offsets", "w", "w_scale", "bias", "r", "y")):
        for bad in (NULL, ODD):
            if bad is NULL and name in ("bias", "r"):
                continue
            args = [OK] * 8
            args[i] = bad
            assert linear(args) == 1 and moe.moe_last_error().startswith(name + " is")


@pytest.mark.parametrize("R,K,type,status,frag", [
    (0, 16, 0, 1, ">= 1"), (1, 0, 0, 1, ">= 1"), (1, 16, 3, 1, "type"), (1, 16, -1, 1, "type"), (1, 24, 0, 2, "multiple of 16"),
    (1, 65552, 1, 2, "65536"), (1 << 40, 16, 1, 2, "2^40"),
])
def test_rows_and_values_refuse_bad_sizes(R, K, type, status, frag):
    L = q8_binding._lib()
    assert L.moe_q8_rows(R, K, type, OK, OK, OK, NULL) == status and frag in moe.moe_last_error()
    assert L.moe_q8_values(R, K, type, OK, OK, OK, NULL) == status and frag in moe.moe_last_error()


def test_rows_and_values_refuse_bad_pointers():
    L = q8_binding._lib()
    for i, names in enumerate((("x", "q"), ("q", "scale"), ("scale", "x"))):
        for bad in (NULL, ODD):
            args = [OK] * 3
            args[i] = bad
            for call, name in zip((L.moe_q8_rows, L.moe_q8_values), names):
                assert call(1, 16, 0, *args, NULL) == 1 and moe.moe_last_error().startswith(name + " is")


def test_norms_refuse_what_has_no_codes():
    L = q8_binding._lib()
    n = moe.NormShape.make(4, 72)
    assert L.moe_norm_before_q8(C.byref(n), *[OK] * 6, NULL) == 2 and "multiple of 16" in moe.moe_last_error()
    assert L.moe_norm_after_q8(C.byref(n), *[OK] * 11, NULL) == 2 and "multiple of 16" in moe.moe_last_error()
    assert L.moe_norm_before_q8(None, *[OK] * 6, NULL) == 1 and L.moe_norm_after_q8(None, *[OK] * 11, NULL) == 1
    n = moe.NormShape.make(0, 64)
    assert L.moe_norm_before_q8(C.byref(n), *[OK] * 6, NULL) == 1
    n = moe.NormShape.make(4, 64)
    for call, names, optional in ((L.moe_norm_before_q8, ("x", "w_next", "b_next", "next", "q", "scale"), ("b_next", "next")),
                                  (L.moe_norm_after_q8, ("x", "z", "w", "b", "gate", "r", "w_next", "b_next", "next", "q", "scale"),
                                   ("b", "gate", "b_next", "next"))):
        for i, name in enumerate(names):
            for bad in (NULL, ODD):
                if bad is NULL and name in optional:
                    continue
                args = [OK] * len(names)
                args[i] = bad
                assert call(C.byref(n), *args, NULL) == 1 and moe.moe_last_error().startswith(name + " is")


def shape(**kw):
    base = dict(T=64, d_model=64, E=4, d_ff=128, k=2, capacity=32, act="silu")
    base.update(kw)
    return moe.Shape.make(**base)


def test_gated_block_sizes_and_refusals():
    L = q8_binding._lib()
    s = shape()
    rows = moe.moe_max_rows(s)
    assert moe.moe_gated_q8_workspace_bytes(s) == rows * 128 * 2 + rows * 128 + -(-rows * 4 // 256) * 256
    for kw, frag in ((dict(dtype="f32"), "bf16"), (dict(d_model=72), "multiples of 16"), (dict(d_ff=72), "multiples of 16"),
                     (dict(d_ff=65552), "65536"), (dict(d_model=32768, d_ff=32768), "2^31"), (dict(E=65), "64"),
                     (dict(T=(1 << 29) - 1, capacity=1 << 29, d_model=65536, d_ff=16), "2^23 tiles")):
        assert moe.moe_gated_q8_workspace_bytes(shape(**kw)) == 0 and frag in moe.moe_last_error()
        assert L.moe_gated_ffn_q8(C.byref(shape(**kw)), *[OK] * 10, NULL) in (1, 2)
    assert L.moe_gated_ffn_q8(None, *[OK] * 10, NULL) == 1
    big = shape(T=1 << 20, d_model=2048, capacity=64)
    assert L.moe_gated_ffn_q8(C.byref(big), *[OK] * 10, NULL) == 2 and "moe_dispatch_q8" in moe.moe_last_error()
    for i, name in enumerate(("x", "x_scale", "src_of", "offsets", "q13", "scale13", "q2", "scale2", "ye", "workspace")):
        for bad in (NULL, ODD):
            if bad is NULL and name == "src_of":
                continue
            args = [OK] * 10
            args[i] = bad
            assert L.moe_gated_ffn_q8(C.byref(s), *args, NULL) == 1 and moe.moe_last_error().startswith(name + " is")


def test_dispatch_refusals():
    L = q8_binding._lib()
    s = shape()
    names = ("x", "x_scale", "expert_idx", "counts", "offsets", "slot_of", "src_of", "xe", "xe_scale", "workspace")
    for i, name in enumerate(names):
        for bad in (NULL, ODD):
            args = [OK] * 10
            args[i] = bad
            assert L.moe_dispatch_q8(C.byref(s), *args, NULL) == 1
            if bad is NULL and name in ("xe", "xe_scale"):
                assert "come together" in moe.moe_last_error()
            else:
                assert moe.moe_last_error().startswith(name + " is")
    assert L.moe_dispatch_q8(None, *[OK] * 10, NULL) == 1
    assert L.moe_dispatch_q8(C.byref(shape(d_model=72)), *[OK] * 10, NULL) == 2 and "multiple of 16" in moe.moe_last_error()


def test_python_calls_check_types_and_sizes():
    with pytest.raises(moe.MoeError, match="x: expected"):
        moe.moe_q8_rows(torch.zeros(2, 16, dtype=torch.float64), None, None)
    with pytest.raises(moe.MoeError, match="x: expected"):
        moe.moe_q8_rows(None, None, None)
    with pytest.raises(moe.MoeError):
        moe.moe_q8_rows(torch.zeros(2, 16), torch.zeros(2, 16, dtype=torch.int8), torch.zeros(2))      # (not on a device)
    with pytest.raises(moe.MoeError, match="x: expected"):
        moe.moe_q8_linear(moe.Q8Shape.make(2, 1, 16, 16), torch.zeros(2, 16), None, None, None, None, None, None, None)


def test_a_residual_of_another_type_may_not_be_the_output():
    s = moe.Q8Shape.make(4, 2, 64, 128, res="f32", y="bf16")
    other = C.c_void_p(8192)
    assert q8_binding._lib().moe_q8_linear(C.byref(s), *[OK] * 6, other, other, NULL) == 1 and "same" in moe.moe_last_error()


def test_kernel_names():
    name = moe.moe_q8_linear_kernel
    assert name(moe.Q8Shape.make(1, 1, 4096, 4096)) == "q8_stream_kernel 16x16 split"
    assert name(moe.Q8Shape.make(16384, 1, 4096, 4096)) == "q8_run_kernel 256x256"
    assert name(moe.Q8Shape.make(16384, 1, 4097, 4096)) == "q8_small_run_kernel 128x128"            # (its ways out are for four columns)
    s = moe.Shape.make(2, 4096, 8, 14336, 1, 2, act="silu")
    assert [moe.moe_gated_q8_kernel(s, w) for w in (0, 1)] == ["q8_stream_kernel 16x32 once", "q8_stream_kernel 16x16 split once"]
    s = moe.Shape.make(32768, 2048, 32, 8192, 1, 32768, act="silu")
    assert [moe.moe_gated_q8_kernel(s, w) for w in (0, 1)] == ["q8_gated_run_kernel 256x256", "q8_run_kernel 256x256"]
    L, buf = q8_binding._lib(), C.create_string_buffer(8)
    q = moe.Q8Shape.make(1, 1, 64, 64)
    assert L.moe_q8_linear_kernel(C.byref(q), None, 8) == 1 and L.moe_q8_linear_kernel(C.byref(q), buf, 0) == 1
    assert L.moe_q8_linear_kernel(None, buf, 8) == 1 and L.moe_gated_q8_kernel(None, 0, buf, 8) == 1
    assert L.moe_q8_linear_kernel(C.byref(q), buf, 8) == 0 and buf.value == b"q8_stre"
    for which in (-1, 2):
        assert L.moe_gated_q8_kernel(C.byref(s), which, buf, 8) == 1
    with pytest.raises(moe.MoeError):
        name(moe.Q8Shape.make(1, 1, 64, 72))


def test_tails_in_kernel_names():
    """Depths of no whole stages of 128, and below four of them where loads run on from tile to tile; kernels for few rows have no such form."""
    linear = lambda R, N, K: moe.moe_q8_linear_kernel(moe.Q8Shape.make(R, 1, N, K))  # noqa: E731
    assert [linear(9000, 4096, K) for K in (256, 384, 512, 528)] == [f"q8_run_kernel 256x256{t}" for t in (" tail", " tail", "", " tail")]
    assert [linear(2600, 1028, K) for K in (640, 656)] == [f"q8_tile_kernel 128x128 deep{t}" for t in ("", " tail")]
    assert not linear(1, 4096, 1040).endswith("tail")
