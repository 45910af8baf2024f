"""CPU-side checks of include/moe_gated.h: sizes, and refusals before anything is enqueued."""
import ctypes as C

import pytest

import paper_2210_17223_amd as moe
from paper_2210_17223_amd import gated_binding


def shape(**kw):
    return moe.Shape.make(**{**dict(T=64, d_model=64, E=4, d_ff=128, k=2, capacity=32, act="silu"), **kw})


def test_sizes():
    s = shape()
    assert moe.moe_gated_packed_bytes(s) == 4 * 64 * 256 * 2
    assert moe.moe_gated_packed_bytes(shape(d_ff=136)) == 4 * 64 * 288 * 2          # the last sixteen columns are padded
    assert moe.moe_gated_packed_bytes(shape(d_ff=132, dtype="f32")) == 4 * 64 * 264 * 4
    assert moe.moe_packed_weight_bytes(s) == 4 * 64 * 128 * 2                        # W2p
    rows = moe.moe_max_rows(s)
    assert moe.moe_gated_workspace_bytes(s) >= rows * 128 * 2
    assert moe.moe_gated_backward_workspace_bytes(s) >= rows * 128 * (4 + 4 + 2)
    assert moe.moe_gated_workspace_bytes(shape(dtype="f32")) >= rows * 128 * 4


@pytest.mark.parametrize("kw,frag", [
    (dict(E=65), "at most 64"), (dict(k=5, E=4), "exceeds"), (dict(d_model=100), "multiples of 16"), (dict(d_ff=4), "multiples of 16"),
    (dict(T=0), ">= 1"), (dict(d_ff=1 << 20), "below 2^20"), (dict(T=1 << 30, capacity=1 << 30, k=2), "31 bits"),
    (dict(T=(1 << 31) - 64, capacity=(1 << 31) - 64, k=1), "31 bits"),
])
def test_bad_shapes_are_refused(kw, frag):
    s = shape(**kw)
    for size in (moe.moe_gated_packed_bytes, moe.moe_gated_workspace_bytes, moe.moe_gated_backward_workspace_bytes):
        assert size(s) == 0 and frag in moe.moe_last_error()


def test_fp32_blocks_have_no_backward_pass():
    s, L, ok = shape(dtype="f32"), gated_binding._lib(), C.c_void_p(4096)
    assert moe.moe_gated_backward_workspace_bytes(s) == 0 and "bf16" in moe.moe_last_error()
    assert L.moe_gated_ffn_backward(C.byref(s), *[ok] * 12, None) == 2
    assert L.moe_gated_ffn(C.byref(s), *[ok] * 8, None) == 2 and "bf16" in moe.moe_last_error()


def test_null_and_misaligned_pointers_are_refused():
    L, s, ok, z, odd = gated_binding._lib(), shape(), C.c_void_p(4096), C.c_void_p(0), C.c_void_p(4100)
    for f, count, optional in ((L.moe_pack_gated_weights, 4, ()), (L.moe_gated_ffn, 8, (5, 6)),
                               (L.moe_gated_ffn_backward, 12, (5, 6))):
        for i in range(count):
            args = [ok] * count
            args[i] = odd
            assert f(C.byref(s), *args, z) == 1 and "aligned" in moe.moe_last_error()
            args[i] = z
            assert f(C.byref(s), *args, z) == 1
            assert ("come together" if i in optional else "is NULL") in moe.moe_last_error()
        assert f(None, *[ok] * count, z) == 1


def test_silu_is_the_gated_blocks_only():
    s, L, ok, z = shape(), moe.lib(), C.c_void_p(4096), C.c_void_p(0)
    assert L.moe_expert_ffn(C.byref(s), ok, ok, ok, z, ok, z, ok, ok, z) == 2 and "gated" in moe.moe_last_error()
    assert L.moe_layer_chunked(C.byref(s), 1, ok, ok, z, 0, *[ok] * 16) == 2 and "gated" in moe.moe_last_error()
    assert moe.moe_padded_workspace_bytes(s, 1) == 0 and moe.moe_offload_workspace_bytes(s) == 0
    assert moe.moe_workspace_bytes(s, 1) > 0                    # its gate, dispatch and combine are the layer's
    bad = shape()
    bad.act = 5
    assert moe.moe_gated_workspace_bytes(bad) == 0 and "activation" in moe.moe_last_error()


def q4(**kw):
    return moe.Q4Shape.make(**{**dict(R=8, E=2, N=48, K=256, group=64), **kw})


@pytest.mark.parametrize("kw,status,frag", [
    (dict(R=0), 1, ">= 1"), (dict(N=0), 1, ">= 1"), (dict(E=65), 2, "at most 64"), (dict(K=1 << 24), 2, "2^24"),
    (dict(N=1 << 24), 2, "2^24"), (dict(R=1 << 30), 2, "2^30"), (dict(group=16), 2, "32, 64 or 128"), (dict(group=0), 2, "32, 64 or 128"),
    (dict(K=96), 2, "divide"), (dict(K=320, group=128), 2, "divide"),
])
def test_q4_linear_refuses_bad_shapes(kw, status, frag):
    L, ok = gated_binding._lib(), C.c_void_p(4096)
    assert L.moe_q4_linear(C.byref(q4(**kw)), *[ok] * 6, None) == status and frag in moe.moe_last_error()


def test_q4_linear_refuses_other_types_and_bad_pointers():
    L, s, ok, z, odd = gated_binding._lib(), q4(), C.c_void_p(4096), C.c_void_p(0), C.c_void_p(4100)
    s.x = 0
    assert L.moe_q4_linear(C.byref(s), *[ok] * 6, None) == 1 and "bf16" in moe.moe_last_error()
    assert L.moe_q4_linear(None, *[ok] * 6, None) == 1
    for i in range(6):
        args = [ok] * 6
        args[i] = odd
        assert L.moe_q4_linear(C.byref(q4()), *args, z) == 1 and "aligned" in moe.moe_last_error()
        args[i] = z
        if i != 4:
            assert L.moe_q4_linear(C.byref(q4()), *args, z) == 1 and "is NULL" in moe.moe_last_error()


def test_gated_ffn_q4_refusals():
    L, ok, z, odd = gated_binding._lib(), C.c_void_p(4096), C.c_void_p(0), C.c_void_p(4100)
    s = shape()
    assert moe.moe_gated_q4_workspace_bytes(s) >= moe.moe_max_rows(s) * 128 * 2
    assert moe.moe_gated_q4_workspace_bytes(shape(dtype="f32")) == 0 and "bf16" in moe.moe_last_error()
    assert L.moe_gated_ffn_q4(C.byref(shape(dtype="f32")), 64, *[ok] * 10, z) == 2
    for group, kw in ((16, {}), (128, {}), (64, dict(d_ff=136)), (32, dict(d_model=72)), (-32, {})):
        assert L.moe_gated_ffn_q4(C.byref(shape(**kw)), group, *[ok] * 10, z) == 2 and "group" in moe.moe_last_error()
    for i in range(10):
        args = [ok] * 10
        args[i] = odd
        assert L.moe_gated_ffn_q4(C.byref(s), 64, *args, z) == 1 and "aligned" in moe.moe_last_error()
        args[i] = z
        if i not in (4, 7):
            assert L.moe_gated_ffn_q4(C.byref(s), 64, *args, z) == 1 and "is NULL" in moe.moe_last_error()
    assert L.moe_gated_ffn_q4(None, 64, *[ok] * 10, z) == 1


def test_another_thread_may_clear_the_table_of_sizes(monkeypatch):
    class Cleared(dict):                              # whatever a call has seen or put there is gone when it looks again
        def __contains__(self, key):
            found = super().__contains__(key)
            self.clear()
            return found

        def __setitem__(self, key, value):
            super().__setitem__(key, value)
            self.clear()

    s = shape()
    want = (moe.moe_max_rows(s), moe.moe_gated_packed_bytes(s), moe.moe_packed_weight_bytes(s), moe.moe_gated_workspace_bytes(s))
    table = Cleared()
    monkeypatch.setattr(gated_binding, "_sizes", table)
    assert gated_binding._sizes_of(s) == want
    dict.__setitem__(table, bytes(s), want)
    assert gated_binding._sizes_of(s) == want


def test_silu_is_refused_by_the_plain_layers_backward_pass():
    s, L, ok, z = shape(), moe.lib(), C.c_void_p(4096), C.c_void_p(0)
    assert moe.moe_backward_workspace_bytes(s) == 0 and "gated" in moe.moe_last_error()
    with pytest.raises(moe.MoeError, match="gated"):
        moe.moe_backward_gemm_kernel(s, 0)
    with pytest.raises(moe.MoeError, match="gated"):
        moe.moe_expert_gemm_kernel(s, 0)
    args = [ok, ok, z, C.c_int32(0), *[ok] * 19, z]
    assert L.moe_layer_backward(C.byref(s), *args) == 2 and "gated" in moe.moe_last_error()
    assert moe.moe_backward_workspace_bytes(shape(act="gelu")) > 0


def test_values_that_lanes_pass_through_lds_have_a_barrier_between():
    """In the 4-bit kernel of few rows a wavefront's lanes write x, codes and sums to LDS that other lanes of it read, with no
    workgroup barrier in between: a handover stands in front of the first write and of the read behind it, whatever the
    compiler knows of the addresses."""
    import os
    path = os.path.join(os.path.dirname(moe.lib_path()), "csrc", "q4.hip")
    with open(path) as f:
        text = f.read()
    body = text[text.index("void q4_stream_kernel("):text.index("many rows per expert")]
    calls = [line.strip() for line in body.splitlines()
             if line.strip().startswith(("lds_handover();", "x_into_lds();", "codes_into_lds(", "use(", "float *mine"))]
    step = ["lds_handover();", "x_into_lds();", "codes_into_lds(", "lds_handover();", "use("]
    assert len(calls) == 12 and all(c.startswith(p) for c, p in zip(calls, step + step + ["lds_handover();", "float *mine"]))


def test_gemm_kernel_names():
    name = moe.moe_gated_gemm_kernel
    s = moe.Shape.make(16384, 2048, 8, 5632, 1, 16384, act="silu")
    assert [name(s, w) for w in range(6)] == ["gated_run_kernel 256x256", "grouped_gemm_mfma_kernel 128x256", "gated_dh_kernel 256x256",
                                              "rows_bf16_run_kernel 128x256", "wgrad_w4_kernel 256x256", "wgrad_w4_kernel 256x256"]
    s = moe.Shape.make(512, 128, 4, 256, 1, 512, act="silu", dtype="f32")
    assert [name(s, w) for w in range(2)] == ["gated_f32_kernel 32x32", "grouped_gemm_f32_kernel 32x32"]
    for bad, frag in ((2, "bf16"), (6, "0..5"), (-1, "0..5")):
        with pytest.raises(moe.MoeError, match=frag):
            name(s, bad)
    with pytest.raises(moe.MoeError):
        name(shape(d_model=100), 0)
    L, buf = gated_binding._lib(), C.create_string_buffer(8)
    assert L.moe_gated_gemm_kernel(C.byref(s), 0, None, 8) == 1 and L.moe_gated_gemm_kernel(C.byref(s), 0, buf, 0) == 1
    assert L.moe_gated_gemm_kernel(None, 0, buf, 8) == 1
    assert L.moe_gated_gemm_kernel(C.byref(s), 0, buf, 8) == 0 and buf.value == b"gated_f"


def test_workspaces_of_calls_that_keep_what_the_backward_pass_reads():
    s = moe.Shape.make(16384, 2048, 8, 5632, 1, 16384, act="silu")
    Rh = moe.moe_max_rows(s) * 5632
    lists = 4 << 20
    assert moe.moe_gated_workspace_bytes(s) >= 2 * Rh and moe.moe_gated_kept_workspace_bytes(s) <= lists
    assert moe.moe_gated_backward_workspace_bytes(s) >= 10 * Rh
    assert 4 * Rh <= moe.moe_gated_kept_backward_workspace_bytes(s) <= 4 * Rh + lists
    f32 = shape(dtype="f32")
    for size in (moe.moe_gated_kept_workspace_bytes, moe.moe_gated_kept_backward_workspace_bytes):
        assert size(f32) == 0 and "bf16" in moe.moe_last_error()


def test_few_rows_of_many_experts_may_be_one_experts():
    """The kernel for few rows of 4-bit weights, which needs no room for rows made ready, takes at most 96 of any number of experts."""
    def ready(R, E):
        s = moe.Shape.make(R, 512, E, 256, 1, R, act="silu")
        hidden = -(-R * 256 * 2 // 256) * 256
        assert moe.moe_gated_q4_workspace_bytes(s) - hidden in (0, -(-R * 512 * 2 // 256) * 256 + -(-R * 4 // 256) * 256)
        return moe.moe_gated_q4_workspace_bytes(s) > hidden
    assert not any(ready(R, E) for R, E in ((1, 1), (16, 1), (80, 8), (96, 10), (96, 64), (16, 64)))
    assert all(ready(R, E) for R, E in ((17, 1), (81, 8), (97, 10), (97, 64), (640, 64)))


def test_tiles_that_leave_through_lds_have_a_barrier_on_both_sides():
    """The epilogues that write a wavefront's accumulators to its own part of LDS and read whole lines of other lanes' values back."""
    import os
    import re
    csrc = os.path.join(os.path.dirname(moe.lib_path()), "csrc")
    for name, start, count in (("gated.hip", "void leave_gated(", 1), ("gemm_w4_run.h", "void leave(", 1), ("bwd.hip", "auto through = ", 2)):
        with open(os.path.join(csrc, name)) as f:
            parts = f.read().split(start)[1:]
        assert len(parts) == count
        for body in parts:
            read = body.index("*reinterpret_cast<const u32x4 *>(")
            end = body.index("\n}\n" if name == "gated.hip" else "};", read)
            assert len(re.findall(r"lds_handover\(\);", body[:read])) == 1 and len(re.findall(r"lds_handover\(\);", body[read:end])) == 1, name
