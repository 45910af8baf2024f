"""Every kernel, tile and form that a gated block's GEMMs run on, at sizes of which moe_gated_gemm_kernel says that they do: against
the formulas in 64 bits, with the bounds of test_gpu_gated.py; and the backward pass beside itself in order and as a graph."""
import pytest
import torch

import paper_2210_17223_amd as moe
from test_gpu_gated import Block, check_backward, check_forward

pytestmark = pytest.mark.gpu
BESIDE = 0                                        # moe_path_calls: weight gradients on a side stream
FIRST, SECOND, DH, DXE, DW2, DW13 = range(6)
RUN, TILE, DX_RUN, DX_TILE = "gated_run_kernel ", "gated_tile_kernel ", "rows_bf16_run_kernel ", "rows_bf16_tile_kernel "

CASES = [
    (dict(R=600, E=16, d=1024, h=2816), {FIRST: RUN + "256x256", DXE: DX_TILE + "128x128 deep", DW2: "wgrad_w4_kernel 256x256", DW13: "wgrad_w4_kernel 256x256"}),
    (dict(R=4000, E=4, d=2048, h=1024, act="gelu"), {FIRST: RUN + "256x256", SECOND: "grouped_gemm_w4_kernel 256x256", DH: "gated_dh_kernel 128x128",
                                                     DXE: DX_RUN + "256x256", DW2: "wgrad_gemm_kernel 128x128", DW13: "wgrad_w4_kernel 256x256"}),
    (dict(R=4000, E=1, d=1024, h=2056), {FIRST: RUN + "256x256", DH: "gated_dh_kernel 256x256", DXE: DX_TILE + "128x128 deep tail"}),
    (dict(R=4000, E=4, d=1024, h=2048, act="gelu_tanh", counts=[0, 3900, 1, 99]), {FIRST: TILE + "128x128", DH: "gated_dh_kernel 256x256", DXE: DX_TILE + "128x128"}),
    (dict(R=8000, E=4, d=2048, h=1544, act="relu"), {FIRST: RUN + "256x256", DH: "gated_dh_kernel 256x256", DXE: DX_RUN + "128x256 tail"}),
    (dict(R=100, E=1, d=2048, h=256), {FIRST: TILE + "128x128 deep", DXE: DX_TILE + "128x128"}),
    (dict(R=100, E=1, d=256, h=1024, act="identity"), {FIRST: TILE + "128x128", DXE: DX_TILE + "128x128 deep"}),
    (dict(R=2400, E=16, d=2048, h=4096), {SECOND: "grouped_gemm_mfma_kernel 128x256", DXE: DX_RUN + "128x256"}),
    (dict(R=600, E=16, d=2048, h=256), {FIRST: TILE + "128x128 deep", SECOND: "grouped_gemm_staged_kernel 64x256"}),
    (dict(R=6000, E=64, d=3080, h=520), {FIRST: RUN + "128x256 tail", DH: "gated_dh_kernel 256x256 tail", DXE: DX_RUN + "256x256 tail"}),
    (dict(R=1200, E=16, d=1024, h=4096, act="gelu"), {SECOND: "grouped_gemm_mfma_kernel 128x128 deep", DH: "gated_dh_kernel 256x256", DXE: DX_TILE + "128x128 deep"}),
    # of the lists beside the formulas' own tests
    (dict(R=2000, E=1, d=3136, h=2056), {FIRST: RUN + "128x256", DXE: DX_RUN + "256x256 tail"}),
    (dict(R=8192, E=2, d=64, h=4096, act="gelu"), {FIRST: RUN + "256x256 tail"}),
    (dict(R=300, E=2, d=2000, h=520), {FIRST: TILE + "128x128 deep tail"}),
    (dict(R=700, E=3, d=1000, h=520), {FIRST: TILE + "128x128 tail", DH: "gated_dh_kernel 128x128 tail", DXE: DX_TILE + "128x128 tail"}),
    (dict(R=40, E=16, d=768, h=2048), {FIRST: "gated_stream_kernel 32x32", SECOND: "grouped_gemm_stream_kernel 32x64"}),
    (dict(R=70, E=4, d=264, h=136, counts=[0, 33, 17, 20]), {FIRST: "gated_stream_kernel 32x32 tail"}),
]


@pytest.mark.parametrize("kw,forms", CASES, ids=lambda v: "-".join(str(x) for x in v.values()) if "R" in v else "")
def test_forward_and_backward(kw, forms):
    b = Block(**kw)
    assert {w: moe.moe_gated_gemm_kernel(b.s, w) for w in forms} == forms
    b.forward(False)
    check_forward(b, False)
    b.ye.fill_(7.0)
    b.forward(True)
    check_forward(b, True)
    kept = b.backward()
    check_backward(b, *kept)
    for t in (b.dxe, b.dW13, b.dW2):
        t.fill_(7.0)
    assert all(torch.equal(p, q) for p, q in zip(kept, b.backward(kept=False)))


def test_every_form_is_among_the_cases():
    """(But for the second GEMM, whose kernels are the plain layer's.)"""
    have = {name for _, forms in CASES for name in forms.values()}
    tiles = [k + t + f for k in (RUN, DX_RUN) for t in ("256x256", "128x256") for f in ("", " tail")]
    tiles += [k + "128x128" + f for k in (TILE, DX_TILE) for f in ("", " tail", " deep", " deep tail")]
    tiles += ["gated_dh_kernel " + t + f for t in ("256x256", "128x128") for f in ("", " tail")]
    tiles += ["wgrad_w4_kernel 256x256", "wgrad_gemm_kernel 128x128", "gated_stream_kernel 32x32", "gated_stream_kernel 32x32 tail"]
    assert set(tiles) <= have, sorted(set(tiles) - have)


@pytest.mark.parametrize("kept", [True, False], ids=["keep", "recompute"])
def test_weight_gradients_beside_the_other_gemms(kept):
    """Rows x d x h above 1.8e9: the weight gradients run on a side stream; in launch order while stages are timed, and in a
    graph.  The same bits each way, on another stream, and from call to call."""
    b = Block(R=2600, E=3, d=768, h=1000, counts=[2000, 0, 600])
    assert 1.8e9 <= moe.moe_max_rows(b.s) * b.d * b.h < 2.7e9
    b.forward(True)
    calls = moe.moe_path_calls(BESIDE)
    want = b.backward(kept)
    assert moe.moe_path_calls(BESIDE) == calls + 1
    check_backward(b, *want)
    outs = (b.dxe, b.dW13, b.dW2)

    def same():
        ok = all(torch.equal(p, q) for p, q in zip(outs, want))
        for t in outs:
            t.fill_(7.0)
        b.dxe[b.R:] = want[0][b.R:]
        return ok

    assert same()
    moe.moe_profile_enable(1, 64)
    try:
        b.backward(kept)
        assert same()
    finally:
        moe.moe_profile_enable(0, 0)
    assert moe.moe_path_calls(BESIDE) == calls + 1
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        b.backward(kept)
    st.synchronize()
    assert same() and moe.moe_path_calls(BESIDE) == calls + 2
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        moe.moe_gated_ffn_backward(b.s, b.xe, b.offsets, b.W13, b.W2, b.W13p, b.pre if kept else None, b.hid if kept else None, b.dye,
                                   b.dxe, b.dW13, b.dW2, b.bws)
    assert moe.moe_path_calls(BESIDE) == calls + 2
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert same()
        b.backward(kept)                          # the program's own eager work in between
        torch.cuda.synchronize()
        assert same()


@pytest.mark.parametrize("kw", [dict(R=40, E=4, d=264, h=136), dict(R=4000, E=4, d=1024, h=2048)], ids=["few", "many"])
def test_what_is_kept_takes_no_workspace(kw):
    """Workspaces of exactly the size for calls that are given pre and hid, and nothing behind them is written."""
    b = Block(**kw)
    b.forward(True)
    ye, want = b.ye.clone(), b.backward()
    for name, size in (("ws", moe.moe_gated_kept_workspace_bytes(b.s)), ("bws", moe.moe_gated_kept_backward_workspace_bytes(b.s))):
        assert 0 < size < getattr(b, name).numel()
        held = torch.full((size + 4096,), 255, dtype=torch.uint8, device=b.xe.device)
        setattr(b, name + "_held", held)
        setattr(b, name, held[:size])
    b.ye[:b.R] = 0.0
    b.forward(True)
    got = b.backward()
    assert torch.equal(b.ye, ye) and all(torch.equal(p, q) for p, q in zip(got, want))
    assert bool((b.ws_held[-4096:] == 255).all()) and bool((b.bws_held[-4096:] == 255).all())
    for call in (lambda: b.forward(False), lambda: b.backward(kept=False)):
        with pytest.raises(moe.MoeError, match="workspace"):
            call()
