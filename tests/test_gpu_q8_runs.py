"""The 8-bit products where a block takes several tiles one after the other: loads that run on into the next tile, another expert's or none, in
every form of the 128 x 128 kernels; and 64 experts, a lane of the tile search for each.  As tests/test_gpu_q8.py holds them otherwise."""
import math

import pytest
import torch

import paper_2210_17223_amd as moe
from gpu_util import DEV
from test_gpu_q8 import EPS, TYPES, act64, codes, expert_of, gelu_room, gen, held, normal, offsets_of, scales, sums

pytestmark = pytest.mark.gpu

AT_ONCE = 512                              # blocks of 128 x 128 tiles that a launch has at once: more tiles than these, and blocks take several

# (rows by expert, N, K)
RUNS = {
    "q8_small_run_kernel 128x128": [([49, 72, 118, 62, 89, 44, 0, 196], 10916, 512), ([163, 310, 0, 233, 506], 10304, 768),
                                    ([46, 89, 0, 37, 41, 148, 54, 33], 12017, 512), ([2246, 1381], 6554, 512)],
    "q8_small_run_kernel 128x128 tail": [([39, 36, 103, 41, 72, 136, 47, 0, 84, 56, 51, 63, 228], 7172, 16), ([139, 57, 73, 104, 230, 64, 0, 52], 12612, 80),
                                         ([73, 81, 0, 176, 291, 66, 108, 132], 6966, 16), ([894, 414, 471, 1456, 338, 673, 372, 0], 3455, 64)],
    "q8_small_run_kernel 128x128 once": [([64, 27, 52, 32, 0, 45, 39, 86, 24, 146, 35, 30, 26], 8820, 640),
                                         ([57, 332, 201, 70, 151, 93, 83, 123, 105, 65, 54, 60, 0], 12044, 512),
                                         ([44, 84, 63, 140, 52, 35, 0, 39], 13454, 640), ([57, 42, 24, 156, 38, 26, 92, 48, 0, 69, 35, 30, 32], 7862, 768)],
    "q8_small_run_kernel 128x128 once tail": [([48, 64, 24, 30, 39, 26, 109, 0], 14228, 624), ([0, 46, 68, 51, 110, 58, 83, 182], 13928, 912),
                                              ([45, 20, 39, 34, 0, 74, 30, 28, 56, 21, 126, 22, 25], 15191, 368),
                                              ([76, 102, 38, 47, 62, 169, 42, 0], 10410, 1424)],
}
RUNS = {f"{name} {i}": case + (name,) for name, cases in RUNS.items() for i, case in enumerate(cases)}
# (rows by expert, d_model, d_ff)
PAIRS = {
    "q8_gated_small_run_kernel 128x128": [([68, 129, 0, 53, 213, 59, 49, 97], 512, 4384), ([519, 0, 1121, 424], 640, 3248)],
    "q8_gated_small_run_kernel 128x128 tail": [([134, 94, 62, 178, 0, 296, 48, 82, 58, 54, 67, 51, 74], 16, 2976), ([0, 560, 421, 344], 64, 5168)],
    "q8_gated_small_run_kernel 128x128 once": [([108, 29, 57, 45, 32, 31, 81, 66, 41, 35, 0, 183, 37], 640, 4160),
                                               ([101, 30, 42, 0, 172, 27, 29, 33, 35, 76, 62, 53, 38], 1408, 3728)],
    "q8_gated_small_run_kernel 128x128 once tail": [([40, 33, 96, 59, 27, 36, 0, 31, 44, 164, 29, 72, 26], 656, 4016),
                                                    ([0, 159, 262, 66, 60, 73, 84, 120], 1008, 4960)],
}
PAIRS = {f"{name} {i}": case + (name,) for name, cases in PAIRS.items() for i, case in enumerate(cases)}


def tiles(counts, columns):
    return sum(-(-c // 128) for c in counts) * -(-columns // 128)


def linear_inputs(counts, N, K, seed, spare=0):
    g, E, R = gen(seed), len(counts), sum(counts) + spare
    return dict(g=g, E=E, R=R, N=N, K=K, rows=sum(counts), x=codes(g, R, K), w=codes(g, E, N, K), xs=scales(g, R, of=1 / 73),
                ws=scales(g, E, N, of=1 / (73 * math.sqrt(K))), offsets=offsets_of(counts))


def check_sums(c):
    """Bit for bit: the whole number, rounded, times both scales; rows behind the last expert are left."""
    y = torch.full((c["R"], c["N"]), 7.0, device=DEV)
    moe.moe_q8_linear(moe.Q8Shape.make(c["R"], c["E"], c["N"], c["K"], y="f32"), c["x"], c["xs"], c["offsets"], c["w"], c["ws"], None, None, y)
    e = expert_of(c["offsets"], c["R"])
    want = sums(c["x"], c["w"], c["offsets"]).float() * c["xs"][:, None] * c["ws"][e]
    want[c["rows"]:] = 7.0
    assert torch.equal(y, want)


def check_epilogue(c, act, out):
    """With bias, activation and a residual in y's place.  Roundings of fp32: the sum, two scales and the bias, taken on by a slope below 1.2; the
    activation's own ((8 + 3 |e|) 2^-24 with silu's e = 1.44 |v|, the erf form's as gelu_room has it); the residual's sum; then the output's."""
    g = c["g"]
    bias, y = normal(g, c["E"], c["N"], std=0.5), normal(g, c["R"], c["N"], std=2.0).to(TYPES[out])
    e = expert_of(c["offsets"], c["R"])
    v = sums(c["x"], c["w"], c["offsets"]) * c["xs"].double()[:, None] * c["ws"][e].double()
    pre = v + bias[e].double()
    value = act64(pre, act)
    want = value + y.double()
    room = 2.0 ** -24 * (4 * v.abs() + 2 * pre.abs()) * 1.2 + (gelu_room(pre, value, out == "f32") if act == "gelu" else (8 + 4.4 * pre.abs()) * 2.0 ** -24 * value.abs())
    room = room + 2.0 ** -24 * want.abs()
    room = room + EPS[out] * (want.abs() + room) + 2.0 ** -25
    moe.moe_q8_linear(moe.Q8Shape.make(c["R"], c["E"], c["N"], c["K"], act=act, res=out, y=out), c["x"], c["xs"], c["offsets"], c["w"], c["ws"],
                      bias, y, y)
    over = (y.double() - want).abs() - room
    assert float(over.max()) <= 0, (float(over.max()), int((over > 0).sum()))


@pytest.mark.parametrize("name", list(RUNS))
def test_products_of_several_tiles_a_block(name):
    counts, N, K, kernel = RUNS[name]
    assert tiles(counts, N) > AT_ONCE + 64
    c = linear_inputs(counts, N, K, seed=N)
    assert moe.moe_q8_linear_kernel(moe.Q8Shape.make(c["R"], c["E"], N, K)) == kernel
    check_sums(c)
    check_epilogue(c, "silu", "f32")
    check_epilogue(c, "gelu", "bf16")
    check_epilogue(c, "gelu", "f32")


def gated_inputs(counts, d, h, seed):
    g, E, R = gen(seed), len(counts), sum(counts)
    return dict(R=R, E=E, d=d, h=h, x=codes(g, R, d), xs=scales(g, R, of=1 / 73), offsets=offsets_of(counts), q13=codes(g, E, 2 * h, d),
                s13=scales(g, E, 2 * h, of=1 / (73 * math.sqrt(d))), q2=codes(g, E, d, h), s2=scales(g, E, d, of=1 / (73 * math.sqrt(h))),
                src=torch.randperm(R, generator=g, device=DEV).int())


def check_block(c, act="silu"):
    """Against 64 bits, as tests/test_gpu_q8.py derives it: 2e-3 of the output's root mean square, a single value 0.14; and rows taken from
    where they stand give the same bits."""
    s = moe.Shape.make(c["R"], c["d"], c["E"], c["h"], 1, c["R"], act=act)
    new = lambda: torch.full((c["R"], c["d"]), 7.0, dtype=torch.float16, device=DEV)  # noqa: E731
    ye, there = new(), new()
    ws = torch.empty(moe.moe_gated_q8_workspace_bytes(s), dtype=torch.uint8, device=DEV)
    rest = (c["offsets"], c["q13"], c["s13"], c["q2"], c["s2"])
    moe.moe_gated_ffn_q8(s, c["x"], c["xs"], None, *rest, ye, ws)
    x, xs = torch.empty_like(c["x"]), torch.empty_like(c["xs"])
    x[c["src"].long()], xs[c["src"].long()] = c["x"], c["xs"]
    moe.moe_gated_ffn_q8(s, x, xs, c["src"], *rest, there, ws)
    assert torch.equal(ye, there)
    o, h = c["offsets"].tolist(), c["h"]
    for e in range(c["E"]):
        lo, hi = o[e], o[e + 1]
        if lo == hi:
            continue
        both = (c["x"][lo:hi].double() @ c["q13"][e].double().T) * c["xs"][lo:hi].double()[:, None] * c["s13"][e].double()
        q, scale = held((act64(both[:, :h], act) * both[:, h:]).half())
        want = (q.double() @ c["q2"][e].double().T) * scale.double()[:, None] * c["s2"][e].double()
        off = (ye[lo:hi].double() - want).abs() - 2.0 ** -11 * want.abs()
        rms = float(want.square().mean().sqrt())
        assert float(off.clamp(min=0).square().mean().sqrt()) <= 2e-3 * rms
        assert float(off.max()) <= 0.14 * rms


@pytest.mark.parametrize("name", list(PAIRS))
def test_blocks_of_several_tiles_a_block(name):
    counts, d, h, kernel = PAIRS[name]
    assert tiles(counts, 2 * h) > AT_ONCE + 64
    c = gated_inputs(counts, d, h, seed=h)
    assert moe.moe_gated_q8_kernel(moe.Shape.make(c["R"], d, c["E"], h, 1, c["R"]), 0) == kernel
    check_block(c)
    check_block(c, "gelu_tanh")


# ---------------------------------------------------------------------------- 64 experts
def spread(rows, empty=()):
    """`rows` rows over 64 experts, unevenly, none to those of `empty`."""
    weight = [0.0 if e in empty else 1.0 + (e * 37 % 64) / 16 for e in range(64)]
    counts = [int(rows * w / sum(weight)) for w in weight]
    counts[max(range(64), key=lambda e: weight[e])] += rows - sum(counts)
    return counts


@pytest.mark.parametrize("counts,N,K,kernel", [
    ([1 if e in (0, 31, 62, 63) else 0 for e in range(64)], 260, 512, "q8_stream_kernel 16x16"), (spread(1200, (0, 5, 63)), 516, 272, "q8_stream_kernel"),
    (spread(7000, (17, 62)), 1028, 1040, "q8_"), (spread(9000, (0, 1, 2)), 1027, 528, "q8_small_run_kernel"),
    (spread(40000, (63,)), 2052, 528, "q8_run_kernel 256x256")])
def test_products_of_64_experts(counts, N, K, kernel):
    c = linear_inputs(counts, N, K, seed=K, spare=2)
    assert moe.moe_q8_linear_kernel(moe.Q8Shape.make(c["R"], 64, N, K)).startswith(kernel)
    check_sums(c)
    check_epilogue(linear_inputs(counts, N, K, seed=K + 1), "silu", "f32")


@pytest.mark.parametrize("counts,d,h,kernel", [
    ([1 if e in (0, 31, 62, 63) else 0 for e in range(64)], 272, 256, "q8_stream_kernel"), (spread(2500, (0, 5, 63)), 272, 512, "q8_"),
    (spread(9000, (17, 62)), 272, 272, "q8_gated_"), (spread(40000, (63,)), 528, 512, "q8_gated_run_kernel 256x256")])
def test_blocks_of_64_experts(counts, d, h, kernel):
    c = gated_inputs(counts, d, h, seed=d)
    assert moe.moe_gated_q8_kernel(moe.Shape.make(c["R"], d, 64, h, 1, c["R"]), 0).startswith(kernel)
    check_block(c)


def test_a_dispatch_over_64_experts():
    """The plan of 8-bit rows is moe_dispatch's, and their codes and scales lie where it says."""
    T, d, E, k = 700, 48, 64, 8
    g = gen(64)
    x, xs = codes(g, T, d), scales(g, T)
    idx = torch.rand(T, E, generator=g, device=DEV).argsort(1)[:, :k].contiguous().int().view(-1)
    s = moe.Shape.make(T, d, E, 32, k, 80)
    rows = moe.moe_max_rows(s)
    i32 = lambda n: torch.full((n,), -7, dtype=torch.int32, device=DEV)  # noqa: E731
    plans = [dict(counts=i32(E), offsets=i32(E + 1), slot_of=i32(T * k), src_of=i32(rows)) for _ in range(2)]
    xe, xes = torch.empty(rows, d, dtype=torch.int8, device=DEV), torch.empty(rows, device=DEV)
    ws = torch.empty(moe.moe_workspace_bytes(s, 1), dtype=torch.uint8, device=DEV)
    moe.moe_dispatch_q8(s, x, xs, idx, *plans[0].values(), xe, xes, ws)
    moe.moe_dispatch(s, x.bfloat16(), idx, *plans[1].values(), torch.empty(rows, d, dtype=torch.bfloat16, device=DEV), ws)
    A = int(plans[1]["offsets"][-1])
    assert 0 < A < T * k                                       # (some were dropped at the capacity)
    for key in ("counts", "offsets", "slot_of"):
        assert torch.equal(plans[0][key], plans[1][key]), key
    assert torch.equal(plans[0]["src_of"][:A], plans[1]["src_of"][:A])
    token = plans[0]["src_of"][:A].long() // k
    assert torch.equal(xe[:A], x[token]) and torch.equal(xes[:A], xs[token])


def test_stages_of_the_8_bit_calls_are_timed():
    """moe_profile_enable's stages: the dispatch's plan and, where rows move, their copies; the block's two products."""
    g = gen(5)
    T, d, E, h, k = 256, 64, 4, 48, 2
    s = moe.Shape.make(T, d, E, h, k, T, act="silu")
    rows = moe.moe_max_rows(s)
    x, xs = codes(g, T, d), scales(g, T)
    idx = torch.rand(T, E, generator=g, device=DEV).argsort(1)[:, :k].contiguous().int().view(-1)
    i32 = lambda n: torch.empty(n, dtype=torch.int32, device=DEV)  # noqa: E731
    plan = [i32(E), i32(E + 1), i32(T * k), i32(rows)]
    xe, xes = torch.empty(rows, d, dtype=torch.int8, device=DEV), torch.empty(rows, device=DEV)
    ws, gws = (torch.empty(n, dtype=torch.uint8, device=DEV) for n in (moe.moe_workspace_bytes(s, 1), moe.moe_gated_q8_workspace_bytes(s)))
    q13, q2, ye = codes(g, E, 2 * h, d), codes(g, E, d, h), torch.empty(rows, d, dtype=torch.float16, device=DEV)
    moe.moe_profile_enable((1 << 12) - 1, 64)
    try:
        moe.moe_dispatch_q8(s, x, xs, idx, *plan, None, None, ws)
        moe.moe_dispatch_q8(s, x, xs, idx, *plan, xe, xes, ws)
        moe.moe_gated_ffn_q8(s, xe, xes, None, plan[1], q13, scales(g, E, 2 * h), q2, scales(g, E, d), ye, gws)
        torch.cuda.synchronize()
        assert [len(moe.moe_profile_read(stage)) for stage in (1, 3, 4, 5)] == [2, 1, 1, 1]
    finally:
        moe.moe_profile_enable(0, 0)


@pytest.mark.parametrize("counts,kernel", [([1, 2], "q8_stream_kernel 16x16"), ([24, 40], "q8_tile_kernel"), ([70, 50], "q8_small_run_kernel"), ([300, 220], "q8_run_kernel")])
def test_weights_past_32_bit_offsets(counts, kernel):
    """Two matrices of 4.3 GB each: the second one's last columns, and some between."""
    N, K, E = (1 << 18) + 260, 16384, 2
    g, R = gen(8), sum(counts)
    assert moe.moe_q8_linear_kernel(moe.Q8Shape.make(R, E, N, K)).startswith(kernel)
    x, xs, ws = codes(g, R, K), scales(g, R, of=1 / 73), scales(g, E, N, of=1 / (73 * 128))
    w = torch.zeros(E, N, K, dtype=torch.int8, device=DEV)
    at = torch.tensor([0, 1, 131071, 131072, N // 2, N - 257, N - 256, N - 2, N - 1], device=DEV)
    some = codes(g, E, len(at), K)
    w[:, at] = some
    y = torch.full((R, N), 7.0, device=DEV)
    offsets = offsets_of(counts)
    moe.moe_q8_linear(moe.Q8Shape.make(R, E, N, K, y="f32"), x, xs, offsets, w, ws, None, None, y)
    e = expert_of(offsets, R)
    assert torch.equal(y[:, at], sums(x, some, offsets).float() * xs[:, None] * ws[e][:, at])
    y[:, at] = 0
    assert not bool(y.any())
