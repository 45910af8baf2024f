"""Rows and weights held in 8 bits, against the formulas in 64 bits: codes, scales and sums of whole numbers are equal to the
last bit; activations, biases and residuals are toleranced by the roundings of fp32 and of the output."""
import math

import pytest
import torch

import paper_2210_17223_amd as moe
from gpu_util import DEV

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def normal(g, *shape, std=1.0, dtype=torch.float32):
    return (torch.randn(*shape, generator=g, device=DEV) * std).to(dtype)


def held(v):
    """Codes and fp32 scales of rows by the definition.  (127 v is exact in 64 bits, and a quotient that lies on no border of two codes is
    further than 2^-33 from it: v and most have 24 digits.)"""
    v = v.double()
    most = v.abs().amax(-1, keepdim=True)
    ok = torch.isfinite(v).all(-1, keepdim=True)
    code = torch.where(ok & (most > 0), torch.round(127 * v / most), 0.0)
    scale = (torch.where(ok, most, math.nan) / 127).float()
    return code.to(torch.int8), scale.squeeze(-1)


def codes(g, *shape):
    return torch.randint(-127, 128, shape, generator=g, device=DEV, dtype=torch.int8)


def scales(g, *shape, of=1.0):
    return (0.5 + torch.rand(*shape, generator=g, device=DEV)) * of


def offsets_of(counts):
    return torch.tensor([0] + list(torch.tensor(counts).cumsum(0)), dtype=torch.int32, device=DEV)


def sums(x, w, offsets):
    """x w^T by expert as fp32 of the exact whole number, [rows, N]; rows behind the last expert 0."""
    out = torch.zeros(x.shape[0], w.shape[1], dtype=torch.float64, device=DEV)
    o = offsets.tolist()
    for e in range(w.shape[0]):
        if o[e + 1] > o[e]:
            out[o[e]:o[e + 1]] = x[o[e]:o[e + 1]].double() @ w[e].double().T
    return out


def expert_of(offsets, rows):
    at = torch.arange(rows, device=DEV, dtype=torch.int32)
    return torch.searchsorted(offsets[1:].contiguous(), at, right=True).clamp(max=offsets.numel() - 2)


def act64(v, name):
    if name == "silu":
        return v * torch.sigmoid(v)
    if name == "gelu":
        return v * torch.special.ndtr(v)
    if name == "gelu_tanh":
        return v * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3))
    return v.clamp(min=0) if name == "relu" else v


# ---------------------------------------------------------------------------- rows
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("R,K", [(1, 16), (5, 48), (64, 1024), (9, 1040), (33, 4096), (3, 4112), (7, 8192), (2, 12304), (2, 16384),
                                 (3, 16400), (2, 65536)])
def test_rows_are_the_rounded_quotients(R, K, dtype):
    x = normal(gen(R + K), R, K, std=3.0).to(TYPES[dtype])
    q = torch.full((R, K), 99, dtype=torch.int8, device=DEV)
    s = torch.full((R,), -1.0, device=DEV)
    moe.moe_q8_rows(x, q, s)
    code, scale = held(x)
    assert torch.equal(q, code) and torch.equal(s, scale)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_values_on_the_border_of_two_codes(dtype):
    """127 v / most = n + 1/2 exactly: ties go to the even code; and the values next to them, which do not tie."""
    most = torch.tensor([[254.0], [127.0], [1.0], [2.0 ** -12], [508.0]], device=DEV)
    n = torch.arange(-127, 127, device=DEV).float() + 0.5
    v = (most * (n / 127))[:, :240]                                # (for 254 and 508 the border itself: 2 n + 1, 4 n + 2)
    v[0], v[4] = 2 * n[:240], 4 * n[:240]
    x = torch.cat([v, most, -most, most * 0.5, most * 0.25], 1).to(TYPES[dtype])
    x = torch.cat([x] + [torch.nextafter(x.float(), torch.full_like(x.float(), t)).to(x.dtype) for t in (-1e9, 1e9)])
    x = torch.cat([x, x[:, :12]], 1).contiguous()
    x = x.clamp(-x[:, 240:241].abs().float(), x[:, 240:241].abs().float()).to(x.dtype) if dtype == "f32" else x
    q, s = torch.empty(x.shape, dtype=torch.int8, device=DEV), torch.empty(x.shape[0], device=DEV)
    assert x.shape[1] % 16 == 0
    moe.moe_q8_rows(x, q, s)
    code, scale = held(x)
    assert torch.equal(q, code) and torch.equal(s, scale)
    assert set(q[0, :240].tolist()) <= {c for c in range(-126, 127, 2)}


def test_rows_of_any_size_and_rows_that_are_not_finite():
    g = gen(3)
    x = normal(g, 12, 320)
    x[0] = 0
    x[1] *= 2.0 ** 120
    x[2] = x[2].sign() * 3.4e38
    x[3] *= 2.0 ** -126
    x[4] *= 2.0 ** -145                       # subnormal numbers
    x[5, 7] = math.nan
    x[6, 319] = math.inf
    x[7, 0] = -math.inf
    x[8] = 0
    x[8, 5] = 2.0 ** -149                     # the smallest there is
    x[9] *= 2.0 ** 64
    x[10] *= 2.0 ** -63
    q, s = torch.empty(12, 320, dtype=torch.int8, device=DEV), torch.empty(12, device=DEV)
    moe.moe_q8_rows(x, q, s)
    code, scale = held(x)
    assert torch.equal(q, code)
    assert torch.equal(torch.isnan(s), torch.isnan(scale)) and torch.equal(s.nan_to_num(7.0), scale.nan_to_num(7.0))
    assert torch.isnan(s).nonzero().flatten().tolist() == [5, 6, 7] and s[0] == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("R,K", [(1, 16), (777, 48), (5, 16400), (3000, 512)])
def test_values_are_codes_times_scales(R, K, dtype):
    g = gen(R)
    q, s = codes(g, R, K), scales(g, R, of=0.01)
    x = torch.empty(R, K, dtype=TYPES[dtype], device=DEV)
    moe.moe_q8_values(q, s, x)
    assert torch.equal(x, (q.float() * s[:, None]).to(TYPES[dtype]))


# ---------------------------------------------------------------------------- linear map
# R counts by expert, N, K: every kernel and form, in the order of q8.hip
LINEAR = {
    "few, one row": ([1], 64, 4096), "few, depth below a stage": ([3, 0, 2], 48, 16), "few, uneven": ([0, 17, 1, 31, 0], 100, 1040),
    "few, odd width": ([5, 16], 37, 272), "few, 32 rows": ([32], 96, 640), "few, wide": ([9], 5001, 128),
    "tiles": ([200, 0, 130], 256, 512), "tiles, tail": ([300], 132, 1008), "tiles, one stage": ([150], 300, 128),
    "tiles, odd width": ([129, 260], 131, 272), "tiles, width 3": ([500], 3, 64),
    "deep": ([100, 60], 384, 4096), "deep, tail": ([140], 388, 4080),
    "wide": ([700, 1, 900], 2048, 1024), "wide, tail": ([2600], 1028, 656), "wide, odd width": ([2600], 1027, 640),
    "128 x 256": ([2100, 1900], 2052, 6144 + 16), "128 x 256, whole": ([4100], 2048, 6400),
    "256 x 256": ([3000, 5, 2500], 4096, 2176), "256 x 256, short": ([9000], 4096, 256),
}


def linear_case(name, seed=0, spare=0):
    counts, N, K = LINEAR[name]
    g, E, R = gen(seed), len(counts), sum(counts) + spare
    x, w = codes(g, R, K), codes(g, E, N, K)
    return dict(R=R, E=E, N=N, K=K, x=x, w=w, xs=scales(g, R, of=1 / 73), ws=scales(g, E, N, of=1 / (73 * math.sqrt(K))),
                offsets=offsets_of(counts), g=g, rows=sum(counts))


@pytest.mark.parametrize("name", list(LINEAR))
def test_sums_are_exact(name):
    """fp32 outputs without bias and activation: the whole number, rounded, times both scales, bit for bit; rows behind the last
    expert are left."""
    c = linear_case(name, spare=3)
    y = torch.full((c["R"], c["N"]), 7.0, device=DEV)
    moe.moe_q8_linear(moe.Q8Shape.make(c["R"], c["E"], c["N"], c["K"], y="f32"), c["x"], c["xs"], c["offsets"], c["w"], c["ws"], None,
                      None, y)
    e = expert_of(c["offsets"], c["R"])
    want = sums(c["x"], c["w"], c["offsets"]).float() * c["xs"][:, None] * c["ws"][e]
    want[c["rows"]:] = 7.0
    assert torch.equal(y, want)


@pytest.mark.parametrize("name", ["few, uneven", "few, odd width", "tiles, tail", "tiles, odd width", "deep", "wide", "wide, tail",
                                  "128 x 256", "256 x 256"])
@pytest.mark.parametrize("act,res,out,in_place", [
    ("identity", "", "bf16", False), ("silu", "f32", "f32", True), ("gelu", "bf16", "bf16", True), ("gelu_tanh", "f16", "f32", False),
    ("relu", "f32", "f16", False), ("gelu", "f16", "f16", True), ("identity", "bf16", "f32", False)])
def test_epilogue(name, act, res, out, in_place):
    c = linear_case(name, seed=1)
    g = c["g"]
    bias = normal(g, c["E"], c["N"], std=0.5) if act != "relu" else None
    r = normal(g, c["R"], c["N"], std=2.0).to(TYPES[res]) if res else None
    e = expert_of(c["offsets"], c["R"])
    v = sums(c["x"], c["w"], c["offsets"]) * c["xs"].double()[:, None] * c["ws"][e].double()
    pre = v if bias is None else v + bias[e].double()
    want = act64(pre, act)
    # roundings of fp32: the sum, two scales, the bias (of what is added); the activation within 7.2e-7 or 2^-20 of its value (relu
    # and identity none: 3 more roundings cover their form); the residual's sum; then the output's
    room = 2.0 ** -24 * (4 * v.abs() + 2 * pre.abs() + 2 * want.abs()) * 1.2 + (7.2e-7 if act == "gelu" else 0.0) + \
        2.0 ** -20 * want.abs()
    if r is not None:
        want = want + r.double()
        room = room + 2.0 ** -24 * want.abs()
    room = room + EPS[out] * want.abs() * (1 + 2.0 ** -8) + 2.0 ** -25
    y = r if in_place else torch.empty(c["R"], c["N"], dtype=TYPES[out], device=DEV)
    moe.moe_q8_linear(moe.Q8Shape.make(c["R"], c["E"], c["N"], c["K"], act=act, res=res or "f32", y=out), c["x"], c["xs"], c["offsets"],
                      c["w"], c["ws"], bias, r, y)
    over = (y.double() - want).abs() - room
    assert float(over.max()) <= 0, (float(over.max()), int((over > 0).sum()))


# ---------------------------------------------------------------------------- gated block
GATED = {
    "one row": ([1], 256, 512), "few, uneven": ([0, 17, 1, 14, 0], 272, 144), "few, 32 rows": ([32, 3], 1040, 528),
    "tiles": ([200, 0, 130], 512, 384), "tiles, tail": ([300, 1], 1008, 208), "deep": ([100, 60], 4096, 320),
    "wide": ([700, 1, 900], 1024, 1024), "wide, tail": ([2600], 656, 1040), "256 x 256": ([3000, 5, 2500], 2176, 2048),
    "256 x 256, tail": ([9000], 304, 1552),
}


def gated_case(name, seed=0, spare=0):
    counts, d, h = GATED[name]
    g, E, R = gen(seed), len(counts), sum(counts) + spare
    return dict(R=R, rows=sum(counts), E=E, d=d, h=h, x=codes(g, R, d), xs=scales(g, R, of=1 / 73), offsets=offsets_of(counts),
                q13=codes(g, E, 2 * h, d), s13=scales(g, E, 2 * h, of=1 / (73 * math.sqrt(d))), q2=codes(g, E, d, h),
                s2=scales(g, E, d, of=1 / (73 * math.sqrt(h))))


def gated_run(c, act, x=None, xs=None, src_of=None, T=None, k=1):
    s = moe.Shape.make(T or c["R"], c["d"], c["E"], c["h"], k, c["R"], act=act)
    ye = torch.full((c["R"], c["d"]), 7.0, dtype=torch.float16, device=DEV)
    ws = torch.empty(moe.moe_gated_q8_workspace_bytes(s), dtype=torch.uint8, device=DEV)
    moe.moe_gated_ffn_q8(s, c["x"] if x is None else x, c["xs"] if xs is None else xs, src_of, c["offsets"], c["q13"], c["s13"], c["q2"],
                         c["s2"], ye, ws)
    return ye


@pytest.mark.parametrize("name", list(GATED))
@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh", "relu", "identity"])
def test_gated_block(name, act):
    """H is off by some 2^-20 of itself before it is rounded, so 2^-8 of its values round to the other neighbour in fp16, which moves
    127 H / most by at most 127 2^-10 = 2^-3: of these an eighth get another code; and a row's largest does so with the same odds,
    when an eighth of the row's codes may change.  So 2^-10 of the codes, each by one step: of a row whose root mean square is at
    least most / 8, sqrt(2^-10) 8 / 127 = 2e-3 of the output, and fp16's rounding, 2^-11.  A single value: all of an eighth of a row's
    codes, six deviations, sqrt(1 / 8) 6 8 / 127 = 0.14 of the output's root mean square."""
    c = gated_case(name, spare=2)
    ye = gated_run(c, act)
    h, rows = c["h"], c["rows"]
    assert bool((ye[rows:] == 7.0).all())
    o = c["offsets"].tolist()
    for e in range(c["E"]):
        lo, hi = o[e], o[e + 1]
        if lo == hi:
            continue
        both = (c["x"][lo:hi].double() @ c["q13"][e].double().T) * c["xs"][lo:hi].double()[:, None] * c["s13"][e].double()
        H = (act64(both[:, :h], act) * both[:, h:]).half()
        q, s = held(H)
        want = (q.double() @ c["q2"][e].double().T) * s.double()[:, None] * c["s2"][e].double()
        off = (ye[lo:hi].double() - want).abs() - 2.0 ** -11 * want.abs()
        rms = float(want.square().mean().sqrt())
        assert float(off.clamp(min=0).square().mean().sqrt()) <= 2e-3 * rms
        assert float(off.max()) <= 0.14 * rms


@pytest.mark.parametrize("T,k,E,d,h,capacity", [(5, 2, 8, 256, 512, 5), (700, 2, 4, 384, 272, 250), (3000, 3, 5, 272, 528, 3000),
                                                (9000, 1, 2, 1024, 1040, 9000)])
def test_rows_taken_where_they_are_and_rows_moved_give_the_same_bits(T, k, E, d, h, capacity):
    g = gen(T)
    x, xs = codes(g, T, d), scales(g, T, of=1 / 73)
    idx = torch.rand(T, E, generator=g, device=DEV).argsort(1)[:, :k].contiguous().int().view(-1)
    s = moe.Shape.make(T, d, E, h, k, capacity, act="silu")
    rows = moe.moe_max_rows(s)
    i32 = lambda n: torch.full((n,), -7, dtype=torch.int32, device=DEV)  # noqa: E731
    plans = [dict(counts=i32(E), offsets=i32(E + 1), slot_of=i32(T * k), src_of=i32(rows)) for _ in range(3)]
    xe, xes = torch.full((rows, d), 5, dtype=torch.int8, device=DEV), torch.full((rows,), -1.0, device=DEV)
    ws = torch.empty(moe.moe_workspace_bytes(s, 1), dtype=torch.uint8, device=DEV)
    moe.moe_dispatch_q8(s, x, xs, idx, *plans[0].values(), xe, xes, ws)
    moe.moe_dispatch_q8(s, x, xs, idx, *plans[1].values(), None, None, ws)
    xe16 = torch.empty(rows, d, dtype=torch.bfloat16, device=DEV)
    moe.moe_dispatch(s, x.bfloat16(), idx, *plans[2].values(), xe16, ws)
    A = int(plans[2]["offsets"][-1])
    for p in plans[:2]:
        for key, v in p.items():
            n = A if key == "src_of" else v.numel()
            assert torch.equal(v[:n], plans[2][key][:n]), key
    token = plans[0]["src_of"][:A].long() // k
    assert torch.equal(xe[:A], x[token]) and torch.equal(xes[:A], xs[token])
    assert bool((xe[A:] == 5).all()) and bool((xes[A:] == -1).all())
    q13, s13 = codes(g, E, 2 * h, d), scales(g, E, 2 * h, of=1 / (73 * math.sqrt(d)))
    q2, s2 = codes(g, E, d, h), scales(g, E, d, of=1 / (73 * math.sqrt(h)))
    gws = torch.empty(moe.moe_gated_q8_workspace_bytes(s), dtype=torch.uint8, device=DEV)
    ye = [torch.full((rows, d), 7.0, dtype=torch.float16, device=DEV) for _ in range(2)]
    moe.moe_gated_ffn_q8(s, xe, xes, None, plans[0]["offsets"], q13, s13, q2, s2, ye[0], gws)
    moe.moe_gated_ffn_q8(s, x, xs, plans[0]["src_of"], plans[0]["offsets"], q13, s13, q2, s2, ye[1], gws)
    assert torch.equal(ye[0], ye[1]) and bool((ye[0][A:] == 7.0).all())


# ---------------------------------------------------------------------------- norms
@pytest.mark.parametrize("T,d", [(1, 16), (3, 96), (70, 512), (5, 2048), (9, 2064), (4, 4096), (3, 8192), (2, 12304), (2, 16384)])
@pytest.mark.parametrize("kind,res,z,bias,gate_tokens", [("rms", "f32", "f16", False, 0), ("layer", "bf16", "bf16", True, 2),
                                                         ("rms", "bf16", "f32", False, 3), ("layer", "f32", "f32", True, 0)])
def test_norms_write_the_codes_of_their_fp32_rows(T, d, kind, res, z, bias, gate_tokens):
    """next in fp32 is what the codes are of, whether it is wanted or not.  r and next against 64 bits: a row's mean and mean square are sums in
    at most 16 + 10 + 4 steps, 2^-19 of the sums of magnitudes, and so is a factor's; of a hat, whose root mean square is one, 2^-18 (1 + |hat|)
    with the roundings of its products; r once more rounded to its type."""
    g = gen(T + d)
    n = moe.NormShape.make(T, d, kind=kind, dtype="f32", res=res, z=z, scale=0.7, gate_tokens=gate_tokens)
    x, zz = normal(g, T, d, std=2.0).to(n.res_torch_dtype), normal(g, T, d).to(n.z_torch_dtype)
    vec = lambda: normal(g, d, std=0.2) + 1.0  # noqa: E731
    w, wn, b, bn = vec(), vec(), vec() if bias else None, vec() if bias else None
    gate = normal(g, n.gates, d, std=0.3) + 0.5
    new = lambda dtype, *s: torch.empty(*s, dtype=dtype, device=DEV)  # noqa: E731

    def hat(v):
        v = v.double()
        v = v - v.mean(1, keepdim=True) if kind == "layer" else v
        return v * torch.rsqrt(v.square().mean(1, keepdim=True) + 1e-5)

    for after in (True, False):
        r = [new(n.res_torch_dtype, T, d) for _ in range(2)]
        nx = new(torch.float32, T, d)
        q, s = [new(torch.int8, T, d) for _ in range(2)], [new(torch.float32, T) for _ in range(2)]
        if after:
            moe.moe_norm_after_q8(n, x, zz, w, b, gate, r[0], wn, bn, nx, q[0], s[0])
            moe.moe_norm_after_q8(n, x, zz, w, b, gate, r[1], wn, bn, None, q[1], s[1])
            assert torch.equal(r[0], r[1])
            zh, gt = hat(zz), 0.7 * gate[torch.arange(T, device=DEV) // (gate_tokens or T)].double()
            want = x.double() + gt * (zh * w + (0 if b is None else b.double()))
            room = 2.0 ** -18 * (1 + zh.abs()) * (gt * w).abs() + 2.0 ** -23 * (x.double().abs() + want.abs()) + 2.0 ** -22
            assert bool(((r[0].double() - want).abs() <= room + (EPS["bf16"] * 1.01 * want.abs() if res == "bf16" else 0)).all())
            rh = hat(r[0])
        else:
            moe.moe_norm_before_q8(n, x, wn, bn, nx, q[0], s[0])
            moe.moe_norm_before_q8(n, x, wn, bn, None, q[1], s[1])
            rh = hat(x)
        want = rh * wn + (0 if bn is None else bn.double())
        room = 2.0 ** -18 * (1 + rh.abs()) * wn.abs() + 2.0 ** -23 * want.abs() + 2.0 ** -22
        assert bool(((nx.double() - want).abs() <= room).all())
        code, scale = held(nx)
        for k in range(2):
            assert torch.equal(q[k], code) and torch.equal(s[k], scale)
