"""moe_q4_linear and moe_gated_ffn_q4 against the formulas in 64 bits.

moe_q4_linear rounds nothing but fp32 sums: of the codes' products with an offset of 128 (bf16 rows) or exactly (fp16
rows) inside a group, then of the groups.  Its bound is K + 8 roundings of 2^-24 of the sum of |x| (|q - z| + 136) s.
The block holds H in fp16 and writes fp16; its weights may be rounded to fp16, too (half a step of 2^-10 each)."""
import math

import numpy as np
import pytest
import torch

import paper_2210_17223_amd as moe
from test_gpu_gated import act64

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U16, U32 = torch.finfo(torch.float16).eps / 2, torch.finfo(torch.float32).eps / 2
TINY16 = 2.0 ** -25


def make_codes(g, E, N, K, group, zeros, std):
    q = torch.randint(0, 256, (E, N, K // 2), generator=g, device=DEV, dtype=torch.uint8)
    s = ((0.5 + torch.rand(E, N, K // group, generator=g, device=DEV)) * std).half()
    z = torch.randint(0, 16, (E, N, K // group), generator=g, device=DEV, dtype=torch.uint8) if zeros else None
    return q, s, z


def wide(q, s, z, e, group):
    """Expert e's codes less their zeros, and scales, [N, K] in 64 bits."""
    c = torch.stack([q[e] & 15, q[e] >> 4], 2).flatten(1).double()
    zero = 8.0 if z is None else z[e].double().repeat_interleave(group, 1)
    return c - zero, s[e].double().repeat_interleave(group, 1)


def offsets_of(R, E, counts, seed):
    if counts is None:
        r = np.random.default_rng(seed)
        counts = r.multinomial(R, r.dirichlet(np.full(E, 0.7)))
    assert sum(counts) == R
    offs = np.concatenate([[0], np.cumsum(counts)])
    return offs, torch.tensor(offs, dtype=torch.int32, device=DEV)


class Linear:
    def __init__(self, R, N, K, group, E=1, x="bf16", zeros=False, counts=None, seed=0, mean=0.0):
        g = torch.Generator(device=DEV).manual_seed(seed)
        self.s = moe.Q4Shape.make(R, E, N, K, group, x=x)
        self.offs, self.offsets = offsets_of(R, E, counts, seed)
        self.x = (torch.randn(R, K, generator=g, device=DEV) + mean).to(self.s.x_torch_dtype)
        self.q, self.sc, self.z = make_codes(g, E, N, K, group, zeros, 0.2 / math.sqrt(K))
        self.guard = torch.full((R * N + 64,), 7.0, device=DEV)
        self.y = self.guard[:R * N].view(R, N)

    def run(self):
        moe.moe_q4_linear(self.s, self.x, self.offsets, self.q, self.sc, self.z, self.y)
        return self.y

    def check(self):
        assert bool((self.guard[-64:] == 7.0).all())
        for e in range(self.s.E):
            rows = slice(int(self.offs[e]), int(self.offs[e + 1]))
            c, s = wide(self.q, self.sc, self.z, e, self.s.group)
            x = self.x[rows].double()
            err = (self.y[rows].double() - x @ (c * s).T).abs()
            bound = (self.s.K + 8) * U32 * (x.abs() @ ((c.abs() + 136) * s).T)
            assert bool((err <= bound + 1e-30).all())
            if err.numel() >= 1000:               # rounded sums of random terms: far below one in 10^4
                assert float(err.square().mean().sqrt()) <= 2e-5 * float((x @ (c * s).T).square().mean().sqrt())


LINEAR = [
    dict(R=1, N=1, K=32, group=32), dict(R=1, N=3, K=64, group=32, zeros=True), dict(R=2, N=17, K=96, group=32, x="f16"),
    dict(R=1, N=4096, K=4096, group=32), dict(R=1, N=1000, K=4224, group=128, zeros=True, x="f16"),
    dict(R=5, N=333, K=192, group=64, E=4, zeros=True), dict(R=16, N=64, K=512, group=64), dict(R=17, N=80, K=256, group=128, x="f16"),
    dict(R=33, N=130, K=1024, group=128, E=3, counts=[0, 16, 17]), dict(R=40, N=100, K=1312, group=32, E=2, zeros=True),
    dict(R=40, N=516, K=1344, group=64, E=4, counts=[1, 0, 39, 0], x="f16", zeros=True),
    dict(R=70, N=200, K=2176, group=128, mean=1.0), dict(R=150, N=520, K=256, group=32, x="f16"),
    dict(R=150, N=520, K=288, group=32, zeros=True), dict(R=300, N=260, K=1088, group=64, E=2, counts=[299, 1]),
    dict(R=300, N=260, K=512, group=64, E=2, x="f16", zeros=True), dict(R=1000, N=1030, K=640, group=128, zeros=True, E=4),
    dict(R=1000, N=129, K=128, group=128, x="f16"), dict(R=513, N=2048, K=768, group=64, E=64), dict(R=100, N=20000, K=256, group=128),
]


@pytest.mark.parametrize("kw", LINEAR, ids=lambda kw: "-".join(str(v) for v in kw.values()))
def test_linear(kw):
    c = Linear(**kw)
    c.run()
    c.check()
    first = c.y.clone()
    c.y.fill_(7.0)
    assert torch.equal(c.run(), first)            # (sums in a fixed order)


@pytest.mark.parametrize("x", ["bf16", "f16"])
@pytest.mark.parametrize("group,K", [(32, 512), (64, 448), (128, 384), (32, 96)])
@pytest.mark.parametrize("R", [1, 50, 200])
def test_linear_every_place_counts_once(R, group, K, x):
    """Whole numbers that fp32 holds exactly: any place that is lost, doubled or mixed up changes the result."""
    c = Linear(R, 48, K, group, x=x, zeros=True, seed=R + K)
    g = torch.Generator(device=DEV).manual_seed(1)
    c.x.copy_(torch.randint(-2, 3, c.x.shape, generator=g, device=DEV))
    c.sc.copy_(torch.randint(1, 3, c.sc.shape, generator=g, device=DEV))
    codes, s = wide(c.q, c.sc, c.z, 0, group)
    assert torch.equal(c.run().double(), c.x.double() @ (codes * s).T)


class Q4Block:
    def __init__(self, R, d, h, group, E=1, act="silu", zeros=False, counts=None, spare=2, seed=0, scale=1.0):
        g = torch.Generator(device=DEV).manual_seed(seed)
        self.R, self.E, self.d, self.h, self.group, self.act = R, E, d, h, group, act
        self.s = moe.Shape.make(R + spare, d, E, h, 1, R + spare, act=act)
        self.offs, self.offsets = offsets_of(R, E, counts, seed)
        self.x = (torch.randn(R + spare, d, generator=g, device=DEV) * scale).bfloat16()
        self.x[R:] = math.nan
        self.w13 = make_codes(g, E, 2 * h, d, group, zeros, 0.2 / math.sqrt(d))
        self.w2 = make_codes(g, E, d, h, group, zeros, 0.2 / math.sqrt(h))
        self.ye = torch.full((R + spare, d), 7.0, dtype=torch.float16, device=DEV)
        self.ws = torch.full((moe.moe_gated_q4_workspace_bytes(self.s),), 255, dtype=torch.uint8, device=DEV)

    def run(self):
        moe.moe_gated_ffn_q4(self.s, self.group, self.x, self.offsets, *self.w13, *self.w2, self.ye, self.ws)
        return self.ye

    def check(self):
        e2 = w2 = n = 0
        for e in range(self.E):
            rows = slice(int(self.offs[e]), int(self.offs[e + 1]))
            if rows.start == rows.stop:
                continue
            x = self.x[rows].double()
            c, s = wide(*self.w13, e, self.group)
            W, h, d = c * s, self.h, self.d
            G, U = x @ W[:h].T, x @ W[h:].T
            # of G and U: fp32 sums, and weights rounded to fp16
            S = (d + 8) * U32 * (x.abs() @ ((c.abs() + 136) * s).T) + x.abs() @ (U16 * W.abs() + TINY16).T
            a, _ = act64(G, self.act)
            H = a * U
            BH = 1.14 * U.abs() * S[:, :h] + a.abs() * S[:, h:] + U.abs() * (1e-6 + 5e-5 * a.abs()) + U16 * H.abs() + TINY16
            c, s = wide(*self.w2, e, self.group)
            W = c * s
            want = H @ W.T
            bound = BH @ W.abs().T + (h + 8) * U32 * (H.abs() @ ((c.abs() + 136) * s).T) + H.abs() @ (U16 * W.abs() + TINY16).T
            err = (self.ye[rows].double() - want).abs()
            assert bool((err <= bound + U16 * want.abs() + TINY16).all())
            e2, w2, n = e2 + float(err.square().sum()), w2 + float(want.square().sum()), n + err.numel()
        if n >= 1000:                             # roundings to fp16: both weights of H (twice), H, the second weight, ye
            assert math.sqrt(e2 / w2) <= math.sqrt(5) * U16
        assert bool((self.ye[self.R:] == 7.0).all())


BLOCKS = [
    dict(R=1, d=32, h=32, group=32), dict(R=2, d=4096, h=1024, group=128, E=8), dict(R=9, d=96, h=160, group=32, E=3, zeros=True, act="gelu"),
    dict(R=64, d=512, h=1344, group=64, E=8, zeros=True), dict(R=50, d=256, h=768, group=128, E=4, counts=[0, 31, 19, 0], act="gelu_tanh"),
    dict(R=200, d=640, h=384, group=64, act="relu"), dict(R=700, d=512, h=1056, group=32, E=2, counts=[699, 1], zeros=True),
    dict(R=1500, d=384, h=1152, group=128, E=5, act="identity"), dict(R=3000, d=1024, h=2048, group=64, E=4, zeros=True, act="gelu"),
    dict(R=2000, d=544, h=1120, group=32, E=1), dict(R=4096, d=512, h=1536, group=128, E=16, act="gelu_tanh"),
]


@pytest.mark.parametrize("kw", BLOCKS, ids=lambda kw: "-".join(str(v) for v in kw.values()))
def test_gated_ffn(kw):
    b = Q4Block(**kw)
    first = b.run().clone()
    b.check()
    b.ye.fill_(7.0)
    assert torch.equal(b.run(), first)


def test_tiny_and_huge_rows():
    """Rows whose values are far apart in size: each is held to its own digits (bf16's range is fp32's)."""
    b = Q4Block(R=600, d=512, h=512, group=128)
    scale = torch.logspace(-30, 2, 600, device=DEV)
    b.x[:600] = (b.x[:600].float() * scale[:, None]).bfloat16()
    b.x[5, :] = 0.0
    b.run()
    b.check()


def test_nan_and_infinite_rows_stay_their_own():
    for R in (20, 700):
        b = Q4Block(R=R, d=256, h=512, group=64)
        clean = b.run().clone()
        b.x[3, 9], b.x[R - 1, 200] = math.nan, math.inf
        b.run()
        rows = torch.ones(R + 2, dtype=torch.bool, device=DEV)
        rows[[3, R - 1]] = False
        assert torch.equal(b.ye[rows], clean[rows]) and not torch.isfinite(b.ye[[3, R - 1]].float()).any()


def test_no_rows_at_all():
    b = Q4Block(R=0, d=64, h=64, group=32, E=3, counts=[0, 0, 0])
    assert bool((b.run() == 7.0).all())
    L = Linear(R=4, N=16, K=64, group=32, E=2, counts=[4, 0])
    L.offsets.zero_()
    assert bool((L.run() == 7.0).all())


def test_another_stream_and_a_graph():
    for kw in (dict(R=12, d=512, h=768, group=64, E=4), dict(R=900, d=512, h=768, group=64, E=2)):
        b = Q4Block(**kw)
        want = b.run().clone()
        st = torch.cuda.Stream()
        b.ye[:b.R] = 0.0
        st.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(st):
            b.run()
        st.synchronize()
        assert torch.equal(b.ye, want)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            b.run()
        for _ in range(3):
            b.ye[:b.R] = 0.0
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(b.ye, want)
            b.run()


# Each tile of the kernels for many rows (32, 64 and 128 rows), and a depth that one, two or four parts of a block share out
TILES = [
    dict(R=40, N=8200, K=256, group=32), dict(R=200, N=4224, K=384, group=64, x="f16", zeros=True), dict(R=35, N=70, K=1184, group=32),
    dict(R=300, N=5000, K=640, group=128, zeros=True), dict(R=300, N=5000, K=96, group=32, x="f16"),
    dict(R=700, N=5000, K=320, group=64), dict(R=800, N=5000, K=320, group=64, x="f16"), dict(R=800, N=5000, K=160, group=32, zeros=True),
    dict(R=2050, N=300, K=384, group=128), dict(R=2050, N=130, K=416, group=32, x="f16", zeros=True),
    dict(R=900, N=2000, K=256, group=128, E=7, counts=[0, 1, 33, 0, 800, 64, 2]), dict(R=24, N=4000, K=512, group=64, zeros=True),
    dict(R=60, N=700, K=640, group=32, E=2, counts=[59, 1], x="f16"),
]


@pytest.mark.parametrize("kw", TILES, ids=lambda kw: "-".join(str(v) for v in kw.values()))
def test_linear_tiles(kw):
    c = Linear(**kw)
    c.run()
    c.check()
    first = c.y.clone()
    c.y.fill_(7.0)
    assert torch.equal(c.run(), first)


BLOCK_TILES = [
    dict(R=100, d=512, h=512, group=128, E=2), dict(R=100, d=96, h=2976, group=32, zeros=True, act="gelu"),
    dict(R=400, d=640, h=3200, group=64), dict(R=1500, d=256, h=4096, group=128, E=8, zeros=True, act="relu"),
    dict(R=2500, d=1056, h=608, group=32, act="gelu_tanh"), dict(R=2100, d=384, h=640, group=128, E=2, counts=[0, 2100], zeros=True),
]


@pytest.mark.parametrize("kw", BLOCK_TILES, ids=lambda kw: "-".join(str(v) for v in kw.values()))
def test_gated_ffn_tiles(kw):
    b = Q4Block(**kw)
    first = b.run().clone()
    b.check()
    b.ye.fill_(7.0)
    assert torch.equal(b.run(), first)


# Few tiles: 32 columns at a time (sixteen gates and their values), widths that end inside them, the depth in eight and four parts
NARROW = [
    dict(R=17, d=96, h=160, group=32, zeros=True), dict(R=40, d=1152, h=1408, group=128), dict(R=90, d=704, h=1088, group=64, act="gelu"),
    dict(R=64, d=352, h=544, group=32, E=3, counts=[33, 0, 31], act="relu"), dict(R=150, d=512, h=1024, group=128, E=2, zeros=True),
]


@pytest.mark.parametrize("kw", NARROW, ids=lambda kw: "-".join(str(v) for v in kw.values()))
def test_gated_ffn_narrow(kw):
    b = Q4Block(**kw)
    first = b.run().clone()
    b.check()
    b.ye.fill_(7.0)
    assert torch.equal(b.run(), first)


# bf16 rows have fp32's range: of every path (few rows, tiles of 32, 64 and 128 rows, a shared depth), with zeros of four and of eight bits
RANGE = [
    dict(R=1, N=100, K=512, group=128), dict(R=16, N=70, K=608, group=32, zeros=True), dict(R=24, N=40, K=512, group=64, E=3, zeros=True),
    dict(R=60, N=300, K=640, group=128, zeros=True), dict(R=200, N=4224, K=384, group=64), dict(R=800, N=5000, K=160, group=32, zeros=True),
    dict(R=2050, N=300, K=384, group=128, zeros=True),
]


@pytest.mark.parametrize("kw,bytes_", [(kw, b) for kw in RANGE for b in ([False, True] if kw.get("zeros") else [False])],
                         ids=lambda v: "-".join(str(x) for x in v.values()) if isinstance(v, dict) else "bytes" if v else "nibbles")
def test_linear_of_rows_of_any_size(kw, bytes_):
    """Rows of 1e-25 to 1e37: what is finite in 64 bits is finite here, and each row is held to its own digits.  (Outputs are below
    1e37 * 255 * 0.3 / sqrt(K) * K < 3.4e38 only with smaller scales: those are taken by 2^-10.)"""
    c = Linear(**kw)
    if bytes_:
        g = torch.Generator(device=DEV).manual_seed(3)
        c.z.copy_(torch.randint(0, 256, c.z.shape, generator=g, device=DEV))
    c.sc.mul_(2.0 ** -10 if c.s.K < 1024 else 2.0 ** -12)
    size = torch.logspace(-25, 37, kw["R"], device=DEV, dtype=torch.float64) if kw["R"] > 1 else torch.tensor([1e37], device=DEV)
    c.x.copy_((c.x.double() * size[:, None]).clamp(-3.3e38, 3.3e38))
    c.run()
    for e in range(c.s.E):
        rows = slice(int(c.offs[e]), int(c.offs[e + 1]))
        codes, s = wide(c.q, c.sc, c.z, e, c.s.group)
        x = c.x[rows].double()
        want = x @ (codes * s).T
        assert bool((want.abs() < 3e38).all())
        bound = (c.s.K + 8) * U32 * (x.abs() @ ((codes.abs() + 136) * s).T)
        assert bool(((c.y[rows].double() - want).abs() <= bound).all())


def test_block_of_few_rows_of_any_size():
    """As test_tiny_and_huge_rows, on the path for few rows.  (H is fp16: a row whose H passes 65504 has no finite output.)"""
    b = Q4Block(R=20, d=512, h=512, group=128, E=2, zeros=True)
    b.x[:20] = (b.x[:20].float() * torch.logspace(-30, 2, 20, device=DEV)[:, None]).bfloat16()
    b.x[5, :] = 0.0
    first = b.run().clone()
    most = torch.zeros(b.R + 2, dtype=torch.float64, device=DEV)
    for e in range(b.E):
        rows = slice(int(b.offs[e]), int(b.offs[e + 1]))
        c, s = wide(*b.w13, e, b.group)
        GU = b.x[rows].double() @ (c * s).T
        most[rows] = (act64(GU[:, :512], "silu")[0] * GU[:, 512:]).abs().amax(1)
    over, near = most > 65504 * 1.01, most > 65504 * 0.99
    assert not torch.isfinite(first[over].float()).any()
    b.x[near] = 0.0
    b.run()
    b.check()
    assert torch.equal(b.ye[~near], first[~near])


# (The bounds above count an offset of the codes of 128 in bf16 sums; it is 16.)
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("R", [1, 16, 50, 200, 2100])
def test_codes_of_bf16_rows_cost_few_digits(R, group):
    """Rows of large whole numbers of one sign among which lie odd ones: a group's sum of (16 + q) x stays below 2^24 and is
    exact in fp32, and so are the totals; a larger offset of the codes would round it.  (A group's x: numbers of 128 .. 255 times
    2048 / group, at most 2^19 together, and one odd number below 256 instead of one of them.)"""
    K = 2 * group
    c = Linear(R, 48, K, group, zeros=True, seed=R)
    g = torch.Generator(device=DEV).manual_seed(R + group)
    x = torch.randint(128, 256, c.x.shape, generator=g, device=DEV) * (2048 // group)
    odd = torch.randint(0, 128, (R, 2), generator=g, device=DEV) * 2 + 1
    x[:, 5], x[:, group + 7] = odd[:, 0], odd[:, 1]
    c.x.copy_(x)
    c.sc.fill_(1.0)
    assert torch.equal(c.x.double(), x.double()) and int(x.view(R, 2, group).sum(2).max()) * 31 < 2 ** 24
    codes, s = wide(c.q, c.sc, c.z, 0, group)
    assert torch.equal(c.run().double(), c.x.double() @ (codes * s).T)


def test_linear_past_2_to_31_bytes_of_a_tiles_rows():
    """128 rows of more than 2^23 values each, whose last stage ends inside 128: what lies past a row's end is zeros, not the
    values 2^31 bytes behind it (infinities here, of a row that has nothing else)."""
    R, N, K, group = 1024, 640, (1 << 23) + 96, 32
    s = moe.Q4Shape.make(R, 1, N, K, group)
    x = torch.zeros(R, K, dtype=torch.bfloat16, device=DEV)
    x[:, ::4099], x[:, K - 1] = 1.0, 3.0
    x[127::128] = math.inf
    q = torch.full((1, N, K // 2), 0x9a, dtype=torch.uint8, device=DEV)     # codes 10, 9, 10, 9, ...
    scale = torch.ones(1, N, K // group, dtype=torch.float16, device=DEV)
    offsets = torch.tensor([0, R], dtype=torch.int32, device=DEV)
    y = torch.full((R, N), 7.0, device=DEV)
    moe.moe_q4_linear(s, x, offsets, q, scale, None, y)
    k = torch.arange(0, K, 4099, device=DEV)
    k = k[k != K - 1]
    want = float(torch.where(k % 2 == 0, 2.0, 1.0).sum()) + 3.0
    rows = torch.ones(R, dtype=torch.bool, device=DEV)
    rows[127::128] = False
    assert bool((y[rows] == want).all()) and not torch.isfinite(y[~rows]).any()


# Few rows of many experts, and the first counts that are too many for that path
@pytest.mark.parametrize("kw", [dict(R=96, N=300, K=608, group=32, E=64, zeros=True), dict(R=97, N=300, K=608, group=32, E=64),
                                dict(R=95, N=72, K=512, group=128, E=16, x="f16", counts=[0, 60] + [0] * 13 + [35])],
                         ids=lambda kw: "-".join(str(v) for v in kw.values() if not isinstance(v, list)))
def test_linear_of_many_experts(kw):
    test_linear(kw)


@pytest.mark.parametrize("R", [96, 97])
def test_block_of_many_experts(R):
    test_gated_ffn(dict(R=R, d=256, h=544, group=32, E=20, zeros=True, spare=0))


def test_block_of_more_rows_than_a_grid_has_wavefronts():
    """Past 2^26 rows (a grid has fewer than 2^32 threads, and a wavefront makes a row ready); checked on rows all over them."""
    R, d, h, group = (1 << 26) + 5, 32, 32, 32
    s = moe.Shape.make(R, d, 1, h, 1, R, act="silu")
    g = torch.Generator(device=DEV).manual_seed(0)
    x = torch.randint(-7, 8, (R, d), generator=g, device=DEV, dtype=torch.int8).bfloat16()
    offsets = torch.tensor([0, R], dtype=torch.int32, device=DEV)
    w13, w2 = make_codes(g, 1, 2 * h, d, group, True, 0.05), make_codes(g, 1, d, h, group, True, 0.05)
    ye = torch.full((R, d), 7.0, dtype=torch.float16, device=DEV)
    ws = torch.full((moe.moe_gated_q4_workspace_bytes(s),), 255, dtype=torch.uint8, device=DEV)
    moe.moe_gated_ffn_q4(s, group, x, offsets, *w13, *w2, ye, ws)
    at = torch.cat([torch.arange(0, R, 1 << 16, device=DEV), torch.arange(R - 300, R, device=DEV)])
    b = Q4Block(R=len(at), d=d, h=h, group=group, zeros=True)
    b.x[:b.R], b.w13, b.w2 = x[at], w13, w2
    b.run()
    b.check()
    assert torch.equal(ye[at], b.ye[:b.R])        # (a row's result does not depend on where it lies)
