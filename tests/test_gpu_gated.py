"""moe_gated_ffn and its backward pass against the formulas in 64 bits.

u(t) = finfo(t).eps / 2 is the most a rounding is off, relative.  Each value is checked twice: every element against a
bound that adds up what each rounding and fp32 sum on its way can do at most, and (of a thousand values or more) the root
mean square of the error against sqrt(n) u, n the roundings to 16 bits on the way (of independent roundings each is at
most u / sqrt(3) in the mean)."""
import math

import numpy as np
import pytest
import torch

import paper_2210_17223_amd as moe

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U16, UB, U32 = (torch.finfo(t).eps / 2 for t in (torch.float16, torch.bfloat16, torch.float32))
TINY16 = 2.0 ** -25                               # half of fp16's smallest step


def act64(v, name):
    """Value and slope."""
    if name == "silu":
        p = torch.sigmoid(v)
        return v * p, p * (1 + v * (1 - p))
    if name == "gelu":
        P = torch.special.ndtr(v)
        return v * P, P + v * torch.exp(-v * v / 2) / math.sqrt(2 * math.pi)
    if name == "gelu_tanh":
        c, a = math.sqrt(2 / math.pi), 0.044715
        t = torch.tanh(c * (v + a * v ** 3))
        return 0.5 * v * (1 + t), 0.5 * (1 + t) + 0.5 * v * (1 - t * t) * c * (1 + 3 * a * v * v)
    if name == "relu":
        return v.clamp(min=0), (v > 0).double()
    return v, torch.ones_like(v)


class Block:
    def __init__(self, R, E, d, h, act="silu", dtype="bf16", counts=None, spare=3, seed=0, scale=1.0):
        g = torch.Generator(device=DEV).manual_seed(seed)
        self.R, self.E, self.d, self.h, self.act = R, E, d, h, act
        self.s = moe.Shape.make(R + spare, d, E, h, 1, R + spare, dtype=dtype, act=act)
        if counts is None:
            r = np.random.default_rng(seed)
            counts = r.multinomial(R, r.dirichlet(np.full(E, 0.7)))
        assert sum(counts) == R
        self.offs = np.concatenate([[0], np.cumsum(counts)])
        self.offsets = torch.tensor(self.offs, dtype=torch.int32, device=DEV)
        t = self.s.torch_dtype
        rnd = lambda *s, std=1.0: (torch.randn(*s, generator=g, device=DEV) * std).to(t)
        n = R + spare
        self.xe, self.dye = rnd(n, d, std=scale), rnd(n, d, std=0.1)
        self.xe[R:] = math.nan                    # (rows past the last expert's are not read)
        self.dye[R:] = math.nan
        self.W13, self.W2 = rnd(E, d, 2 * h, std=1 / math.sqrt(d)), rnd(E, h, d, std=1 / math.sqrt(h))
        new = lambda *s, t, v=7.0: torch.full(s, v, dtype=t, device=DEV)
        self.W13p = torch.empty(moe.moe_gated_packed_bytes(self.s), dtype=torch.uint8, device=DEV)
        self.W2p = torch.empty(moe.moe_packed_weight_bytes(self.s), dtype=torch.uint8, device=DEV)
        self.ws = torch.full((moe.moe_gated_workspace_bytes(self.s),), 255, dtype=torch.uint8, device=DEV)
        self.ye = new(n, d, t=self.s.ye_dtype)
        if dtype == "bf16":
            self.pre, self.hid = new(n, 2 * h, t=torch.float16), new(n, h, t=torch.float16)
            self.dxe = new(n, d, t=torch.bfloat16)
            self.dW13, self.dW2 = new(E, d, 2 * h, t=torch.bfloat16), new(E, h, d, t=torch.bfloat16)
            self.bws = torch.full((moe.moe_gated_backward_workspace_bytes(self.s),), 255, dtype=torch.uint8, device=DEV)
        moe.moe_pack_gated_weights(self.s, self.W13, self.W2, self.W13p, self.W2p)

    def forward(self, keep):
        moe.moe_gated_ffn(self.s, self.xe, self.offsets, self.W13p, self.W2p, self.ye, self.pre if keep else None,
                          self.hid if keep else None, self.ws)

    def backward(self, kept=True):
        moe.moe_gated_ffn_backward(self.s, self.xe, self.offsets, self.W13, self.W2, self.W13p, self.pre if kept else None,
                                   self.hid if kept else None, self.dye, self.dxe, self.dW13, self.dW2, self.bws)
        return self.dxe.clone(), self.dW13.clone(), self.dW2.clone()

    def experts(self):
        for e in range(self.E):
            lo, hi = int(self.offs[e]), int(self.offs[e + 1])
            yield e, slice(lo, hi)


class Errors:
    """Elementwise bounds now, root mean squares over all experts at the end."""
    def __init__(self):
        self.sums = {}

    def add(self, what, got, want, bound, roundings, u):
        # (a value past its type's largest is infinite; one within a hundredth of it may be either)
        largest = torch.finfo(got.dtype).max
        assert bool(torch.isinf(got[want.abs() > 1.01 * largest]).all()), what
        inside = want.abs() < 0.99 * largest
        got, want, bound = got[inside], want[inside], bound[inside]
        err = (got.double() - want).abs()
        assert torch.isfinite(err).all(), what
        assert bool((err <= bound + 1e-30).all()), (what, float((err / (bound + 1e-30)).max()))
        s = self.sums.setdefault(what, [0.0, 0.0, 0, math.sqrt(roundings) * u])
        s[0] += float(err.square().sum())
        s[1] += float(want.square().sum())
        s[2] += err.numel()

    def close(self):
        for what, (e, w, n, limit) in self.sums.items():
            if n >= 1000:
                assert math.sqrt(e) <= limit * math.sqrt(w), (what, math.sqrt(e / w) / limit)


def check_forward(b, keep):
    d, h = b.d, b.h
    errors = Errors()
    for e, rows in b.experts():
        x = b.xe[rows].double()
        if not len(x):
            continue
        Wg, Wu, W2 = b.W13[e, :, :h].double(), b.W13[e, :, h:].double(), b.W2[e].double()
        G, U = x @ Wg, x @ Wu
        SG, SU = (d + 8) * U32 * (x.abs() @ Wg.abs()), (d + 8) * U32 * (x.abs() @ Wu.abs())
        if keep:
            pre = b.pre[rows]
            errors.add("G", pre[:, :h], G, U16 * G.abs() + SG + TINY16, 1, U16)
            errors.add("U", pre[:, h:], U, U16 * U.abs() + SU + TINY16, 1, U16)
        a, _ = act64(G, b.act)
        H = a * U
        # the activation's own error: 1e-6, and 5e-5 of its value
        BH = 1.14 * U.abs() * SG + a.abs() * SU + U.abs() * (1e-6 + 5e-5 * a.abs()) + U16 * H.abs() + TINY16
        if keep:
            errors.add("hid", b.hid[rows], H, BH, 1, U16)
        bound = BH @ W2.abs() + (h + 8) * U32 * (H.abs() @ W2.abs()) + H.abs().sum(1, keepdim=True) * TINY16
        want = H @ W2
        errors.add("ye", b.ye[rows], want, bound + U16 * want.abs() + TINY16, 2, U16)
    errors.close()
    assert bool((b.ye[b.R:] == 7.0).all())
    if keep:
        assert bool((b.pre[b.R:] == 7.0).all()) and bool((b.hid[b.R:] == 7.0).all())


def check_backward(b, dxe, dW13, dW2):
    d, h = b.d, b.h
    errors = Errors()
    for e, rows in b.experts():
        x, dy = b.xe[rows].double(), b.dye[rows].double()
        n = len(x)
        if n == 0:
            assert not dW13[e].any() and not dW2[e].any()
            continue
        # (from G, U, H as they were kept: what their roundings do to the gradients is not counted again)
        G, U, H = b.pre[rows, :h].double(), b.pre[rows, h:].double(), b.hid[rows].double()
        W2, W13 = b.W2[e].double(), b.W13[e].double()
        dH = dy @ W2.T
        SH = (d + 8) * U32 * (dy.abs() @ W2.abs().T)
        a, s = act64(G, b.act)
        dG, dU = dH * U * s, dH * a
        # the slope's own error: 5e-6; the value's as above
        BG = SH * (U * s).abs() + (dH * U).abs() * 5e-6 + (UB + 4 * U32) * dG.abs()
        BU = SH * a.abs() + dH.abs() * (1e-6 + 5e-5 * a.abs()) + (UB + 4 * U32) * dU.abs()
        dGU, BGU = torch.cat([dG, dU], 1), torch.cat([BG, BU], 1)
        want = dGU @ W13.T
        bound = BGU @ W13.abs().T + (2 * h + 8) * U32 * (dGU.abs() @ W13.abs().T) + UB * want.abs()
        errors.add("dxe", dxe[rows], want, bound, 2, UB)
        want = x.T @ dGU
        bound = x.abs().T @ BGU + (n + 8) * U32 * (x.abs().T @ dGU.abs()) + UB * want.abs()
        errors.add("dW13", dW13[e], want, bound, 2, UB)
        want = H.T @ dy
        bound = (UB + (n + 8) * U32) * (H.abs().T @ dy.abs()) + UB * want.abs()
        errors.add("dW2", dW2[e], want, bound, 2, UB)
    errors.close()
    assert bool((dxe[b.R:] == 7.0).all())


FORWARD = [
    # decode steps: one row, odd sizes, empty experts, both row groups of an item
    dict(R=1, E=1, d=8, h=8), dict(R=3, E=8, d=72, h=40, act="gelu"), dict(R=40, E=16, d=768, h=2048),
    dict(R=70, E=4, d=264, h=136, counts=[0, 33, 17, 20], act="gelu_tanh"), dict(R=5, E=64, d=136, h=24, act="relu"),
    # 128 x 128 tiles; the same with five stages on their way; widths that end inside a tile
    dict(R=700, E=3, d=1000, h=520), dict(R=900, E=64, d=264, h=264, act="gelu"), dict(R=300, E=2, d=2000, h=520),
    dict(R=300, E=1, d=2056, h=264, act="gelu_tanh"), dict(R=3000, E=2, d=1032, h=8, act="identity"),
    # 128 x 256 and 256 x 256 tiles, a depth below four stages, depths that end inside a stage
    dict(R=2000, E=1, d=3136, h=2056), dict(R=8192, E=2, d=64, h=4096, act="gelu"),
    dict(R=9400, E=3, d=1096, h=2600, counts=[9100, 0, 300], act="relu"),
]


@pytest.mark.parametrize("keep", [False, True], ids=["serve", "keep"])
@pytest.mark.parametrize("kw", FORWARD, ids=lambda kw: "-".join(str(v) for v in kw.values()))
def test_forward(kw, keep):
    b = Block(**kw)
    b.forward(keep)
    check_forward(b, keep)


BACKWARD = [
    dict(R=1, E=1, d=8, h=8), dict(R=3, E=8, d=72, h=40, act="gelu"), dict(R=70, E=4, d=264, h=136, counts=[0, 33, 17, 20], act="gelu_tanh"),
    dict(R=700, E=3, d=1000, h=520), dict(R=900, E=64, d=264, h=264, act="relu"), dict(R=300, E=1, d=2056, h=264),
    dict(R=2000, E=4, d=512, h=1000, act="gelu"),              # dxe: five stages on their way
    dict(R=2000, E=4, d=3000, h=1600, act="identity"),         # dxe: 128 x 256; weight gradients on 256 x 256
    dict(R=9400, E=3, d=1096, h=2600, counts=[9100, 0, 300]),  # 256 x 256 throughout
    dict(R=8300, E=3, d=40, h=8200, counts=[8171, 1, 128]),    # dH: one stage, 256 x 256
]


@pytest.mark.parametrize("kw", BACKWARD, ids=lambda kw: "-".join(str(v) for v in kw.values()))
def test_backward(kw):
    b = Block(**kw)
    b.forward(True)
    kept = b.backward()
    check_backward(b, *kept)
    for t in (b.dxe, b.dW13, b.dW2):
        t.fill_(7.0)
    again = b.backward(kept=False)                # the same values computed again: the same bits
    assert all(torch.equal(p, q) for p, q in zip(kept, again))


@pytest.mark.parametrize("kw", [dict(R=1, E=1, d=4, h=4), dict(R=37, E=3, d=52, h=100, act="gelu"), dict(R=512, E=4, d=128, h=256),
                                dict(R=900, E=5, d=420, h=636, counts=[0, 31, 33, 0, 836], act="gelu_tanh"),
                                dict(R=4096, E=2, d=512, h=1028, act="relu"), dict(R=90, E=2, d=132, h=68, act="identity")],
                         ids=lambda kw: "-".join(str(v) for v in kw.values()))
def test_forward_f32(kw):
    b = Block(dtype="f32", **kw)
    moe.moe_gated_ffn(b.s, b.xe, b.offsets, b.W13p, b.W2p, b.ye, None, None, b.ws)
    for e, rows in b.experts():
        x = b.xe[rows].double()
        Wg, Wu, W2 = b.W13[e, :, :b.h].double(), b.W13[e, :, b.h:].double(), b.W2[e].double()
        G, U = x @ Wg, x @ Wu
        a, _ = act64(G, b.act)
        # sums of d products; the activation is good to 16 units of its value's last place
        BH = (b.d + 8) * U32 * (1.14 * U.abs() * (x.abs() @ Wg.abs()) + a.abs() * (x.abs() @ Wu.abs())) + 17 * U32 * (a * U).abs() + 4 * U32 * U.abs()
        bound = BH @ W2.abs() + (b.h + 8) * U32 * ((a * U).abs() @ W2.abs())
        err = (b.ye[rows].double() - (a * U) @ W2).abs()
        assert bool((err <= bound + 1e-30).all())
    assert bool((b.ye[b.R:] == 7.0).all())


def test_gradient_against_differences():
    """d loss along a direction of x, W13 and W2 by central differences of the formulas in 64 bits."""
    b = Block(R=50, E=2, d=48, h=72, counts=[30, 20], seed=5)
    b.forward(True)
    dxe, dW13, dW2 = b.backward()
    g = torch.Generator(device=DEV).manual_seed(1)
    x, W13, W2 = b.xe[:50].double(), b.W13.double(), b.W2.double()

    def loss(x, W13, W2):
        total = 0.0
        for e, rows in b.experts():
            a, _ = act64(x[rows] @ W13[e, :, :b.h], b.act)
            total += float((((a * (x[rows] @ W13[e, :, b.h:])) @ W2[e]) * b.dye[rows].double()).sum())
        return total

    for i, grad in enumerate((dxe[:50], dW13, dW2)):
        leaves = [x, W13, W2]
        v = torch.randn(leaves[i].shape, generator=g, device=DEV, dtype=torch.float64)
        step, sides = 1e-4, []
        for sign in (1, -1):
            moved = list(leaves)
            moved[i] = leaves[i] + sign * step * v
            sides.append(loss(*moved))
        want, terms = (sides[0] - sides[1]) / (2 * step), grad.double() * v
        # each value is within 3 roundings to bf16 in the mean; what they add up to along v in the square
        assert abs(float(terms.sum()) - want) <= 4 * 3 * UB * math.sqrt(float(terms.square().sum())) + 1e-6 * abs(want)


def test_no_rows_at_all():
    b = Block(R=0, E=3, d=128, h=64, counts=[0, 0, 0], spare=5)
    b.forward(True)
    dxe, dW13, dW2 = b.backward()
    assert bool((b.ye == 7.0).all()) and bool((dxe == 7.0).all()) and not dW13.any() and not dW2.any()


def test_packed_weights_hold_what_the_header_says():
    b = Block(R=4, E=2, d=40, h=24, counts=[2, 2])
    p = b.W13p.view(torch.bfloat16).view(2, 64, 40)
    for e in range(2):
        for c in range(24):
            assert torch.equal(p[e, c // 16 * 32 + c % 16], b.W13[e, :, c])
            assert torch.equal(p[e, c // 16 * 32 + 16 + c % 16], b.W13[e, :, 24 + c])
        for c in range(24, 32):
            assert not p[e, c // 16 * 32 + c % 16].any() and not p[e, c // 16 * 32 + 16 + c % 16].any()
    assert torch.equal(b.W2p.view(torch.float16).view(2, 40, 24), b.W2.transpose(1, 2).half())
    m, W1p, W2p = 2 * 24 * 40, torch.empty_like(b.W2p), torch.empty_like(b.W2p)
    moe.moe_pack_weights(b.s, b.W2.view(-1)[:m].view(2, 40, 24).contiguous(), b.W2, W1p, W2p)
    assert torch.equal(W2p, b.W2p)                # (as moe_pack_weights writes it)


def test_large_gates_and_infinities():
    """Gates far below and above where the activation's exponential over- and underflows.  H is fp16: where it passes
    65504 it is infinite, and so is its row of ye; what is infinite stays in its row."""
    b = Block(R=64, E=1, d=64, h=64, scale=200.0)
    b.forward(True)
    G, U = b.pre[:64, :64].double(), b.pre[:64, 64:].double()
    assert float(G.abs().max()) > 500
    H = act64(G, "silu")[0] * U
    over, near = H.abs() > 65504 * (1 + 1e-2), H.abs() > 65504 * (1 - 1e-2)
    hid = b.hid[:64]
    assert bool(over.any()) and bool(torch.isinf(hid[over]).all()) and bool((torch.sign(hid[over]) == torch.sign(H[over])).all())
    assert bool(torch.isfinite(hid[~near]).all())
    rows = ~near.any(1)
    assert bool(rows.any()) and not bool(torch.isfinite(b.ye[:64][over.any(1)]).any())
    small = Block(R=int(rows.sum()), E=1, d=64, h=64)         # the others, by themselves, against the formulas
    small.xe[:small.R] = b.xe[:64][rows]
    for name in ("W13", "W2", "W13p", "W2p"):
        setattr(small, name, getattr(b, name))
    small.forward(True)
    check_forward(small, True)
    assert torch.equal(small.ye[:small.R], b.ye[:64][rows])
    clean, bad = b.ye.clone(), int(torch.nonzero(rows)[0])
    b.xe[bad, 3] = math.inf
    b.forward(True)
    others = torch.arange(67, device=DEV) != bad
    finite = others & torch.isfinite(clean).all(1)
    assert torch.equal(b.ye[finite], clean[finite]) and not torch.isfinite(b.ye[bad]).any()


def test_another_stream_and_a_graph():
    b = Block(R=900, E=4, d=512, h=520, counts=[300, 0, 599, 1])
    b.forward(True)
    ye, pre, hid = b.ye.clone(), b.pre.clone(), b.hid.clone()
    want = b.backward()
    outs = (b.ye, b.pre, b.hid, b.dxe, b.dW13, b.dW2)
    want = (ye, pre, hid) + want

    def same():
        ok = all(torch.equal(p, q) for p, q in zip(outs, want))
        for t in outs[:4]:
            t[:900] = 0.0
        return ok

    st = torch.cuda.Stream()
    for t in outs:
        t[:900] = 0.0
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        b.forward(True)
        b.backward()
    st.synchronize()
    assert same()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        moe.moe_gated_ffn(b.s, b.xe, b.offsets, b.W13p, b.W2p, b.ye, b.pre, b.hid, b.ws)
        moe.moe_gated_ffn_backward(b.s, b.xe, b.offsets, b.W13, b.W2, b.W13p, b.pre, b.hid, b.dye, b.dxe, b.dW13, b.dW2, b.bws)
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert same()
        b.forward(True)                           # the program's own eager work in between
        b.backward()
        torch.cuda.synchronize()
        assert same()


@pytest.mark.parametrize("size", [dict(R=50, d=64, h=72), dict(R=2000, d=128, h=1096), dict(R=4000, d=1024, h=2056)], ids=["few", "128", "256"])
@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh", "relu"])
def test_gates_that_fp16_does_not_hold(act, size):
    """Every other gate lies far below -65504 in every row, and the values of some of these gates past 65504: kept in fp16
    they are infinite.  These gates are closed, so the forward pass is finite, and what they give to any gradient is 0.  One
    row has an open gate past 65504 and a gradient of 0."""
    b = Block(E=1, act=act, **size)
    R, h = b.R, b.h
    assert moe.moe_gated_gemm_kernel(b.s, 2) == "gated_dh_kernel " + ("256x256" if R == 4000 else "128x128")
    b.xe[:R] = b.xe[:R].abs() + 0.5
    b.W13[0, :, :h:2] = -b.W13[0, :, :h:2].abs() * 1e5 - 2e4
    b.W13[0, :, h:2 * h:4] *= 1e6
    b.W13[0, 0, 1] = 6e4                              # gate 1: open, past 65504 in the last row alone
    b.xe[:R, 0], b.xe[R - 1, 0] = 0.0, 4.0
    b.W13[0, :, h + 1] *= 1e-4
    b.dye[R - 1] = 0.0
    moe.moe_pack_gated_weights(b.s, b.W13, b.W2, b.W13p, b.W2p)
    b.forward(True)
    G, U = b.pre[:R, :h], b.pre[:R, h:]
    assert bool((G[:, ::2] == -math.inf).all()) and bool(torch.isinf(U[:, ::4]).any()) and bool(torch.isfinite(b.ye[:R]).all())
    assert float(G[R - 1, 1]) == math.inf and bool(torch.isfinite(G[:R - 1, 1::2]).all())
    kept = b.backward()
    again = b.backward(kept=False)
    assert all(torch.equal(p, q) for p, q in zip(kept, again))
    b.pre[:R] = b.pre[:R].clamp(-65504, 65504)        # (as the formulas take them)
    check_backward(b, *kept)
