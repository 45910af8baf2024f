"""moe_norm_* against the formulas in 64 bits.

A rounding is off by at most half a step, relative: u(t) = finfo(t).eps / 2.  Statistics are sums of d fp32 values in a
tree of at most EPT + 10 roundings a path, so that hats are within 64 u(f32) of their size and results within that plus
one rounding to their type; row-wise gradients subtract two means that are at most as large as the row's largest term, so
they are bounded relative to the row's largest magnitude; vector gradients are sums over T rows in chains of at most
per_run + runs / 16 + 16 additions, bounded relative to the sum of magnitudes."""
import math

import numpy as np
import pytest
import torch

import paper_2210_17223_amd as moe

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def half_step(t):
    return torch.finfo(t).eps / 2


U32 = half_step(torch.float32)


class Case:
    def __init__(self, T, d, kind="rms", dtype="bf16", res="f32", z="f32", gate_tokens=0, bias=None, gate=True,
                 eps=1e-5, scale=0.7, seed=0, z_std=1.0):
        self.n = moe.NormShape.make(T, d, kind=kind, dtype=dtype, res=res, z=z, eps=eps, scale=scale,
                                    gate_tokens=gate_tokens)
        bias = kind == "layer" if bias is None else bias
        g = torch.Generator().manual_seed(seed)
        rnd = lambda *s, std=1.0, mean=0.0, t=torch.float32: (torch.randn(*s, generator=g) * std + mean).to(t).to(DEV)
        self.x = rnd(T, d, std=2.0, mean=0.3, t=TYPES[res])
        self.zz = rnd(T, d, std=z_std, mean=-0.2, t=TYPES[z])
        self.w, self.w_next = rnd(d, std=0.3, mean=1.0), rnd(d, std=0.3, mean=1.0)
        self.b, self.b_next = (rnd(d, std=0.3), rnd(d, std=0.3)) if bias else (None, None)
        self.gate = rnd(self.n.gates, d, std=0.4, mean=0.5) if gate else None
        self.dr = rnd(T, d, std=0.1, t=TYPES[res])
        self.dnext = rnd(T, d, std=0.1, t=TYPES[dtype])
        self.ws = torch.empty(moe.moe_norm_workspace_bytes(self.n), dtype=torch.uint8, device=DEV)
        self.at = torch.arange(T, device=DEV) // (gate_tokens or T)

    def after(self):
        n = self.n
        r = torch.full((n.T, n.d), 7.0, dtype=n.res_torch_dtype, device=DEV)
        nx = torch.full((n.T, n.d), 7.0, dtype=n.torch_dtype, device=DEV)
        moe.moe_norm_after(n, self.x, self.zz, self.w, self.b, self.gate, r, self.w_next, self.b_next, nx)
        return r, nx

    def after_backward(self, r):
        n = self.n
        new = lambda *s, t=torch.float32: torch.full(s, 7.0, dtype=t, device=DEV)
        o = dict(dx=new(n.T, n.d, t=n.res_torch_dtype), dz=new(n.T, n.d, t=n.dz_torch_dtype), dw=new(n.d),
                 dw_next=new(n.d), db=new(n.d) if self.b is not None else None,
                 db_next=new(n.d) if self.b is not None else None,
                 dgate=new(n.gates, n.d) if self.gate is not None else None)
        self.ws.fill_(0xff)                       # (NaN: nothing is read that was not written)
        moe.moe_norm_after_backward(n, self.zz, r, self.w, self.b, self.gate, self.w_next, self.dr, self.dnext, o["dx"],
                                    o["dz"], o["dw"], o["db"], o["dgate"], o["dw_next"], o["db_next"], self.ws)
        return o


def hat64(v, n):
    m = v.mean(1, keepdim=True) if n.kind == 1 else torch.zeros_like(v[:, :1])
    f = 1 / torch.sqrt((v - m).square().mean(1, keepdim=True) + float(np.float32(n.eps)))
    return (v - m) * f, f


def through64(g, hat, f, n):
    return f * (g - (g.mean(1, keepdim=True) if n.kind == 1 else 0.0) - hat * (g * hat).mean(1, keepdim=True))


def check_rows(got, want, size, what):
    """|got - want| against one rounding of the value and 64 fp32 roundings of what it is made of."""
    u = half_step(got.dtype)
    err = (got.double() - want).abs()
    assert torch.isfinite(err).all(), what
    bound = 1.01 * u * want.abs() + 64 * U32 * size + torch.finfo(got.dtype).tiny
    assert bool((err <= bound).all()), (what, float((err / bound).max()))


def check_sums(got, want, magnitude, chain, what):
    err = (got.double() - want).abs()
    bound = (chain + 64) * U32 * magnitude + 1e-30
    assert torch.isfinite(err).all() and bool((err <= bound).all()), (what, float((err / bound).max()))


def forward64(c):
    n, D = c.n, lambda t: None if t is None else t.double()
    zhat, zf = hat64(D(c.zz), n)
    norm = zhat * D(c.w) + (0 if c.b is None else D(c.b))
    gate = torch.ones(1, n.d, dtype=torch.float64, device=DEV) if c.gate is None else D(c.gate)
    s = float(np.float32(n.scale)) * gate[c.at if c.gate is not None else torch.zeros_like(c.at)]
    return zhat, zf, norm, s


def run_after(c):
    n, D = c.n, lambda t: t.double()
    r, nx = c.after()
    zhat, zf, norm, s = forward64(c)
    size_z = s.abs() * (zhat.abs() * D(c.w).abs() + (0 if c.b is None else D(c.b).abs()) + 1)
    check_rows(r, D(c.x) + s * norm, D(c.x).abs() + size_z, "r")
    rhat, rf = hat64(D(r), n)                     # (of r as it is stored)
    size = rhat.abs() * D(c.w_next).abs() + D(r).abs().amax(1, keepdim=True) * rf + (0 if c.b is None else D(c.b_next).abs())
    check_rows(nx, rhat * D(c.w_next) + (0 if c.b is None else D(c.b_next)), size, "next")
    return r


def run_after_backward(c, r):
    n, D = c.n, lambda t: t.double()
    o = c.after_backward(r)
    zhat, zf, norm, s = forward64(c)
    rhat, rf = hat64(D(r), n)
    dn = D(c.dnext)
    u = dn * D(c.w_next)
    dr = D(c.dr) + through64(u, rhat, rf, n)
    big = lambda t: t.abs().amax(1, keepdim=True)
    size = D(c.dr).abs() + rf * big(u) * (1 + rhat.abs())
    check_rows(o["dx"], dr, size, "dx")
    a = s * dr
    v = a * D(c.w)
    size_a = s.abs() * big(size) + big(a)
    check_rows(o["dz"], through64(v, zhat, zf, n), zf * big(size_a * D(c.w).abs()) * (1 + zhat.abs()), "dz")
    chain = n.T
    tot = lambda t: t.sum(0)
    check_sums(o["dw_next"], tot(dn * rhat), tot(dn.abs() * (rhat.abs() + 1)), chain, "dw_next")
    check_sums(o["dw"], tot(a * zhat), tot(size_a * (zhat.abs() + 1)), chain, "dw")
    if c.b is not None:
        check_sums(o["db_next"], tot(dn), tot(dn.abs()), chain, "db_next")
        check_sums(o["db"], tot(a), tot(size_a), chain, "db")
    if c.gate is not None:
        sc = float(np.float32(n.scale))
        groups = torch.zeros(n.gates, n.d, dtype=torch.float64, device=DEV)
        want = groups.clone().index_add_(0, c.at, sc * dr * norm)
        mag = groups.clone().index_add_(0, c.at, abs(sc) * big(size) * (norm.abs() + 1 + (0 if c.b is None else 2 * D(c.b).abs())))
        check_sums(o["dgate"], want, mag, chain, "dgate")
    return o


CASES = [
    dict(T=1, d=8), dict(T=3, d=8, kind="layer", dtype="f32"),
    dict(T=5, d=72, kind="layer", res="bf16", z="f16"), dict(T=37, d=512, res="bf16", z="bf16"),
    dict(T=33, d=520, kind="layer", z="f16"), dict(T=16, d=4096, res="bf16", z="f16"),
    dict(T=9, d=2048, dtype="f32"), dict(T=9, d=2056, kind="layer", res="bf16", z="bf16"),
    dict(T=7, d=4104, kind="layer"), dict(T=5, d=8192, res="bf16", z="f32"), dict(T=3, d=8200, kind="layer", z="bf16"),
    dict(T=2, d=16384, kind="layer", res="bf16", z="bf16"),
    dict(T=3001, d=136, kind="layer", gate_tokens=100), dict(T=3001, d=136, gate_tokens=1, res="bf16", z="f16"),
    dict(T=2500, d=1000, kind="layer", gate_tokens=7, z="bf16"), dict(T=4099, d=520, gate_tokens=1031, bias=True),
    dict(T=700, d=2048, gate_tokens=699), dict(T=700, d=2048, gate_tokens=10 ** 9, kind="layer", bias=False),
    dict(T=600, d=4096, gate=False, kind="layer", res="bf16", z="bf16"), dict(T=5000, d=64, gate_tokens=2500),
]


@pytest.mark.parametrize("kw", CASES, ids=lambda kw: "-".join(str(v) for v in kw.values()))
def test_after_and_its_gradients(kw):
    c = Case(**kw)
    r = run_after(c)
    o = run_after_backward(c, r)
    again = c.after_backward(r)                   # (a fixed order of sums: the same bits)
    assert all(o[k] is None or torch.equal(o[k], again[k]) for k in o)


@pytest.mark.parametrize("kw", CASES[:12] + [dict(T=3001, d=1000, kind="layer"), dict(T=5000, d=64, res="bf16", z="bf16")],
                         ids=lambda kw: "-".join(str(v) for v in kw.values()))
def test_before_and_its_gradients(kw):
    c = Case(**kw)
    n, D = c.n, lambda t: t.double()
    nx = torch.full((n.T, n.d), 7.0, dtype=n.torch_dtype, device=DEV)
    moe.moe_norm_before(n, c.x, c.w_next, c.b_next, nx)
    hat, f = hat64(D(c.x), n)
    bn = 0 if c.b is None else D(c.b_next)
    check_rows(nx, hat * D(c.w_next) + bn, hat.abs() * D(c.w_next).abs() + D(c.x).abs().amax(1, keepdim=True) * f + abs(bn), "next")
    dx = torch.full((n.T, n.d), 7.0, dtype=n.res_torch_dtype, device=DEV)
    dw, db = torch.full((n.d,), 7.0, device=DEV), None if c.b is None else torch.full((n.d,), 7.0, device=DEV)
    c.ws.fill_(0xff)
    moe.moe_norm_before_backward(n, c.x, c.w_next, c.dnext, c.dr, dx, dw, db, c.ws)
    dn = D(c.dnext)
    u = dn * D(c.w_next)
    check_rows(dx, D(c.dr) + through64(u, hat, f, n), D(c.dr).abs() + f * u.abs().amax(1, keepdim=True) * (1 + hat.abs()), "dx")
    check_sums(dw, (dn * hat).sum(0), (dn.abs() * (hat.abs() + 1)).sum(0), n.T, "dw_next")
    if db is not None:
        check_sums(db, dn.sum(0), dn.abs().sum(0), n.T, "db_next")


def test_gradients_against_differences():
    """d loss along a direction of every input, by central differences of the fp32 forward pass in 64 bits."""
    c = Case(T=24, d=40, kind="layer", dtype="f32", gate_tokens=5, seed=3)
    r, _ = c.after()
    o = c.after_backward(r)
    g = torch.Generator().manual_seed(9)
    leaves = {"dx": "x", "dz": "zz", "dw": "w", "db": "b", "dgate": "gate", "dw_next": "w_next", "db_next": "b_next"}

    def loss():
        zhat, _, norm, s = forward64(c)
        r = c.x.double() + s * norm
        nx = hat64(r, c.n)[0] * c.w_next.double() + c.b_next.double()
        return float((r * c.dr.double()).sum() + (nx * c.dnext.double()).sum())

    for grad, name in leaves.items():
        v = getattr(c, name)
        step = torch.randn(v.shape, generator=g).to(DEV).double()
        h, sides = 1e-5, []
        for sign in (1, -1):
            setattr(c, name, v.double() + sign * h * step)
            sides.append(loss())
        setattr(c, name, v)
        want = (sides[0] - sides[1]) / (2 * h)
        got = float((o[grad].double() * step).sum())
        # differences: h^2 of third derivatives of order one; gradients: fp32 sums, r rounded to fp32
        assert abs(got - want) <= 1e-5 * float((o[grad].double() * step).abs().sum()) + 1e-6, (grad, got, want)


def test_residual_in_place_and_another_stream():
    c = Case(T=1500, d=1000, kind="layer", res="bf16", z="f16", gate_tokens=64)
    r, nx = c.after()
    o = c.after_backward(r)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    x, dr, n = c.x.clone(), c.dr.clone(), c.n
    nx2 = torch.empty_like(nx)
    with torch.cuda.stream(st):
        moe.moe_norm_after(n, x, c.zz, c.w, c.b, c.gate, x, c.w_next, c.b_next, nx2)
        dz = torch.empty_like(o["dz"])
        vec = [torch.empty_like(o[k]) for k in ("dw", "db", "dgate", "dw_next", "db_next")]
        moe.moe_norm_after_backward(n, c.zz, x, c.w, c.b, c.gate, c.w_next, dr, c.dnext, dr, dz, *vec, c.ws)
    st.synchronize()
    assert torch.equal(x, r) and torch.equal(nx2, nx) and torch.equal(dr, o["dx"]) and torch.equal(dz, o["dz"])
    assert all(torch.equal(v, o[k]) for v, k in zip(vec, ("dw", "db", "dgate", "dw_next", "db_next")))


def test_infinities_and_nans_stay_in_their_rows():
    c = Case(T=40, d=1000, kind="layer", dtype="f32")
    clean = c.after()[1].clone()
    c.zz[3, 17], c.zz[11, 0] = math.inf, math.nan
    nx = c.after()[1]
    rows = torch.ones(40, dtype=torch.bool, device=DEV)
    rows[[3, 11]] = False
    assert torch.equal(nx[rows], clean[rows]) and not torch.isfinite(nx[~rows]).any()


def test_rows_of_zeros_and_far_means():
    """A row of zeros has norm b; a row whose mean is 300 times its spread keeps its digits (mean first)."""
    c = Case(T=4, d=2048, kind="layer", dtype="f32")
    c.x.zero_()
    c.zz.zero_()
    _, nx = c.after()
    s = float(np.float32(0.7)) * c.gate.double()
    hat, _ = hat64(s * c.b.double(), c.n)
    assert torch.allclose(nx[0].double(), (hat * c.w_next.double() + c.b_next.double())[0], rtol=0, atol=64 * U32 * 40)
    nx2 = torch.empty_like(nx)
    x = torch.randn(4, 2048, device=DEV) + 300.0
    moe.moe_norm_before(c.n, x, c.w_next, c.b_next, nx2)
    hat, f = hat64(x.double(), c.n)
    want = hat * c.w_next.double() + c.b_next.double()
    assert float((nx2.double() - want).abs().max()) <= 4 * U32 * 304 * 2.5 + 64 * U32 * float(want.abs().max())


def test_captured_into_a_graph_replays_the_same_bits():
    c = Case(T=300, d=2048, kind="layer", res="bf16", z="bf16", gate_tokens=50)
    r, nx = c.after()
    o = c.after_backward(r)
    n = c.n
    outs = {k: torch.zeros_like(v) for k, v in o.items()}
    r2, nx2 = torch.zeros_like(r), torch.zeros_like(nx)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        moe.moe_norm_after(n, c.x, c.zz, c.w, c.b, c.gate, r2, c.w_next, c.b_next, nx2)
        moe.moe_norm_after_backward(n, c.zz, r2, c.w, c.b, c.gate, c.w_next, c.dr, c.dnext, outs["dx"], outs["dz"],
                                    outs["dw"], outs["db"], outs["dgate"], outs["dw_next"], outs["db_next"], c.ws)
    for _ in range(4):
        for v in (r2, nx2, *outs.values()):
            v.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(r2, r) and torch.equal(nx2, nx) and all(torch.equal(outs[k], o[k]) for k in o)
        c.after_backward(r)                       # the program's own eager work in between


# next in fp32 beside a residual in bf16: pieces of eight columns of which next has sixteen bytes twice
WIDE_NEXT = [
    dict(T=3, d=8, kind="layer", dtype="f32", res="bf16", z="f16"), dict(T=37, d=512, dtype="f32", res="bf16", z="bf16"),
    dict(T=300, d=1000, kind="layer", dtype="f32", res="bf16", z="f16", gate_tokens=7), dict(T=16, d=4096, dtype="f32", res="bf16", z="bf16"),
    dict(T=9, d=4104, kind="layer", dtype="f32", res="bf16", z="f16"), dict(T=5, d=8200, dtype="f32", res="bf16", z="bf16"),
    dict(T=3, d=16384, kind="layer", dtype="f32", res="bf16", z="f16"), dict(T=9, d=2056, dtype="f32", res="bf16"),
]


@pytest.mark.parametrize("kw", WIDE_NEXT, ids=lambda kw: "-".join(str(v) for v in kw.values()))
def test_next_in_fp32_beside_a_bf16_residual(kw):
    test_after_and_its_gradients(kw)
    test_before_and_its_gradients(kw)
