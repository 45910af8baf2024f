"""The 8-bit operators of a block of gated experts as timed cases, in plain form and through the library.

  norm        the step between two blocks, r = x + scale * gate * norm(z), next = norm(r), with next also as 8-bit codes and a
              scale for every row; or the norm in front of the first block.  The codes come back as the values they stand for
  norm_linear the same, and the projection that reads its codes
  linear      y = act(x W^T + bias) + r of rows and weights in 8 bits, for one matrix or one of several; `raw`: x comes in 16 bits
  gated       the gated feed-forward block of experts whose weights are held in 8 bits, (act(x Wg) * (x Wu)) W2, on 8-bit rows
  layer       the same behind a router: tokens to their experts, the block, and the weighted sum back

A row in 8 bits is codes of -127 .. 127 and scale = its largest magnitude / 127: code = round(127 value / largest), ties to even.
The block's hidden row act(G) * U is rounded to 16 bits and held so, too.

`own` false: elementary torch operations in 32 bits, rounded where the definition says and once at the end.  `own` true: the
library's calls.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS, SCALE = 1e-5, 0.7


# ---------------------------------------------------------------------------- the cases
def _norm(name, T, d, kind="rms", res="f32", z="f16", gate_tokens=0, part="after", N=0, y="f16"):
    """N: of the projection behind it, 0: none."""
    return dict(name=name, op="norm_linear" if N else "norm", T=T, d=d, kind=kind, res=res, z=z, gate_tokens=gate_tokens,
                part=part, N=N, y=y)


def _linear(name, R, N, K, E=1, act="identity", bias=False, res="", y="bf16", raw="", skew=0.0):
    """res: type of the residual, "": none; raw: type in which x comes, "": in 8 bits."""
    return dict(name=name, op="linear", R=R, N=N, K=K, E=E, act=act, bias=bias, res=res, y=y, raw=raw, skew=skew)


def _gated(name, R, d, h, E, act="silu", skew=0.0):
    return dict(name=name, op="gated", R=R, d=d, h=h, E=E, act=act, skew=skew)


def _layer(name, T, d, h, E, k, act="silu", skew=0.0):
    return dict(name=name, op="layer", R=T * k, T=T, k=k, d=d, h=h, E=E, act=act, skew=skew)


def listed():
    return [
        # between two blocks: a decode step of 16 sequences; a prompt
        _norm("norm_decode", 16, 4096, res="bf16"),
        _norm("norm_prompt", 32768, 2048),
        # a decode step's norm and the projection behind it
        _norm("norm_linear_step", 32, 4096, N=6144),
        # one token through one map; the logits of a step; a prompt through a dense layer with all of the epilogue; several
        # matrices of odd sizes on few, uneven rows that come in 16 bits
        _linear("linear_vector", 1, 4096, 4096, y="f32"),
        _linear("linear_logits", 64, 32000, 4096, y="f32", raw="bf16"),
        _linear("linear_prompt", 16384, 4096, 4096, act="gelu", bias=True, res="bf16"),
        _linear("linear_ragged", 1003, 1999, 1008, E=5, act="silu", bias=True, res="f32", y="f32", raw="f16", skew=0.5),
        # serving: one token through two of eight experts; a step of 32 tokens; a prompt with uneven experts, one of them
        # without rows; odd sizes
        _gated("gated_one_token", 2, 4096, 14336, 8),
        _gated("gated_decode", 64, 4096, 14336, 8),
        _gated("gated_prompt", 32768, 2048, 8192, 32, skew=0.5),
        _gated("gated_ragged", 6002, 1008, 2608, 13, act="gelu", skew=0.5),
        # a small layer behind its router
        _layer("layer", 4096, 768, 2048, 16, 2),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _mult(v, m):
    return max(m, (int(v) + m // 2) // m * m)


def draw(rng):
    op = rng.choice(["norm", "norm", "norm_linear", "linear", "linear", "linear", "gated", "gated", "gated", "layer"])
    act = rng.choice(["silu", "silu", "gelu", "gelu_tanh", "relu"])
    skew = rng.choice([0.0, 0.5])
    if op in ("norm", "norm_linear"):
        d = _mult(_log_int(rng, 64, 8192), 16)
        T = min(_log_int(rng, 1, 65536), 32768 * 2048 // d)
        N = 0 if op == "norm" else min(_log_int(rng, 64, 8192), max(64, int(2.7e11 / (T * d))))
        return _norm("", T, d, rng.choice(["rms", "rms", "layer"]), rng.choice(["f32", "bf16"]),
                     rng.choice(["f32", "f16", "bf16"]), rng.choice([0, 0, _log_int(rng, 1, T)]),
                     rng.choice(["after", "after", "before"]), N, rng.choice(["f16", "bf16"]))
    if op == "linear":
        K = _mult(_log_int(rng, 128, 8192), rng.choice([16, 128]))
        N = _log_int(rng, 100, 16384)
        R = min(_log_int(rng, 1, 32768), max(1, int(2.7e11 / (N * K))))
        return _linear("", R, N, K, rng.choice([1, 1, 4, 16]), rng.choice(["identity", act]), rng.random() < 0.5,
                       rng.choice(["", "", "f32", "bf16", "f16"]), rng.choice(["f32", "bf16", "f16"]),
                       rng.choice(["", "", "f32", "bf16", "f16"]), skew)
    step = rng.choice([16, 128])
    d = _mult(_log_int(rng, 128, 4096), step)
    h = _mult(d * rng.uniform(1.0, 4.0), step)
    E = rng.choice([1, 4, 8, 13, 16, 32, 64]) if op == "gated" else rng.choice([4, 8, 13, 16, 32])
    while E * d * h > 32 * 2048 * 8192:
        E = max(1, E // 2)
    most = max(1, min(32768, int(5.4e11 / (d * h))))
    if op == "gated":
        return _gated("", _log_int(rng, 1, most), d, h, E, act, skew)
    k = min(E, rng.choice([1, 2, 2, 4]))
    return _layer("", _log_int(rng, 1, max(most // k, 2)), d, h, E, k, act, skew)


# ---------------------------------------------------------------------------- what a program has in hand
def _normal(g, *shape, std=1.0, dtype=torch.float32):
    return (torch.randn(*shape, generator=g, device=DEV) * std).to(dtype)


def _codes(g, *shape):
    """Of normally distributed values whose row's largest is a little under four deviations."""
    out = torch.empty(*shape, dtype=torch.int8, device=DEV)
    for part in out.view(-1, shape[-1]).split(1 << 14):        # (a part's normal numbers at a time)
        part.copy_(torch.randn(part.shape, generator=g, device=DEV).mul_(33.0).round_().clamp_(-127, 127))
    return out


def _scales(g, *shape, of=1.0):
    return (0.5 + torch.rand(*shape, generator=g, device=DEV)) * (of / 33.0)


def _weights(g, E, N, K):
    return dict(q=_codes(g, E, N, K), s=_scales(g, E, N, of=1 / math.sqrt(K)))


def _popularity(case, r):
    E = case["E"]
    p = (1.0 + np.arange(E)) ** -case["skew"]
    if case["skew"] and E > 8:
        p[-1] = 0.0
    return r.permutation(p / p.sum())


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    r = np.random.default_rng(seed)
    st = dict(case=case)
    op = case["op"]
    if op in ("norm", "norm_linear"):
        T, d = case["T"], case["d"]
        G = -(-T // case["gate_tokens"]) if case["gate_tokens"] else 1
        layer = case["kind"] == "layer"
        vec = lambda std, mean=0.0: _normal(g, d, std=std) + mean  # noqa: E731
        st.update(x=_normal(g, T, d, std=2.0, dtype=TYPES[case["res"]]), w_next=vec(0.2, 1.0),
                  b_next=vec(0.2) if layer else None)
        if case["part"] == "after":
            st.update(z=_normal(g, T, d, dtype=TYPES[case["z"]]), w=vec(0.2, 1.0), b=vec(0.2) if layer else None,
                      gate=_normal(g, G, d, std=0.3) + 0.5)
        if op == "norm_linear":
            st.update(W=_weights(g, 1, case["N"], d), offsets=torch.tensor([0, T], dtype=torch.int32, device=DEV), most=T)
    elif op == "layer":
        T, E, k = case["T"], case["E"], case["k"]
        # k experts of every token, distinct, by popularity; and their weights, which add up to one
        with np.errstate(divide="ignore"):
            z = np.log(_popularity(case, r))[None] - np.log(-np.log(r.uniform(1e-12, 1, (T, E))))
        idx = np.argsort(-z, axis=1)[:, :k].astype(np.int32)
        gate = r.dirichlet(np.full(k, 2.0), T).astype(np.float32)
        st.update(x=dict(q=_codes(g, T, case["d"]), s=_scales(g, T)), expert_idx=torch.from_numpy(idx.reshape(-1)).to(DEV),
                  gate=torch.from_numpy(gate.reshape(-1)).to(DEV), most=int(np.bincount(idx.reshape(-1), minlength=E).max()))
    else:
        counts = r.multinomial(case["R"], _popularity(case, r))
        st.update(offsets=torch.from_numpy(np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)).to(DEV),
                  most=int(counts.max()))
        R = case["R"]
        if op == "linear":
            K, N = case["K"], case["N"]
            st["x"] = _normal(g, R, K, dtype=TYPES[case["raw"]]) if case["raw"] else dict(q=_codes(g, R, K), s=_scales(g, R))
            st.update(W=_weights(g, case["E"], N, K), bias=_normal(g, case["E"], N, std=0.3) if case["bias"] else None,
                      r=_normal(g, R, N, dtype=TYPES[case["res"]]) if case["res"] else None)
        else:
            st["x"] = dict(q=_codes(g, R, case["d"]), s=_scales(g, R))
    if op in ("gated", "layer"):
        E, d, h = case["E"], case["d"], case["h"]
        st.update(w13=_weights(g, E, 2 * h, d), w2=_weights(g, E, d, h))
    if own:
        _hold(st)
    return st


def _hold(st):
    """What a program of the library's keeps besides: shapes, output buffers, workspaces."""
    import paper_2210_17223_amd as moe
    c = st["case"]
    new = lambda *shape, dtype: torch.empty(*shape, dtype=dtype, device=DEV)  # noqa: E731
    if c["op"] in ("norm", "norm_linear"):
        T, d = c["T"], c["d"]
        n = st["shape"] = moe.NormShape.make(T, d, kind=c["kind"], res=c["res"], z=c["z"], eps=EPS, scale=SCALE,
                                             gate_tokens=c["gate_tokens"])
        st.update(r_out=new(T, d, dtype=n.res_torch_dtype), next=new(T, d, dtype=n.torch_dtype),
                  q=new(T, d, dtype=torch.int8), s=new(T, dtype=torch.float32))
        if c["N"]:
            st.update(linear=moe.Q8Shape.make(T, 1, c["N"], d, y=c["y"]), y=new(T, c["N"], dtype=TYPES[c["y"]]))
        else:
            st["values"] = new(T, d, dtype=torch.bfloat16)
        return
    R = c["R"]
    if c["op"] == "linear":
        st["shape"] = moe.Q8Shape.make(R, c["E"], c["N"], c["K"], act=c["act"], res=c["res"] or "f32", y=c["y"])
        st["y"] = new(R, c["N"], dtype=TYPES[c["y"]])
        if c["raw"]:
            st.update(q=new(R, c["K"], dtype=torch.int8), s=new(R, dtype=torch.float32))
        return
    layer = c["op"] == "layer"
    s = st["shape"] = moe.Shape.make(c["T"] if layer else R, c["d"], c["E"], c["h"], c["k"] if layer else 1,
                                     c["T"] if layer else R, act=c["act"])
    st.update(ye=new(R, c["d"], dtype=torch.float16), workspace=new(moe.moe_gated_q8_workspace_bytes(s), dtype=torch.uint8))
    if layer:
        i32 = torch.int32
        st.update(counts=new(c["E"], dtype=i32), offsets=new(c["E"] + 1, dtype=i32), slot_of=new(R, dtype=i32),
                  src_of=new(R, dtype=i32), plan_workspace=new(moe.moe_workspace_bytes(s, 1), dtype=torch.uint8),
                  y=new(c["T"], c["d"], dtype=torch.float32), y_act=new(c["T"], c["d"], dtype=torch.bfloat16))


# ---------------------------------------------------------------------------- one pass
def run(st):
    op = st["case"]["op"]
    if own:
        return _run_own(st)
    return {"norm": _norm_plain, "norm_linear": _norm_plain, "linear": _linear_plain, "gated": _gated_plain,
            "layer": _layer_plain}[op](st)


def _run_own(st):
    import paper_2210_17223_amd as moe
    c = st["case"]
    op = c["op"]
    if op in ("norm", "norm_linear"):
        n = st["shape"]
        if c["part"] == "before":
            moe.moe_norm_before_q8(n, st["x"], st["w_next"], st["b_next"], st["next"], st["q"], st["s"])
            out = {"next": st["next"]}
        else:
            moe.moe_norm_after_q8(n, st["x"], st["z"], st["w"], st["b"], st["gate"], st["r_out"], st["w_next"], st["b_next"],
                                  st["next"], st["q"], st["s"])
            out = {"r": st["r_out"], "next": st["next"]}
        if c["N"]:
            moe.moe_q8_linear(st["linear"], st["q"], st["s"], st["offsets"], st["W"]["q"], st["W"]["s"], None, None, st["y"])
            return {**out, "scale": st["s"], "y": st["y"]}
        moe.moe_q8_values(st["q"], st["s"], st["values"])
        return {**out, "scale": st["s"], "values": st["values"]}
    if op == "linear":
        if c["raw"]:
            moe.moe_q8_rows(st["x"], st["q"], st["s"])
            q, s = st["q"], st["s"]
        else:
            q, s = st["x"]["q"], st["x"]["s"]
        moe.moe_q8_linear(st["shape"], q, s, st["offsets"], st["W"]["q"], st["W"]["s"], st["bias"], st["r"], st["y"])
        return st["y"]
    s, x, a, b = st["shape"], st["x"], st["w13"], st["w2"]
    if op == "gated":
        moe.moe_gated_ffn_q8(s, x["q"], x["s"], None, st["offsets"], a["q"], a["s"], b["q"], b["s"], st["ye"], st["workspace"])
        return st["ye"]
    # (the first product takes the tokens' rows where they are)
    moe.moe_dispatch_q8(s, x["q"], x["s"], st["expert_idx"], st["counts"], st["offsets"], st["slot_of"], st["src_of"], None,
                        None, st["plan_workspace"])
    moe.moe_gated_ffn_q8(s, x["q"], x["s"], st["src_of"], st["offsets"], a["q"], a["s"], b["q"], b["s"], st["ye"],
                         st["workspace"])
    moe.moe_combine(s, st["ye"], st["slot_of"], st["gate"], st["y"], st["y_act"])
    return st["y_act"]


# ---------------------------------------------------------------------------- plain forms
def _act(v, name):
    if name == "identity":
        return v
    if name == "silu":
        return v / (1 + torch.exp(-v))
    if name == "gelu":
        return 0.5 * v * (1 + torch.erf(v * math.sqrt(0.5)))
    if name == "gelu_tanh":
        return 0.5 * v * (1 + torch.tanh(math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3)))
    return torch.where(v > 0, v, torch.zeros_like(v))


def _in_8_bits(v):
    """Codes (as 32-bit numbers) and scales of v's rows.  (In 64 bits: 16-bit values lie on the border of two codes often.)"""
    most = v.abs().amax(-1, keepdim=True)
    code = torch.where(most > 0, torch.round(v.double() * 127 / most), 0.0)
    return code.float(), most / 127


def _by_expert(offsets, E, most, rows):
    """Expert of every row, and rows -> [E, most rows, width] with zeros behind an expert's rows, and back."""
    at = torch.arange(rows, device=DEV, dtype=offsets.dtype)
    e = torch.searchsorted(offsets[1:], at, right=True)
    place = (at - offsets[e]).long()

    def spread(v):
        out = torch.zeros(E, most, v.shape[1], device=DEV)
        out[e, place] = v.float()
        return out

    return e, spread, lambda v: v[e, place]


def _product(x, sx, W):
    """Of rows by expert [E, rows, K] with their scales [E, rows, 1]."""
    return torch.bmm(x, W["q"].float().transpose(1, 2)) * sx * W["s"][:, None, :]


def _hat(v, kind):
    if kind == "layer":
        v = v - v.mean(1, keepdim=True)
    return v / torch.sqrt((v * v).mean(1, keepdim=True) + EPS)


def _norm_plain(st):
    c = st["case"]
    r = st["x"].float()
    out = {}
    if c["part"] == "after":
        at = torch.arange(c["T"], device=DEV) // (c["gate_tokens"] or c["T"])
        n = _hat(st["z"].float(), c["kind"]) * st["w"]
        n = n if st["b"] is None else n + st["b"]
        out["r"] = (r + SCALE * st["gate"][at] * n).to(TYPES[c["res"]])
        r = out["r"].float()                   # (of what the next block's residual is read as)
    nx = _hat(r, c["kind"]) * st["w_next"]
    nx = nx if st["b_next"] is None else nx + st["b_next"]
    code, scale = _in_8_bits(nx)
    out.update(next=nx.bfloat16(), scale=scale[:, 0])
    if c["N"]:
        out["y"] = _product(code[None], scale[None], st["W"])[0].to(TYPES[c["y"]])
    else:
        out["values"] = (code * scale).bfloat16()
    return out


def _linear_plain(st):
    c = st["case"]
    e, spread, gather = _by_expert(st["offsets"], c["E"], st["most"], c["R"])
    code, scale = _in_8_bits(st["x"].float()) if c["raw"] else (st["x"]["q"].float(), st["x"]["s"][:, None])
    v = gather(_product(spread(code), spread(scale), st["W"]))
    v = _act(v if st["bias"] is None else v + st["bias"][e], c["act"])
    return (v if st["r"] is None else v + st["r"].float()).to(TYPES[c["y"]])


def _block(st, x, sx):
    c = st["case"]
    GU = _product(x, sx, st["w13"])
    H = (_act(GU[..., :c["h"]], c["act"]) * GU[..., c["h"]:]).half().float()
    return _product(*_in_8_bits(H), st["w2"])


def _gated_plain(st):
    c = st["case"]
    _, spread, gather = _by_expert(st["offsets"], c["E"], st["most"], c["R"])
    return gather(_block(st, spread(st["x"]["q"]), spread(st["x"]["s"][:, None]))).half()


def _layer_plain(st):
    c = st["case"]
    # the assignments by expert, those of an expert in their order
    order = torch.sort(st["expert_idx"], stable=True)[1]
    offsets = torch.zeros(c["E"] + 1, dtype=torch.int64, device=DEV)
    offsets[1:] = torch.cumsum(torch.bincount(st["expert_idx"], minlength=c["E"]), 0)
    _, spread, gather = _by_expert(offsets, c["E"], st["most"], c["R"])
    token = order // c["k"]
    ye = gather(_block(st, spread(st["x"]["q"][token]), spread(st["x"]["s"][token][:, None])))
    back = torch.empty_like(ye)
    back[order] = ye * st["gate"][order][:, None]
    return back.view(c["T"], c["k"], c["d"]).sum(1).bfloat16()


# ---------------------------------------------------------------------------- work and exact values
def work(case):
    c, size = case, {"": 0, "f32": 4, "bf16": 2, "f16": 2}
    if c["op"] in ("norm", "norm_linear"):
        n, r = c["T"] * c["d"], size[c["res"]]
        b = n * (r + 2 + 1) if c["part"] == "before" else n * (2 * r + size[c["z"]] + 2 + 1)
        f = (10 if c["part"] == "before" else 22) * n
        if c["N"]:
            b, f = b + n + c["d"] * c["N"] + c["T"] * c["N"] * size[c["y"]], f + 2 * n * c["N"]
        return {"bytes": b, "flops": f}
    R, E = c["R"], c["E"]
    used = min(R, E)
    if c["op"] == "linear":
        return {"bytes": R * c["K"] * (size[c["raw"]] or 1) + used * c["N"] * c["K"] + R * c["N"] * (size[c["res"]] + size[c["y"]]),
                "flops": 2 * R * c["N"] * c["K"]}
    m = c["d"] * c["h"]
    rows = c["T"] * c["d"] * 3 if c["op"] == "layer" else R * c["d"] * 3
    return {"bytes": rows + 3 * used * m, "flops": 6 * R * m}


def _exact_act(v, name):
    if name == "silu":
        return v * torch.sigmoid(v)
    if name == "gelu":
        return v * torch.special.ndtr(v)
    if name == "gelu_tanh":
        return v * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (v + 0.044715 * v * v * v))
    return v.clamp(min=0) if name == "relu" else v


def _exact_rows(v):
    """What v's rows (64 bits) are in 8 bits."""
    most = v.abs().max(-1, keepdim=True).values
    return torch.where(most > 0, torch.round(127 * v / most), torch.zeros_like(v)) * most / 127


def _exact_matrix(W, e):
    return W["q"][e].double() * W["s"][e].double()[:, None]


def exact(case, seed):
    c, st = case, prepare(case, seed)
    f64 = torch.float64
    if c["op"] in ("norm", "norm_linear"):
        return _norm_exact(c, st)
    if c["op"] == "layer":
        idx = st["expert_idx"].view(c["T"], c["k"])
        gate = st["gate"].double().view(c["T"], c["k"])
        x = st["x"]["q"].double() * st["x"]["s"].double()[:, None]
        y = torch.zeros(c["T"], c["d"], dtype=f64, device=DEV)
        for e in range(c["E"]):
            t, j = torch.nonzero(idx == e, as_tuple=True)
            if len(t):
                y.index_add_(0, t, _exact_block(c, st, e, x[t]) * gate[t, j][:, None])
        return y
    offs, R = st["offsets"].tolist(), c["R"]
    y = torch.zeros(R, c["N"] if c["op"] == "linear" else c["d"], dtype=f64, device=DEV)
    for e in range(c["E"]):
        lo, hi = offs[e], offs[e + 1]
        if hi == lo:
            continue
        if c["op"] == "linear" and c["raw"]:
            x = _exact_rows(st["x"][lo:hi].double())
        else:
            x = st["x"]["q"][lo:hi].double() * st["x"]["s"][lo:hi].double()[:, None]
        if c["op"] == "gated":
            y[lo:hi] = _exact_block(c, st, e, x)
            continue
        v = x @ _exact_matrix(st["W"], e).T
        if st["bias"] is not None:
            v = v + st["bias"][e].double()
        y[lo:hi] = _exact_act(v, c["act"])
        if st["r"] is not None:
            y[lo:hi] += st["r"][lo:hi].double()
    return y


def _exact_block(c, st, e, x):
    both = x @ _exact_matrix(st["w13"], e).T
    H = _exact_act(both[:, :c["h"]], c["act"]) * both[:, c["h"]:]
    return _exact_rows(H.half().double()) @ _exact_matrix(st["w2"], e).T


def _norm_exact(c, st):
    def norm(v, w, b):
        m = v.mean(1, keepdim=True) if c["kind"] == "layer" else 0.0
        y = (v - m) * torch.rsqrt((v - m).square().mean(1, keepdim=True) + EPS) * w.double()
        return y if b is None else y + b.double()

    out, r = {}, st["x"].double()
    if c["part"] == "after":
        per = c["gate_tokens"] or c["T"]
        gate = st["gate"].double()[torch.div(torch.arange(c["T"], device=DEV), per, rounding_mode="floor")]
        out["r"] = r + SCALE * gate * norm(st["z"].double(), st["w"], st["b"])
        r = out["r"].to(TYPES[c["res"]]).double()      # as it is stored
    nx = norm(r, st["w_next"], st["b_next"])
    held = _exact_rows(nx)
    out.update(next=nx, scale=nx.abs().max(1).values / 127)
    if c["N"]:
        out["y"] = held @ _exact_matrix(st["W"], 0).T
    else:
        out["values"] = held
    return out
