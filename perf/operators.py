"""The gated block's operators as timed cases, in plain form and through the library.

  gated   the gated feed-forward block on expert-major rows, G = x Wg, U = x Wu, y = (act(G) * U) W2, forward, or
          one training step of it: weights packed, forward that keeps what the backward pass reads, backward pass
  q4      products with weights held as 4-bit codes with group scales (and zero points): the gated block of a serving
          program, or one linear map
  norm    the step between two blocks, r = x + scale * gate * norm(z), next = norm(r); forward, or forward and
          backward; and the norm in front of the first block

`own` false: elementary torch operations in 32 bits, rounded once at the end.  `own` true: the library's calls.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


# ---------------------------------------------------------------------------- the cases
def _gated(name, R, d, h, E, act="silu", dtype="bf16", skew=0.0, train=False):
    return dict(name=name, op="gated", R=R, d=d, h=h, E=E, act=act, dtype=dtype, skew=skew, train=train)


def _q4_ffn(name, R, d, h, E, group, act="silu", zeros=False, skew=0.0):
    return dict(name=name, op="q4_ffn", R=R, d=d, h=h, E=E, group=group, act=act, zeros=zeros, skew=skew)


def _q4_linear(name, R, N, K, E, group, x="bf16", zeros=False, skew=0.0):
    return dict(name=name, op="q4_linear", R=R, N=N, K=K, E=E, group=group, x=x, zeros=zeros, skew=skew)


def _norm(name, T, d, kind="rms", dtype="bf16", res="f32", z="f32", gate_tokens=0, train=False, part="after"):
    return dict(name=name, op="norm", T=T, d=d, kind=kind, dtype=dtype, res=res, z=z, gate_tokens=gate_tokens,
                train=train, part=part)


def listed():
    return [
        # the correctness-sized fp32 layer with gated experts: launches and host time
        _gated("gated_tiny_f32", 512, 128, 256, 4, dtype="f32"),
        # a decode step of 16 sequences, two of 16 small experts each
        _gated("gated_decode", 32, 768, 2048, 16),
        # prefill of the large layer, uneven experts, one of them without rows
        _gated("gated_prefill", 32768, 2048, 8192, 32, skew=0.5),
        # training steps: experts of ordinary size; odd sizes and the GeLU form; a dense block
        _gated("gated_train", 16384, 2048, 5632, 8, train=True),
        _gated("gated_train_ragged", 6002, 1000, 2600, 13, act="gelu", skew=0.5, train=True),
        # serving with 4-bit experts: one token through two of eight, a step of 32 tokens, a prompt
        _q4_ffn("q4_one_token", 2, 4096, 14336, 8, 128),
        _q4_ffn("q4_decode", 64, 4096, 14336, 8, 64, zeros=True),
        _q4_ffn("q4_prompt", 4096, 2048, 8192, 8, 128, act="gelu_tanh"),
        # one linear map of one token
        _q4_linear("q4_vector", 1, 4096, 4096, 1, 32),
        # between two blocks: a decode step; a prompt; a training step with a gate per sequence
        _norm("norm_decode", 16, 4096, res="bf16", z="f16"),
        _norm("norm_prompt", 32768, 2048),
        _norm("norm_train", 16384, 4096, kind="layer", res="bf16", z="bf16", gate_tokens=2048, train=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _mult(v, m):
    return max(m, (int(v) + m // 2) // m * m)


def draw(rng):
    op = rng.choice(["gated", "gated", "gated_f32", "gated_train", "gated_train", "q4_ffn", "q4_ffn", "q4_linear",
                     "norm", "norm", "norm_train"])
    act = rng.choice(["silu", "silu", "gelu", "gelu_tanh", "relu"])
    if op == "gated_f32":
        d, E = _mult(_log_int(rng, 64, 1024), 4), rng.randint(1, 16)
        return _gated("", _log_int(rng, 16, 4096), d, _mult(d * rng.uniform(1.5, 3.0), 4), E, act, "f32",
                      rng.choice([0.0, 0.5]))
    if op in ("gated", "gated_train"):
        train = op == "gated_train"
        step = rng.choice([8, 64])
        d = _mult(_log_int(rng, 128, 4096), step)
        h = _mult(d * rng.uniform(1.0, 4.0), step)
        E = rng.choice([1, 4, 8, 13, 16, 32, 64])
        while E * d * h > 32 * 2048 * 8192 * (0.5 if train else 1):
            E = max(1, E // 2)
        most = min(32768, int(5.4e11 * (0.35 if train else 1) / (d * h)))
        return _gated("", _log_int(rng, 64 if train else 1, max(most, 65)), d, h, E, act, skew=rng.choice([0.0, 0.5]),
                      train=train)
    group = rng.choice([32, 64, 128])
    if op == "q4_ffn":
        d = _mult(_log_int(rng, 512, 4096), group)
        h = _mult(d * rng.uniform(1.5, 3.5), group)
        E, R = rng.choice([1, 4, 8, 16]), _log_int(rng, 1, 4096)
        return _q4_ffn("", min(R, int(6.5e10 / (d * h))), d, h, E, group, act, rng.random() < 0.5,
                       rng.choice([0.0, 0.5]))
    if op == "q4_linear":
        K = _mult(_log_int(rng, 256, 8192), group)
        return _q4_linear("", _log_int(rng, 1, 1024), _log_int(rng, 200, 16384), K, rng.choice([1, 1, 4]), group,
                          rng.choice(["bf16", "f16"]), rng.random() < 0.5, rng.choice([0.0, 0.5]))
    d = _mult(_log_int(rng, 64, 8192), 8)
    T = min(_log_int(rng, 1, 65536), 32768 * 2048 // d)
    f32 = rng.random() < 0.2
    return _norm("", T, d, rng.choice(["rms", "rms", "layer"]), "f32" if f32 else "bf16",
                 "f32" if f32 else rng.choice(["f32", "bf16"]), "f32" if f32 else rng.choice(["f32", "f16", "bf16"]),
                 rng.choice([0, 0, _log_int(rng, 1, T)]), op == "norm_train", rng.choice(["after", "after", "before"]))


# ---------------------------------------------------------------------------- what a program has in hand
def _normal(g, *shape, std=1.0, dtype=torch.float32):
    return (torch.randn(*shape, generator=g, device=DEV) * std).to(dtype)


def _offsets(case, seed):
    """Rows per expert: multinomial, popularity by rank ** -skew in an order of the seed's; skewed ones leave one empty."""
    r = np.random.default_rng(seed)
    E = case["E"]
    p = (1.0 + np.arange(E)) ** -case["skew"]
    if case["skew"] and E > 2:
        p[-1] = 0.0
    counts = r.multinomial(case["R"], r.permutation(p / p.sum()))
    return np.concatenate([[0], np.cumsum(counts)]).astype(np.int32), int(counts.max())


def _codes(g, E, N, K, group, zeros):
    return dict(q=torch.randint(0, 256, (E, N, K // 2), generator=g, device=DEV, dtype=torch.uint8),
                s=((0.5 + torch.rand(E, N, K // group, generator=g, device=DEV)) * (0.2 / math.sqrt(K))).half(),
                z=torch.randint(4, 12, (E, N, K // group), generator=g, device=DEV, dtype=torch.uint8) if zeros else None)


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    st = dict(case=case)
    op = case["op"]
    if op == "norm":
        T, d = case["T"], case["d"]
        dt, rt, zt = TYPES[case["dtype"]], TYPES[case["res"]], TYPES[case["z"]]
        G = -(-T // case["gate_tokens"]) if case["gate_tokens"] else 1
        layer = case["kind"] == "layer"
        vec = lambda std, mean=0.0: _normal(g, d, std=std) + mean  # noqa: E731
        st.update(x=_normal(g, T, d, std=2.0, dtype=rt), w_next=vec(0.2, 1.0), b_next=vec(0.2) if layer else None)
        if case["part"] == "after":
            st.update(z=_normal(g, T, d, dtype=zt), w=vec(0.2, 1.0), b=vec(0.2) if layer else None,
                      gate=_normal(g, G, d, std=0.3) + 0.5)
        if case["train"]:
            st.update(dr=_normal(g, T, d, std=0.1, dtype=rt), dnext=_normal(g, T, d, std=0.1, dtype=dt))
    else:
        offs, most = _offsets(case, seed)
        st.update(offsets=torch.from_numpy(offs).to(DEV), most=most)
        R, E = case["R"], case["E"]
        if op == "gated":
            d, h, dt = case["d"], case["h"], TYPES[case["dtype"]]
            st.update(x=_normal(g, R, d, dtype=dt), W13=_normal(g, E, d, 2 * h, std=1 / math.sqrt(d), dtype=dt),
                      W2=_normal(g, E, h, d, std=1 / math.sqrt(h), dtype=dt))
            if case["train"]:
                st["dy"] = _normal(g, R, d, std=0.1, dtype=dt)
        elif op == "q4_ffn":
            d, h = case["d"], case["h"]
            st.update(x=_normal(g, R, d, dtype=torch.bfloat16), w13=_codes(g, E, 2 * h, d, case["group"], case["zeros"]),
                      w2=_codes(g, E, d, h, case["group"], case["zeros"]))
        else:
            st.update(x=_normal(g, R, case["K"], dtype=TYPES[case["x"]]),
                      w=_codes(g, E, case["N"], case["K"], case["group"], case["zeros"]))
    if own:
        _hold(st)
    return st


def _hold(st):
    """What a program of the library's keeps besides: shapes, output buffers, workspaces; a serving one its packed weights."""
    import paper_2210_17223_amd as moe
    c = st["case"]
    new = lambda *shape, dtype: torch.empty(*shape, dtype=dtype, device=DEV)  # noqa: E731
    if c["op"] == "norm":
        T, d = c["T"], c["d"]
        n = st["shape"] = moe.NormShape.make(T, d, kind=c["kind"], dtype=c["dtype"], res=c["res"], z=c["z"], eps=EPS,
                                             scale=SCALE, gate_tokens=c["gate_tokens"])
        st.update(r=new(T, d, dtype=n.res_torch_dtype), next=new(T, d, dtype=n.torch_dtype))
        if c["train"]:
            st.update(dx=new(T, d, dtype=n.res_torch_dtype), dz=new(T, d, dtype=n.dz_torch_dtype),
                      **{"d" + k: torch.empty_like(st[k]) for k in ("w", "b", "gate", "w_next", "b_next")
                         if st.get(k) is not None},
                      workspace=new(moe.moe_norm_workspace_bytes(n), dtype=torch.uint8))
        return
    R = c["R"]
    if c["op"] == "q4_linear":
        st["shape"] = moe.Q4Shape.make(R, c["E"], c["N"], c["K"], c["group"], x=c["x"])
        st["y"] = new(R, c["N"], dtype=torch.float32)
        return
    s = st["shape"] = moe.Shape.make(R, c["d"], c["E"], c["h"], 1, R, dtype=c.get("dtype", "bf16"), act=c["act"])
    st["ye"] = new(R, c["d"], dtype=s.ye_dtype)
    if c["op"] == "q4_ffn":
        st["workspace"] = new(moe.moe_gated_q4_workspace_bytes(s), dtype=torch.uint8)
        return
    st.update(workspace=new(moe.moe_gated_workspace_bytes(s), dtype=torch.uint8),
              W13p=new(moe.moe_gated_packed_bytes(s), dtype=torch.uint8),
              W2p=new(moe.moe_packed_weight_bytes(s), dtype=torch.uint8))
    if c["train"]:
        st.update(pre=new(R, 2 * c["h"], dtype=torch.float16), hid=new(R, c["h"], dtype=torch.float16),
                  dxe=new(R, c["d"], dtype=torch.bfloat16), dW13=torch.empty_like(st["W13"]),
                  dW2=torch.empty_like(st["W2"]),
                  bwd_workspace=new(moe.moe_gated_backward_workspace_bytes(s), dtype=torch.uint8))
    else:
        moe.moe_pack_gated_weights(s, st["W13"], st["W2"], st["W13p"], st["W2p"])


# ---------------------------------------------------------------------------- one pass
EPS, SCALE = 1e-5, 0.7


def run(st):
    op = st["case"]["op"]
    if own:
        return _run_own(st)
    return {"gated": _gated_plain, "q4_ffn": _q4_ffn_plain, "q4_linear": _q4_linear_plain, "norm": _norm_plain}[op](st)


def _run_own(st):
    import paper_2210_17223_amd as moe
    c = st["case"]
    if c["op"] == "gated":
        s = st["shape"]
        if not c["train"]:
            moe.moe_gated_ffn(s, st["x"], st["offsets"], st["W13p"], st["W2p"], st["ye"], None, None, st["workspace"])
            return st["ye"]
        # (the weights are new in every step)
        moe.moe_pack_gated_weights(s, st["W13"], st["W2"], st["W13p"], st["W2p"])
        moe.moe_gated_ffn(s, st["x"], st["offsets"], st["W13p"], st["W2p"], st["ye"], st["pre"], st["hid"],
                          st["workspace"])
        moe.moe_gated_ffn_backward(s, st["x"], st["offsets"], st["W13"], st["W2"], st["W13p"], st["pre"], st["hid"],
                                   st["dy"], st["dxe"], st["dW13"], st["dW2"], st["bwd_workspace"])
        return {k: st[k] for k in ("ye", "dxe", "dW13", "dW2")}
    if c["op"] == "q4_ffn":
        a, b = st["w13"], st["w2"]
        moe.moe_gated_ffn_q4(st["shape"], c["group"], st["x"], st["offsets"], a["q"], a["s"], a["z"], b["q"], b["s"],
                             b["z"], st["ye"], st["workspace"])
        return st["ye"]
    if c["op"] == "q4_linear":
        w = st["w"]
        moe.moe_q4_linear(st["shape"], st["x"], st["offsets"], w["q"], w["s"], w["z"], st["y"])
        return st["y"]
    n = st["shape"]
    if c["part"] == "before":
        moe.moe_norm_before(n, st["x"], st["w_next"], st["b_next"], st["next"])
        if not c["train"]:
            return st["next"]
        moe.moe_norm_before_backward(n, st["x"], st["w_next"], st["dnext"], st["dr"], st["dx"], st["dw_next"],
                                     st.get("db_next"), st["workspace"])
        return {k: st[k] for k in ("next", "dx", "dw_next", "db_next") if st.get(k) is not None}
    moe.moe_norm_after(n, st["x"], st["z"], st["w"], st["b"], st["gate"], st["r"], st["w_next"], st["b_next"], st["next"])
    if not c["train"]:
        return {"r": st["r"], "next": st["next"]}
    moe.moe_norm_after_backward(n, st["z"], st["r"], st["w"], st["b"], st["gate"], st["w_next"], st["dr"], st["dnext"],
                                st["dx"], st["dz"], st["dw"], st.get("db"), st["dgate"], st["dw_next"],
                                st.get("db_next"), st["workspace"])
    return {k: st[k] for k in ("r", "next", "dx", "dz", "dw", "db", "dgate", "dw_next", "db_next")
            if st.get(k) is not None}


# ---------------------------------------------------------------------------- plain forms
def _act(v, name):
    if name == "silu":
        return v / (1 + torch.exp(-v))
    if name == "gelu":
        return 0.5 * v * (1 + torch.erf(v * math.sqrt(0.5)))
    if name == "gelu_tanh":
        return 0.5 * v * (1 + torch.tanh(math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3)))
    return torch.where(v > 0, v, torch.zeros_like(v))


def _act_slope(v, name):
    if name == "silu":
        p = 1 / (1 + torch.exp(-v))
        return p * (1 + v * (1 - p))
    if name == "gelu":
        return 0.5 * (1 + torch.erf(v * math.sqrt(0.5))) + v * torch.exp(-0.5 * v * v) / math.sqrt(2 * math.pi)
    if name == "gelu_tanh":
        t = torch.tanh(math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3))
        return 0.5 * (1 + t) + 0.5 * v * (1 - t * t) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * v * v)
    return (v > 0).to(v.dtype)


def _by_expert(st, rows):
    """Expert and place of every row, and rows -> [E, most rows, width] with zeros behind an expert's rows."""
    at = torch.arange(rows, device=DEV, dtype=torch.int32)
    e = torch.searchsorted(st["offsets"][1:], at, right=True)
    place = (at - st["offsets"][e]).long()

    def spread(v):
        out = torch.zeros(st["case"]["E"], st["most"], v.shape[1], device=DEV)
        out[e, place] = v.float()
        return out

    return spread, lambda v: v[e, place]


def _gated_plain(st):
    c = st["case"]
    out = torch.float32 if c["dtype"] == "f32" else torch.float16
    spread, gather = _by_expert(st, c["R"])
    h, x, W13, W2 = c["h"], spread(st["x"]), st["W13"].float(), st["W2"].float()
    GU = torch.bmm(x, W13)
    a = _act(GU[..., :h], c["act"])
    H = a * GU[..., h:]
    ye = gather(torch.bmm(H, W2)).to(out)
    if not c["train"]:
        return ye
    dy = spread(st["dy"])
    dH = torch.bmm(dy, W2.transpose(1, 2))
    dW2 = torch.bmm(H.transpose(1, 2), dy)
    dGU = torch.cat([dH * GU[..., h:] * _act_slope(GU[..., :h], c["act"]), dH * a], 2)
    dx = gather(torch.bmm(dGU, W13.transpose(1, 2)))
    dW13 = torch.bmm(x.transpose(1, 2), dGU)
    b = torch.bfloat16
    return {"ye": ye, "dxe": dx.to(b), "dW13": dW13.to(b), "dW2": dW2.to(b)}


def _weights(w, group):
    """[E, K, N] in 32 bits."""
    q = torch.stack([w["q"] & 15, w["q"] >> 4], 3).flatten(2).float()
    z = 8.0 if w["z"] is None else w["z"].float().repeat_interleave(group, 2)
    return ((q - z) * w["s"].float().repeat_interleave(group, 2)).transpose(1, 2)


def _q4_ffn_plain(st):
    c = st["case"]
    spread, gather = _by_expert(st, c["R"])
    GU = torch.bmm(spread(st["x"]), _weights(st["w13"], c["group"]))
    H = _act(GU[..., :c["h"]], c["act"]) * GU[..., c["h"]:]
    return gather(torch.bmm(H, _weights(st["w2"], c["group"]))).half()


def _q4_linear_plain(st):
    c = st["case"]
    spread, gather = _by_expert(st, c["R"])
    return gather(torch.bmm(spread(st["x"]), _weights(st["w"], c["group"])))


def _hat(v, kind):
    """The row with its mean taken off (layer) and its length divided out, and the factor that did the latter."""
    if kind == "layer":
        v = v - v.mean(1, keepdim=True)
    f = 1 / torch.sqrt((v * v).mean(1, keepdim=True) + EPS)
    return v * f, f


def _hat_gradient(dv, hat, f, kind):
    out = dv - hat * (dv * hat).mean(1, keepdim=True)
    if kind == "layer":
        out = out - dv.mean(1, keepdim=True)
    return out * f


def _norm_plain(st):
    c = st["case"]
    kind, dt, rt = c["kind"], TYPES[c["dtype"]], TYPES[c["res"]]
    x, w2 = st["x"].float(), st["w_next"]
    if c["part"] == "before":
        hat, f = _hat(x, kind)
        out = {"next": (hat * w2 if st["b_next"] is None else hat * w2 + st["b_next"]).to(dt)}
        if not c["train"]:
            return out["next"]
        dn = st["dnext"].float()
        out["dx"] = (st["dr"].float() + _hat_gradient(dn * w2, hat, f, kind)).to(rt)
        out["dw_next"] = (dn * hat).sum(0)
        if kind == "layer":
            out["db_next"] = dn.sum(0)
        return out
    gate = st["gate"]
    T, G = c["T"], gate.shape[0]
    at = torch.arange(T, device=DEV) // (c["gate_tokens"] or T)
    zhat, zf = _hat(st["z"].float(), kind)
    n = zhat * st["w"] if st["b"] is None else zhat * st["w"] + st["b"]
    r = (x + SCALE * gate[at] * n).to(rt)
    rhat, rf = _hat(r.float(), kind)       # (of what the next block's residual is read as)
    nx = rhat * w2 if st["b_next"] is None else rhat * w2 + st["b_next"]
    out = {"r": r, "next": nx.to(dt)}
    if not c["train"]:
        return out
    dn = st["dnext"].float()
    dr = st["dr"].float() + _hat_gradient(dn * w2, rhat, rf, kind)
    da = SCALE * gate[at] * dr
    zt = torch.float32 if c["z"] == "f32" else torch.bfloat16
    out.update(dx=dr.to(rt), dz=_hat_gradient(da * st["w"], zhat, zf, kind).to(zt), dw=(da * zhat).sum(0),
               dgate=torch.zeros_like(gate).index_add_(0, at, SCALE * dr * n), dw_next=(dn * rhat).sum(0))
    if kind == "layer":
        out.update(db=da.sum(0), db_next=dn.sum(0))
    return out


# ---------------------------------------------------------------------------- work and exact values
def work(case):
    c = case
    if c["op"] == "norm":
        n, size = c["T"] * c["d"], {"f32": 4, "bf16": 2, "f16": 2}
        r, z, o = size[c["res"]], size[c["z"]], size[c["dtype"]]
        b = n * (r + o) if c["part"] == "before" else n * (2 * r + z + o)
        f = (8 if c["part"] == "before" else 20) * n
        if c["train"]:
            # (r and z are read again: the loss lies between the two passes)
            b += n * (3 * r + o) if c["part"] == "before" else n * (3 * r + 2 * z + o)
            f *= 3
        return {"bytes": b, "flops": f}
    R, E = c["R"], c["E"]
    used = min(R, E)
    if c["op"] == "gated":
        e, m = (4 if c["dtype"] == "f32" else 2), c["d"] * c["h"]
        b, f = 2 * R * c["d"] * e + 3 * used * m * e, 6 * R * m
        if c["train"]:
            b, f = b + 2 * R * c["d"] * e + 3 * E * m * e, 3 * f
        return {"bytes": b, "flops": f}
    per = 0.5 + 2 / c["group"] + (1 / c["group"] if c["zeros"] else 0)
    if c["op"] == "q4_ffn":
        m = c["d"] * c["h"]
        return {"bytes": 4 * R * c["d"] + 3 * used * m * per, "flops": 6 * R * m}
    return {"bytes": R * (2 * c["K"] + 4 * c["N"]) + used * c["N"] * c["K"] * per, "flops": 2 * R * c["N"] * c["K"]}


def _exact_weights(w, e, group):
    """Expert e's [N, K] in 64 bits, a code at a time of every byte."""
    N, half = w["q"][e].shape
    m = torch.empty(N, 2 * half, dtype=torch.float64, device=DEV)
    m[:, 0::2] = (w["q"][e] % 16).double()
    m[:, 1::2] = torch.div(w["q"][e], 16, rounding_mode="floor").double()
    m = m.view(N, -1, group)
    m -= 8.0 if w["z"] is None else w["z"][e].double()[:, :, None]
    return (m * w["s"][e].double()[:, :, None]).view(N, 2 * half)


def exact(case, seed):
    c, st = case, prepare(case, seed)
    f64 = torch.float64
    if c["op"] == "norm":
        return _norm_exact(c, st)
    offs, R = st["offsets"].tolist(), c["R"]

    def act(v):              # value and slope
        v = v.detach().requires_grad_(True)
        if c["act"] == "silu":
            y = v * torch.sigmoid(v)
        elif c["act"] == "gelu":
            y = v * torch.special.ndtr(v)
        elif c["act"] == "gelu_tanh":
            y = v * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (v + 0.044715 * v * v * v))
        else:
            y = v.clamp(min=0)
        return y.detach(), torch.autograd.grad(y.sum(), v)[0]

    if c["op"] == "q4_linear":
        y = torch.zeros(R, c["N"], dtype=f64, device=DEV)
        for e in range(c["E"]):
            lo, hi = offs[e], offs[e + 1]
            if hi > lo:
                y[lo:hi] = st["x"][lo:hi].double() @ _exact_weights(st["w"], e, c["group"]).T
        return y
    d, h = c["d"], c["h"]
    train = c.get("train", False)
    ye = torch.zeros(R, d, dtype=f64, device=DEV)
    if train:
        dx, dW13, dW2 = torch.zeros_like(ye), torch.zeros(st["W13"].shape, dtype=f64, device=DEV), \
            torch.zeros(st["W2"].shape, dtype=f64, device=DEV)
    for e in range(c["E"]):
        lo, hi = offs[e], offs[e + 1]
        if hi == lo:
            continue
        x = st["x"][lo:hi].double()
        if c["op"] == "gated":
            Wg, Wu, W2 = st["W13"][e, :, :h].double(), st["W13"][e, :, h:].double(), st["W2"][e].double()
        else:
            both = _exact_weights(st["w13"], e, c["group"])
            Wg, Wu, W2 = both[:h].T, both[h:].T, _exact_weights(st["w2"], e, c["group"]).T
        U = x @ Wu
        a, slope = act(x @ Wg)
        ye[lo:hi] = (a * U) @ W2
        if train:
            dy = st["dy"][lo:hi].double()
            dH = dy @ W2.T
            dG, dU = dH * U * slope, dH * a
            dW2[e] = (a * U).T @ dy
            dW13[e, :, :h], dW13[e, :, h:] = x.T @ dG, x.T @ dU
            dx[lo:hi] = dG @ Wg.T + dU @ Wu.T
    return {"ye": ye, "dxe": dx, "dW13": dW13, "dW2": dW2} if train else ye


def _norm_exact(c, st):
    f64, T = torch.float64, c["T"]
    D = lambda k: None if st.get(k) is None else st[k].double().requires_grad_(True)  # noqa: E731

    def norm(v, w, b):
        m = v.mean(1, keepdim=True) if c["kind"] == "layer" else 0.0
        var = (v - m).square().mean(1, keepdim=True)
        y = (v - m) * torch.rsqrt(var + EPS) * w
        return y if b is None else y + b

    leaves = {k: D(k) for k in ("x", "z", "w", "b", "gate", "w_next", "b_next")}
    L = type("L", (), leaves)
    with torch.enable_grad():
        if c["part"] == "before":
            r = L.x
        else:
            per = c["gate_tokens"] or T
            gate = L.gate[torch.div(torch.arange(T, device=DEV), per, rounding_mode="floor")]
            r = L.x + SCALE * gate * norm(L.z, L.w, L.b)
            # as it is stored
            r = r + (r.detach().to(TYPES[c["res"]]).double() - r.detach())
        nx = norm(r, L.w_next, L.b_next)
    out = {"next": nx.detach()} if c["part"] == "before" else {"r": r.detach(), "next": nx.detach()}
    if not c["train"]:
        return out if c["part"] == "after" else out["next"]
    loss = (nx * st["dnext"].double()).sum() + (r * st["dr"].double()).sum()
    want = [k for k in leaves if leaves[k] is not None]
    out.update(zip(("d" + k for k in want), torch.autograd.grad(loss, [leaves[k] for k in want])))
    return out
