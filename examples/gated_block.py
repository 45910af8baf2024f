"""A residual block of gated experts, as it is trained and as it is served.

    python examples/gated_block.py [--tokens T] [--width D] [--hidden H] [--steps N]

TrainBlock: norm, one gated feed-forward block, gate and residual sum, next norm, and back, with 16-bit weights.
ServeBlock: the same around experts whose weights are 4-bit codes, between the framework's gate, dispatch and combine, and
a 4-bit projection of the result; a whole step is captured into one graph.
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2210_17223_amd as moe


def weight(*shape, std, seed, device="cuda:0"):
    g = torch.Generator(device=device).manual_seed(seed)
    return torch.randn(*shape, generator=g, device=device) * std


class TrainBlock:
    """next = norm(x + scale * norm(ffn(norm(x)))); T tokens of width d, hidden width h."""

    def __init__(self, T, d, h, act="silu", scale=0.5, seed=0, device="cuda:0"):
        def new(*shape, dtype=torch.bfloat16):
            return torch.empty(*shape, dtype=dtype, device=device)
        self.s = s = moe.Shape.make(T, d, 1, h, 1, T, act=act)
        self.n = n = moe.NormShape.make(T, d, z="f16", scale=scale)
        self.offsets = torch.tensor([0, T], dtype=torch.int32, device=device)
        # fp32 masters, and the 16-bit weights that the products read
        self.master = dict(W13=weight(1, d, 2 * h, std=d ** -0.5, seed=seed, device=device),
                           W2=weight(1, h, d, std=h ** -0.5, seed=seed + 1, device=device))
        self.W13, self.W2 = (self.master[k].bfloat16() for k in ("W13", "W2"))
        self.w0, self.w1, self.w2 = (torch.ones(d, device=device) for _ in range(3))
        self.W13p, self.W2p = new(moe.moe_gated_packed_bytes(s), dtype=torch.uint8), new(moe.moe_packed_weight_bytes(s), dtype=torch.uint8)
        self.xn, self.ye, self.r, self.out = new(T, d), new(T, d, dtype=torch.float16), new(T, d, dtype=torch.float32), new(T, d)
        self.pre, self.hid = new(T, 2 * h, dtype=torch.float16), new(T, h, dtype=torch.float16)
        self.dr, self.dx, self.dz, self.dxn = new(T, d, dtype=torch.float32), new(T, d, dtype=torch.float32), new(T, d), new(T, d)
        self.dW13, self.dW2 = torch.empty_like(self.W13), torch.empty_like(self.W2)
        self.dw0, self.dw1, self.dw2 = (torch.empty_like(self.w0) for _ in range(3))
        # (of calls that are given pre and hid)
        self.ws = new(moe.moe_gated_kept_workspace_bytes(s), dtype=torch.uint8)
        self.bwd_ws = new(moe.moe_gated_kept_backward_workspace_bytes(s), dtype=torch.uint8)
        self.norm_ws = new(moe.moe_norm_workspace_bytes(n), dtype=torch.uint8)

    def forward(self, x):
        moe.moe_pack_gated_weights(self.s, self.W13, self.W2, self.W13p, self.W2p)
        moe.moe_norm_before(self.n, x, self.w0, None, self.xn)
        moe.moe_gated_ffn(self.s, self.xn, self.offsets, self.W13p, self.W2p, self.ye, self.pre, self.hid, self.ws)
        moe.moe_norm_after(self.n, x, self.ye, self.w1, None, None, self.r, self.w2, None, self.out)
        return self.out

    def backward(self, x, dout):
        """Gradients of everything for a loss whose gradient with respect to out is dout (bf16) and to r nothing."""
        self.dr.zero_()
        moe.moe_norm_after_backward(self.n, self.ye, self.r, self.w1, None, None, self.w2, self.dr, dout, self.dx, self.dz,
                                    self.dw1, None, None, self.dw2, None, self.norm_ws)
        moe.moe_gated_ffn_backward(self.s, self.xn, self.offsets, self.W13, self.W2, self.W13p, self.pre, self.hid, self.dz,
                                   self.dxn, self.dW13, self.dW2, self.bwd_ws)
        # dx so far is the residual path's
        moe.moe_norm_before_backward(self.n, x, self.w0, self.dxn, self.dx, self.dx, self.dw0, None, self.norm_ws)
        return self.dx

    def step(self, x, target, lr):
        """One step of gradient descent on the mean square distance from target; the loss before it."""
        diff = self.forward(x).float() - target
        self.backward(x, (diff * (2.0 / diff.numel())).bfloat16())
        for w, dw in ((self.w0, self.dw0), (self.w1, self.dw1), (self.w2, self.dw2)):
            w -= lr * dw
        for k, dw in (("W13", self.dW13), ("W2", self.dW2)):
            self.master[k] -= lr * dw.float()
            getattr(self, k).copy_(self.master[k])
        return diff.square().mean()


def quantise(w, group):
    """fp32 [E, N, K] to 4-bit codes with scales and zeros for every `group` of K: (q, scale, zero)."""
    E, N, K = w.shape
    g = w.reshape(E, N, K // group, group)
    low, high = g.amin(-1).clamp(max=0.0), g.amax(-1).clamp(min=0.0)
    scale = ((high - low) / 15).clamp(min=2.0 ** -14).half()
    zero = (-low / scale.float()).round().clamp(0, 15)
    q = (g / scale.float()[..., None] + zero[..., None]).round().clamp(0, 15).to(torch.uint8).reshape(E, N, K)
    return q[..., 0::2] | q[..., 1::2] << 4, scale, zero.to(torch.uint8)


def dequantise(q, scale, zero):
    c = torch.stack([q & 15, q >> 4], -1).flatten(-2).double()
    group = c.shape[-1] // scale.shape[-1]
    return (c - zero.double().repeat_interleave(group, -1)) * scale.double().repeat_interleave(group, -1)


class ServeBlock:
    """out, logits of T tokens: E experts, k of them per token, and `vocab` rows of the projection."""

    def __init__(self, T, d, h, E, k, vocab, group=64, act="silu", scale=0.5, seed=0, device="cuda:0"):
        self.s = s = moe.Shape.make(T, d, E, h, k, T, act=act, renorm_topk=True)
        self.n = moe.NormShape.make(T, d, scale=scale)
        self.group = group
        self.head = moe.Q4Shape.make(T, 1, vocab, d, group)
        self.w13 = quantise(weight(E, 2 * h, d, std=d ** -0.5, seed=seed, device=device), group)
        self.w2 = quantise(weight(E, d, h, std=h ** -0.5, seed=seed + 1, device=device), group)
        self.w_head = quantise(weight(1, vocab, d, std=d ** -0.5, seed=seed + 2, device=device), group)
        self.Wg = weight(d, E, std=d ** -0.5, seed=seed + 3, device=device).bfloat16()
        self.w0, self.w1, self.w_out = (torch.ones(d, device=device) for _ in range(3))
        self.b = moe.alloc_buffers(s, 1, device)
        moe.moe_pack_gate(s, self.Wg, self.b["Wgp"])
        self.ws = torch.empty(moe.moe_gated_q4_workspace_bytes(s), dtype=torch.uint8, device=device)
        self.all_rows = torch.tensor([0, T], dtype=torch.int32, device=device)
        self.x = torch.empty(T, d, device=device)
        self.xn, self.out = (torch.empty(T, d, dtype=torch.bfloat16, device=device) for _ in range(2))
        self.logits = torch.empty(T, vocab, device=device)
        self.graph = None

    def forward(self):
        """From self.x (the residual stream, updated in place) to self.out and self.logits."""
        s, b = self.s, self.b
        moe.moe_norm_before(self.n, self.x, self.w0, None, self.xn)
        moe.moe_route(s, self.xn, b["Wgp"], None, 0, b["expert_idx"], b["gate"])
        moe.moe_dispatch(s, self.xn, b["expert_idx"], b["counts"], b["offsets"], b["slot_of"], b["src_of"], b["xe"], b["workspace"])
        moe.moe_gated_ffn_q4(s, self.group, b["xe"], b["offsets"], *self.w13, *self.w2, b["ye"], self.ws)
        moe.moe_combine(s, b["ye"], b["slot_of"], b["gate"], b["y"])
        moe.moe_norm_after(self.n, self.x, b["y"], self.w1, None, None, self.x, self.w_out, None, self.out)
        moe.moe_q4_linear(self.head, self.out, self.all_rows, *self.w_head, self.logits)

    def capture(self):
        """One graph of forward(); step() replays it from then on."""
        self.x.zero_()
        self.forward()                            # (launches everything once outside)
        torch.cuda.synchronize()
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(self.graph):
            self.forward()

    def step(self, x):
        """Logits for the tokens x [T, d] fp32."""
        self.x.copy_(x)
        self.forward() if self.graph is None else self.graph.replay()
        return self.logits


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("tokens", 2048), ("width", 1024), ("hidden", 2816), ("steps", 50)):
        ap.add_argument("--" + name, type=int, default=value)
    a = ap.parse_args()
    x = weight(a.tokens, a.width, std=1.0, seed=7)
    target = weight(a.tokens, a.width, std=1.0, seed=8)
    block = TrainBlock(a.tokens, a.width, a.hidden)
    for i in range(a.steps):
        loss = block.step(x, target, lr=0.05 * math.sqrt(a.tokens * a.width))
        if i % 10 == 0 or i == a.steps - 1:
            print(f"step {i:4d}  loss {float(loss):.4f}", flush=True)
    serve = ServeBlock(16, a.width, a.hidden // 64 * 64, 8, 2, 32000)
    serve.capture()
    serve.step(x[:16])
    start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    start.record()
    for _ in range(100):
        serve.step(x[:16])
    end.record()
    end.synchronize()
    print(f"decode step of 16 tokens, 8 experts: {start.elapsed_time(end) * 10:.1f} us", flush=True)


if __name__ == "__main__":
    main()
