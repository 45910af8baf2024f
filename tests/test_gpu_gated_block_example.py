"""The example of a block of gated experts: gradients against automatic differentiation in 64 bits, and served logits
against the formulas on the same codes.

Tolerances.  Every tensor that the block stores in bf16 (norm outputs, gradients) is off by at most 2^-8 of a value where it is
rounded to, in fp16 by 2^-11; a rounded sum of independent terms by less in the mean (2^-8 / sqrt(3)).  Between an input and the
logits lie two bf16 roundings in a row and fewer than four of fp16, between a weight's gradient and the loss at most eight
of bf16: relative root-mean-square errors below 2 * 2^-8 and 8 * 2^-8."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HALF_STEP = torch.finfo(torch.bfloat16).eps / 2


@pytest.fixture(scope="module")
def example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "gated_block.py")
    spec = importlib.util.spec_from_file_location("gated_block", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def rms_norm(v, w):
    return w * v / torch.sqrt(v.square().mean(-1, keepdim=True) + 1e-5)


def rel(a, want):
    a, want = a.detach().double().cpu(), want.detach().double().cpu()
    return float(((a - want).square().mean() / want.square().mean()).sqrt())


def test_training_gradients_and_progress(example):
    T, d, h = 300, 256, 712
    block = example.TrainBlock(T, d, h)
    x, target = example.weight(T, d, std=1.0, seed=3), example.weight(T, d, std=1.0, seed=4)
    diff = block.forward(x).float() - target
    block.backward(x, (diff * (2.0 / diff.numel())).bfloat16())

    leaf = {k: v.detach().double().cpu().requires_grad_(True)
            for k, v in dict(x=x, W13=block.W13[0], W2=block.W2[0], w0=block.w0, w1=block.w1, w2=block.w2).items()}
    G, U = (rms_norm(leaf["x"], leaf["w0"]) @ leaf["W13"]).split(h, 1)
    z = (G * torch.sigmoid(G) * U) @ leaf["W2"]
    out = rms_norm(leaf["x"] + 0.5 * rms_norm(z, leaf["w1"]), leaf["w2"])
    assert rel(block.out, out) <= 2 * HALF_STEP
    (out - target.double().cpu()).square().mean().backward()
    for name, got in dict(x=block.dx, W13=block.dW13[0], W2=block.dW2[0], w0=block.dw0, w1=block.dw1, w2=block.dw2).items():
        assert rel(got, leaf[name].grad) <= 8 * HALF_STEP, name

    losses = [float(block.step(x, target, lr=0.2 * (T * d) ** 0.5)) for _ in range(20)]
    assert losses[-1] < 0.9 * losses[0]


@pytest.mark.parametrize("T", [1, 16, 400])
def test_served_logits(example, T):
    d, h, E, k = 256, 640, 4, 2
    block = example.ServeBlock(T, d, h, E, k, vocab=1000)
    x = example.weight(T, d, std=1.0, seed=5)
    got = block.step(x).clone()
    xd = x.double().cpu()
    w13, w2, head = (example.dequantise(*(t.cpu() for t in w)) for w in (block.w13, block.w2, block.w_head))
    xn = rms_norm(xd, 1.0)
    idx, gate = block.b["expert_idx"].view(T, k).cpu(), block.b["gate"].view(T, k).double().cpu()
    # the experts that the gate chose are the largest of its logits, but for ties within its own rounding
    z = xn @ block.Wg.double().cpu()
    assert bool((z.gather(1, idx.long()).amin(1) >= z.topk(k, 1).values[:, -1] - 0.05).all())
    y = torch.zeros_like(xd)
    for e in range(E):
        G, U = (xn @ w13[e].T).split(h, 1)
        y += (gate * (idx == e)).sum(1, keepdim=True) * ((G * torch.sigmoid(G) * U) @ w2[e].T)
    want = rms_norm(xd + 0.5 * rms_norm(y, 1.0), 1.0) @ head[0].T
    assert rel(got, want) <= 2 * HALF_STEP
    # as one graph
    block.capture()
    for _ in range(3):
        block.logits.fill_(7.0)
        assert torch.equal(block.step(x), got)
        torch.cuda.synchronize()
        x.mul_(1.0)                               # the program's own work
