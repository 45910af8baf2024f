"""The example's block in 8 bits: its parts' results against the formulas in 64 bits, from the values that the parts were given.

Tolerances.  The experts' sum: codes of the rows are the oracle's but for one in a thousand (fp32's norm against 64 bits at a border of two codes; a
code is a thirty-sixth of a row's root mean square), 9e-4 of it in the mean; so is H off, and has as many other codes as lie that near
to a border: sqrt(1e-3 / 36) = 5e-3, with 2e-3 of its own rounding to fp16: below 1e-2.  The last rows' codes stand for their values within
half a code and fp32's roundings; the logits are exact sums, scaled twice: 2 roundings and the comparison's own."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "gated_block.py")
    spec = importlib.util.spec_from_file_location("gated_block", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def rms_norm(v):
    return v / torch.sqrt(v.square().mean(-1, keepdim=True) + 1e-5)


def held(v):
    most = v.abs().amax(-1, keepdim=True)
    return torch.round(127 * v / most) * (most / 127)


def values(w):
    return w[0].double().cpu() * w[1].double().cpu()[..., None]


@pytest.mark.parametrize("T", [1, 16, 700])
def test_served_logits_in_8_bits(example, T):
    d, h, E, k = 256, 640, 4, 2
    block = example.Serve8Block(T, d, h, E, k, vocab=1001)
    x = example.weight(T, d, std=1.0, seed=5)
    got = block.step(x).clone()
    rows, y, last = block.x.double().cpu(), block.b["y"].view(T, d).double().cpu(), values((block.q, block.q_scale))
    xd = x.double().cpu()
    w13, w2, head = (values(w) for w in (block.w13, block.w2, block.w_head))
    idx, gate = block.b["expert_idx"].view(T, k).cpu(), block.b["gate"].view(T, k).double().cpu()
    xn, want = held(rms_norm(xd)), torch.zeros_like(xd)
    for e in range(E):
        G, U = (xn @ w13[e].T).split(h, 1)
        want += (gate * (idx == e)).sum(1, keepdim=True) * (held((G * torch.sigmoid(G) * U).half().double()) @ w2[e].T)
    assert float((y - want).square().mean().sqrt()) <= 1e-2 * float(want.square().mean().sqrt())
    r = xd + 0.5 * rms_norm(y)
    assert float((rows - r).abs().max()) <= 2.0 ** -18 * (1 + float(r.abs().max()))
    assert bool(((last - rms_norm(rows)).abs() <= (0.5 + 2.0 ** -10) * block.q_scale.double().cpu()[:, None]).all())
    want = last @ head[0].T
    assert bool(((got.double().cpu() - want).abs() <= 2.0 ** -21 * want.abs() + 1e-12).all())
    # as one graph
    block.capture()
    for _ in range(3):
        block.logits.fill_(7.0)
        assert torch.equal(block.step(x), got)
        torch.cuda.synchronize()
        x.mul_(1.0)                               # the program's own work
