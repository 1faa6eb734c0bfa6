"""The norm, dropout and 8-bit operators with the layer operators and the compressor: the example's gradients, and that it runs."""
import math
import os
import sys

import pytest
import torch

import paper_2009_09271_b200 as sc
from block_util import dropped64

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import train_block  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("act,blocks,width,hidden,p", [("silu", 1, 96, 200, 0.0), ("gelu", 2, 96, 200, 0.25), ("gelu_tanh", 2, 77, 131, 0.1)])
def test_gradients_of_the_example_against_autograd(act, blocks, width, hidden, p):
    """Whole-network gradients in 64 bits, the rounding to 8 bits left out.  A step of an 8-bit row is 1/127 of its largest value, about three
    deviations: 0.024 deviations, an error of 0.7 % at random in each operand, 1 % in a product, 0.8 % in a checkpoint.  Two blocks
    have four products on the way forward and four operands read back: under 4 % of a gradient's norm together with the 16-bit
    roundings; half as much again is allowed."""
    net = train_block.Network(width, hidden, 40, blocks, act, p, seed=5)
    ctx = sc.Context(max_n=net.n)
    g = torch.Generator(device="cuda").manual_seed(9)
    x = torch.randn(300, width, generator=g, device="cuda").to(torch.bfloat16)
    target = torch.randn(300, 40, generator=g, device="cuda")
    for i, t in enumerate(net.views(net.params)):
        if t.dim() == 1:
            t.add_(torch.randn(t.shape, generator=g, device="cuda") * 0.1)
    prepared = net.prepare(ctx)
    row = torch.full((net.n,), float("nan"), device="cuda")
    loss = net.forward_backward(ctx, prepared, x, target, 12345, row)
    w = [t.double().requires_grad_() for t in prepared[0]]
    fns = {"silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu, "gelu_tanh": lambda z: torch.nn.functional.gelu(z, approximate="tanh")}

    def norm(h, gamma):
        return h * (h.square().mean(1, keepdim=True) + train_block.EPS).rsqrt() * gamma

    h = x.double()
    for b in range(blocks):
        gamma, w1, b1, w2, b2 = w[5 * b:5 * b + 5]
        out = fns[act](norm(h, gamma) @ w1.t() + b1) @ w2.t() + b2
        mask = dropped64(torch.ones(300, width, device="cuda"), 12345 + b + 1, p) if p else 1.0
        h = h + out * mask
    want = (norm(h, w[-2]) @ w[-1].t() - target.double()).square().mean()
    want.backward()
    assert abs(float(loss) - float(want.detach())) <= 0.02 * float(want.detach())
    for got, ref in zip(net.views(row), w):
        assert float((got.double() - ref.grad).norm() / ref.grad.norm()) <= 0.06
    assert ctx.sc_sync_status() == 0
    ctx.close()


@pytest.mark.parametrize("blocks,dropout", [(1, 0.0), (3, 0.2)])
def test_example_runs(blocks, dropout):
    losses = train_block.train(steps=4, blocks=blocks, workers=2, tokens=130, dropout=dropout)
    assert len(losses) == 4 and all(math.isfinite(v) for v in losses)
