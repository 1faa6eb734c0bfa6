"""Residual feed-forward blocks trained by sparsified SGD with error feedback, their products in 8-bit integers.

    python examples/train_block.py [--steps 20] [--blocks 2] [--workers 2] [--tokens 512] [--dropout 0.1]

A block is h <- h + dropout(W2 act(W1 norm(h) + b1) + b2).  The norm that follows a block takes the block's output, drops, adds the residual
and normalises in one call, straight to 8-bit rows, which the next product reads; the weights are rounded to 8-bit rows once a step, from
the fp32 parameters where they lie.  Between its forward and backward pass a worker keeps a block's input h in 16 bits and, in 8 bits, the
inputs of both products and the pre-activation; dropout keeps its seed.  The gradients land in the worker's row of the gradient matrix,
which one sc_step_apply call compresses, averages and subtracts from the parameters.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2009_09271_b200 as sc  # noqa: E402
import workloads as wl  # noqa: E402

BF16 = torch.bfloat16
EPS = 1e-5


def _empty(rows: int, cols: int, dtype=BF16) -> torch.Tensor:
    return torch.empty(rows, cols, dtype=dtype, device="cuda")


class Network:
    """Blocks, a norm and a linear head, with all parameters in one flat fp32 vector, one segment per tensor."""

    def __init__(self, width: int, hidden: int, width_out: int, blocks: int, act: str = "silu", dropout: float = 0.1, seed: int = 0):
        self.blocks, self.dropout, self.act = blocks, dropout, sc.ACTIVATIONS[act]
        self.shapes = [s for _ in range(blocks) for s in ((width,), (hidden, width), (hidden,), (width, hidden), (width,))] + [(width,), (width_out, width)]
        self.sizes = [torch.Size(s).numel() for s in self.shapes]
        self.n = sum(self.sizes)
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.params = torch.zeros(self.n, device="cuda")
        for i, p in enumerate(self.views(self.params)):
            if p.dim() == 2:
                p.copy_(torch.randn(p.shape, generator=g, device="cuda") * p.shape[1] ** -0.5)
            elif i % 5 == 0:                                            # a norm's gamma; the others are biases
                p.fill_(1.0)

    def views(self, flat: torch.Tensor):
        """The tensors inside a flat vector (parameters or a worker's gradient row)."""
        out, at = [], 0
        for shape, size in zip(self.shapes, self.sizes):
            out.append(flat[at:at + size].view(shape))
            at += size
        return out

    def prepare(self, ctx):
        """What a step's workers share: the parameters in 16 bits, and the blocks' matrices as 8-bit rows, from the fp32 vector."""
        tensors = self.views(self.params)
        eight = {}
        for i, p in enumerate(tensors[:-1]):
            if p.dim() == 2:
                eight[i] = sc.quantized_buffers(*p.shape)
                ctx.sc_quantize(p, *eight[i])
        return [p.to(BF16) for p in tensors], eight

    def forward_backward(self, ctx, prepared, x, target, seed: int, grad_row) -> torch.Tensor:
        """Loss of one worker's batch; its gradient is written into grad_row (every element of it)."""
        weights, eight = prepared
        grads = self.views(grad_row)
        tokens, width = x.shape
        p, kept = self.dropout, []
        h, out = x, None
        for b in range(self.blocks):
            gamma, w1, b1, w2, b2 = weights[5 * b:5 * b + 5]
            hidden = w1.shape[0]
            norm8, hidden8 = sc.quantized_buffers(tokens, width), sc.quantized_buffers(tokens, hidden)
            z = sc.checkpoint_buffers(tokens, hidden)
            if out is None:
                ctx.sc_rms_norm(h, gamma, EPS, q=norm8[0], scales=norm8[1])
            else:                                                       # closes the block before
                h = self._close(ctx, out, h, gamma, seed + b, q=norm8[0], scales=norm8[1])
            a, out = _empty(tokens, hidden), _empty(tokens, width)
            ctx.sc_linear_quantized(self.act, *norm8, *eight[5 * b + 1], a, bias=b1, q=z[0], scales=z[1])
            ctx.sc_quantize(a, *hidden8)
            ctx.sc_linear_quantized(sc.SC_ACT_NONE, *hidden8, *eight[5 * b + 3], out, bias=b2)
            kept.append((h, norm8, z, hidden8))
        gamma, head = weights[-2:]
        last, y = _empty(tokens, width), _empty(tokens, head.shape[0])
        h = self._close(ctx, out, h, gamma, seed + self.blocks, y=last)
        ctx.sc_linear(sc.SC_ACT_NONE, last, head, y)
        error = y.float() - target
        dy = (error * (2.0 / error.numel())).to(BF16)

        dnorm, dh, dout = _empty(tokens, width), _empty(tokens, width), _empty(tokens, width)
        ctx.sc_linear_grad_weight(dy, grads[-1], x=last)
        ctx.sc_linear_grad_input(dy, head, dnorm)
        ctx.sc_rms_norm_grad(dnorm, h, gamma, EPS, dh, dgamma=grads[-2], dx=dout, p=p, seed=seed + self.blocks)
        for b in reversed(range(self.blocks)):
            gamma, w1, b1, w2, b2 = weights[5 * b:5 * b + 5]
            dgamma, dw1, db1, dw2, db2 = grads[5 * b:5 * b + 5]
            h, norm8, z, hidden8 = kept.pop()
            hidden = w1.shape[0]
            held, dz = _empty(tokens, hidden), _empty(tokens, hidden)
            ctx.sc_dequantize(*hidden8, held)
            ctx.sc_activation_grad(sc.SC_ACT_NONE, dout, None, None, None, db2)
            ctx.sc_linear_grad_weight(dout, dw2, x=held)
            ctx.sc_linear_grad_input(dout, w2, dz, act=self.act, q=z[0], scales=z[1])
            held = _empty(tokens, width)
            ctx.sc_dequantize(*norm8, held)
            ctx.sc_activation_grad(sc.SC_ACT_NONE, dz, None, None, None, db1)
            ctx.sc_linear_grad_weight(dz, dw1, x=held)
            ctx.sc_linear_grad_input(dz, w1, dnorm)
            # the norm's gradient joins the residual's; the gradient of the block before passes its dropout
            ctx.sc_rms_norm_grad(dnorm, h, gamma, EPS, dh, dgamma=dgamma, residual=dh, dx=dout if b else None, p=p, seed=seed + b)
        return error.square().mean()

    def _close(self, ctx, out, h, gamma, seed, **to):
        """The residual stream after a block, and its norm."""
        after = torch.empty_like(h)
        ctx.sc_rms_norm(out, gamma, EPS, residual=h, h=after, p=self.dropout, seed=seed, **to)
        return after


def train(steps: int = 20, blocks: int = 2, workers: int = 2, tokens: int = 512, width: int = 256, hidden: int = 1000, width_out: int = 64,
          dropout: float = 0.1, act: str = "silu", lr: float = 0.3, density=(1, 10)) -> list:
    """Losses of the steps.  The data is a fixed random linear teacher."""
    net = Network(width, hidden, width_out, blocks, act, dropout, seed=1)
    segs = wl.segment_table(net.sizes, *density)
    K = sum(s.k for s in segs)
    ctx = sc.Context(max_n=net.n, max_W=workers, max_segments=len(segs))
    ctx.sc_layer_reserve(tokens, hidden, width)
    ctx.sc_set_gamma(lr)
    grads, residuals = torch.empty(workers, net.n, device="cuda"), torch.zeros(workers, net.n, device="cuda")
    vals, idx = torch.empty(workers, K, device="cuda"), torch.empty(workers, K, device="cuda", dtype=torch.int32)
    g = torch.Generator(device="cuda").manual_seed(3)
    teacher = torch.randn(width_out, width, generator=g, device="cuda") * width ** -0.5
    losses = []
    for step in range(steps):
        prepared = net.prepare(ctx)
        loss = torch.zeros((), device="cuda")
        for w in range(workers):
            x = torch.randn(tokens, width, generator=g, device="cuda").to(BF16)
            loss += net.forward_backward(ctx, prepared, x, x.float() @ teacher.t(), wl.step_seed(0, step, w), grads[w]) / workers
        ctx.sc_step_apply(sc.SC_TOPK, grads, residuals, segs, [wl.step_seed(0, step)] * workers, vals, idx, net.params)
        losses.append(loss)
    status = ctx.sc_sync_status()
    if status != 0:
        raise RuntimeError(f"device status {status}: {sc.strerror(status)}")
    ctx.close()
    return [float(v) for v in losses]


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--blocks", type=int, default=2)
    ap.add_argument("--workers", type=int, default=2)
    ap.add_argument("--tokens", type=int, default=512)
    ap.add_argument("--dropout", type=float, default=0.1)
    a = ap.parse_args()
    for step, loss in enumerate(train(a.steps, a.blocks, a.workers, a.tokens, dropout=a.dropout)):
        print(f"step {step:4d}  loss {loss:.6f}")


if __name__ == "__main__":
    main()
