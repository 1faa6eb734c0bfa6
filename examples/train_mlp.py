"""A two-layer network trained by sparsified SGD with error feedback, its activations kept in 8 bits.

    python examples/train_mlp.py [--steps 30] [--workers 4] [--tokens 512] [--act gelu] [--scheme topk]

Each simulated worker runs its own batch forward and backward through the layer operators; the weight and bias gradients
land in its row of the gradient matrix, which one sc_step_apply call compresses (k of n per tensor, the rest goes to the
residual), averages and subtracts from the fp32 parameters.  What a worker keeps between its forward and backward pass is one
byte an element and one byte per 32: the layer inputs x and h, and the pre-activation z.
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


class Mlp:
    """y = W2 act(W1 x + b1) + b2 with its parameters in one flat fp32 vector, one segment per tensor."""

    def __init__(self, width_in: int, width: int, width_out: int, act: str, seed: int = 0):
        self.shapes = [(width, width_in), (width,), (width_out, width), (width_out,)]
        self.sizes = [torch.Size(s).numel() for s in self.shapes]
        self.n = sum(self.sizes)
        self.act = sc.ACTIVATIONS[act]
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.params = torch.zeros(self.n, device="cuda")
        w1, _, w2, _ = self.views(self.params)
        w1.copy_(torch.randn(w1.shape, generator=g, device="cuda") * width_in ** -0.5)
        w2.copy_(torch.randn(w2.shape, generator=g, device="cuda") * width ** -0.5)

    def views(self, flat: torch.Tensor):
        """The four tensors inside a flat vector (parameters or a worker's gradient row)."""
        out, at = [], 0
        for shape, size in zip(self.shapes, self.sizes):
            out.append(flat[at:at + size].view(shape))
            at += size
        return out

    def forward_backward(self, ctx, weights, x, target, grad_row) -> torch.Tensor:
        """Loss of one worker's batch; its gradient is written into grad_row (every element of it)."""
        w1, b1, w2, b2 = weights                                   # bf16
        tokens = x.shape[0]
        new = lambda rows, cols: torch.empty(rows, cols, dtype=BF16, device="cuda")  # noqa: E731
        x_kept, z_kept, h_kept = (sc.checkpoint_buffers(tokens, c) for c in (x.shape[1], w1.shape[0], w1.shape[0]))
        h, y = new(tokens, w1.shape[0]), new(tokens, w2.shape[0])
        ctx.sc_checkpoint_pack(x, *x_kept)
        ctx.sc_linear(self.act, x, w1, h, bias=b1, q=z_kept[0], scales=z_kept[1])
        ctx.sc_checkpoint_pack(h, *h_kept)
        ctx.sc_linear(sc.SC_ACT_NONE, h, w2, y, bias=b2)
        del h                                                       # from here on only the 8-bit copies are needed
        error = y.float() - target
        dy = (error * (2.0 / error.numel())).to(BF16)

        dw1, db1, dw2, db2 = self.views(grad_row)
        dz = new(tokens, w1.shape[0])
        ctx.sc_activation_grad(sc.SC_ACT_NONE, dy, None, None, None, db2)
        ctx.sc_linear_grad_weight(dy, dw2, q=h_kept[0], scales=h_kept[1])
        ctx.sc_linear_grad_input(dy, w2, dz, act=self.act, q=z_kept[0], scales=z_kept[1])
        ctx.sc_activation_grad(sc.SC_ACT_NONE, dz, None, None, None, db1)
        ctx.sc_linear_grad_weight(dz, dw1, q=x_kept[0], scales=x_kept[1])
        return error.square().mean()


def train(steps: int = 30, workers: int = 4, tokens: int = 512, act: str = "gelu", scheme: str = "topk", lr: float = 0.3,
          width_in: int = 256, width: int = 1000, width_out: int = 64, density=(1, 10)) -> list:
    """Losses of the steps.  The data is a fixed random teacher of the same shape."""
    net, teacher = Mlp(width_in, width, width_out, act, seed=1), Mlp(width_in, width, width_out, act, seed=2)
    segs = wl.segment_table(net.sizes, *density)
    K = sum(s.k for s in segs)
    ctx = sc.Context(max_n=net.n, max_W=workers, max_segments=len(segs))
    ctx.sc_layer_reserve(tokens, width, max(width_in, width))
    ctx.sc_set_gamma(lr)
    grads = torch.empty(workers, net.n, device="cuda")
    residuals = torch.zeros(workers, net.n, device="cuda")
    vals = torch.empty(workers, K, device="cuda")
    idx = torch.empty(workers, K, device="cuda", dtype=torch.int32)
    g = torch.Generator(device="cuda").manual_seed(3)
    t1, _, t2, _ = teacher.views(teacher.params)
    losses = []
    for step in range(steps):
        weights = [p.to(BF16) for p in net.views(net.params)]
        loss = torch.zeros((), device="cuda")
        for w in range(workers):
            x = torch.randn(tokens, width_in, generator=g, device="cuda").to(BF16)
            target = torch.nn.functional.gelu(x.float() @ t1.t()) @ t2.t()
            loss += net.forward_backward(ctx, weights, x, target, grads[w]) / workers
        ctx.sc_step_apply(sc.SCHEMES[scheme], grads, residuals, segs, [wl.step_seed(0, step)] * workers, vals, idx, net.params)
        losses.append(loss)
    status = ctx.sc_sync_status()
    if status != 0:
        raise RuntimeError(f"device status {status}: {sc.strerror(status)}")
    ctx.close()
    return [float(v) for v in losses]


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=30)
    ap.add_argument("--workers", type=int, default=4)
    ap.add_argument("--tokens", type=int, default=512)
    ap.add_argument("--act", choices=sorted(sc.ACTIVATIONS), default="gelu")
    ap.add_argument("--scheme", choices=sorted(sc.SCHEMES), default="topk")
    ap.add_argument("--lr", type=float, default=0.3, help="step size; a random block wants about a sixth of top-k's")
    a = ap.parse_args()
    for step, loss in enumerate(train(a.steps, a.workers, a.tokens, a.act, a.scheme, a.lr)):
        print(f"step {step:4d}  loss {loss:.6f}")


if __name__ == "__main__":
    main()
