"""Checkpoints of another matrix's shape are refused, although they have as many elements."""
import pytest
import torch

import paper_2009_09271_b200 as sc

pytestmark = pytest.mark.gpu


def test_a_checkpoint_of_the_transposed_shape_is_refused():
    ctx = sc.Context(max_n=1)
    rows, cols = 64, 128
    x = torch.randn(rows, cols, device="cuda").to(torch.bfloat16)
    q, scales = sc.checkpoint_buffers(cols, rows)                   # as many bytes of both
    w, y, dw = (torch.zeros(r, c, dtype=t, device="cuda") for r, c, t in ((cols, 8, x.dtype), (rows, 8, x.dtype), (8, cols, torch.float32)))
    launches = ctx.launch_count
    for call in (lambda: ctx.sc_checkpoint_pack(x, q, scales), lambda: ctx.sc_checkpoint_unpack(q, scales, x),
                 lambda: ctx.sc_activation_grad(sc.SC_ACT_RELU, x, q, scales, x), lambda: ctx.sc_linear(sc.SC_ACT_RELU, y, w, x, q=q, scales=scales),
                 lambda: ctx.sc_linear_grad_input(y, w.t().contiguous(), x, act=sc.SC_ACT_RELU, q=q, scales=scales),
                 lambda: ctx.sc_linear_grad_weight(y, dw, q=q, scales=scales),
                 lambda: ctx.sc_checkpoint_pack(x, q.view(rows, cols), scales)):
        with pytest.raises(ValueError):
            call()
    assert ctx.launch_count == launches
    flat, marks = q.view(-1), scales.view(-1)                       # flat buffers say nothing about a shape
    ctx.sc_checkpoint_pack(x, flat, marks)
    want = sc.checkpoint_buffers(rows, cols)
    ctx.sc_checkpoint_pack(x, *want)
    assert torch.equal(flat.view(rows, cols), want[0]) and torch.equal(marks.view(rows, -1), want[1])
    ctx.close()
