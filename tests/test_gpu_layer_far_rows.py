"""Rows so many and so far apart that element offsets pass 2^32, through the tensor tiles, their copies of unaligned rows, their
stores, and the elementwise operators; results are those of the same call on dense rows."""
import pytest
import torch

import paper_2009_09271_b200 as sc

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16
ROWS, FAR = 300, 1 << 24                           # 300 rows of 2^24 elements: offsets up to 5.0e9


@pytest.fixture(scope="module")
def ctx():
    c = sc.Context(max_n=1)
    yield c
    assert c.sc_sync_status() == 0
    c.close()


def normal(seed, rows, cols):
    return torch.randn(rows, cols, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(BF16)


def far_view(store, cols, step, offset=0):
    return store.as_strided((ROWS, cols), (step, 1), offset)


@pytest.fixture(scope="module")
def store():
    """10 GB of bf16, used by one case after another."""
    torch.cuda.empty_cache()
    return torch.zeros(ROWS * (FAR + 8) + 4096, dtype=BF16, device="cuda")


@pytest.mark.parametrize("step,offset", [(FAR + 8, 0), (FAR + 7, 0), (FAR + 2, 4), (FAR + 8, 1)])
def test_far_inputs(ctx, store, step, offset):
    far = far_view(store, 200, step, offset)
    far.copy_(normal(1, ROWS, 200))
    dense = far.clone()
    w, v, x = normal(2, 72, 200), normal(3, 200, 72), normal(4, ROWS, 72)
    y, want = torch.empty(ROWS, 72, dtype=BF16, device="cuda"), torch.empty(ROWS, 72, dtype=BF16, device="cuda")
    for out, a in ((y, far), (want, dense)):
        ctx.sc_linear(sc.SC_ACT_SILU, a, w, out)
    assert torch.equal(y, want) and bool(y.any())
    for out, a in ((y, far), (want, dense)):
        ctx.sc_linear_grad_input(a, v, out)
    assert torch.equal(y, want) and bool(y.any())
    wide, wide2 = torch.empty(72, ROWS, dtype=BF16, device="cuda"), torch.empty(72, ROWS, dtype=BF16, device="cuda")
    for out, a in ((wide, far), (wide2, dense)):                        # as the weights
        ctx.sc_linear(sc.SC_ACT_NONE, w, a, out)
    assert torch.equal(wide, wide2) and bool(wide.any())
    back, back2 = torch.empty(72, 200, dtype=BF16, device="cuda"), torch.empty(72, 200, dtype=BF16, device="cuda")
    for out, a in ((back, far), (back2, dense)):
        ctx.sc_linear_grad_input(wide, a, out)
    assert torch.equal(back, back2) and bool(back.any())
    dw, dw2 = torch.empty(200, 72, device="cuda"), torch.empty(200, 72, device="cuda")
    for out, a in ((dw, far), (dw2, dense)):
        ctx.sc_linear_grad_weight(a, out, x=x)
    assert torch.equal(dw, dw2) and bool(dw.any())
    dv, dv2 = torch.empty(72, 200, device="cuda"), torch.empty(72, 200, device="cuda")
    for out, a in ((dv, far), (dv2, dense)):
        ctx.sc_linear_grad_weight(x, out, x=a)
    assert torch.equal(dv, dv2) and bool(dv.any())
    for out, a in ((y, far[:, :72]), (want, dense[:, :72])):            # residuals
        ctx.sc_linear(sc.SC_ACT_NONE, x, v[:72, :72].contiguous(), out, residual=a)
    assert torch.equal(y, want)
    q, scales, q2, scales2 = *sc.checkpoint_buffers(ROWS, 200), *sc.checkpoint_buffers(ROWS, 200)
    ctx.sc_checkpoint_pack(far, q, scales)
    ctx.sc_checkpoint_pack(dense, q2, scales2)
    assert torch.equal(q, q2) and torch.equal(scales, scales2) and bool(q.any())
    dz, dz2, db, db2 = torch.empty_like(dense), torch.empty_like(dense), torch.empty(200, device="cuda"), torch.empty(200, device="cuda")
    ctx.sc_activation_grad(sc.SC_ACT_SILU, far, q, scales, dz, db)
    ctx.sc_activation_grad(sc.SC_ACT_SILU, dense, q, scales, dz2, db2)
    assert torch.equal(dz, dz2) and torch.equal(db, db2) and bool(dz.any())


@pytest.mark.parametrize("cols,step,offset", [(72, FAR + 8, 0), (72, FAR + 8, 1), (200, FAR + 7, 0), (77, FAR + 2, 2)])
def test_far_outputs(ctx, store, cols, step, offset):
    x, w, dz, v = normal(5, ROWS, 136), normal(6, cols, 136), normal(7, ROWS, 40), normal(8, 40, cols)
    out, want = far_view(store, cols, step, offset), torch.empty(ROWS, cols, dtype=BF16, device="cuda")
    q, scales, q2, scales2 = *sc.checkpoint_buffers(ROWS, cols), *sc.checkpoint_buffers(ROWS, cols)
    out.fill_(7)
    ctx.sc_linear(sc.SC_ACT_GELU, x, w, out, q=q, scales=scales)
    ctx.sc_linear(sc.SC_ACT_GELU, x, w, want, q=q2, scales=scales2)
    assert torch.equal(out, want) and torch.equal(q, q2) and torch.equal(scales, scales2)
    ctx.sc_linear_grad_input(dz, v, out)
    ctx.sc_linear_grad_input(dz, v, want)
    assert torch.equal(out, want)
    ctx.sc_linear_grad_input(dz, v, out, residual=out)                  # in place
    ctx.sc_linear_grad_input(dz, v, want, residual=want)
    assert torch.equal(out, want)
    ctx.sc_checkpoint_unpack(q, scales, out)
    ctx.sc_checkpoint_unpack(q, scales, want)
    assert torch.equal(out, want)
    ctx.sc_activation_grad(sc.SC_ACT_GELU, want, q, scales, out)
    ctx.sc_activation_grad(sc.SC_ACT_GELU, want, q, scales, want)
    assert torch.equal(out, want)


@pytest.mark.parametrize("cols,step,offset", [(72, FAR + 4, 0), (72, FAR + 5, 0), (77, FAR + 8, 3)])
def test_far_weight_gradients(ctx, cols, step, offset):
    torch.cuda.empty_cache()
    row = torch.zeros(ROWS * (FAR + 8) + 64, device="cuda")              # 20 GB
    dw, want = row.as_strided((ROWS, cols), (step, 1), offset), torch.zeros(ROWS, cols, device="cuda")
    for tokens in (7, 70, 5000):
        dz, x = normal(9, tokens, ROWS), normal(10, tokens, cols)
        for accumulate in (False, True):
            ctx.sc_linear_grad_weight(dz, dw, x=x, accumulate=accumulate)
            ctx.sc_linear_grad_weight(dz, want, x=x, accumulate=accumulate)
            assert torch.equal(dw, want) and bool(want.any())
    del row, dw


def test_checkpoints_past_32_bits_in_the_activation_gradient(ctx):
    """4.4e9 elements of dy and q: the last rows against the same rows alone."""
    torch.cuda.empty_cache()
    rows, cols = 2100, (1 << 21) + 32
    dy = torch.ones(rows, cols, dtype=BF16, device="cuda")
    q = torch.zeros(rows, cols, dtype=torch.int8, device="cuda")
    scales = torch.full((rows, cols // 32), 127 - 5, dtype=torch.uint8, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(3)
    q[-3:] = torch.randint(-127, 128, (3, cols), generator=g, device="cuda").to(torch.int8)
    dy[-3:] = torch.randn(3, cols, generator=g, device="cuda").to(BF16)
    last, want = dy[-3:].clone(), torch.empty(3, cols, dtype=BF16, device="cuda")
    ctx.sc_activation_grad(sc.SC_ACT_SILU, last, q[-3:].contiguous(), scales[-3:].contiguous(), want)
    db = torch.empty(cols, device="cuda")
    ctx.sc_activation_grad(sc.SC_ACT_SILU, dy, q, scales, dy, db)
    assert torch.equal(dy[-3:], want)
    assert bool((dy[:-3] == 0.5).all())
    sums = 0.5 * (rows - 3) + want.double().sum(0)                       # want is rounded, the sums are taken before
    assert bool(((db.double() - sums).abs() <= 2.0 ** -8 * want.double().abs().sum(0) + (rows + 2) * 2.0 ** -23 * 0.5 * rows + 1e-3).all())
