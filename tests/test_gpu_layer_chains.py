"""Layer calls back to back, each reading what the one before it has just written: a kernel that begins while its predecessor ends
must not read before the predecessor's results are there.  Every round writes other data to the same buffers, so that anything
read too early is the round before's; the same calls with a wait after each are the reference."""
import pytest
import torch

import paper_2009_09271_b200 as sc

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16
ROUNDS = 24


@pytest.fixture(scope="module")
def ctx():
    c = sc.Context(max_n=1)
    c.sc_layer_reserve(3000, 1040, 1040)
    yield c
    assert c.sc_sync_status() == 0
    c.close()


def compare(step, rounds, outs):
    """step(i) makes the calls of round i and returns nothing; outs[i] are what it leaves for good."""
    for i in range(rounds):
        step(i, torch.cuda.synchronize)
    want = [[t.clone() for t in o] for o in outs]
    for o in outs:
        for t in o:
            t.zero_()
    torch.cuda.synchronize()
    for _ in range(3):
        for i in range(rounds):
            step(i, lambda: None)
    torch.cuda.synchronize()
    for got, ref in zip(outs, want):
        for a, b in zip(got, ref):
            assert torch.equal(a, b)


def pool(seed, *shape):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.randn(*shape, generator=g, device="cuda").to(BF16) for _ in range(ROUNDS)]


@pytest.mark.parametrize("M,N,K", [(1, 1000, 264), (3, 520, 264), (8, 256, 1032), (200, 264, 136), (2100, 1032, 520), (1500, 256, 1024), (7, 333, 77)])
def test_linear_then_unpack_then_gradients(ctx, M, N, K):
    xs, w, dys = pool(M, M, K), pool(N, N, K)[0], pool(K, M, N)
    q, scales = sc.checkpoint_buffers(M, N)
    y, dz = torch.empty(M, N, dtype=BF16, device="cuda"), torch.empty(M, N, dtype=BF16, device="cuda")
    qx, sx = sc.checkpoint_buffers(M, K)
    outs = [(torch.empty(M, N, dtype=BF16, device="cuda"), torch.empty(M, K, dtype=BF16, device="cuda"), torch.empty(N, K, device="cuda"),
             torch.empty(N, device="cuda"), torch.empty(N, K, device="cuda")) for _ in range(ROUNDS)]

    def step(i, wait):
        held, dx, dw, db, dense = outs[i]
        for call in (lambda: ctx.sc_checkpoint_pack(xs[i], qx, sx),
                     lambda: ctx.sc_linear(sc.SC_ACT_SILU, xs[i], w, y, q=q, scales=scales),
                     lambda: ctx.sc_checkpoint_unpack(q, scales, held),
                     lambda: ctx.sc_activation_grad(sc.SC_ACT_SILU, dys[i], q, scales, dz, db),
                     lambda: ctx.sc_linear_grad_weight(dz, dw, q=qx, scales=sx),
                     lambda: ctx.sc_linear_grad_input(dz, w, dx),
                     lambda: ctx.sc_linear_grad_weight(dz, dense, x=dx)):
            call()
            wait()

    compare(step, ROUNDS, outs)


@pytest.mark.parametrize("M,K", [(1, 264), (5, 1032), (8, 4096), (700, 1000), (63, 77)])
def test_pack_then_weight_gradient_and_unpack(ctx, M, K):
    N = 96
    xs, dzs = pool(M, M, K), pool(K, M, N)
    q, scales = sc.checkpoint_buffers(M, K)
    held = torch.empty(M, K, dtype=BF16, device="cuda")
    outs = [(torch.empty(N, K, device="cuda"), torch.empty(N, K, device="cuda"), torch.empty(M, N, dtype=BF16, device="cuda")) for _ in range(ROUNDS)]
    w = pool(3, N, K)[0]

    def step(i, wait):
        dw, dense, y = outs[i]
        for call in (lambda: ctx.sc_checkpoint_pack(xs[i], q, scales),
                     lambda: ctx.sc_linear_grad_weight(dzs[i], dw, q=q, scales=scales),
                     lambda: ctx.sc_checkpoint_unpack(q, scales, held),
                     lambda: ctx.sc_linear_grad_weight(dzs[i], dense, x=held),
                     lambda: ctx.sc_checkpoint_pack(xs[(i + 1) % ROUNDS], q, scales),
                     lambda: ctx.sc_checkpoint_unpack(q, scales, held),
                     lambda: ctx.sc_linear(sc.SC_ACT_NONE, held, w, y)):
            call()
            wait()

    compare(step, ROUNDS, outs)


def test_in_place_chain(ctx):
    """Results that replace their inputs: residuals in place, the activation's gradient in place, read again at once."""
    M, N, K = 8, 264, 520
    xs, w, dys = pool(1, M, K), pool(2, N, K)[0], pool(3, M, N)
    q, scales = sc.checkpoint_buffers(M, N)
    outs = [(torch.empty(M, N, dtype=BF16, device="cuda"), torch.empty(N, K, device="cuda")) for _ in range(ROUNDS)]
    y, dz = torch.zeros(M, N, dtype=BF16, device="cuda"), torch.empty(M, N, dtype=BF16, device="cuda")

    def step(i, wait):
        held, dw = outs[i]
        for call in (lambda: ctx.sc_linear(sc.SC_ACT_NONE, xs[i], w, y),
                     lambda: ctx.sc_linear(sc.SC_ACT_GELU, xs[i], w, y, residual=y, q=q, scales=scales),
                     lambda: ctx.sc_activation_grad(sc.SC_ACT_GELU, y, q, scales, y),
                     lambda: ctx.sc_linear_grad_weight(y, dw, x=xs[i]),
                     lambda: ctx.sc_activation_grad(sc.SC_ACT_GELU, dys[i], q, scales, dz),
                     lambda: ctx.sc_linear_grad_weight(dz, dw, x=xs[i], accumulate=True),
                     lambda: ctx.sc_checkpoint_unpack(q, scales, held)):
            call()
            wait()

    compare(step, ROUNDS, outs)
