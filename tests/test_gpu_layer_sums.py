"""Long sums of the 16-bit products, as a whole instead of element by element.

The tensor cores add 16 products at a time to an fp32 accumulator and cut what does not fit, so that n steps lose at most n 2^-23 of
the largest running sum.  With sums of one sign that is n 2^-23 of the result; with random signs the running sum grows as the square root of
the step and stays below the result's own size on average, so the same bound holds for the norm."""
import math

import pytest
import torch

import paper_2009_09271_b200 as sc
from layer_util import GROUP, UNIT

pytestmark = pytest.mark.gpu

TYPES = (torch.bfloat16, torch.float16)


@pytest.fixture(scope="module")
def ctx():
    c = sc.Context(max_n=1)
    yield c
    assert c.sc_sync_status() == 0
    c.close()


def inputs(dtype, M, N, K, seed, one_sign):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x, w = torch.randn(M, K, generator=g, device="cuda"), torch.randn(N, K, generator=g, device="cuda") / math.sqrt(K)
    return (x.abs().to(dtype), (w.abs() / math.sqrt(K)).to(dtype)) if one_sign else (x.to(dtype), w.to(dtype))


def run(ctx, kind, dtype, x, w, kept=None):
    M, N = x.shape[0], w.shape[0]
    y = torch.empty(M, N, dtype=dtype, device="cuda")
    if kind == "forward":
        q, scales = kept or (None, None)
        ctx.sc_linear(sc.SC_ACT_NONE, x, w, y, q=q, scales=scales)
    else:
        ctx.sc_linear_grad_input(x, w.t().contiguous(), y)
    return y


LONG = [(300, 264, 4096), (130, 72, 16384), (1100, 1032, 16384), (9, 64, 32768), (520, 512, 32768)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", ["forward", "input"])
@pytest.mark.parametrize("M,N,K", LONG)
def test_long_sums_as_a_whole(ctx, kind, dtype, M, N, K):
    """The error's norm is at most that of rounding 64-bit results to the type, plus the accumulator's."""
    x, w = inputs(dtype, M, N, K, M + K, False)
    y = run(ctx, kind, dtype, x, w).double()
    want = x.double() @ w.double().t()
    rounded = (want.to(dtype).double() - want).norm()
    assert float((y - want).norm()) <= float(rounded) + K / 16 * 2.0 ** -23 * float(want.norm())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", ["forward", "input"])
@pytest.mark.parametrize("M,N,K", LONG)
def test_long_sums_of_one_sign(ctx, kind, dtype, M, N, K):
    """Element by element: half a step of the type and n 2^-23 of the sum; the forward product's checkpoint half a step of its own."""
    x, w = inputs(dtype, M, N, K, M + K, True)
    kept = sc.checkpoint_buffers(M, N) if kind == "forward" else None
    y = run(ctx, kind, dtype, x, w, kept).double()
    want = x.double() @ w.double().t()
    lost = K / 16 * 2.0 ** -23 * want
    rel, tiny = UNIT[dtype]
    assert bool(((y - want).abs() <= lost * (1 + rel) + rel * want + tiny).all())
    if kept:
        held = torch.empty(M, N, dtype=dtype, device="cuda")
        ctx.sc_checkpoint_unpack(*kept, held)
        step = torch.exp2(kept[1].double() - 127).repeat_interleave(GROUP, 1)[:, :N]
        assert bool(((held.double() - want).abs() <= lost + 0.5 * step).all())


@pytest.mark.parametrize("kind", ["forward", "input"])
def test_products_repeat_bit_for_bit(ctx, kind):
    for M, N, K in ((250, 1000, 512), (1024, 2048, 4096), (509, 2048, 1000)):
        x, w = inputs(torch.bfloat16, M, N, K, M, False)
        kept, again = sc.checkpoint_buffers(M, N), sc.checkpoint_buffers(M, N)
        first = run(ctx, kind, torch.bfloat16, x, w, kept)
        for _ in range(3):
            assert torch.equal(run(ctx, kind, torch.bfloat16, x, w, again), first)
            assert kind != "forward" or (torch.equal(kept[0], again[0]) and torch.equal(kept[1], again[1]))
