"""What follows the sums of an 8-bit product, on every path: tiles of each shape, split sums, rows of any alignment, the kernels for few tokens."""
import pytest
import torch

import paper_2009_09271_b200 as sc
from layer_util import assert_close, strided

pytestmark = pytest.mark.gpu

TILES = [(256, 256), (128, 256), (128, 128), (128, 64)]


@pytest.fixture(scope="module")
def ctx():
    c = sc.Context(max_n=1)
    yield c
    c.sc_debug_layer_tiles()
    assert c.sc_sync_status() == 0
    c.close()


def paths(M, K):
    """(tile, parts, further elements between rows, offset) of the calls that reach one form of the epilogue each."""
    yield (0, 0), 0, 0, 0                                               # the library's choice: up to 32 tokens without tiles
    for tile in TILES:
        for parts in (1, 3):
            if tile[0] <= 128 or M > 128:
                yield tile, parts, 0, 0                                 # whole accesses, or the join of the parts
    yield (128, 128), 1, 2, 2                                           # pairs of elements
    yield (128, 64), 1, 3, 1                                            # single elements
    yield (128, 64), 2, 3, 1


@pytest.mark.parametrize("M,N,K", [(1, 40, 64), (2, 136, 272), (7, 64, 400), (30, 72, 400), (150, 264, 400), (300, 512, 400)])
def test_scales_far_from_one(ctx, M, N, K):
    """Rows whose sums times the row's scale, or the columns', leave fp32's range while the result is well within: three products, each off by
    2^-24 of its result, and a bias."""
    g = torch.Generator(device="cuda").manual_seed(M)
    x, w = (torch.randint(-127, 128, (r, K), generator=g, device="cuda").to(torch.int8) for r in (M, N))
    bias = torch.randn(N, generator=g, device="cuda").bfloat16()
    for x_size, w_size in ((2.0 ** 120, 2.0 ** -100), (2.0 ** 66, 2.0 ** -80), (2.0 ** -100, 2.0 ** 120), (2.0 ** 62, 2.0 ** 30)):
        xs, ws = (s * (0.5 + torch.rand(n, generator=g, device="cuda")) for s, n in ((x_size, M), (w_size, N)))
        want = (x.double() @ w.double().t()) * xs.double()[:, None] * ws.double()
        slack = want.abs() * 4 * 2.0 ** -24
        want = want + bias.double()
        for tile, parts, extra, offset in paths(M, K):
            ctx.sc_debug_layer_tiles(*tile, parts)
            y = strided(torch.zeros(M, N, device="cuda", dtype=torch.bfloat16), extra, offset)
            ctx.sc_linear_quantized(sc.SC_ACT_NONE, x, xs, w, ws, y, bias=bias)
            assert_close(y, want, slack + want.abs() * 2.0 ** -24, torch.bfloat16, f"scales {x_size} {w_size}, tiles {tile} x {parts}")
    # the largest scale that sc_quantize makes, beside sums of zero
    xs, ws = torch.full((M,), 2.6793883890187504e+36, device="cuda"), torch.full((N,), 2.6793883890187504e+36, device="cuda")
    for tile, parts, extra, offset in paths(M, K):
        ctx.sc_debug_layer_tiles(*tile, parts)
        y = strided(torch.zeros(M, N, device="cuda", dtype=torch.bfloat16), extra, offset)
        ctx.sc_linear_quantized(sc.SC_ACT_NONE, torch.zeros_like(x), xs, w, ws, y, bias=bias)
        assert torch.equal(y, bias.expand(M, N))
    ctx.sc_debug_layer_tiles()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("act", ["none", "relu", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("M,N,K", [(1, 40, 64), (2, 136, 272), (7, 64, 400), (30, 72, 400), (150, 264, 400), (300, 513, 1024)])
def test_every_path_gives_the_same_bits(ctx, dtype, act, M, N, K):
    """y and the checkpoint of z, zeros' signs among them, with and without bias and residual.  z reaches from where the activations are curved
    to where they have become 0 or z."""
    g = torch.Generator(device="cuda").manual_seed(N)
    x, w = (torch.randint(-127, 128, (r, K), generator=g, device="cuda").to(torch.int8) for r in (M, N))
    x[-1] = 0 if M > 1 else x[-1]
    xs = torch.exp2(torch.randint(-14, -4, (M,), generator=g, device="cuda").float()) * (1 + torch.rand(M, generator=g, device="cuda"))
    ws = torch.rand(N, generator=g, device="cuda") / K ** 0.5
    ws[3] = -ws[3]
    bias = torch.randn(N, generator=g, device="cuda").to(dtype)
    bias[:2] = torch.tensor([0.0, -0.0])
    residual = torch.randn(M, N, generator=g, device="cuda").to(dtype)
    residual[:, 1:4] = torch.tensor([0.0, -0.0, 0.0], device="cuda").to(dtype)
    for b in (None, bias):
        for r in (None, residual):
            want, kept = None, None
            for tile, parts, extra, offset in paths(M, K):
                ctx.sc_debug_layer_tiles(*tile, parts)
                for keep in (False, True):
                    y = strided(torch.zeros(M, N, device="cuda", dtype=dtype), extra, offset)
                    q, scales = sc.checkpoint_buffers(M, N) if keep else (None, None)
                    ctx.sc_linear_quantized(sc.ACTIVATIONS[act], x, xs, w, ws, y, bias=b, residual=None if r is None else strided(r, extra, offset), q=q, scales=scales)
                    y, path = y.contiguous().view(torch.int16), (tile, parts, extra, offset, b is not None, r is not None, keep)
                    want = y if want is None else want
                    differing = int((y != want).sum())
                    assert differing == 0, path
                    if keep:
                        kept = (q, scales) if kept is None else kept
                        assert torch.equal(q, kept[0]) and torch.equal(scales, kept[1]), path
    ctx.sc_debug_layer_tiles()
