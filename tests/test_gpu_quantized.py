"""8-bit rows and the linear layer on them.

Rows are compared bit for bit with their definition in IEEE fp32.  The product's sums are exact integers; three fp32 multiplications
(the conversion, two scales) and the bias follow, each off by at most 2^-24 of its result, then the activation, whose slope and value are
computed to 2^-18 of their size, as in sc_linear."""
import math

import pytest
import torch

import paper_2009_09271_b200 as sc
from block_util import rows_in_8_bits
from layer_util import ACTS, GROUP, act64, assert_close, strided

pytestmark = pytest.mark.gpu

TYPES = (torch.bfloat16, torch.float16)
ACT_ERR, LIPSCHITZ = 2.0 ** -18, 1.13
TILES = [(256, 256), (128, 256), (128, 128), (128, 64)]


@pytest.fixture(scope="module")
def ctx():
    c = sc.Context(max_n=1)
    yield c
    c.sc_debug_layer_tiles()
    assert c.sc_sync_status() == 0
    c.close()


def rng(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


# -- rows ------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", TYPES + (torch.float32,))
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 7), (3, 8), (5, 33), (70, 256), (7, 1000), (2, 1024), (9, 2049), (33, 4096), (3, 8200), (2, 16391), (1, 70001)])
def test_rows_bits(ctx, dtype, rows, cols):
    g = rng(rows * 7919 + cols)
    x = (normal(g, rows, cols) * torch.exp2(torch.randint(-20, 12, (rows, 1), generator=g, device="cuda").float())).to(dtype)
    if rows > 1:
        x[1] = 0
    wq, ws = rows_in_8_bits(x)
    for extra, offset in ((0, 0), (8, 8), (16, 4), (3, 1), (2, 2)):
        xs = strided(x, extra, offset)
        q, scales = strided(torch.zeros(rows, cols, dtype=torch.int8, device="cuda"), extra, offset), torch.empty(rows, device="cuda")
        ctx.sc_quantize(xs, q, scales)
        assert torch.equal(q.cpu(), wq) and torch.equal(scales.cpu(), ws)
        out = strided(torch.zeros(rows, cols, device="cuda", dtype=dtype), extra, offset)
        ctx.sc_dequantize(q, scales, out)
        assert torch.equal(out.cpu(), (wq.float() * ws[:, None]).to(dtype))
    assert bool(((wq.double() * ws.double()[:, None] - x.double().cpu()).abs() <= ws.double()[:, None] * 0.50001).all())


@pytest.mark.parametrize("dtype", TYPES + (torch.float32,))
def test_rows_special_values(ctx, dtype):
    info, inf, nan = torch.finfo(dtype), float("inf"), float("nan")
    rows = [[0.0, -0.0, 1.0, -1.0], [inf, 1.0, -2.0, 0.5], [nan, 3.0, 1.0, 0.25], [-inf, inf, nan, 0.0], [info.max, -info.max, 1.0, 0.0],
            [info.smallest_normal, -info.smallest_normal, 0.0, 0.0], [info.smallest_normal / 4, 0.0, 0.0, 0.0], [0.0] * 4, [-0.0] * 4,
            [127.0, 126.5, 125.5, -126.5], [254.0, 127.0, -253.0, 1.0], [2.0 ** -20, 1.0, 0.5, -0.25], [2.0 ** -100, 2.0 ** -101, 0.0, 0.0],
            [2.0 ** -101, -(2.0 ** -102), 0.0, 0.0]]
    for wide in (3, 300, 2600):                       # 12, 1200 and 10400 columns
        x = torch.tensor(rows, dtype=torch.float64).to(dtype).repeat(1, wide).cuda()
        x[:, 4:] = torch.where(torch.isfinite(x[:, 4:]), x[:, 4:], 0.0)             # one element that is not finite is enough
        q, scales = sc.quantized_buffers(*x.shape)
        ctx.sc_quantize(x, q, scales)
        wq, ws = rows_in_8_bits(x)
        assert torch.equal(q.cpu(), wq) and torch.equal(torch.nan_to_num(scales.cpu(), nan=-1.0), torch.nan_to_num(ws, nan=-1.0))
        out = torch.empty_like(x)
        ctx.sc_dequantize(q, scales, out)
        lost = ~torch.isfinite(x).all(1)
        assert bool(torch.isnan(out[lost]).all()) and bool(torch.isfinite(out[~lost]).all())


def test_rows_offsets_past_32_bits(ctx):
    rows, cols = 3, (1 << 31) - 32
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    tail = normal(rng(5), rows, 4096).to(torch.bfloat16)
    x[:, -4096:] = tail
    q, scales = sc.quantized_buffers(rows, cols)
    ctx.sc_quantize(x, q, scales)
    wq, ws = rows_in_8_bits(tail)
    assert torch.equal(q[:, -4096:].cpu(), wq) and torch.equal(scales.cpu(), ws) and not bool(q[:, :4096].any())
    x.fill_(3)
    ctx.sc_dequantize(q, scales, x)
    assert torch.equal(x[:, -4096:].cpu(), (wq.float() * ws[:, None]).to(x.dtype)) and not bool(x[:, :4096].any())


# -- the product -----------------------------------------------------------------------------------------------------
def eight_bits(g, rows, cols, size, extra=0, offset=0):
    q = (normal(g, rows, cols) * 40).round().clamp(-127, 127).to(torch.int8)
    return strided(q, extra, offset), size * (0.5 + torch.rand(rows, generator=g, device="cuda"))


def check_linear(ctx, dtype, act, M, N, K, bias=False, residual=False, keep=False, extra=0, offset=0, given=None):
    g = rng(M * 31 + N * 7 + K)
    (x, xs), (w, ws) = eight_bits(g, M, K, 1 / 40, extra, offset), eight_bits(g, N, K, 1 / 40 / math.sqrt(max(K, 1)), extra, offset)
    if given is not None:
        x, xs, w, ws = given(x, xs, w, ws)
    b = (normal(g, N) * 0.3).to(dtype) if bias else None
    r = strided(normal(g, M, N).to(dtype), extra, offset) if residual else None
    y = strided(torch.zeros(M, N, device="cuda").to(dtype), extra, offset)
    q, scales = sc.checkpoint_buffers(M, N) if keep else (None, None)
    ctx.sc_linear_quantized(sc.ACTIVATIONS[act], x, xs, w, ws, y, bias=b, residual=r, q=q, scales=scales)
    z = (x.double() @ w.double().t()) * xs.double()[:, None] * ws.double()
    slack = z.abs() * 4 * 2.0 ** -24
    if b is not None:
        z = z + b.double()
        slack = slack + z.abs() * 2.0 ** -24
    want = act64(z, act)
    y_slack = LIPSCHITZ * slack + z.abs() * ACT_ERR
    if r is not None:
        want = want + r.double()
        y_slack = y_slack + want.abs() * 2.0 ** -23
    assert_close(y, want, y_slack, dtype, "y")
    if keep:
        held = torch.empty(M, N, dtype=dtype, device="cuda")
        ctx.sc_checkpoint_unpack(q, scales, held)
        step = torch.exp2(scales.double() - 127).repeat_interleave(GROUP, 1)[:, :N]
        fine = torch.isfinite(z)
        assert bool(((held.double() - z).abs() <= 0.5 * step + slack)[fine].all())
        # the scale is the least for the group's largest, or for a value within its slack
        top = torch.nn.functional.pad(torch.where(fine, z, 0.0).abs(), (0, -N % GROUP)).view(M, -1, GROUP).amax(2)
        s = torch.exp2(scales.double() - 127)
        assert bool((top * (1 - 2.0 ** -20) <= 127 * s).all())
        assert bool(((top * (1 + 2.0 ** -20) > 63.5 * s) | (scales.int() - 127 == (-126 if dtype == torch.bfloat16 else -24))).all())
    return y


SIZES = [(1, 1, 1), (1, 64, 16), (1, 100, 257), (2, 40, 4096), (3, 1000, 520), (4, 33, 64), (5, 65, 96), (8, 200, 1000), (9, 128, 128), (16, 72, 2048),
         (17, 300, 131), (64, 512, 512), (127, 129, 127), (128, 256, 1024), (250, 1000, 520), (129, 264, 4104), (513, 70, 48), (1000, 1200, 272)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N,K", SIZES)
def test_linear_sizes(ctx, dtype, M, N, K):
    ctx.sc_debug_layer_tiles()
    check_linear(ctx, dtype, "none", M, N, K)
    check_linear(ctx, dtype, "gelu", M, N, K, True, True, True)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("bias,residual,keep", [(True, False, True), (False, True, False), (False, False, True)])
@pytest.mark.parametrize("M,N,K", [(1, 136, 80), (6, 100, 72), (200, 320, 136)])
def test_linear_epilogue(ctx, dtype, act, bias, residual, keep, M, N, K):
    check_linear(ctx, dtype, act, M, N, K, bias, residual, keep)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("extra,offset", [(16, 0), (16, 16), (1, 0), (0, 1), (2, 2), (3, 5), (4, 8), (64, 2)])
@pytest.mark.parametrize("M,N,K", [(1, 96, 64), (7, 96, 64), (140, 264, 80), (33, 65, 129)])
def test_linear_strides(ctx, dtype, extra, offset, M, N, K):
    check_linear(ctx, dtype, "silu", M, N, K, True, True, True, extra, offset)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tile", TILES)
@pytest.mark.parametrize("parts", [1, 2, 3])
@pytest.mark.parametrize("M,N,K", [(300, 520, 400), (517, 640, 656), (389, 333, 300), (258, 388, 144), (1025, 128, 1027)])
def test_every_tile_shape(ctx, dtype, tile, parts, M, N, K):
    ctx.sc_debug_layer_tiles(*tile, parts)
    before = ctx.launch_count
    check_linear(ctx, dtype, "none", M, N, K)
    assert ctx.launch_count - before == 1 + (K % 16 != 0) + (parts > 1)
    check_linear(ctx, dtype, "gelu_tanh", M, N, K, True, True, True)
    check_linear(ctx, dtype, "relu", M, N, K, True, False, True, 16, 16)
    check_linear(ctx, dtype, "silu", M, N, K, False, True, True, 3, 1)
    ctx.sc_debug_layer_tiles()


@pytest.mark.parametrize("tile", TILES)
def test_more_tiles_than_ctas(ctx, tile):
    ctx.sc_debug_layer_tiles(*tile, 1)
    M, N = {(256, 256): (3400, 3600), (128, 256): (2100, 5000), (128, 128): (2100, 2600), (128, 64): (1300, 2100)}[tile]
    check_linear(ctx, torch.bfloat16, "silu", M, N, 272, True, True, True)
    check_linear(ctx, torch.float16, "relu", M, N + 5, 144, True, False, True)
    ctx.sc_debug_layer_tiles()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N,K", [(1024, 4096, 1024), (1100, 4104, 1000), (900, 3001, 777), (32, 4096, 4096), (4, 4096, 4096)])
def test_sizes_of_real_layers(ctx, dtype, M, N, K):
    ctx.sc_debug_layer_tiles()
    check_linear(ctx, dtype, "gelu", M, N, K, True, True, True)


def test_sums_are_exact_at_their_largest(ctx):
    """All terms at their largest, of one sign: 131071 products of 127^2 (and of 128^2, bytes that sc_quantize does not make) fit 32 bits."""
    K = 131071
    for M in (1, 3, 6, 40):
        for value in (127, -128):
            x, w = torch.full((M, K), value, dtype=torch.int8, device="cuda"), torch.full((33, K), value, dtype=torch.int8, device="cuda")
            y = torch.empty(M, 33, dtype=torch.bfloat16, device="cuda")
            ones = torch.ones(64, device="cuda")
            ctx.sc_linear_quantized(sc.SC_ACT_NONE, x, ones[:M], w, ones[:33], y)
            assert bool((y == torch.tensor(float(value * value * K)).to(torch.bfloat16)).all())
    with pytest.raises(sc.SparseCommError) as e:
        big = torch.zeros(1, K + 1, dtype=torch.int8, device="cuda")
        ctx.sc_linear_quantized(sc.SC_ACT_NONE, big, ones[:1], big, ones[:1], torch.empty(1, 1, dtype=torch.bfloat16, device="cuda"))
    assert e.value.code == -2


@pytest.mark.parametrize("M", [1, 5, 150])
def test_scales_that_are_not_finite_reach_their_row_and_column_only(ctx, M):
    def given(x, xs, w, ws):
        xs, ws = xs.clone(), ws.clone()
        xs[M // 2], ws[7] = float("nan"), float("nan")
        xs[0] = 0.0 if M > 1 else xs[0]
        return x, xs, w, ws
    for act in ("none", "silu"):
        check_linear(ctx, torch.bfloat16, act, M, 200, 96, True, True, True, given=given)


def test_empty_sizes(ctx):
    bf = torch.bfloat16
    new8 = lambda r, c: torch.zeros(r, c, dtype=torch.int8, device="cuda")  # noqa: E731
    nan = lambda n: torch.full((n,), float("nan"), device="cuda")  # noqa: E731
    b, r = (torch.arange(40, device="cuda") / 8 - 2).to(bf), torch.ones(6, 40, dtype=bf, device="cuda")
    y = torch.full((6, 40), 9.0, dtype=bf, device="cuda")
    q, scales = sc.checkpoint_buffers(6, 40)
    ctx.sc_linear_quantized(sc.SC_ACT_RELU, new8(6, 0), nan(6), new8(40, 0), nan(40), y, bias=b, residual=r, q=q, scales=scales)     # an empty sum
    assert torch.equal(y, (torch.relu(b.float()) + 1).to(bf).expand(6, 40))
    launches = ctx.launch_count
    ctx.sc_linear_quantized(sc.SC_ACT_NONE, new8(0, 8), nan(0), new8(40, 8), nan(40), y[:0])
    ctx.sc_linear_quantized(sc.SC_ACT_NONE, new8(6, 8), nan(6), new8(0, 8), nan(0), y[:, :0])
    for rows, cols in ((0, 5), (5, 0), (0, 0)):
        x = torch.empty(rows, cols, dtype=bf, device="cuda")
        ctx.sc_quantize(x, new8(rows, cols), nan(rows))
        ctx.sc_dequantize(new8(rows, cols), nan(rows), x)
    assert ctx.launch_count == launches


def test_gradients_through_the_rounding(ctx):
    """The documented backward pass: the layer's 16-bit weights and the 8-bit rows' values."""
    M, N, K, bf = 130, 72, 264, torch.bfloat16
    g = rng(11)
    x, w, dz = normal(g, M, K).to(bf), (normal(g, N, K) / 16).to(bf), normal(g, M, N).to(bf)
    q, s = sc.quantized_buffers(M, K)
    ctx.sc_quantize(x, q, s)
    held, dw, dx = torch.empty_like(x), torch.empty(N, K, device="cuda"), torch.empty_like(x)
    ctx.sc_dequantize(q, s, held)
    ctx.sc_linear_grad_weight(dz, dw, x=held)
    ctx.sc_linear_grad_input(dz, w, dx)
    values = q.double() * s.double()[:, None]
    bound = (dz.double().abs().t() @ values.abs())
    assert bool(((dw.double() - dz.double().t() @ values).abs() <= (2.0 ** -8 + (M + 2) * 2.0 ** -23) * bound).all())
    assert_close(dx, dz.double() @ w.double(), (N + 2) * 2.0 ** -23 * (dz.double().abs() @ w.double().abs()), bf, "dx")


def test_refusals(ctx):
    bf = torch.bfloat16
    x8, w8, xs, ws = (torch.zeros(s, dtype=t, device="cuda") for s, t in (((6, 32), torch.int8), ((40, 32), torch.int8), (6, torch.float32), (40, torch.float32)))
    y, x = torch.zeros(6, 40, dtype=bf, device="cuda"), torch.zeros(6, 32, dtype=bf, device="cuda")
    q, scales = sc.checkpoint_buffers(6, 40)
    launches = ctx.launch_count
    linear = ctx.sc_linear_quantized
    for call in (lambda: linear(0, x8, xs, w8, ws, y.float()), lambda: linear(0, x8.float(), xs, w8, ws, y), lambda: linear(0, x8, xs.half(), w8, ws, y),
                 lambda: linear(0, x8, xs[:5], w8, ws, y), lambda: linear(0, x8, xs, w8[:, :31], ws, y), lambda: linear(0, x8, xs, w8[:39], ws, y),
                 lambda: linear(0, x8, None, w8, ws, y), lambda: linear(0, None, xs, w8, ws, y), lambda: linear(0, x8.cpu(), xs, w8, ws, y),
                 lambda: linear(0, x8, xs, w8, ws, y, bias=ws), lambda: linear(0, x8, xs, w8, ws, y, residual=y[:5]), lambda: linear(0, x8, xs, w8, ws, y, q=q),
                 lambda: linear(0, x8, xs, w8, ws, y, q=scales, scales=q), lambda: linear(0, x8.t(), xs, w8, ws, y), lambda: linear(9, x8, xs, w8, ws, y),
                 lambda: ctx.sc_quantize(x.double(), x8, xs), lambda: ctx.sc_quantize(x, x8[:5], xs), lambda: ctx.sc_quantize(x, x8, xs[:5]),
                 lambda: ctx.sc_quantize(x, x8.view(torch.uint8), xs), lambda: ctx.sc_quantize(x, x8, None), lambda: ctx.sc_quantize(x[0], x8, xs),
                 lambda: ctx.sc_dequantize(x8, xs, x[:, ::2]), lambda: ctx.sc_dequantize(None, xs, x), lambda: ctx.sc_dequantize(x8, xs.cpu(), x),
                 lambda: ctx.sc_quantize(x, x8[:1].expand(6, 32), xs)):
        with pytest.raises((TypeError, ValueError, sc.SparseCommError)):
            call()
    assert ctx.launch_count == launches


@pytest.mark.parametrize("M", [1, 2, 3, 8, 9, 16, 17, 32, 33])
@pytest.mark.parametrize("N,K", [(1, 16), (15, 48), (40, 1024), (1000, 80), (33, 4112)])
def test_few_tokens(ctx, M, N, K):
    ctx.sc_debug_layer_tiles()
    before = ctx.launch_count
    check_linear(ctx, torch.bfloat16, "gelu", M, N, K, True, True, False)
    assert ctx.launch_count - before == 1 or M == 33                    # no copies, no join
    check_linear(ctx, torch.float16, "none", M, N, K, False, False, True, 16, 16)


def test_sums_of_few_tokens_are_exact_at_their_largest(ctx):
    """A multiple of 16 near the largest sum, which these sizes' kernels take; the result is the exact sum rounded once to 24 bits and once to 8."""
    K = 131056
    ones = torch.ones(64, device="cuda")
    for M in (1, 2, 5, 12, 30):
        for a, b in ((127, 127), (-128, -128), (-128, 127)):
            x, w = torch.full((M, K), a, dtype=torch.int8, device="cuda"), torch.full((37, K), b, dtype=torch.int8, device="cuda")
            x[:, 5], w[:, K - 3] = 1, 1
            y = torch.empty(M, 37, dtype=torch.bfloat16, device="cuda")
            ctx.sc_linear_quantized(sc.SC_ACT_NONE, x, ones[:M], w, ones[:37], y)
            assert bool((y == torch.tensor(float(a * b * (K - 2) + b + a)).to(torch.bfloat16)).all())


def test_sums_of_few_tokens_term_by_term(ctx):
    """Large sums that cancel: every single term is seen in the result."""
    K = 4096
    g = rng(3)
    x = torch.randint(-128, 128, (32, K), generator=g, device="cuda").to(torch.int8)
    w = torch.randint(-128, 128, (64, K // 2), generator=g, device="cuda").to(torch.int8)
    w = torch.cat((w, torch.where(w == -128, 127, -w).to(torch.int8)), 1)
    x = torch.cat((x[:, :K // 2], x[:, :K // 2]), 1)
    exact = x.double() @ w.double().t()                                 # small: only where w was -128 the halves differ
    ones = torch.ones(64, device="cuda")
    for M in (1, 2, 6, 16, 32):
        y = torch.empty(M, 64, dtype=torch.float16, device="cuda")
        ctx.sc_linear_quantized(sc.SC_ACT_NONE, x[:M], ones[:M], w, ones, y)
        assert torch.equal(y, exact[:M].to(torch.float16))


@pytest.mark.parametrize("offset", [0, 1, 7, 15])
@pytest.mark.parametrize("M,N,K", [(9, 40, 127), (9, 40, 129), (1, 33, 2047), (40, 1, 2049), (33, 65, 4097), (3, 20, 131071)])
def test_rows_of_bytes_at_any_alignment(ctx, M, N, K, offset):
    """The operands' copies: rows that begin anywhere in 16 bytes, among bytes that are not theirs, of one and of several runs a warp."""
    ctx.sc_debug_layer_tiles()
    g = rng(K + offset)
    x, w = (strided(torch.randint(-127, 128, (r, K), generator=g, device="cuda").to(torch.int8), 5 if offset else 0, offset) for r in (M, N))
    y, ones = torch.empty(M, N, device="cuda", dtype=torch.bfloat16), [torch.ones(n, device="cuda") for n in (M, N)]
    ctx.sc_linear_quantized(sc.ACTIVATIONS["none"], x, ones[0], w, ones[1], y)
    assert torch.equal(y, (x.double() @ w.double().T).float().bfloat16())
