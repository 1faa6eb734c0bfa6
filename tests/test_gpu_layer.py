"""Layer operators (checkpoints, activation gradient, linear layer forward and backward) against 64-bit statements.

Tolerances: an output is within its type's rounding of the 64-bit value plus the bound of an fp32 sum of its products
(layer_util.product_slack) carried through the activation, whose slope and value are computed to 2^-18 of their size.
Checkpoints are compared bit for bit."""
import math

import pytest
import torch

import paper_2009_09271_b200 as sc
from layer_util import (ACTS, GROUP, act64, assert_close, checkpoint64, product_slack, slope64, strided)

pytestmark = pytest.mark.gpu

TYPES = (torch.bfloat16, torch.float16)
ACT_ERR = 2.0 ** -18
LIPSCHITZ = 1.13                                     # largest slope of the activations
CURVATURE = 1.13                                     # and of the slopes (gelu: 0.8 at 0; the others below)


@pytest.fixture(scope="module")
def ctx():
    c = sc.Context(max_n=1 << 20, max_W=2, max_segments=8)
    yield c
    assert c.sc_sync_status() == 0
    c.close()


def rng(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def kept_of(g, rows, cols, spread=2):
    q = (normal(g, rows, cols) * 40).round().clamp(-127, 127).to(torch.int8)
    e = torch.randint(-6, -6 + spread, (rows, -(-cols // GROUP)), generator=g, device="cuda")
    scales = (e + 127).to(torch.uint8)
    values = q.double() * torch.exp2(e.double()).repeat_interleave(GROUP, 1)[:, :cols]
    return q, scales, values


# -- checkpoints -----------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", TYPES + (torch.float32,))
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 31), (3, 32), (5, 33), (2, 64), (7, 1000), (65, 1024), (1, 4099), (301, 8)])
def test_checkpoint_bits(ctx, dtype, rows, cols):
    g = rng(rows * 7919 + cols)
    x = (normal(g, rows, cols) * torch.exp2(torch.randint(-20, 12, (rows, 1), generator=g, device="cuda").float())).to(dtype)
    if rows > 1:
        x[1] = 0
    for extra, offset in ((0, 0), (8, 8), (3, 1)):
        xs = strided(x, extra, offset)
        q, scales = sc.checkpoint_buffers(rows, cols)
        ctx.sc_checkpoint_pack(xs, q, scales)
        wq, ws, wv = checkpoint64(x, dtype)
        assert torch.equal(q.cpu(), wq) and torch.equal(scales.cpu(), ws)
        out = strided(torch.zeros(rows, cols, device="cuda", dtype=dtype), extra, offset)
        ctx.sc_checkpoint_unpack(q, scales, out)
        assert torch.equal(out.double().cpu(), wv)
    # the stored value is within half a step of the input, a step being at most 2/127 of the group's largest
    assert bool(((wv - x.double().cpu()).abs() <= x.double().abs().amax(1, keepdim=True).cpu() / 126 + 1e-30).all())


@pytest.mark.parametrize("dtype", TYPES + (torch.float32,))
def test_checkpoint_special_values(ctx, dtype):
    info = torch.finfo(dtype)
    inf, nan = float("inf"), float("nan")
    rows = [[0.0, -0.0, 1.0, -1.0], [inf, 1.0, -2.0, 0.5], [nan, 3.0, -inf, 0.25], [info.max, -info.max, 1.0, 0.0],
            [info.smallest_normal, -info.smallest_normal, 0.0, 0.0], [info.smallest_normal / 4, 0.0, 0.0, 0.0], [nan] * 4, [-inf] * 4,
            [127.0, 126.5, 125.5, -126.5], [127.5, 63.5, -0.5, 1.5], [info.max / 2, info.max, -info.max * 0.99, 1e-3],
            [254.0, 127.0, -253.0, 1.0]]
    x = torch.tensor(rows, dtype=torch.float64).to(dtype).repeat(1, 12).cuda()        # 48 columns: a whole group and a part
    q, scales = sc.checkpoint_buffers(*x.shape)
    ctx.sc_checkpoint_pack(x, q, scales)
    wq, ws, wv = checkpoint64(x, dtype)
    assert torch.equal(q.cpu(), wq) and torch.equal(scales.cpu(), ws)
    out = torch.empty_like(x)
    ctx.sc_checkpoint_unpack(q, scales, out)
    assert torch.equal(torch.nan_to_num(out.double().cpu(), nan=12345.0), torch.nan_to_num(wv, nan=12345.0))
    assert torch.equal(torch.isnan(out), ~torch.isfinite(x))
    assert bool(torch.isfinite(out[torch.isfinite(x)]).all())


def test_checkpoint_offsets_past_32_bits(ctx):
    rows, cols = 3, (1 << 31) - 32                     # 6.4e9 elements, 12.9 GB
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    g = rng(5)
    tail = normal(g, rows, 4096).to(torch.bfloat16)
    x[:, -4096:] = tail
    q, scales = sc.checkpoint_buffers(rows, cols)
    ctx.sc_checkpoint_pack(x, q, scales)
    wq, ws, wv = checkpoint64(tail, torch.bfloat16)
    assert torch.equal(q[:, -4096:].cpu(), wq) and torch.equal(scales[:, -128:].cpu(), ws)
    x.fill_(3)
    ctx.sc_checkpoint_unpack(q, scales, x)
    assert torch.equal(x[:, -4096:].double().cpu(), wv) and not bool(x[:, :4096].any())


# -- activation gradient ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("rows,cols,extra,offset", [(1, 1, 0, 0), (1, 257, 0, 0), (33, 64, 8, 0), (509, 1000, 0, 0), (2050, 40, 3, 1), (70, 4104, 0, 8)])
def test_activation_grad(ctx, dtype, act, rows, cols, extra, offset):
    g = rng(rows + cols)
    dy = strided(normal(g, rows, cols).to(dtype), extra, offset)
    q, scales, z = kept_of(g, rows, cols)
    want = dy.double() * slope64(z, act)
    slack = dy.double().abs() * (1 + z.abs()) * ACT_ERR
    dz = strided(torch.zeros(rows, cols, device="cuda").to(dtype), extra, offset)
    db = torch.full((cols,), 9.0, device="cuda")
    ctx.sc_activation_grad(sc.ACTIVATIONS[act], dy, q, scales, dz, db)
    assert_close(dz, want, slack, dtype, "dz")
    sums = slack.sum(0) + (rows + 2) * 2.0 ** -23 * want.abs().sum(0)
    assert_close(db, want.sum(0), sums, torch.float32, "db")
    db2 = torch.full((cols,), 2.0, device="cuda")
    ctx.sc_activation_grad(sc.ACTIVATIONS[act], dy, q, scales, None, db2, accumulate=True)
    assert torch.equal(db2, db + 2.0)                                  # the same sums every time, in the same order
    only = torch.empty_like(dz)
    ctx.sc_activation_grad(sc.ACTIVATIONS[act], dy, q, scales, only)
    assert torch.equal(only, dz)
    inplace = strided(dy, extra, offset)
    ctx.sc_activation_grad(sc.ACTIVATIONS[act], inplace, q, scales, inplace)
    assert torch.equal(inplace, dz)


@pytest.mark.parametrize("act", ACTS[1:])
def test_activation_grad_extremes(ctx, act):
    """NaN in a checkpoint passes on, large magnitudes saturate, dy's own infinities follow the formula."""
    z = torch.tensor([0.0, 1e-30, -1e-30, 3e4, -3e4, 1e30, -1e30, 88.0, -88.0, 20.0, -20.0, 3.0, -3.0, float("nan"), 0.5, -0.5])
    z = z.view(-1, 1).repeat(1, 40).cuda()
    q, scales = sc.checkpoint_buffers(*z.shape)
    ctx.sc_checkpoint_pack(z, q, scales)
    held = torch.empty_like(z)
    ctx.sc_checkpoint_unpack(q, scales, held)
    dy = torch.ones(*z.shape, dtype=torch.bfloat16, device="cuda")
    dz = torch.empty_like(dy)
    ctx.sc_activation_grad(sc.ACTIVATIONS[act], dy, q, scales, dz)
    want = slope64(held.double(), act)
    assert bool(torch.isnan(dz[13]).all())
    assert_close(dz, want, (1 + held.abs().double().clamp(max=8)) * ACT_ERR, torch.bfloat16, "dz")


# -- the linear layer ------------------------------------------------------------------------------------------------
SIZES = [(1, 1, 1), (1, 8, 8), (1, 33, 31), (1, 1024, 520), (3, 130, 64), (7, 64, 96), (17, 1000, 512), (64, 256, 128), (65, 72, 4104),
         (128, 256, 64), (129, 257, 65), (250, 1000, 512), (300, 136, 200), (513, 264, 1032), (1, 4096, 4096), (40, 512, 8192)]


def layer_inputs(dtype, M, N, K, seed, extra=0, offset=0):
    g = rng(seed)
    x = strided(normal(g, M, K).to(dtype), extra, offset)
    w = strided((normal(g, N, K) / math.sqrt(K)).to(dtype), extra, offset)
    return g, x, w


def check_linear(ctx, dtype, act, M, N, K, bias, residual, keep, extra=0, offset=0, x_w=None):
    g, x, w = layer_inputs(dtype, M, N, K, M * 31 + N * 7 + K, extra, offset)
    if x_w is not None:
        x, w = x_w
    b = (normal(g, N) * 0.3).to(dtype) if bias else None
    r = strided(normal(g, M, N).to(dtype), extra, offset) if residual else None
    y = strided(torch.zeros(M, N, device="cuda").to(dtype), extra, offset)
    q, scales = sc.checkpoint_buffers(M, N) if keep else (None, None)
    ctx.sc_linear(sc.ACTIVATIONS[act], x, w, y, bias=b, residual=r, q=q, scales=scales)
    z = x.double() @ w.double().t()
    slack = product_slack(x, w.t(), K)
    if b is not None:
        z = z + b.double()
    z_slack = slack + z.abs() * 2.0 ** -23
    want = act64(z, act)
    y_slack = LIPSCHITZ * z_slack + z.abs() * ACT_ERR
    if r is not None:
        want = want + r.double()
        y_slack = y_slack + want.abs() * 2.0 ** -23
    assert_close(y, want, y_slack, dtype, "y")
    if keep:
        held = torch.empty(M, N, dtype=dtype, device="cuda")
        ctx.sc_checkpoint_unpack(q, scales, held)
        # half a step of the group's scale, and the scale is the definition's for some z within its slack
        step = torch.exp2(scales.double() - 127).repeat_interleave(GROUP, 1)[:, :N]
        assert bool(((held.double() - z).abs() <= 0.5 * step + z_slack).all())
        pad = -N % GROUP
        top = torch.nn.functional.pad(z.abs(), (0, pad)).view(M, -1, GROUP).amax(2)
        top_slack = torch.nn.functional.pad(z_slack, (0, pad)).view(M, -1, GROUP).amax(2)
        s = torch.exp2(scales.double() - 127)
        assert bool((top - top_slack <= 127 * s).all())
        lo = -126 if dtype == torch.bfloat16 else -24
        assert bool(((top + top_slack > 63.5 * s) | (scales.int() - 127 == lo)).all())
    return y


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N,K", SIZES)
def test_linear_sizes(ctx, dtype, M, N, K):
    check_linear(ctx, dtype, "none", M, N, K, False, False, False)
    check_linear(ctx, dtype, "gelu", M, N, K, True, True, True)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("bias,residual,keep", [(True, False, True), (False, True, False), (False, False, True)])
@pytest.mark.parametrize("M,N,K", [(5, 100, 72), (200, 320, 136)])
def test_linear_epilogue(ctx, dtype, act, bias, residual, keep, M, N, K):
    check_linear(ctx, dtype, act, M, N, K, bias, residual, keep)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("extra,offset", [(8, 0), (8, 8), (1, 0), (0, 1), (3, 5), (64, 2)])
@pytest.mark.parametrize("M,N,K", [(2, 96, 64), (140, 264, 72), (33, 65, 129)])
def test_linear_strides(ctx, dtype, extra, offset, M, N, K):
    check_linear(ctx, dtype, "silu", M, N, K, True, True, True, extra, offset)
    check_input_grad(ctx, dtype, "gelu_tanh", M, N, K, True, extra, offset)
    check_weight_grad(ctx, dtype, M, N, K, "kept", extra, offset)
    check_weight_grad(ctx, dtype, M, N, K, "dense", extra, offset)


def check_input_grad(ctx, dtype, act, M, N, K, residual, extra=0, offset=0):
    g, _, w = layer_inputs(dtype, M, N, K, M + N * 13 + K * 5, extra, offset)
    dz = strided(normal(g, M, N).to(dtype), extra, offset)
    r = strided(normal(g, M, K).to(dtype), extra, offset) if residual else None
    dx = strided(torch.zeros(M, K, device="cuda").to(dtype), extra, offset)
    q, scales, z = kept_of(g, M, K)
    if act == "none":
        ctx.sc_linear_grad_input(dz, w, dx, residual=r)
    else:
        ctx.sc_linear_grad_input(dz, w, dx, residual=r, act=sc.ACTIVATIONS[act], q=q, scales=scales)
    want = dz.double() @ w.double()
    slack = product_slack(dz, w, N)
    if r is not None:
        want = want + r.double()
        slack = slack + want.abs() * 2.0 ** -23
    slack = slack * LIPSCHITZ + want.abs() * (1 + z.abs()) * ACT_ERR
    assert_close(dx, want * slope64(z, act), slack, dtype, "dx")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N,K", SIZES)
def test_linear_grad_input(ctx, dtype, M, N, K):
    check_input_grad(ctx, dtype, "none", M, N, K, False)
    check_input_grad(ctx, dtype, "silu", M, N, K, True)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("residual", [False, True])
def test_linear_grad_input_acts(ctx, act, residual):
    check_input_grad(ctx, torch.bfloat16, act, 150, 136, 264, residual)
    check_input_grad(ctx, torch.float16, act, 3, 200, 100, residual)


def check_weight_grad(ctx, dtype, M, N, K, how, extra=0, offset=0):
    g = rng(M * 3 + N + K * 17)
    dz = strided(normal(g, M, N).to(dtype), extra, offset)
    q, scales, xv = kept_of(g, M, K, 9)
    given = {"q": q, "scales": scales}
    if how == "dense":
        x = strided(xv.to(dtype), extra, offset)
        xv = x.double()
        given = {"x": x}
    row = torch.full((N * (K + extra) + offset + 7,), 5.0, device="cuda")
    dw = row[offset:offset + N * (K + extra)].view(N, K + extra)[:, :K]
    want = dz.double().t() @ xv
    slack = product_slack(dz.t(), xv, M)
    ctx.sc_linear_grad_weight(dz, dw, **given)
    assert_close(dw, want, slack, torch.float32, "dw")
    first = dw.clone()
    ctx.sc_linear_grad_weight(dz, dw, accumulate=True, **given)
    assert_close(dw, 2 * want, 2 * slack + want.abs() * 2.0 ** -22, torch.float32, "dw accumulated")
    again = torch.empty_like(first)
    ctx.sc_linear_grad_weight(dz, again, **given)
    assert torch.equal(again, first)                                   # no order that changes from run to run
    guard = row.clone()
    guard[offset:offset + N * (K + extra)].view(N, K + extra)[:, :K] = 5.0
    assert bool((guard == 5.0).all())                                  # nothing outside the matrix was touched


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("how", ["kept", "dense"])
@pytest.mark.parametrize("M,N,K", SIZES)
def test_linear_grad_weight(ctx, dtype, how, M, N, K):
    check_weight_grad(ctx, dtype, M, N, K, how)


@pytest.mark.parametrize("offset", [1, 2, 3])
def test_linear_grad_weight_at_any_offset_of_a_gradient_row(ctx, offset):
    check_weight_grad(ctx, torch.bfloat16, 70, 200, 136, "kept", 0, offset)


@pytest.mark.parametrize("M,N,K", [(5000, 130, 72), (20011, 256, 256)])
def test_linear_grad_weight_long_sums(ctx, M, N, K):
    """Many tokens, few tiles: the sum is split and joined.  The error of the whole, not of the worst element alone: rounding
    errors of M / 16 steps of random sign would give 2^-24 sqrt(M / 16); four times that is allowed."""
    check_weight_grad(ctx, torch.bfloat16, M, N, K, "kept")
    g = rng(M)
    dz = normal(g, M, N).to(torch.bfloat16)
    q, scales, xv = kept_of(g, M, K, 9)
    dw = torch.empty(N, K, device="cuda")
    ctx.sc_linear_grad_weight(dz, dw, q=q, scales=scales)
    want = dz.double().t() @ xv
    assert float((dw.double() - want).norm() / want.norm()) <= 4 * 2.0 ** -24 * math.sqrt(M / 16)


def test_split_sums_with_one_sign(ctx):
    """Products of one sign: a sum that is cut at each addition drifts.  At most 2^-20 of the sum is allowed."""
    for M, N, K in ((4096, 128, 128), (16384, 1000, 1024)):
        g = rng(M)
        dz = normal(g, M, N).abs().to(torch.bfloat16)
        x = normal(g, M, K).abs().to(torch.bfloat16)
        dw = torch.empty(N, K, device="cuda")
        ctx.sc_linear_grad_weight(dz, dw, x=x)
        want = dz.double().t() @ x.double()
        assert float(((dw.double() - want) / want).abs().max()) <= 2.0 ** -20


def test_empty_sizes(ctx):
    bf = torch.bfloat16
    new = lambda r, c, t=bf, v=0.0: torch.full((r, c), v, device="cuda").to(t)  # noqa: E731
    b, r = (torch.arange(40, device="cuda") / 8 - 2).to(bf), new(6, 40, v=1.0)
    y = new(6, 40, v=9.0)
    q, scales = sc.checkpoint_buffers(6, 40)
    ctx.sc_linear(sc.SC_ACT_RELU, new(6, 0), new(40, 0), y, bias=b, residual=r, q=q, scales=scales)      # an empty sum
    assert torch.equal(y, (torch.relu(b.float()) + 1).to(bf).expand(6, 40))
    held = new(6, 40)
    ctx.sc_checkpoint_unpack(q, scales, held)
    assert bool(((held.float() - b.float()).abs() <= 0.5 * 2.0 ** -4).all())
    ctx.sc_linear(sc.SC_ACT_NONE, new(0, 8), new(40, 8), new(0, 40))
    ctx.sc_linear(sc.SC_ACT_NONE, new(6, 8), new(0, 8), new(6, 0))
    dx = new(6, 8, v=9.0)
    ctx.sc_linear_grad_input(new(6, 0), new(0, 8), dx)
    assert not bool(dx.any())
    dw = torch.full((40, 8), 3.0, device="cuda")
    ctx.sc_linear_grad_weight(new(0, 40), dw, x=new(0, 8), accumulate=True)
    assert bool((dw == 3).all())
    ctx.sc_linear_grad_weight(new(0, 40), dw, x=new(0, 8))
    assert not bool(dw.any())
    db = torch.full((40,), 3.0, device="cuda")
    ctx.sc_activation_grad(sc.SC_ACT_NONE, new(0, 40), None, None, None, db, accumulate=True)
    assert bool((db == 3).all())
    ctx.sc_activation_grad(sc.SC_ACT_NONE, new(0, 40), None, None, None, db)
    assert not bool(db.any())
    q0, s0 = sc.checkpoint_buffers(0, 8)
    ctx.sc_checkpoint_pack(new(0, 8), q0, s0)
    assert ctx.sc_sync_status() == 0


def test_not_finite_stays_in_its_row(ctx):
    """An infinity or NaN of one token reaches that token's outputs alone."""
    g, x, w = layer_inputs(torch.bfloat16, 200, 264, 136, 3)
    x[17, 5], x[130, 0] = float("nan"), float("inf")
    y = torch.empty(200, 264, dtype=torch.bfloat16, device="cuda")
    q, scales = sc.checkpoint_buffers(200, 264)
    ctx.sc_linear(sc.SC_ACT_SILU, x, w, y, q=q, scales=scales)
    fine = torch.ones(200, dtype=torch.bool, device="cuda")
    fine[17] = fine[130] = False
    assert bool(torch.isfinite(y[fine]).all()) and bool(torch.isnan(y[17]).all())
    assert bool((q[17] == -128).all()) and bool((q[fine] != -128).all())
    z = x[130].double() @ w.double().t()
    assert bool((q[130] == -128).all()) and not bool(torch.isfinite(z).any())


def test_in_place_residual_and_other_stream(ctx):
    g, x, w = layer_inputs(torch.float16, 300, 520, 264, 8)
    r = normal(g, 300, 520).half()
    want = torch.empty_like(r)
    ctx.sc_linear(sc.SC_ACT_GELU, x, w, want, residual=r)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    same = r.clone()
    dw, dw2 = torch.empty(520, 264, device="cuda"), torch.empty(520, 264, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        ctx.sc_linear(sc.SC_ACT_GELU, x, w, same, residual=same)
        ctx.sc_linear_grad_weight(same, dw, x=x)
    side.synchronize()
    assert torch.equal(same, want)
    ctx.sc_linear_grad_weight(want, dw2, x=x, stream=torch.cuda.current_stream())
    assert torch.equal(dw, dw2)


def test_capture_in_a_graph(ctx):
    """Layer calls replay from a CUDA graph once their workspace is reserved; without it they refuse."""
    M, N, K = 1500, 264, 136
    g, x, w = layer_inputs(torch.bfloat16, M, N, K, 21)
    dz = normal(g, M, N).to(torch.bfloat16)
    q, scales, _ = kept_of(g, M, K)
    own = sc.Context(max_n=1)
    dw, dx, db = torch.empty(N, K, device="cuda"), torch.empty(M, K, dtype=torch.bfloat16, device="cuda"), torch.empty(N, device="cuda")

    def step():
        own.sc_linear_grad_weight(dz, dw, q=q, scales=scales)
        own.sc_linear_grad_input(dz, w, dx)
        own.sc_activation_grad(sc.SC_ACT_NONE, dz, None, None, None, db)

    graph = torch.cuda.CUDAGraph()
    refused = False
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        try:
            own.sc_linear_grad_weight(dz, dw, q=q, scales=scales)
        except sc.SparseCommError as e:
            refused = e.code == -3
    assert refused
    own.sc_layer_reserve(M, N, K)
    held = own.scratch_bytes
    step()
    torch.cuda.synchronize()
    assert own.scratch_bytes == held
    want = [t.clone() for t in (dw, dx, db)]
    for t in (dw, dx, db):
        t.fill_(0)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    for got, ref in zip((dw, dx, db), want):
        assert torch.equal(got, ref)
    own.sc_layer_reserve(4 * M, N, K)                       # a larger workspace leaves the graph's own in place
    for t in (dw, dx, db):
        t.fill_(0)
    torch.empty(1 << 28, device="cuda", dtype=torch.uint8).fill_(255)
    graph.replay()
    torch.cuda.synchronize()
    for got, ref in zip((dw, dx, db), want):
        assert torch.equal(got, ref)
    del graph
    own.close()


def test_rows_past_32_bits(ctx):
    """Rows so far apart that element offsets pass 2^32, in every product, and the same through the copies of unaligned rows."""
    for step in ((1 << 31) - 1024, (1 << 31) - 1023):
        store = torch.zeros(2 * step + 4096, dtype=torch.bfloat16, device="cuda")           # 8.6 GB
        g = rng(4)
        far = store.as_strided((3, 200), (step, 1))
        far.copy_(normal(g, 3, 200).to(torch.bfloat16))
        w = (normal(g, 72, 200) / 14).to(torch.bfloat16)
        xs = far.clone()
        for rows in (3,):
            y, want = torch.empty(rows, 72, dtype=torch.bfloat16, device="cuda"), torch.empty(rows, 72, dtype=torch.bfloat16, device="cuda")
            ctx.sc_linear(sc.SC_ACT_NONE, far, w, y)
            ctx.sc_linear(sc.SC_ACT_NONE, xs, w, want)
            assert torch.equal(y, want)
            v = (normal(g, 200, 72) / 14).to(torch.bfloat16)
            ctx.sc_linear_grad_input(far, v, y)
            ctx.sc_linear_grad_input(xs, v, want)
            assert torch.equal(y, want)
            dw, dww = torch.empty(200, 72, device="cuda"), torch.empty(200, 72, device="cuda")
            ctx.sc_linear_grad_weight(far, dw, x=want)
            ctx.sc_linear_grad_weight(xs, dww, x=want)
            assert torch.equal(dw, dww)
        out = store.as_strided((3, 72), (step, 1))
        ctx.sc_linear(sc.SC_ACT_NONE, xs, w, out)
        ctx.sc_linear(sc.SC_ACT_NONE, xs, w, want)
        assert torch.equal(out, want)
        del store, far, out


@pytest.mark.parametrize("M,N,K", [(5181, 264, 88), (2500, 640, 72), (20000, 64, 64)])
def test_many_narrow_tiles_a_cta(ctx, M, N, K):
    """Short sums over more tiles than CTAs: the accumulators, the output buffers and the copies from them all take turns."""
    for _ in range(3):
        check_linear(ctx, torch.bfloat16, "relu", M, N, K, True, False, True)
        check_input_grad(ctx, torch.float16, "silu", M, K, N, True)


def test_tokens_and_tiles_agree_at_the_border(ctx):
    """One or two tokens, and four of short calls, take the kernel without tiles, five the tensor tiles: the same sums within their
    bounds."""
    for M in (1, 2, 3, 4, 5):
        for N, K in ((1000, 8), (33, 5000), (4096, 264), (4096, 2056)):
            check_linear(ctx, torch.bfloat16, "gelu_tanh", M, N, K, True, True, True)
            check_linear(ctx, torch.float16, "relu", M, N, K, False, False, False, 1, 1)


@pytest.mark.parametrize("M", [1, 4, 5, 8, 9, 17])
@pytest.mark.parametrize("N,K", [(1000, 33), (70, 260), (2049, 129)])
def test_weight_gradient_of_few_tokens(ctx, M, N, K):
    """Up to eight tokens take the kernel without tiles, nine the tensor tiles."""
    for how, extra, offset in (("kept", 0, 0), ("dense", 0, 0), ("kept", 3, 1), ("dense", 8, 3)):
        check_weight_grad(ctx, torch.bfloat16, M, N, K, how, extra, offset)
        check_weight_grad(ctx, torch.float16, M, N, K, how, extra, offset)


def test_weight_gradient_passes_nan_of_a_checkpoint(ctx):
    for M in (3, 40):
        x = torch.ones(M, 70, device="cuda")
        x[1, 5], x[2, 69] = float("inf"), float("nan")
        q, scales = sc.checkpoint_buffers(M, 70)
        ctx.sc_checkpoint_pack(x, q, scales)
        dw = torch.empty(36, 70, device="cuda")
        ctx.sc_linear_grad_weight(torch.ones(M, 36, dtype=torch.bfloat16, device="cuda"), dw, q=q, scales=scales)
        bad = torch.zeros(70, dtype=torch.bool, device="cuda")
        bad[5] = bad[69] = True
        assert bool(torch.isnan(dw[:, bad]).all()) and bool((dw[:, ~bad] == M).all())


@pytest.mark.parametrize("length,ld", [(35, 40), (999, 1000), (1002, 1008), (65, 128), (130, 136), (37, 37)])
def test_nothing_between_input_rows_is_read(ctx, length, ld):
    """NaN between the rows of every input leaves the outputs alone."""
    for dtype in TYPES:
        def spaced(t):
            store = torch.full((t.shape[0], ld), float("nan"), dtype=dtype, device="cuda")
            store[:, :length] = t
            return store[:, :length]

        g = rng(length)
        for rows in (3, 150):
            a, b = normal(g, rows, length).to(dtype), normal(g, 72, length).to(dtype)
            y, want = torch.empty(rows, 72, dtype=dtype, device="cuda"), torch.empty(rows, 72, dtype=dtype, device="cuda")
            ctx.sc_linear(sc.SC_ACT_NONE, spaced(a), spaced(b), y)
            ctx.sc_linear(sc.SC_ACT_NONE, a, b, want)
            assert bool(torch.isfinite(y).all())
            assert_close(y, want.double(), product_slack(a, b.t(), length), dtype, "y")
            dx, wide = torch.empty(rows, length, dtype=dtype, device="cuda"), torch.empty(rows, length, dtype=dtype, device="cuda")
            ctx.sc_linear_grad_input(want, spaced(b), dx, residual=spaced(a))
            ctx.sc_linear_grad_input(want, b, wide, residual=a)
            assert bool(torch.isfinite(dx).all())
            assert_close(dx, wide.double(), product_slack(want, b, 72), dtype, "dx")
            dw, dense = torch.empty(length, length, device="cuda"), torch.empty(length, length, device="cuda")
            ctx.sc_linear_grad_weight(spaced(a), dw, x=spaced(a))
            ctx.sc_linear_grad_weight(a, dense, x=a)
            assert bool(torch.isfinite(dw).all())
            assert_close(dw, dense.double(), product_slack(a.t(), a, rows), torch.float32, "dw")
            q, scales = sc.checkpoint_buffers(rows, length)
            q2, scales2 = sc.checkpoint_buffers(rows, length)
            ctx.sc_checkpoint_pack(spaced(a), q, scales)
            ctx.sc_checkpoint_pack(a, q2, scales2)
            assert torch.equal(q, q2) and torch.equal(scales, scales2)
            dz, db, db2 = torch.empty_like(a), torch.empty(length, device="cuda"), torch.empty(length, device="cuda")
            ctx.sc_activation_grad(sc.SC_ACT_GELU, spaced(a), q, scales, dz, db)
            ctx.sc_activation_grad(sc.SC_ACT_GELU, a, q, scales, None, db2)
            assert bool(torch.isfinite(dz).all()) and torch.equal(db, db2)


@pytest.mark.parametrize("cols", [1, 2, 4, 6, 12, 1002, 1004, 999])
@pytest.mark.parametrize("extra,offset", [(0, 0), (2, 2), (4, 4), (1, 0), (7, 8), (8, 4)])
def test_nothing_is_written_between_or_behind_rows(ctx, cols, extra, offset):
    """Outputs inside a larger buffer: what lies between their rows, and behind the last, stays as it was."""
    for rows in (1, 5, 150):
        for dtype in TYPES:
            g = rng(rows + cols)
            x, w = normal(g, rows, 72).to(dtype), normal(g, cols, 72).to(dtype)
            dz, v = normal(g, rows, 40).to(dtype), normal(g, 40, cols).to(dtype)
            q, scales, _ = kept_of(g, rows, cols)

            def guarded(call, t=dtype):
                ld = cols + extra
                store = torch.full((offset + rows * ld + 64,), 3.0, device="cuda").to(t)
                call(store[offset:offset + rows * ld].view(rows, ld)[:, :cols])
                store[offset:offset + rows * ld].view(rows, ld)[:, :cols] = 3
                assert bool((store == 3).all())

            guarded(lambda out: ctx.sc_linear(sc.SC_ACT_GELU, x, w, out, residual=out))
            guarded(lambda out: ctx.sc_linear_grad_input(dz, v, out))
            guarded(lambda out: ctx.sc_checkpoint_unpack(q, scales, out))
            guarded(lambda out: ctx.sc_activation_grad(sc.SC_ACT_SILU, normal(g, rows, cols).to(dtype), q, scales, out))
            for tokens in (6, 40, 700):
                a, b = normal(g, tokens, rows).to(dtype), normal(g, tokens, cols).to(dtype)
                guarded(lambda out: ctx.sc_linear_grad_weight(a, out, x=b), torch.float32)
                guarded(lambda out: ctx.sc_linear_grad_weight(a, out, x=b, accumulate=True), torch.float32)
            kept = torch.full((rows * cols + 64,), 9, dtype=torch.int8, device="cuda")
            marks = torch.full((rows * -(-cols // GROUP) + 64,), 9, dtype=torch.uint8, device="cuda")
            kq, ks = kept[:rows * cols].view(rows, cols), marks[:rows * -(-cols // GROUP)].view(rows, -1)
            y = torch.empty(rows, cols, dtype=dtype, device="cuda")
            for call in (lambda: ctx.sc_linear(sc.SC_ACT_RELU, x, w, y, q=kq, scales=ks), lambda: ctx.sc_checkpoint_pack(y, kq, ks)):
                call()
                assert bool((kept[rows * cols:] == 9).all()) and bool((marks[rows * -(-cols // GROUP):] == 9).all())


@pytest.mark.parametrize("cols", [1, 2, 4, 6, 12, 1002, 1004, 999])
@pytest.mark.parametrize("extra,offset", [(0, 0), (2, 2), (4, 4), (1, 0), (7, 8), (8, 4)])
def test_every_alignment_of_rows(ctx, cols, extra, offset):
    """Rows aligned to 2, 4, 8 and 16 bytes, dense or apart, in every elementwise operator and both products' epilogues."""
    rows = 37
    g = rng(cols + extra)
    for dtype in TYPES:
        x = normal(g, rows, cols).to(dtype)
        q, scales = sc.checkpoint_buffers(rows, cols)
        ctx.sc_checkpoint_pack(strided(x, extra, offset), q, scales)
        wq, ws, wv = checkpoint64(x, dtype)
        assert torch.equal(q.cpu(), wq) and torch.equal(scales.cpu(), ws)
        out = strided(torch.zeros_like(x), extra, offset)
        ctx.sc_checkpoint_unpack(q, scales, out)
        assert torch.equal(out.double().cpu(), wv)
        dz, ref = strided(torch.zeros_like(x), extra, offset), torch.empty(rows, cols, dtype=dtype, device="cuda")
        ctx.sc_activation_grad(sc.SC_ACT_SILU, strided(x, extra, offset), q, scales, dz)
        ctx.sc_activation_grad(sc.SC_ACT_SILU, x, q, scales, ref)
        assert torch.equal(dz, ref)
    check_linear(ctx, torch.bfloat16, "relu", rows, cols, 72, True, True, True, extra, offset)
    check_input_grad(ctx, torch.float16, "silu", rows, 40, cols, True, extra, offset)


def test_product_wait_runs_out_and_the_context_stays_usable():
    own = sc.Context(max_n=1)
    own.sc_debug_set_poll_limits(2000, 2000)
    own.sc_debug_wait_probe(2)
    assert own.sc_sync_status() == -5
    assert own.sc_sync_status() == 0
    check_linear(own, torch.bfloat16, "silu", 130, 264, 136, True, False, True)
    assert own.sc_sync_status() == 0
    own.close()


def test_a_closed_context_is_refused():
    own = sc.Context(max_n=1)
    own.close()
    x = torch.zeros(8, 64, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(sc.SparseCommError) as e:
        own.sc_linear(0, x, x, torch.zeros(8, 8, dtype=torch.bfloat16, device="cuda"))
    assert e.value.code == -1


def test_broadcast_and_transposed_inputs_are_refused(ctx):
    row = torch.zeros(1, 64, dtype=torch.bfloat16, device="cuda")
    y, w = torch.zeros(8, 32, dtype=torch.bfloat16, device="cuda"), torch.zeros(32, 64, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(TypeError):
        ctx.sc_linear(0, row.expand(8, 64), w, y)
    with pytest.raises(TypeError):
        ctx.sc_activation_grad(0, row.expand(8, 64), None, None, torch.zeros(8, 64, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(TypeError):
        ctx.sc_linear_grad_input(y, w.t().contiguous().t(), torch.zeros(8, 64, dtype=torch.bfloat16, device="cuda"))


# -- gradients against differences -----------------------------------------------------------------------------------
@pytest.mark.parametrize("act", ACTS[1:])
def test_gradients_against_differences(ctx, act):
    """L = sum(c * act(x W^T + b)) in 64 bits, differentiated by central differences along random directions.  The inputs are
    small multiples of powers of two, so that z and x are exactly what their checkpoints hold; what is left is the 16-bit
    rounding of dz and dx (2^-9 an element, at random: 2^-9 of the norm is a bound) and the difference's own error."""
    M, N, K = 48, 96, 64
    g = rng(77)
    bf = torch.bfloat16
    x = torch.randint(-4, 5, (M, K), generator=g, device="cuda").to(bf) / 4
    w = torch.randint(-2, 3, (N, K), generator=g, device="cuda").to(bf) / 8
    b = torch.randint(-3, 4, (N,), generator=g, device="cuda").to(bf) / 32 + 1 / 64      # keeps relu off its kink
    c = normal(g, M, N).to(bf)
    z = x.double() @ w.double().t() + b.double()
    assert bool((z * 64 == torch.round(z * 64)).all())
    qx, sx = sc.checkpoint_buffers(M, K)
    ctx.sc_checkpoint_pack(x, qx, sx)
    y = torch.empty(M, N, dtype=bf, device="cuda")
    qz, sz = sc.checkpoint_buffers(M, N)
    ctx.sc_linear(sc.ACTIVATIONS[act], x, w, y, bias=b, q=qz, scales=sz)
    held = torch.empty(M, N, device="cuda")
    ctx.sc_checkpoint_unpack(qz, sz, held)
    dz, db = torch.empty(M, N, dtype=bf, device="cuda"), torch.empty(N, device="cuda")
    ctx.sc_activation_grad(sc.ACTIVATIONS[act], c, qz, sz, dz, db)
    dx, dw = torch.empty(M, K, dtype=bf, device="cuda"), torch.empty(N, K, device="cuda")
    ctx.sc_linear_grad_input(dz, w, dx)
    ctx.sc_linear_grad_weight(dz, dw, q=qx, scales=sx)
    # where z needs more than the checkpoint's bits the loss is taken around the kept value
    shift = held.double() - z

    def loss(x_, w_, b_):
        return float((c.double() * act64(x_ @ w_.t() + b_ + shift, act)).sum())

    xd, wd, bd = x.double(), w.double(), b.double()
    h = 2.0 ** -12
    for seed in range(3):
        gg = rng(seed)
        ux, uw, ub = (torch.randn(t.shape, generator=gg, device="cuda").double() for t in (xd, wd, bd))
        for grad, plus, minus, norm, exact in (
                (dx, (xd + h * ux, wd, bd), (xd - h * ux, wd, bd), ux, False),
                (dw, (xd, wd + h * uw, bd), (xd, wd - h * uw, bd), uw, False),
                (db, (xd, wd, bd + h * ub), (xd, wd, bd - h * ub), ub, True)):
            got = float((grad.double() * norm).sum())
            want = (loss(*plus) - loss(*minus)) / (2 * h)
            bound = float(grad.double().norm() * norm.norm()) * (2.0 ** -16 if exact else 2.0 ** -8)
            if act == "relu":
                bound += 2.0 ** -6 * float(grad.double().norm() * norm.norm())     # kinks that the step crosses
            assert abs(got - want) <= bound, (act, seed, got, want, bound)


# -- refusals --------------------------------------------------------------------------------------------------------
def test_refusals(ctx):
    bf = torch.bfloat16
    new = lambda r, c, t=bf: torch.zeros(r, c, dtype=t, device="cuda")  # noqa: E731
    x, w, y = new(4, 64), new(32, 64), new(4, 32)
    q, scales = sc.checkpoint_buffers(4, 32)
    with pytest.raises(TypeError):
        ctx.sc_linear(0, x.float(), w.float(), y.float())
    with pytest.raises(TypeError):
        ctx.sc_linear(0, x, w.half(), y)
    with pytest.raises(TypeError):
        ctx.sc_linear(0, x.cpu(), w, y)
    with pytest.raises(TypeError):
        ctx.sc_linear(0, new(64, 4).t(), w, y)
    with pytest.raises(ValueError):
        ctx.sc_linear(0, x, new(32, 65), y)
    with pytest.raises(ValueError):
        ctx.sc_linear(0, x, w, new(4, 33))
    with pytest.raises(ValueError):
        ctx.sc_linear(0, x, w, y, bias=torch.zeros(31, dtype=bf, device="cuda"))
    with pytest.raises(ValueError):
        ctx.sc_linear(0, x, w, y, q=q)
    with pytest.raises(sc.SparseCommError) as e:
        ctx.sc_linear(9, x, w, y)
    assert e.value.code == -1
    with pytest.raises(ValueError):
        ctx.sc_checkpoint_pack(x, q, scales)
    with pytest.raises(ValueError):
        ctx.sc_linear_grad_weight(new(4, 32), torch.zeros(32, 64, device="cuda"))
    with pytest.raises(ValueError):
        ctx.sc_linear_grad_weight(new(4, 32), torch.zeros(32, 64, device="cuda"), x=x, q=q, scales=scales)
    with pytest.raises(TypeError):
        ctx.sc_linear_grad_weight(new(4, 32), new(32, 64), x=x)
    with pytest.raises(ValueError):
        ctx.sc_activation_grad(sc.SC_ACT_RELU, y, None, None, y)
    lib, h = sc.load_library(), ctx._h
    p = lambda t: t.data_ptr()  # noqa: E731
    before = y.fill_(4.0).clone()
    launches = ctx.launch_count
    bad = [(None, 0, 0, p(x), 64, p(w), 64, None, None, 0, 4, 32, 64, p(y), 32, None, None, None, -1),
           (h, 2, 0, p(x), 64, p(w), 64, None, None, 0, 4, 32, 64, p(y), 32, None, None, None, -6),
           (h, 0, 0, None, 64, p(w), 64, None, None, 0, 4, 32, 64, p(y), 32, None, None, None, -1),
           (h, 0, 0, p(x) + 1, 64, p(w), 64, None, None, 0, 4, 32, 64, p(y), 32, None, None, None, -1),
           (h, 0, 0, p(x), 63, p(w), 64, None, None, 0, 4, 32, 64, p(y), 32, None, None, None, -1),
           (h, 0, 0, p(x), 64, p(w), 64, None, None, 0, 1 << 31, 32, 64, p(y), 32, None, None, None, -2),
           (h, 0, 0, p(x), 64, p(w), 64, None, None, 0, 4, 32, 64, p(y), 32, p(q), None, None, -1),
           (h, 0, 0, p(x), 64, p(w), 64, None, None, 0, 4, 32, 64, None, 32, None, None, None, -1)]
    for *args, code in bad:
        assert lib.sc_linear(*args) == code, args
    dw = torch.zeros(32, 64, device="cuda")
    assert lib.sc_linear_grad_weight(h, 0, p(y), 32, None, 64, None, None, 4, 32, 64, p(dw), 64, 0, None) == -1
    assert lib.sc_linear_grad_weight(h, 0, p(y), 32, p(x), 64, None, None, 4, 32, 64, p(dw) + 2, 64, 0, None) == -1
    assert lib.sc_linear_grad_input(h, 0, 1, p(y), 32, p(w), 64, None, 0, None, None, 4, 32, 64, p(x), 64, None) == -1
    assert lib.sc_activation_grad(h, 0, 0, p(y), 32, None, None, 4, 32, None, 32, None, 0, None) == -1
    assert lib.sc_checkpoint_pack(h, 7, p(x), 64, 4, 64, p(q), p(scales), None) == -6
    assert lib.sc_checkpoint_unpack(h, 0, None, p(scales), 4, 32, p(y), 32, None) == -1
    assert lib.sc_layer_reserve(h, 1 << 31, 1, 1) == -2
    torch.cuda.synchronize()
    assert torch.equal(y, before) and ctx.launch_count == launches
