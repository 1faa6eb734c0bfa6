"""Root-mean-square norm forward and backward, and dropout, against 64-bit statements.

A row's sum of squares goes through block_util.depth() additions, each off by at most 2^-24 of the sum so far (all terms are positive);
the root halves that.  h is made by two fp32 operations."""
import numpy as np
import pytest
import torch

import paper_2009_09271_b200 as sc
from block_util import SALT_DROPOUT, depth, dropped64, kept_mask, mix64, norm64, norm_grad64, rows_in_8_bits
from layer_util import assert_close, strided

pytestmark = pytest.mark.gpu

TYPES = (torch.bfloat16, torch.float16)
EPS = 1e-5
SIZES = [(1, 1), (1, 8), (3, 7), (2, 257), (33, 64), (5, 1000), (70, 1001), (2, 1024), (9, 2050), (1, 4096), (300, 520), (3, 8200), (2, 16391), (1, 70001)]
LAYOUTS = [(0, 0), (8, 8), (3, 1), (2, 2), (4, 12)]


@pytest.fixture(scope="module")
def ctx():
    c = sc.Context(max_n=1)
    yield c
    assert c.sc_sync_status() == 0
    c.close()


def rng(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def inputs(dtype, rows, cols, extra=0, offset=0):
    g = rng(rows * 131 + cols)
    loud = torch.where(torch.rand(cols, generator=g, device="cuda") < 0.02, 9.0, 1.0)
    x, r = (strided((normal(g, rows, cols) * loud).to(dtype), extra, offset) for _ in range(2))
    return x, r, (1 + 0.2 * normal(g, cols)).to(dtype), g


def check_norm(ctx, dtype, rows, cols, residual, p, extra=0, offset=0, x=None, eps=EPS):
    given, r, gamma, _ = inputs(dtype, rows, cols, extra, offset)
    x = given if x is None else x
    r = r if residual else None
    new = lambda t=dtype: strided(torch.zeros(rows, cols, device="cuda").to(t), extra, offset)  # noqa: E731
    h, y, q, scales = new(), new(), new(torch.int8), torch.empty(rows, device="cuda")
    seed = rows * 65537 + cols
    ctx.sc_rms_norm(x, gamma, eps, y=y, q=q, scales=scales, residual=r, h=h, p=p, seed=seed)
    wh, wy = norm64(x, r, gamma, eps, seed, p)
    h_slack = (wh.abs() + (wh - (0 if r is None else r.double())).abs()) * 2.0 ** -24
    assert_close(h, wh, h_slack, dtype, "h")
    rms = (wh * wh).mean(1, keepdim=True).add(eps).sqrt()
    # an error of h enters y directly and through the norm, by at most its share of it
    y_slack = wy.abs() * depth(cols) * 2.0 ** -24 + gamma.double().abs() * (h_slack + wh.abs() * (h_slack / rms).amax(1, keepdim=True)) / rms
    assert_close(y, wy, y_slack, dtype, "y")
    top = wy.abs().amax(1)
    assert bool(((scales.double() * 127 - top).abs() <= top * 2.0 ** -22 + y_slack.amax(1)).all())
    step = scales.double()[:, None]
    assert bool(((q.double() * step - wy).abs() <= step * 0.5 + y_slack + 127 * step * 2.0 ** -22).all())
    assert int(q.abs().max()) == 127 or not bool(top.any())
    # the outputs one at a time are the same
    for name in ("y", "q"):
        only = {"y": new()} if name == "y" else {"q": new(torch.int8), "scales": torch.empty(rows, device="cuda")}
        ctx.sc_rms_norm(x, gamma, eps, residual=r, p=p, seed=seed, **only)
        assert torch.equal(only[name], y if name == "y" else q)
    return h, y


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("residual,p", [(False, 0.0), (True, 0.0), (True, 0.25), (False, 0.1)])
def test_norm(ctx, dtype, rows, cols, residual, p):
    check_norm(ctx, dtype, rows, cols, residual, p)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("extra,offset", LAYOUTS[1:])
@pytest.mark.parametrize("rows,cols", [(5, 264), (70, 1001), (3, 4098), (2, 16400)])
def test_norm_strides(ctx, dtype, extra, offset, rows, cols):
    check_norm(ctx, dtype, rows, cols, True, 0.5, extra, offset)


@pytest.mark.parametrize("cols", [40, 1001, 4096, 20000])
def test_norm_in_place(ctx, cols):
    x, r, gamma, _ = inputs(torch.bfloat16, 37, cols)
    h, y = torch.empty_like(x), torch.empty_like(x)
    ctx.sc_rms_norm(x, gamma, EPS, y=y, residual=r, h=h, p=0.3, seed=5)
    a, b = x.clone(), r.clone()
    ctx.sc_rms_norm(a, gamma, EPS, y=a, residual=b, h=b, p=0.3, seed=5)
    assert torch.equal(a, y) and torch.equal(b, h)
    a, b = x.clone(), r.clone()
    ctx.sc_rms_norm(a, gamma, EPS, y=b, residual=b, h=a, p=0.3, seed=5)
    assert torch.equal(b, y) and torch.equal(a, h)


@pytest.mark.parametrize("cols", [40, 1001, 4096, 20000])
def test_norm_rows_that_are_zero_or_not_finite(ctx, cols):
    """Each such row is on its own; zeros give zeros, what is not finite gives NaN in y and in the scale."""
    dtype = torch.bfloat16
    x, _, gamma, _ = inputs(dtype, 9, cols)
    clean = x.clone()
    x[2], x[4, cols // 2], x[5, cols - 1], x[7] = 0.0, float("inf"), float("nan"), 3e38
    y, q, scales = torch.empty_like(x), torch.empty(9, cols, dtype=torch.int8, device="cuda"), torch.empty(9, device="cuda")
    ctx.sc_rms_norm(x, gamma, EPS, y=y, q=q, scales=scales)
    lost = [4, 5, 7]
    fine = [0, 1, 3, 6, 8]
    assert bool(torch.isnan(y[lost]).all()) and bool(torch.isnan(scales[lost]).all()) and not bool(q[lost].any())
    assert not bool(y[2].any()) and scales[2] == 0 and not bool(q[2].any())
    want, wq, ws = torch.empty_like(x), torch.empty_like(q), torch.empty_like(scales)
    ctx.sc_rms_norm(clean, gamma, EPS, y=want, q=wq, scales=ws)
    assert torch.equal(y[fine], want[fine]) and torch.equal(q[fine], wq[fine]) and torch.equal(scales[fine], ws[fine])
    # dropped elements are 0 whatever they were
    mask, _ = kept_mask(3, 9, cols, 0.5)
    x = torch.where(mask.cuda(), clean, torch.full_like(clean, float("nan")))
    h, h2, y2 = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    ctx.sc_rms_norm(x, gamma, EPS, y=y, h=h, p=0.5, seed=3)
    ctx.sc_rms_norm(clean, gamma, EPS, y=y2, h=h2, p=0.5, seed=3)
    assert torch.equal(h, h2) and torch.equal(y, y2)


@pytest.mark.parametrize("scale", [2.0 ** -30, 2.0 ** 30])
def test_norm_of_small_and_large_rows(ctx, scale):
    x, _, _, _ = inputs(torch.bfloat16, 4, 1000)
    check_norm(ctx, torch.bfloat16, 4, 1000, False, 0.0, x=(x.float() * scale).to(torch.bfloat16), eps=1e-6)
    if scale > 1:
        check_norm(ctx, torch.bfloat16, 4, 1000, False, 0.0, x=(x.float() * scale).to(torch.bfloat16), eps=0.0)


@pytest.mark.parametrize("cols", [40, 1001, 4096, 20000])
def test_norm_to_8_bits_where_h_gamma_is_next_to_the_smallest_numbers(ctx, cols):
    """The largest h gamma is 2^-121.6, and 127 over it no fp32 number; the row itself is around 2^-72.  Elements of 2^-6 and more of the largest
    are normal numbers, the others are off by 2^-150, 2^-28 of the largest, at most."""
    g = rng(cols)
    x = torch.randint(-80, 81, (3, cols), generator=g, device="cuda").to(torch.bfloat16) * 2.0 ** -56
    x[:, 0], x[:, 1] = 80 * 2.0 ** -56, 0.0
    gamma = torch.full((cols,), 2.0 ** -72, device="cuda", dtype=torch.bfloat16)
    _, wy = norm64(x, None, gamma, 0.0)
    y, q, only, scales = torch.empty_like(x), torch.empty_like(x, dtype=torch.int8), torch.empty_like(x, dtype=torch.int8), torch.empty(3, device="cuda")
    ctx.sc_rms_norm(x, gamma, 0.0, q=only, scales=scales)
    ctx.sc_rms_norm(x, gamma, 0.0, y=y, q=q, scales=scales)
    assert torch.equal(q, only) and bool((q[:, 0] == 127).all()) and bool((q[:, 1] == 0).all())
    slack, step = wy.abs() * depth(cols) * 2.0 ** -24 + wy.abs().amax(1, keepdim=True) * 2.0 ** -28, scales.double()[:, None]
    assert bool(((q.double() * step - wy).abs() <= step * 0.5 + slack + 127 * step * 2.0 ** -22).all())
    assert_close(y, wy, slack, torch.bfloat16, "y")


# -- backward --------------------------------------------------------------------------------------------------------
def check_grad(ctx, dtype, rows, cols, residual, p, extra=0, offset=0, eps=EPS):
    h, r, gamma, g = inputs(dtype, rows, cols, extra, offset)
    r = r if residual else None
    dy = strided((normal(g, rows, cols) * 0.1).to(dtype), extra, offset)
    dh, dx = (strided(torch.zeros(rows, cols, device="cuda").to(dtype), extra, offset) for _ in range(2))
    row = torch.full((cols + 9,), 5.0, device="cuda")
    dgamma, seed = row[offset % 4:offset % 4 + cols], rows * 77 + cols
    ctx.sc_rms_norm_grad(dy, h, gamma, eps, dh, dgamma=dgamma, residual=r, dx=dx, p=p, seed=seed)
    (wh, wg), (h_slack, g_slack) = norm_grad64(dy, h, gamma, eps, r)
    assert_close(dh, wh, h_slack, dtype, "dh")
    assert_close(dgamma, wg, g_slack, torch.float32, "dgamma")
    if p:
        assert_close(dx, dropped64(wh, seed, p), dropped64(h_slack + wh.abs() * 2.0 ** -23, seed, p), dtype, "dx")
    else:
        assert torch.equal(dx, dh)
    guard = row.clone()
    guard[offset % 4:offset % 4 + cols] = 5.0
    assert bool((guard == 5.0).all())
    first = dgamma.clone()
    ctx.sc_rms_norm_grad(dy, h, gamma, eps, dgamma=dgamma, accumulate=True)
    assert torch.equal(dgamma, first + first)                         # the same sums every time, in the same order
    only = torch.zeros_like(dh)
    ctx.sc_rms_norm_grad(dy, h, gamma, eps, only, residual=r)
    assert torch.equal(only, dh)
    ctx.sc_rms_norm_grad(dy, h, gamma, eps, dx=only, residual=r, p=p, seed=seed)
    assert torch.equal(only, dx)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", SIZES + [(1021, 72), (2500, 8), (4100, 1000)])
@pytest.mark.parametrize("residual,p", [(False, 0.0), (True, 0.0), (True, 0.25)])
def test_norm_grad(ctx, dtype, rows, cols, residual, p):
    check_grad(ctx, dtype, rows, cols, residual, p)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("extra,offset", LAYOUTS[1:])
@pytest.mark.parametrize("rows,cols", [(5, 264), (170, 1001), (3, 4098), (2, 16400)])
def test_norm_grad_strides(ctx, dtype, extra, offset, rows, cols):
    check_grad(ctx, dtype, rows, cols, True, 0.5, extra, offset)


@pytest.mark.parametrize("cols", [40, 1001, 4096, 20000])
def test_norm_grad_in_place(ctx, cols):
    h, r, gamma, g = inputs(torch.float16, 41, cols)
    dy = (normal(g, 41, cols) * 0.1).half()
    dh, dx, dgamma = torch.empty_like(h), torch.empty_like(h), torch.empty(cols, device="cuda")
    ctx.sc_rms_norm_grad(dy, h, gamma, EPS, dh, dgamma=dgamma, residual=r, dx=dx, p=0.3, seed=5)
    for a, b in (("dy", "h"), ("r", "dy"), ("h", "r")):
        given = {"dy": dy.clone(), "h": h.clone(), "r": r.clone()}
        sums = torch.empty_like(dgamma)
        ctx.sc_rms_norm_grad(given["dy"], given["h"], gamma, EPS, given[a], dgamma=sums, residual=given["r"], dx=given[b], p=0.3, seed=5)
        assert torch.equal(given[a], dh) and torch.equal(given[b], dx) and torch.equal(sums, dgamma)


def test_norm_grad_by_differences(ctx):
    """The gradient of sum(c y) by central differences of the 64-bit forward formula, at a few elements and for every gamma."""
    rows, cols = 3, 24
    x, _, gamma, g = inputs(torch.float16, rows, cols)
    c = normal(g, rows, cols).half()
    dh, dgamma = torch.empty_like(x), torch.empty(cols, device="cuda")
    ctx.sc_rms_norm_grad(c, x, gamma, EPS, dh, dgamma=dgamma)
    step = 1e-4

    def loss(xv, gv):
        r = ((xv * xv).mean(1, keepdim=True) + EPS).rsqrt()
        return (c.double() * xv * r * gv).sum()

    for i in range(rows):
        for j in range(0, cols, 5):
            at = torch.zeros(rows, cols, dtype=torch.float64, device="cuda")
            at[i, j] = step
            want = float(loss(x.double() + at, gamma.double()) - loss(x.double() - at, gamma.double())) / (2 * step)
            assert abs(float(dh[i, j]) - want) <= 2.0 ** -11 * abs(want) + 1e-5
    for j in range(cols):
        at = torch.zeros(cols, dtype=torch.float64, device="cuda")
        at[j] = step
        want = float(loss(x.double(), gamma.double() + at) - loss(x.double(), gamma.double() - at)) / (2 * step)
        assert abs(float(dgamma[j]) - want) <= 1e-5


def test_norm_empty_sizes(ctx):
    bf = torch.bfloat16
    new = lambda r, c: torch.full((r, c), 3.0, dtype=bf, device="cuda")  # noqa: E731
    launches = ctx.launch_count
    for rows, cols in ((0, 8), (4, 0), (0, 0)):
        x, gamma = new(rows, cols), torch.ones(cols, dtype=bf, device="cuda")
        ctx.sc_rms_norm(x, gamma, EPS, y=new(rows, cols), h=new(rows, cols), residual=x, p=0.5)
        ctx.sc_dropout(x, new(rows, cols), 0.5, 1)
        for accumulate in (False, True):
            dgamma = torch.full((cols,), 7.0, device="cuda")
            ctx.sc_rms_norm_grad(x, x, gamma, EPS, new(rows, cols), dgamma=dgamma, accumulate=accumulate)
            assert bool((dgamma == (7.0 if accumulate else 0.0)).all())
    assert ctx.launch_count == launches


# -- dropout ---------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("p", [0.0, 1e-6, 0.1, 0.5, 0.999, 1.0])
@pytest.mark.parametrize("rows,cols,extra,offset", [(1, 1, 0, 0), (3, 7, 0, 0), (70, 1001, 0, 0), (64, 1024, 8, 8), (5, 4098, 2, 2), (33, 260, 3, 1), (1, 70001, 0, 0)])
def test_dropout(ctx, dtype, p, rows, cols, extra, offset):
    x, r, _, _ = inputs(dtype, rows, cols, extra, offset)
    seed = (1 << 63) + rows * 31 + cols
    y = strided(torch.zeros(rows, cols, device="cuda").to(dtype), extra, offset)
    ctx.sc_dropout(x, y, p, seed)
    want = dropped64(x, seed, p)
    assert_close(y, want, want.abs() * 2.0 ** -23, dtype, "y")
    assert bool((y[want == 0] == 0).all())
    if p <= 1e-6:
        assert torch.equal(y, x)                                       # the cut is 0: nothing is dropped or scaled
    ctx.sc_dropout(x, y, p, seed, residual=r)
    assert_close(y, want + r.double(), want.abs() * 2.0 ** -23 + (want + r.double()).abs() * 2.0 ** -24, dtype, "y with a residual")
    a, b = x.clone(), r.clone()
    ctx.sc_dropout(a, a, p, seed, residual=r)
    ctx.sc_dropout(x, b, p, seed, residual=b)
    assert torch.equal(a, y) and torch.equal(b, y)


def test_dropout_statistics(ctx):
    """The share of what is kept is 1 - p within five standard deviations, over all, by column and from one seed to the next."""
    rows, cols, p = 4096, 1024, 0.3
    x, y = torch.ones(rows, cols, dtype=torch.float16, device="cuda"), torch.empty(rows, cols, dtype=torch.float16, device="cuda")
    masks = []
    for seed in (1, 2, 1 << 40):
        ctx.sc_dropout(x, y, p, seed)
        masks.append(y != 0)
        off = (masks[-1].double().mean(0) - (1 - p)).abs()
        assert float(off.max()) <= 5.5 * (p * (1 - p) / rows) ** 0.5
        assert abs(float(masks[-1].double().mean()) - (1 - p)) <= 5 * (p * (1 - p) / rows / cols) ** 0.5
    both = (masks[0] & masks[1]).double().mean()
    assert abs(float(both) - (1 - p) ** 2) <= 5 * (0.25 / rows / cols) ** 0.5


def test_dropout_offsets_past_32_bits(ctx):
    rows, cols = 3, (1 << 31) - 32
    x = torch.ones(rows, cols, dtype=torch.bfloat16, device="cuda")
    ctx.sc_dropout(x, x, 0.5, 9)
    mask, _ = kept_mask(9, 1, cols // 64, 0.5)                          # the first columns of row 0
    assert torch.equal(x[0, :cols // 64].cpu() != 0, mask[0])
    per_row = cols // 4
    words = mix64(mix64(9, SALT_DROPOUT), np.arange(3 * per_row - 1024, 3 * per_row, dtype=np.uint64))
    bits = np.stack([(words >> np.uint64(16 * i)) & np.uint64(0xFFFF) for i in range(4)], 1).reshape(-1)
    assert torch.equal(x[2, -4096:].cpu() != 0, torch.from_numpy(bits >= 32768))
    assert bool(((x[1, :4096] == 0) | (x[1, :4096] == 2)).all())


def test_refusals(ctx):
    bf = torch.bfloat16
    x, y, gamma = torch.ones(6, 32, dtype=bf, device="cuda"), torch.ones(6, 32, dtype=bf, device="cuda"), torch.ones(32, dtype=bf, device="cuda")
    q, s, f = torch.zeros(6, 32, dtype=torch.int8, device="cuda"), torch.zeros(6, device="cuda"), torch.zeros(32, device="cuda")
    launches = ctx.launch_count
    norm, grad, drop = ctx.sc_rms_norm, ctx.sc_rms_norm_grad, ctx.sc_dropout
    nan = float("nan")
    for call in (lambda: norm(x, gamma, EPS), lambda: norm(x, gamma, EPS, h=y), lambda: norm(x.float(), gamma, EPS, y=y), lambda: norm(x, f, EPS, y=y),
                 lambda: norm(x, gamma[:31], EPS, y=y), lambda: norm(x, gamma, -1.0, y=y), lambda: norm(x, gamma, nan, y=y), lambda: norm(x, gamma, float("inf"), y=y),
                 lambda: norm(x, gamma, EPS, y=y.half()), lambda: norm(x, gamma, EPS, y=y[:5]), lambda: norm(x, gamma, EPS, q=q), lambda: norm(x, gamma, EPS, scales=s),
                 lambda: norm(x, gamma, EPS, q=q, scales=s[:5]), lambda: norm(x, gamma, EPS, y=y, p=1.5), lambda: norm(x, gamma, EPS, y=y, p=-0.1),
                 lambda: norm(x, gamma, EPS, y=y, p=nan), lambda: norm(x, gamma, EPS, y=y, residual=x.cpu()), lambda: norm(x, gamma.cpu(), EPS, y=y),
                 lambda: norm(x[0], gamma, EPS, y=y), lambda: norm(x, gamma, EPS, y=y.t()), lambda: norm(x, gamma, EPS, y=y, h=y[:, ::2]),
                 lambda: grad(x, y, gamma, EPS), lambda: grad(x, y, gamma, EPS, x, dgamma=gamma), lambda: grad(x, y[:5], gamma, EPS, x),
                 lambda: grad(x, y, gamma, -EPS, x), lambda: grad(x, y, gamma, EPS, x, p=2), lambda: grad(x, y, gamma, EPS, x.half()),
                 lambda: grad(x, y, gamma, EPS, x, residual=x[:, :31]), lambda: grad(x, y, gamma, EPS, x, dgamma=f[:31]),
                 lambda: drop(x, y, 1.01, 0), lambda: drop(x, y, nan, 0), lambda: drop(x, y[:5], 0.1, 0), lambda: drop(x.float(), y, 0.1, 0),
                 lambda: drop(x, y, 0.1, 0, residual=f), lambda: drop(x, y.cpu(), 0.1, 0)):
        with pytest.raises((TypeError, ValueError, sc.SparseCommError)):
            call()
    assert ctx.launch_count == launches


@pytest.mark.parametrize("rows,cols", [(9, 264), (40, 1001), (300, 1000), (5, 2050), (3, 4099), (1, 9)])
@pytest.mark.parametrize("which", ["x", "residual", "gamma", "out", "8 bits"])
def test_rows_of_several_alignments(ctx, rows, cols, which):
    """One operand lies apart from the others: the results are those of dense ones, bit for bit where only a result lies apart."""
    x, r, gamma, g = inputs(torch.bfloat16, rows, cols)
    new = lambda t=x.dtype: torch.zeros(rows, cols, device="cuda").to(t)  # noqa: E731
    apart = lambda t: strided(t, 3, 5)  # noqa: E731
    want = {"h": new(), "y": new(), "q": new(torch.int8), "scales": torch.empty(rows, device="cuda")}
    ctx.sc_rms_norm(x, gamma, EPS, residual=r, p=0.3, seed=5, **want)
    given = {"h": new(), "y": new(), "q": new(torch.int8), "scales": torch.empty(rows, device="cuda")}
    if which == "out":
        given["h"], given["y"] = apart(given["h"]), strided(given["y"], 1, 2)
    if which == "8 bits":
        given["q"] = apart(given["q"])
    xs, rs = (apart(x) if which == "x" else x), (apart(r) if which == "residual" else r)
    gs = strided(gamma.view(1, -1), 0, 3).view(-1) if which == "gamma" else gamma
    ctx.sc_rms_norm(xs, gs, EPS, residual=rs, p=0.3, seed=5, **given)
    wh, wy = norm64(x, r, gamma, EPS, 5, 0.3)
    assert torch.equal(given["h"], want["h"])                          # elementwise: no sums
    assert bool(((given["y"].double() - want["y"].double()).abs() <= wy.abs() * (2.0 ** -7 + depth(cols) * 2.0 ** -23) + 1e-30).all())
    if which in ("out", "8 bits"):
        assert all(torch.equal(given[k], want[k]) for k in want)
    assert int((given["q"].int() - want["q"].int()).abs().max()) <= 1

    dy = (normal(g, rows, cols) * 0.1).to(x.dtype)
    outs = [{"dh": new(), "dx": new(), "dgamma": torch.empty(cols, device="cuda")} for _ in range(2)]
    ctx.sc_rms_norm_grad(dy, x, gamma, EPS, residual=r, p=0.3, seed=5, **outs[0])
    if which == "out":
        outs[1]["dh"], outs[1]["dx"] = apart(outs[1]["dh"]), strided(outs[1]["dx"], 1, 2)
    ctx.sc_rms_norm_grad(apart(dy) if which == "8 bits" else dy, xs, gs, EPS, residual=rs, p=0.3, seed=5, **outs[1])
    (dh, dg), (dh_slack, dg_slack) = norm_grad64(dy, x, gamma, EPS, r)
    for o in outs:
        assert_close(o["dh"], dh, dh_slack, x.dtype, "dh")
        assert_close(o["dgamma"], dg, dg_slack, torch.float32, "dgamma")
        assert_close(o["dx"], dropped64(dh, 5, 0.3), dropped64(dh_slack + dh.abs() * 2.0 ** -23, 5, 0.3), x.dtype, "dx")

    y, z = new(), apart(new())
    ctx.sc_dropout(x, y, 0.3, 5, residual=r)
    ctx.sc_dropout(xs, z if which == "out" else y.clone().copy_(y), 0.3, 5, residual=rs)
    if which == "out":
        assert torch.equal(z, y)


@pytest.mark.parametrize("cols", [1, 2, 5, 6, 7, 9, 15])
@pytest.mark.parametrize("rows", [1, 2, 3, 8, 9, 40])
def test_short_rows_and_their_neighbours(ctx, rows, cols):
    """Rows shorter than an access: what lies before, between and behind them is neither read nor written."""
    for dtype in TYPES:
        check_norm(ctx, dtype, rows, cols, True, 0.3, 0, 1)
        check_grad(ctx, dtype, rows, cols, True, 0.3, 0, 3)
        x, r, gamma, _ = inputs(dtype, rows, cols, 3, 5)
        store = torch.full((rows * (cols + 3) + 40,), float("nan"), device="cuda").to(dtype)

        def among_nan(t):
            v = store.clone()[5:5 + rows * (cols + 3)].view(rows, cols + 3)[:, :cols]
            v.copy_(t)
            return v

        a, b = among_nan(x), among_nan(r)
        y, h, z = (among_nan(torch.zeros_like(x)) for _ in range(3))
        ctx.sc_rms_norm(a, gamma, EPS, y=y, h=h, residual=b, p=0.3, seed=2)
        want_h, want_y = torch.empty(rows, cols, dtype=dtype, device="cuda"), torch.empty(rows, cols, dtype=dtype, device="cuda")
        ctx.sc_rms_norm(x.contiguous(), gamma, EPS, y=want_y, h=want_h, residual=r.contiguous(), p=0.3, seed=2)
        assert torch.equal(h, want_h) and bool(torch.isfinite(y).all())
        ctx.sc_dropout(a, z, 0.3, 2, residual=b)
        assert torch.equal(z, want_h)
        for t in (y, h, z):                                             # the rest of the storage is as it was
            whole = t.as_strided((rows * (cols + 3) + 40 - 5,), (1,), 5)
            outside = torch.ones(whole.shape, dtype=torch.bool, device="cuda")
            outside[:rows * (cols + 3)].view(rows, cols + 3)[:, :cols] = False
            assert bool(torch.isnan(whole[outside]).all())


# -- rows as long as a kernel's threads hold, and their ends ----------------------------------------------------------------
LONGEST = [(9, 255), (9, 263), (9, 519), (9, 1031), (2500, 1031), (5, 2055), (5, 4103), (3, 8199), (2, 16391), (2, 16399), (1, 32775), (1, 32776)]


@pytest.mark.parametrize("extra,offset", [(0, 0), (3, 1)])
@pytest.mark.parametrize("rows,cols", LONGEST)
def test_longest_rows_of_each_kernel(ctx, rows, cols, extra, offset):
    check_norm(ctx, torch.bfloat16, rows, cols, True, 0.25, extra, offset)
    check_grad(ctx, torch.float16, rows, cols, True, 0.25, extra, offset)
    g = rng(cols)
    x = strided(normal(g, rows, cols).bfloat16(), extra, offset)
    y = strided(torch.zeros(rows, cols, device="cuda").bfloat16(), extra, offset)
    ctx.sc_dropout(x, y, 0.3, 11)
    mask, scale = kept_mask(11, rows, cols, 0.3)
    want = torch.where(mask.cuda(), x.float() * np.float32(scale), torch.zeros((), device="cuda")).bfloat16()
    assert torch.equal(y, want)
    q, scales = strided(torch.zeros(rows, cols, device="cuda").to(torch.int8), extra, offset), torch.empty(rows, device="cuda")
    ctx.sc_quantize(x, q, scales)
    wq, ws = rows_in_8_bits(x)
    assert torch.equal(q.cpu(), wq) and torch.equal(scales.cpu(), ws)
    ctx.sc_dequantize(q, scales, y)
    assert torch.equal(y, (q.float() * scales[:, None]).bfloat16())


def test_one_row_as_long_as_sizes_go(ctx):
    """2^31 - 1 columns that begin off a boundary: both ends, and the middle, of dropout and of 8-bit rows there and back."""
    cols = 2 ** 31 - 1
    base = torch.empty(cols + 1, device="cuda", dtype=torch.bfloat16).normal_(generator=rng(1))
    x, y = base[1:].view(1, cols), torch.zeros(cols + 1, device="cuda", dtype=torch.bfloat16)
    y[0] = 7.0
    places = [slice(c, c + 4096) for c in (0, 2 ** 30 - 2048, cols - 4096 - cols % 4)] + [slice(cols - cols % 4 - 4, cols)]
    ctx.sc_dropout(x, y[1:].view(1, cols), 0.5, 3)
    assert float(y[0]) == 7.0
    key = mix64(3, SALT_DROPOUT)
    for s in places:
        words = mix64(key, np.arange(s.start // 4, -(-s.stop // 4), dtype=np.uint64))
        bits = np.stack([(words >> np.uint64(16 * i)) & np.uint64(0xFFFF) for i in range(4)], 1).reshape(-1)[:s.stop - s.start]
        kept = torch.from_numpy(bits >= np.uint64(32768)).cuda()
        assert torch.equal(y[1:][s], torch.where(kept, x[0, s] * 2, torch.zeros_like(x[0, s])))
    q, scales = torch.zeros(1, cols, device="cuda", dtype=torch.int8), torch.empty(1, device="cuda")
    ctx.sc_quantize(x, q, scales)
    top = torch.maximum(x.max(), -x.min()).float()
    assert float(scales) == float(top / torch.full_like(top, 127.0))
    ctx.sc_dequantize(q, scales, y[1:].view(1, cols))
    for s in places:
        want = torch.round(x[0, s].float() * (127 * (1 / top)))
        assert torch.equal(q[0, s].float(), want)
        assert torch.equal(y[1:][s], (want * scales).bfloat16())
