"""8-bit rows, norm and dropout between matrices that lie differently, and what lies around the matrices that they write.

Bytes, their values and dropout are made element by element: they are the same wherever rows begin.  A row of the norm and of its gradient is summed in an
order that its first operand's place decides, so these are compared only where that stays."""
import pytest
import torch

import paper_2009_09271_b200 as sc
from block_util import dropped64, rows_in_8_bits
from layer_util import assert_close

pytestmark = pytest.mark.gpu

EPS = 1e-5


@pytest.fixture(scope="module")
def ctx():
    c = sc.Context(max_n=1)
    yield c
    assert c.sc_sync_status() == 0
    c.close()


def rng(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


class Placed:
    """A matrix inside a storage whose every other element holds one value: rows `extra` elements further apart, the first one `offset` in."""

    def __init__(self, rows, cols, dtype, extra, offset, fill, values=None):
        self.store = torch.full((offset + rows * (cols + extra) + 32,), fill, device="cuda").to(dtype)
        self.at = self.store[offset:offset + rows * (cols + extra)].view(rows, cols + extra)[:, :cols]
        if values is not None:
            self.at.copy_(values)
        self.inside = torch.zeros_like(self.store, dtype=torch.bool)
        self.inside[offset:offset + rows * (cols + extra)].view(rows, cols + extra)[:, :cols] = True
        self.before = self.store.clone()

    def kept(self):
        """Nothing but the matrix has changed, before, between and behind its rows."""
        now, before = (t.masked_fill(self.inside, 0) for t in (self.store, self.before))
        return bool((now == before).all())


NAN = float("nan")
SIZES = [(3, 1), (9, 5), (40, 7), (5, 9), (2, 15), (70, 33), (9, 257), (30, 1001), (5, 4099), (3, 20001)]
PLACES = [(0, 0), (0, 1), (3, 2), (5, 3), (1, 4), (0, 5), (2, 6), (7, 7), (16, 8)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("rows,cols", SIZES + [(2, 40000)])
def test_eight_bit_rows_between_any_two_places(ctx, dtype, rows, cols):
    """Values at every offset to dense bytes, as fp32 parameters out of one flat vector are rounded; and the other way about."""
    g = rng(rows * 31 + cols)
    x = (torch.randn(rows, cols, generator=g, device="cuda") * torch.exp2(torch.randint(-9, 9, (rows, 1), generator=g, device="cuda").float())).to(dtype)
    wq, ws = (t.cuda() for t in rows_in_8_bits(x))
    values = (wq.float() * ws[:, None]).to(dtype)
    for i, place in enumerate(PLACES):
        for other in ((0, 0), PLACES[(i + 4) % len(PLACES)]):
            a, q = Placed(rows, cols, dtype, *place, NAN, x), Placed(rows, cols, torch.int8, *other, 77)
            scales = Placed(1, rows, torch.float32, 0, 1 + i % 3, 77)
            ctx.sc_quantize(a.at, q.at, scales.at[0])
            assert torch.equal(q.at, wq) and torch.equal(scales.at[0], ws) and q.kept() and scales.kept()
            for b, out in ((q, Placed(rows, cols, dtype, *place, 77)), (Placed(rows, cols, torch.int8, *place, 77, wq), Placed(rows, cols, dtype, *other, 77))):
                ctx.sc_dequantize(b.at, scales.at[0], out.at)
                assert torch.equal(out.at, values) and out.kept()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_dropout_between_any_places(ctx, dtype, rows, cols):
    g = rng(cols)
    x, r = (torch.randn(rows, cols, generator=g, device="cuda").to(dtype) for _ in range(2))
    dense = [torch.empty_like(x) for _ in range(2)]
    ctx.sc_dropout(x, dense[0], 0.3, 5)
    ctx.sc_dropout(x, dense[1], 0.3, 5, residual=r)
    want = dropped64(x, 5, 0.3)
    assert_close(dense[0], want, want.abs() * 2.0 ** -23, dtype, "y")
    assert_close(dense[1], want + r.double(), want.abs() * 2.0 ** -23 + (want + r.double()).abs() * 2.0 ** -24, dtype, "y with a residual")
    for i, place in enumerate(PLACES):
        for places in ((place, (0, 0), (0, 0)), ((0, 0), place, (0, 0)), ((0, 0), (0, 0), place), (place, PLACES[i - 1], PLACES[i - 3])):
            a, b = Placed(rows, cols, dtype, *places[0], NAN, x), Placed(rows, cols, dtype, *places[1], NAN, r)
            for add, ref in zip((None, b.at), dense):
                y = Placed(rows, cols, dtype, *places[2], 77)
                ctx.sc_dropout(a.at, y.at, 0.3, 5, residual=add)
                assert torch.equal(y.at, ref) and y.kept()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,cols", SIZES + [(2500, 1001), (2, 33001)])
def test_norm_and_its_gradient_keep_to_their_rows(ctx, dtype, rows, cols):
    """Results at any place are those of dense results of the same x (or dy); inputs lie among NaN, results among what has to stay."""
    g = rng(cols + 1)
    x, r, dy = (torch.randn(rows, cols, generator=g, device="cuda").to(dtype) for _ in range(3))
    gamma = Placed(1, cols, dtype, 0, 3, NAN, (1 + 0.2 * torch.randn(cols, generator=g, device="cuda")).to(dtype)[None])
    for i, place in enumerate(PLACES[:6]):
        places = [PLACES[(i + k) % len(PLACES)] for k in (1, 3, 5)]
        a, b, d = (Placed(rows, cols, dtype, *place, NAN, t) for t in (x, r, dy))
        h, y, q, scales = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x, dtype=torch.int8), torch.empty(rows, device="cuda")
        ctx.sc_rms_norm(a.at, gamma.at[0], EPS, y=y, q=q, scales=scales, residual=b.at, h=h, p=0.3, seed=9)
        assert bool(torch.isfinite(h).all() & torch.isfinite(y).all() & torch.isfinite(scales).all())
        results = [Placed(rows, cols, t, *p, 77) for t, p in zip((dtype, dtype, torch.int8), places)] + [Placed(1, rows, torch.float32, 0, 1, 77)]
        ctx.sc_rms_norm(a.at, gamma.at[0], EPS, y=results[1].at, q=results[2].at, scales=results[3].at[0], residual=b.at, h=results[0].at, p=0.3, seed=9)
        for got, want in zip(results, (h, y, q, scales[None])):
            assert torch.equal(got.at, want) and got.kept()
        dh, dx, dgamma = torch.empty_like(x), torch.empty_like(x), torch.empty(cols, device="cuda")
        ctx.sc_rms_norm_grad(d.at, a.at, gamma.at[0], EPS, dh, dgamma=dgamma, residual=b.at, dx=dx, p=0.3, seed=9)
        assert bool(torch.isfinite(dh).all() & torch.isfinite(dx).all() & torch.isfinite(dgamma).all())
        results = [Placed(rows, cols, dtype, *p, 77) for p in places[:2]] + [Placed(1, cols, torch.float32, 0, 3, 77)]
        ctx.sc_rms_norm_grad(d.at, a.at, gamma.at[0], EPS, results[0].at, dgamma=results[2].at[0], residual=b.at, dx=results[1].at, p=0.3, seed=9)
        for got, want in zip(results, (dh, dx, dgamma[None])):
            assert torch.equal(got.at, want) and got.kept()


@pytest.mark.parametrize("M,N,K", [(1, 40, 64), (5, 33, 47), (30, 65, 128), (40, 7, 129), (300, 131, 272)])
def test_product_keeps_to_its_rows(ctx, M, N, K):
    """Operands among bytes that are not theirs, results among what has to stay."""
    g = rng(K)
    x, w = (torch.randint(-127, 128, (n, K), generator=g, device="cuda").to(torch.int8) for n in (M, N))
    xs, ws = torch.rand(M, generator=g, device="cuda") / 64, torch.rand(N, generator=g, device="cuda") / 64
    r = torch.randn(M, N, generator=g, device="cuda").bfloat16()
    want, kept = torch.empty_like(r), sc.checkpoint_buffers(M, N)
    ctx.sc_linear_quantized(sc.SC_ACT_SILU, x, xs, w, ws, want, residual=r, q=kept[0], scales=kept[1])
    for i, place in enumerate(PLACES):
        other = PLACES[(i + 4) % len(PLACES)]
        a, b, c = Placed(M, K, torch.int8, *place, 77, x), Placed(N, K, torch.int8, *other, 77, w), Placed(M, N, torch.bfloat16, *place, NAN, r)
        y, q, s = Placed(M, N, torch.bfloat16, *other, 77), Placed(1, M * N, torch.int8, 0, 5, 77), Placed(1, kept[1].numel(), torch.uint8, 0, 3, 77)
        ctx.sc_linear_quantized(sc.SC_ACT_SILU, a.at, xs, b.at, ws, y.at, residual=c.at, q=q.at.view(M, N), scales=s.at.view(M, -1))
        assert torch.equal(y.at, want) and torch.equal(q.at.view(M, N), kept[0]) and torch.equal(s.at.view(M, -1), kept[1])
        assert y.kept() and q.kept() and s.kept()


@pytest.mark.parametrize("M", [1, 7, 30, 300])
@pytest.mark.parametrize("N,K", [(72, 400), (33, 129)])
def test_product_onto_its_residual(ctx, M, N, K):
    g = rng(M + N)
    x, w = (torch.randint(-127, 128, (n, K), generator=g, device="cuda").to(torch.int8) for n in (M, N))
    xs, ws = torch.rand(M, generator=g, device="cuda") / 64, torch.rand(N, generator=g, device="cuda") / 64
    r = torch.randn(M, N, generator=g, device="cuda").bfloat16()
    want = torch.empty_like(r)
    ctx.sc_linear_quantized(sc.SC_ACT_GELU, x, xs, w, ws, want, residual=r)
    for tile, parts in (((0, 0), 0), ((128, 64), 1), ((128, 128), 2), ((256, 256), 1)):
        ctx.sc_debug_layer_tiles(*tile, parts)
        for extra, offset in ((0, 0), (2, 2), (3, 1)):
            y = Placed(M, N, torch.bfloat16, extra, offset, 77, r)
            ctx.sc_linear_quantized(sc.SC_ACT_GELU, x, xs, w, ws, y.at, residual=y.at)
            assert torch.equal(y.at, want) and y.kept()
    ctx.sc_debug_layer_tiles()


@pytest.mark.parametrize("cols,ld", [(1000, 2 ** 30 + 8), (1001, 2 ** 30 + 9), (40001, 2 ** 30 + 8)])
def test_rows_further_apart_than_32_bits_reach(ctx, cols, ld):
    """Four rows, the last one 3 * 2^30 elements in: norm, gradient, dropout, 8-bit rows and a product, against the same rows close together and alike cut."""
    rows, g = 4, rng(cols)

    def far(values):
        t = torch.empty(3 * ld + cols, dtype=values.dtype, device="cuda").as_strided((rows, cols), (ld, 1))
        t.copy_(values)
        return t

    near = lambda values: Placed(rows, cols, values.dtype, (ld - cols) % 16, 0, 77, values).at  # noqa: E731
    x, r, gamma = (torch.randn(*s, generator=g, device="cuda").bfloat16() for s in ((rows, cols), (rows, cols), (cols,)))
    a, b, c, d = far(x), far(r), far(torch.zeros_like(x)), far(torch.zeros_like(x, dtype=torch.int8))
    na, nb, want, wq = near(x), near(r), near(torch.zeros_like(x)), near(torch.zeros_like(x, dtype=torch.int8))
    s, ws = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    ctx.sc_rms_norm(a, gamma, EPS, y=c, q=d, scales=s, residual=b, p=0.2, seed=3)
    ctx.sc_rms_norm(na, gamma, EPS, y=want, q=wq, scales=ws, residual=nb, p=0.2, seed=3)
    assert torch.equal(c, want) and torch.equal(d, wq) and torch.equal(s, ws)
    dgamma, wg = torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    ctx.sc_rms_norm_grad(b, a, gamma, EPS, c, dgamma=dgamma, residual=a, p=0.2, seed=3)
    ctx.sc_rms_norm_grad(nb, na, gamma, EPS, want, dgamma=wg, residual=na, p=0.2, seed=3)
    assert torch.equal(c, want) and torch.equal(dgamma, wg)
    ctx.sc_dropout(a, c, 0.3, 4, residual=b)
    ctx.sc_dropout(na, want, 0.3, 4, residual=nb)
    assert torch.equal(c, want)
    ctx.sc_quantize(b, d, s)
    ctx.sc_dequantize(d, s, c)
    q, ref = rows_in_8_bits(r)
    assert torch.equal(d.cpu(), q) and torch.equal(s.cpu(), ref) and torch.equal(c.cpu(), (q.float() * ref[:, None]).bfloat16())
    w, y = q.cuda(), [torch.empty(rows, rows, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    ctx.sc_linear_quantized(sc.SC_ACT_NONE, d, s, w, s, y[0])
    ctx.sc_linear_quantized(sc.SC_ACT_NONE, w, s, d, s, y[1])
    exact = (w.double() @ w.double().t()) * s.double()[:, None] * s.double()
    for got in y:
        assert_close(got, exact, exact.abs() * 4 * 2.0 ** -24, torch.bfloat16, "product")
