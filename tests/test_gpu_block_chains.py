"""The norm, dropout and 8-bit operators as they are used: call after call without a wait between, captured and replayed, on another stream, and
through the compiled caller and without it.  The same calls with a wait after each are the reference; what they compute is tested elsewhere."""
import numpy as np
import pytest
import torch

import paper_2009_09271_b200 as sc

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


@pytest.fixture(scope="module")
def ctx():
    c = sc.Context(max_n=1)
    c.sc_layer_reserve(3000, 1040, 1040)
    yield c
    assert c.sc_sync_status() == 0
    c.close()


def normal(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(BF16)


class Block:
    """One block's forward and backward pass on buffers of its own; every result is kept."""

    def __init__(self, ctx, M, N, K, seed):
        self.ctx, self.M = ctx, M
        new = lambda r, c, t=BF16: torch.empty(r, c, dtype=t, device="cuda")  # noqa: E731
        self.x, self.res, self.gamma = normal(seed, M, K), normal(seed + 1, M, K), normal(seed + 2, K)
        self.w, self.bias, self.dy = (normal(seed + 3, N, K).float() / K ** 0.5).to(BF16), normal(seed + 4, N), normal(seed + 5, M, N)
        self.h, self.q, self.w8, self.z = new(M, K), sc.quantized_buffers(M, K), sc.quantized_buffers(N, K), sc.checkpoint_buffers(M, N)
        self.y, self.y8, self.back, self.dropped = new(M, N), sc.quantized_buffers(M, N), new(M, N), new(M, N)
        self.dz, self.held, self.dw, self.dn, self.dh, self.dx = new(M, N), new(M, K), new(N, K, torch.float32), new(M, K), new(M, K), new(M, K)
        self.dgamma = torch.empty(K, device="cuda")

    def calls(self, stream=None):
        c, at = self.ctx, {"stream": stream}
        yield lambda: c.sc_quantize(self.w, *self.w8, **at)
        yield lambda: c.sc_rms_norm(self.x, self.gamma, 1e-5, q=self.q[0], scales=self.q[1], residual=self.res, h=self.h, p=0.2, seed=7, **at)
        yield lambda: c.sc_linear_quantized(sc.SC_ACT_SILU, *self.q, *self.w8, self.y, bias=self.bias, q=self.z[0], scales=self.z[1], **at)
        yield lambda: c.sc_quantize(self.y, *self.y8, **at)
        yield lambda: c.sc_dequantize(*self.y8, self.back, **at)
        yield lambda: c.sc_dropout(self.back, self.dropped, 0.3, 11, residual=self.y, **at)
        yield lambda: c.sc_activation_grad(sc.SC_ACT_SILU, self.dy, *self.z, self.dz, **at)
        yield lambda: c.sc_dequantize(*self.q, self.held, **at)
        yield lambda: c.sc_linear_grad_weight(self.dz, self.dw, x=self.held, **at)
        yield lambda: c.sc_linear_grad_input(self.dz, self.w, self.dn, **at)
        yield lambda: c.sc_rms_norm_grad(self.dn, self.h, self.gamma, 1e-5, self.dh, dgamma=self.dgamma, residual=self.res, dx=self.dx, p=0.2, seed=7, **at)

    def results(self):
        return [self.h, *self.q, *self.w8, *self.z, self.y, *self.y8, self.back, self.dropped, self.dz, self.held, self.dw, self.dn, self.dh, self.dx, self.dgamma]

    def run(self, wait=None, stream=None):
        for call in self.calls(stream):
            call()
            if wait:
                wait()


SHAPES = [(1, 264, 520), (2, 264, 528), (5, 272, 1024), (30, 264, 512), (77, 131, 77), (300, 264, 1001), (2500, 1032, 520), (64, 1040, 1040)]


@pytest.mark.parametrize("M,N,K", SHAPES)
def test_without_waits(ctx, M, N, K):
    blocks = [Block(ctx, M, N, K, 100 * i) for i in range(6)]
    for b in blocks:
        b.run(torch.cuda.synchronize)
    want = [[t.clone() for t in b.results()] for b in blocks]
    for b in blocks:
        for t in b.results():
            t.zero_()
    torch.cuda.synchronize()
    for _ in range(3):
        for b in blocks:
            b.run()
    torch.cuda.synchronize()
    for b, ref in zip(blocks, want):
        for got, r in zip(b.results(), ref):
            assert torch.equal(got, r)


@pytest.mark.parametrize("M,N,K", [(1, 264, 520), (130, 136, 1001), (600, 264, 2064)])
def test_two_captured_graphs_of_one_context(M, N, K):
    """Graphs share the context's workspace: replayed in turn, each gives what its calls gave; growing the workspace afterwards hurts neither."""
    own = sc.Context(max_n=1)
    own.sc_layer_reserve(M, max(N, K), max(N, K))
    blocks = [Block(own, M, N, K, 7), Block(own, M, N, K, 70)]
    graphs, want = [], []
    for b in blocks:
        b.run(torch.cuda.synchronize)
        want.append([t.clone() for t in b.results()])
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g):
            b.run()
        graphs.append(g)
    own.sc_layer_reserve(4 * M + 3000, 4096, 4096)
    for _ in range(3):
        for b in blocks:
            for t in b.results():
                t.zero_()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for b, ref in zip(blocks, want):
            for got, r in zip(b.results(), ref):
                assert torch.equal(got, r)
    assert own.sc_sync_status() == 0
    del graphs, g
    own.close()


def test_a_capture_without_workspace_is_refused():
    own = sc.Context(max_n=1)
    b = Block(own, 300, 264, 520, 3)
    codes = []
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        own.sc_dropout(b.x, b.dx, 0.5, 1)                              # needs none
        own.sc_rms_norm(b.x, b.gamma, 1e-5, y=b.h)
        try:
            own.sc_rms_norm_grad(b.res, b.x, b.gamma, 1e-5, b.dh, dgamma=b.dgamma)
        except sc.SparseCommError as e:
            codes.append(e.code)
        own.sc_rms_norm_grad(b.res, b.x, b.gamma, 1e-5, b.dh)          # without dgamma there is nothing to join
    assert codes == [-3]
    graph.replay()
    torch.cuda.synchronize()
    del graph
    own.close()


def test_on_another_stream(ctx):
    b = Block(ctx, 300, 264, 520, 21)
    b.run(torch.cuda.synchronize)
    want = [t.clone() for t in b.results()]
    for given in (True, False):
        for t in b.results():
            t.zero_()
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        if given:
            b.run(stream=side)
        else:
            with torch.cuda.stream(side):
                b.run()
        side.synchronize()
        for got, r in zip(b.results(), want):
            assert torch.equal(got, r)


@pytest.mark.parametrize("M,N,K", [(1, 264, 528), (33, 131, 77)])
def test_without_the_compiled_caller(ctx, M, N, K):
    """The binding's own checks and the compiled caller's end in the same calls."""
    b = Block(ctx, M, N, K, 5)
    b.run()
    torch.cuda.synchronize()
    want = [t.clone() for t in b.results()]
    direct, ctx._direct = ctx._direct, None
    try:
        for t in b.results():
            t.zero_()
        b.run()
    finally:
        ctx._direct = direct
    torch.cuda.synchronize()
    for got, r in zip(b.results(), want):
        assert torch.equal(got, r)


def test_what_only_the_bindings_checks_take(ctx):
    """Seeds of other integer types, matrices of one row or column with any stride, vectors as matrices: the compiled caller passes them on."""
    x, gamma = normal(1, 1, 64), normal(2, 64)
    far = torch.empty(64 * 3, dtype=BF16, device="cuda").as_strided((1, 64), (3, 1))
    far.copy_(x)
    y, want = torch.empty_like(x), torch.empty_like(x)
    ctx.sc_rms_norm(x, gamma, 1e-5, y=want, p=0.5, seed=-3)
    for seed in (np.int64(-3), 2 ** 64 - 3):
        y.zero_()
        ctx.sc_rms_norm(far, gamma.view(1, 64), 1e-5, y=y, p=np.float64(0.5), seed=seed)
        assert torch.equal(y, want)
    column = normal(3, 50, 1)
    q, s = sc.quantized_buffers(50, 1)
    ctx.sc_quantize(column.expand(50, 1), q, s.view(50, 1))
    assert torch.equal(q, torch.where(column == 0, 0, torch.where(column < 0, -127, 127)).to(torch.int8))


def test_tensors_of_another_device_are_refused(ctx):
    """The context's device is what counts, not the current one (here the context believes to be elsewhere)."""
    x, y, q, s = normal(1, 4, 64), normal(2, 4, 64), *sc.quantized_buffers(4, 64)
    home, ctx._device = ctx._device, ctx._device + 1
    stream = torch.cuda.current_stream()
    launches = ctx.launch_count
    try:
        for call in (lambda: ctx.sc_dropout(x, y, 0.5, 1, stream=stream), lambda: ctx.sc_quantize(x, q, s, stream=stream), lambda: ctx.sc_dequantize(q, s, y, stream=stream),
                     lambda: ctx.sc_rms_norm(x, y[0], 1e-5, y=y, stream=stream), lambda: ctx.sc_rms_norm_grad(x, y, y[0], 1e-5, x, stream=stream),
                     lambda: ctx.sc_linear_quantized(0, q, s, q, s, y[:, :4].contiguous(), stream=stream)):
            with pytest.raises(ValueError, match="device"):
                call()
    finally:
        ctx._device = home
    assert ctx.launch_count == launches
