"""Layer calls and their workspace: which calls need one, how large it may become, what is refused."""
import pytest
import torch

import paper_2009_09271_b200 as sc

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


def normal(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(BF16)


@pytest.mark.parametrize("rows", [1, 20, 70])
def test_column_sums_of_very_wide_rows(rows):
    """More strips of 256 columns than the tickets that joins of several runs of rows use."""
    cols = 4194304 + 257
    own = sc.Context(max_n=1)
    dy = normal(1, rows, cols)
    db = torch.empty(cols, device="cuda")
    own.sc_activation_grad(sc.SC_ACT_NONE, dy, None, None, None, db)
    want = dy.double().sum(0)
    assert bool(((db.double() - want).abs() <= (rows + 2) * 2.0 ** -23 * dy.double().abs().sum(0)).all())
    assert own.sc_sync_status() == 0
    own.close()


def test_calls_without_workspace_are_captured_on_a_new_context():
    """Aligned rows, one part, one run of rows: nothing to allocate, so nothing to refuse while a stream is captured."""
    M, N, K = 200, 256, 64
    x, w, dz, v = normal(2, M, K), normal(3, N, K), normal(4, M, K), normal(5, K, N)
    few = normal(6, 64, N), normal(7, 64, K)
    outs = [torch.empty(M, N, dtype=BF16, device="cuda"), torch.empty(M, N, dtype=BF16, device="cuda"), torch.empty(N, K, device="cuda"),
            torch.empty(N, device="cuda")]

    def step(c):
        c.sc_linear(sc.SC_ACT_SILU, x, w, outs[0])
        c.sc_linear_grad_input(dz, v, outs[1])
        c.sc_linear_grad_weight(few[0], outs[2], x=few[1])
        c.sc_activation_grad(sc.SC_ACT_NONE, few[0][:32], None, None, None, outs[3])

    other = sc.Context(max_n=1)
    other.sc_layer_reserve(M, N, K)
    step(other)
    torch.cuda.synchronize()
    want = [t.clone() for t in outs]
    for t in outs:
        t.zero_()
    own = sc.Context(max_n=1)
    held = own.scratch_bytes
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    refused = None
    with torch.cuda.graph(graph):
        try:
            step(own)
        except sc.SparseCommError as e:
            refused = e.code
    assert refused is None
    assert own.scratch_bytes == held
    graph.replay()
    torch.cuda.synchronize()
    for got, ref in zip(outs, want):
        assert torch.equal(got, ref)
    assert own.sc_sync_status() == 0
    del graph
    own.close()
    other.close()


def test_a_reservation_beyond_64_bits_is_refused():
    """Three copies of matrices of this size add up to 2^64 bytes and a little more."""
    M, N, K = 1753412483, 1753409644, 1753417036
    total = (64 << 20) + sum(-(-rows * -(-cols // 8) * 16 // 256) * 256 for rows, cols in ((M, K), (N, K), (M, N)))
    assert 2 ** 64 <= total < 2 ** 64 + 2 ** 32
    own = sc.Context(max_n=1)
    held = own.scratch_bytes
    code = sc.load_library().sc_layer_reserve(own._h, M, N, K)
    assert code == -3 and own.scratch_bytes == held
    own.close()
