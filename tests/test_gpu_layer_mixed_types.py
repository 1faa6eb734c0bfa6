"""A checkpoint made from one type and read in calls of another: its values are rounded to the type of the call, whatever kernel reads them."""
import pytest
import torch

import paper_2009_09271_b200 as sc

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M", [1, 4, 7, 40, 300])
def test_weight_gradient_reads_a_checkpoint_as_unpack_does(M):
    """Values past fp16's range read as infinity and those below half its smallest step as 0, for few tokens and many."""
    N, K = 36, 96
    x = torch.ones(M, K, device="cuda")
    x[0, :32] = 1e6
    x[0, 32:64] = 2.0 ** -40
    x[:, 64:] *= 1.5
    ctx = sc.Context(max_n=1)
    q, scales = sc.checkpoint_buffers(M, K)
    ctx.sc_checkpoint_pack(x, q, scales)
    held = torch.empty(M, K, dtype=torch.float16, device="cuda")
    ctx.sc_checkpoint_unpack(q, scales, held)
    assert bool(torch.isinf(held[0, :32]).all()) and not bool(held[0, 32:64].any())
    dz = torch.ones(M, N, dtype=torch.float16, device="cuda")
    got, want = torch.empty(N, K, device="cuda"), torch.empty(N, K, device="cuda")
    ctx.sc_linear_grad_weight(dz, got, q=q, scales=scales)
    ctx.sc_linear_grad_weight(dz, want, x=held)
    assert torch.equal(got, want) and bool(torch.isinf(got[:, :32]).all())
    assert bool((got[:, 32:64] == M - 1).all()) and bool((got[:, 64:] == 1.5 * M).all())
    assert ctx.sc_sync_status() == 0
    ctx.close()
