"""The 8-bit rows that the norm writes are those of its fp32 y, bit for bit.

x holds integers of magnitude up to 15, so that h gamma and a row's sum of squares (below 2^24) are exact in fp32 whatever the order of the
sum.  What follows is IEEE fp32 but for the root's start, CUDA's rsqrtf: r = s (1.5 - (v s / 2) s) with the last product and the difference
rounded once (in 64 bits both are exact), y = (h gamma) r, and the 8-bit rows of y."""
import pytest
import torch

import paper_2009_09271_b200 as sc
from block_util import rows_in_8_bits
from layer_util import strided

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = sc.Context(max_n=1)
    yield c
    assert c.sc_sync_status() == 0
    c.close()


def differing(a, b):
    return int((a != b).sum())


def root(sums, cols):
    """fp32 (sum / cols)^(-1/2) as the norm takes it, eps = 0."""
    mean = torch.ones((), device="cuda") / torch.full((), float(cols), device="cuda")
    v = (sums.double() * mean.double()).float()
    s = torch.rsqrt(v)
    return s * ((-0.5 * v * s).double() * s.double() + 1.5).float()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,cols,extra,offset", [(3000, 40, 0, 0), (1500, 257, 0, 0), (700, 1001, 0, 0), (700, 1001, 3, 1), (300, 4096, 0, 0), (70, 20000, 0, 0),
                                                    (40, 33000, 0, 0), (30, 40001, 0, 0)])
def test_bytes_are_those_of_the_fp32_result(ctx, dtype, rows, cols, extra, offset):
    g = torch.Generator(device="cuda").manual_seed(cols)
    x = torch.randint(-15, 16, (rows, cols), generator=g, device="cuda")
    x[:, 0] = 15
    gamma = (1 + 0.2 * torch.randn(cols, generator=g, device="cuda")).to(dtype)
    product = x.float() * gamma.float()
    r = root(x.square().sum(1), cols)[:, None]
    want = product * r
    q, scales = strided(torch.zeros(rows, cols, device="cuda").to(torch.int8), extra, offset), torch.empty(rows, device="cuda")
    y, only = strided(torch.zeros(rows, cols, device="cuda").to(dtype), extra, offset), torch.zeros(rows, cols, device="cuda", dtype=torch.int8)
    xs = strided(x.to(dtype), extra, offset)
    ctx.sc_rms_norm(xs, gamma, 0.0, y=y, q=q, scales=scales)
    wq, ws = rows_in_8_bits(want)
    assert differing(y, want.to(dtype)) == 0
    assert differing(scales.cpu(), ws) == 0
    assert differing(q.cpu(), wq) == 0
    ctx.sc_rms_norm(xs, gamma, 0.0, q=only, scales=scales)
    assert differing(only.cpu(), wq) == 0
    # bytes made with one factor for r and the scale, or from (h r) gamma, are others: the inputs tell them apart
    inv = (127.0 * (1.0 / want.abs().amax(1, keepdim=True)))
    if rows * cols > 700000:
        assert differing(torch.round(product * (inv * r)).to(torch.int8).cpu(), wq) > 0
        assert differing(torch.round(x.float() * r * gamma.float() * inv).to(torch.int8).cpu(), wq) > 0
