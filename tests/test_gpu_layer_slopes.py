"""Slopes of the activations relative to their own size: a worker whose pre-activations lie in the negative tail gets gradients
of a few millionths, and those have to be right in their leading digits too."""
import math

import pytest
import torch

import paper_2009_09271_b200 as sc
from layer_util import slope64

pytestmark = pytest.mark.gpu


def exponent(z, act):
    """|log| of the exponential that the slope's tail is made of."""
    if act == "gelu":
        return z * z / 2
    if act == "gelu_tanh":
        return (math.sqrt(8 / math.pi) * (z + 0.044715 * z ** 3)).abs()
    return z.abs()


def magnitudes(z, act):
    """The sum of the magnitudes of the slope's terms: what rounding errors are relative to."""
    if act == "gelu":
        return 0.5 * torch.special.erfc(-z / math.sqrt(2)) + z.abs() * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    v = math.sqrt(8 / math.pi) * (z + 0.044715 * z ** 3) if act == "gelu_tanh" else z
    inner = math.sqrt(8 / math.pi) * (1 + 0.134145 * z * z) if act == "gelu_tanh" else 1.0
    s, rest = torch.sigmoid(v), torch.sigmoid(-v)
    return s + z.abs() * s * rest * inner


def slope(z, act):
    """slope64, but tanh's form through the logistic function: 1 + tanh(u) is 0 in 64 bits below u = -19."""
    if act != "gelu_tanh":
        return slope64(z, act)
    v = math.sqrt(8 / math.pi) * (z + 0.044715 * z ** 3)
    s = torch.sigmoid(v)
    return s + z * s * torch.sigmoid(-v) * math.sqrt(8 / math.pi) * (1 + 0.134145 * z * z)


@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("e", [-8, -5, -4, -3])
def test_slopes_keep_their_leading_digits(act, e):
    """Every value q 2^e of a checkpoint.  The column sums of one row of ones are the slopes in fp32, before any rounding to 16 bits.
    An exponential of argument t is off by 2^-22 t of its value (four roundings on the way to t), the other steps together by less than 2^-20; results below
    2^-120 may be lost."""
    q = torch.arange(-127, 128, device="cuda").to(torch.int8).view(1, -1)
    cols = q.shape[1]
    scales = torch.full((1, -(-cols // 32)), 127 + e, dtype=torch.uint8, device="cuda")
    z = q.double() * 2.0 ** e
    ctx = sc.Context(max_n=1)
    got = torch.empty(cols, device="cuda")
    dy = torch.ones(1, cols, dtype=torch.bfloat16, device="cuda")
    ctx.sc_activation_grad(sc.ACTIVATIONS[act], dy, q, scales, None, got)
    want = slope(z, act)
    slack = (2.0 ** -20 + exponent(z, act) * 2.0 ** -22) * magnitudes(z, act) + 2.0 ** -120
    over = ((got.double() - want).abs() / slack).view(-1)
    at = int(over.argmax())
    assert float(over[at]) <= 1, (float(z[0, at]), float(got[at]), float(want[0, at]), float(over[at]))
    assert ctx.sc_sync_status() == 0
    ctx.close()
