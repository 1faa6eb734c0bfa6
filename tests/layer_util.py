"""Plain 64-bit statements of the layer operators and the error bounds their tests use."""
from __future__ import annotations

import math

import torch

GROUP = 32
ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")
RANGES = {torch.bfloat16: (-126, 122), torch.float16: (-24, 10), torch.float32: (-126, 122)}
# half a step of the type, relative to the value (8 and 11 significant bits), and half its smallest step
UNIT = {torch.bfloat16: (2.0 ** -8, 2.0 ** -134), torch.float16: (2.0 ** -11, 2.0 ** -25)}


def act64(z, name):
    if name == "relu":
        return torch.where(z < 0, torch.zeros_like(z), z)
    if name == "gelu":
        return 0.5 * z * torch.special.erfc(-z / math.sqrt(2))
    if name == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    if name == "silu":
        return z / (1 + torch.exp(-z))
    return z


def slope64(z, name):
    if name == "relu":
        return torch.where(z > 0, 1.0, torch.where(z <= 0, 0.0, z))
    if name == "gelu":
        return 0.5 * torch.special.erfc(-z / math.sqrt(2)) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if name == "gelu_tanh":
        z = z.clamp(-64, 64)
        t = torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * z * z)
    if name == "silu":
        s = torch.sigmoid(z)
        return s + z.clamp(-300, 300) * s * (1 - s)
    return torch.ones_like(z)


def checkpoint64(x, dtype):
    """(q, scale bytes, values) of x [rows, cols] by the definition: e by trying every exponent from below."""
    lo, hi = RANGES[dtype]
    x = x.double().cpu()
    rows, cols = x.shape
    groups = -(-cols // GROUP)
    q = torch.zeros(rows, cols, dtype=torch.int8)
    scales = torch.zeros(rows, groups, dtype=torch.uint8)
    values = torch.zeros(rows, cols, dtype=torch.float64)
    for g in range(groups):
        part = x[:, g * GROUP:(g + 1) * GROUP]
        fine = torch.isfinite(part)
        top = torch.where(fine, part.abs(), 0.0).amax(1, keepdim=True)
        e = torch.full_like(top, hi)
        for k in range(hi, lo - 1, -1):
            e = torch.where(top <= 127 * 2.0 ** k, float(k), e)
        most = torch.where(e == hi, 63.0, 127.0)
        v = torch.round(torch.where(fine, part, 0.0) * torch.exp2(-e))
        v = torch.minimum(torch.maximum(v, -most), most)
        q[:, g * GROUP:(g + 1) * GROUP] = torch.where(fine, v, -128.0).to(torch.int8)
        scales[:, g] = (e[:, 0] + 127).to(torch.uint8)
        values[:, g * GROUP:(g + 1) * GROUP] = torch.where(fine, v * torch.exp2(e), float("nan"))
    return q, scales, values


def product_slack(a, b, terms):
    """Bound on the error of an fp32 sum of `terms` exact products in any order, with sums that may be cut instead of
    rounded: each of at most `terms` additions loses at most 2^-23 of the sum of magnitudes."""
    return (terms + 2) * 2.0 ** -23 * (a.double().abs() @ b.double().abs())


def assert_close(got, want, slack, dtype, what):
    """|got - want| within the slack plus the rounding to the type; not finite exactly where want is not."""
    got, want = got.double(), want.double()
    if dtype in UNIT:
        rel, tiny = UNIT[dtype]
        slack = slack * (1 + rel) + want.abs() * rel + tiny
    fine = torch.isfinite(want)
    if not torch.equal(torch.isnan(got), torch.isnan(want)):
        raise AssertionError(f"{what}: NaN in other places")
    over = (got - want).abs() - slack
    over = torch.where(fine, over, torch.where(got == want, -1.0, 1.0))
    over = torch.where(torch.isnan(want), torch.full_like(over, -1.0), over)
    if over.numel() and bool((over > 0).any()):
        at = int(over.argmax())
        raise AssertionError(f"{what}: {int((over > 0).sum())} of {over.numel()} outside, worst at {at}: got {got.reshape(-1)[at].item()!r} "
                             f"want {want.reshape(-1)[at].item()!r} slack {slack.reshape(-1)[at].item()!r}")


def strided(t, ld_extra=0, offset=0):
    """The same matrix with rows `ld_extra` further apart, starting `offset` elements into its storage."""
    rows, cols = t.shape
    store = torch.full((offset + rows * (cols + ld_extra) + 64,), 7.0, device=t.device).to(t.dtype)
    out = store[offset:offset + rows * (cols + ld_extra)].view(rows, cols + ld_extra)[:, :cols]
    out.copy_(t)
    return out
