"""Plain statements of 8-bit rows, the root-mean-square norm and dropout, and the error bounds their tests use."""
from __future__ import annotations

import numpy as np
import torch

SALT_DROPOUT = 0x64726F70
_GOLDEN, _A, _B = 0x9E3779B97F4A7C15, 0xBF58476D1CE4E5B9, 0x94D049BB133111EB


def mix64(a, b):
    """The generator on arrays of unsigned 64-bit counters b."""
    with np.errstate(over="ignore"):
        z = np.asarray(a, np.uint64) + (np.asarray(b, np.uint64) + np.uint64(1)) * np.uint64(_GOLDEN)
        z = (z ^ (z >> np.uint64(30))) * np.uint64(_A)
        z = (z ^ (z >> np.uint64(27))) * np.uint64(_B)
        return z ^ (z >> np.uint64(31))


def kept_mask(seed, rows, cols, p, first_row=0):
    """(mask [rows, cols] on the host, scale) of dropout, for rows from first_row."""
    cut = int(np.rint(p * 65536))
    per_row = -(-cols // 4)
    key = mix64(seed % 2 ** 64, SALT_DROPOUT)
    counters = np.arange(first_row * per_row, (first_row + rows) * per_row, dtype=np.uint64)
    words = mix64(key, counters) if counters.size else counters
    bits = np.stack([(words >> np.uint64(16 * i)) & np.uint64(0xFFFF) for i in range(4)], 1).reshape(rows, per_row * 4)[:, :cols]
    return torch.from_numpy(bits >= np.uint64(cut)), (65536 / (65536 - cut) if cut < 65536 else 0.0)


def dropped64(x, seed, p):
    mask, scale = kept_mask(seed, *x.shape, p)
    return torch.where(mask.to(x.device), x.double() * scale, torch.zeros((), dtype=torch.float64, device=x.device))


def rows_in_8_bits(x):
    """(q, scales) of x by the definition, in IEEE fp32 on the host."""
    v = x.detach().float().cpu().numpy()
    with np.errstate(all="ignore"):
        m = np.abs(v).max(1, initial=0.0)
        m = np.where(np.isfinite(v).all(1), m, np.float32(np.nan)).astype(np.float32)
        scale, inv = m / np.float32(127), np.float32(127) * (np.float32(1) / m)
        small, lost = m < np.float32(2.0 ** -100), np.isnan(m)
        scale = np.minimum(scale, np.float32(2.6793883890187504e+36))                      # 127 times more is not a number
        scale = np.where(small, np.float32(0), scale).astype(np.float32)
        q = np.rint(v * inv[:, None])
        q[small | lost] = 0
    return torch.from_numpy(q.astype(np.int8)), torch.from_numpy(scale)


def depth(cols):
    """Additions on the way from a square to a row's sum: at least 32 threads share a row, eight elements at a time; the joins of lanes
    and warps, and the operations around the sum, are below 40."""
    return cols / 32 + 40


def norm64(x, residual, gamma, eps, seed=0, p=0.0):
    """(h, y) in 64 bits."""
    h = dropped64(x, seed, p) if p else x.double()
    if residual is not None:
        h = h + residual.double()
    r = ((h * h).mean(1, keepdim=True) + eps).rsqrt()
    return h, h * r * gamma.double()


def norm_grad64(dy, h, gamma, eps, residual=None):
    """((dh, dgamma), (slack of dh, slack of dgamma)): a term loses at most depth 2^-23 of what it is made of."""
    dy, h, gamma = dy.double(), h.double(), gamma.double()
    r = ((h * h).mean(1, keepdim=True) + eps).rsqrt()
    g, u = gamma * dy, h * r
    dh = r * (g - u * (g * u).mean(1, keepdim=True))
    part = depth(h.shape[1]) * 2.0 ** -23
    slack = part * r * (g.abs() + u.abs() * (g * u).abs().mean(1, keepdim=True))
    if residual is not None:
        dh = dh + residual.double()
        slack = slack + dh.abs() * 2.0 ** -23
    return (dh, (dy * u).sum(0)), (slack, (part + h.shape[0] * 2.0 ** -23) * (dy * u).abs().sum(0))
