"""Cases that measure the operators of residual feed-forward blocks: 8-bit products, root-mean-square norm, dropout.

Operators (``case["op"]``):

``quantize``   x is rounded to 8 bits with one scale a row, and the values that it stands for are read back
``linear``     y = act((xq wq^T) sx sw + b) + r: both operands in 8 bits, a scale for each token and each output channel
``norm``       h = r + dropout(x), y = h / rms(h) * gamma, with y in 16 bits, or in 8 bits with one scale a token
``norm_grad``  dh = r + (gradient of the norm at h), dx = dropout(dh), dgamma in 32 bits
``dropout``    y = r + dropout(x): forward onto a residual, backward without one

Dropout draws 16 bits an element from a counter-based generator (the seed is an input) and stores no mask.
M counts tokens, N features (of a linear layer: outputs), K a linear layer's inputs.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BIG_M, BIG_N, BIG_K = 8192, 16384, 4096
BIG_ROWS, BIG_COLS = 16384, 8192
ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")
EPS = 1e-6


def listed():
    return [
        # a handful of tokens of an odd-sized layer: what a call costs when there is nothing to do
        {"name": "quantize 5x1000 f16", "op": "quantize", "dtype": "f16", "M": 5, "N": 1000},
        # the weights of a wide layer, laid out in 8 bits: bandwidth
        {"name": "quantize 16384x4096 bf16", "op": "quantize", "dtype": "bf16", "M": 16384, "N": 4096},
        # one new token through a projection with its residual: latency and the weights' bandwidth
        {"name": "linear 1x4096x4096 bf16", "op": "linear", "dtype": "bf16", "M": 1, "N": 4096, "K": 4096,
         "act": "none", "bias": True, "residual": True},
        # a ragged batch through a classifier-sized layer
        {"name": "linear 250x1000x520 f16 relu", "op": "linear", "dtype": "f16", "M": 250, "N": 1000, "K": 520,
         "act": "relu", "bias": True, "residual": False},
        # the widening half of a feed-forward block over a long batch: the tensor cores
        {"name": "linear 8192x16384x4096 bf16", "op": "linear", "dtype": "bf16", "M": BIG_M, "N": BIG_N, "K": BIG_K,
         "act": "gelu_tanh", "bias": True, "residual": False},
        # one new token on its way into an 8-bit projection: latency
        {"name": "norm 1x4096 bf16 to 8 bits", "op": "norm", "dtype": "bf16", "M": 1, "N": 4096, "p": 0.0, "residual": True, "out": "q"},
        # a ragged batch of an odd width, no residual, into an 8-bit projection
        {"name": "norm 1021x1001 f16 to 8 bits", "op": "norm", "dtype": "f16", "M": 1021, "N": 1001, "p": 0.0, "residual": False, "out": "q"},
        # between two blocks in training: dropout, residual, norm
        {"name": "norm 16384x8192 bf16 p 0.1", "op": "norm", "dtype": "bf16", "M": BIG_ROWS, "N": BIG_COLS, "p": 0.1, "residual": True, "out": "y"},
        # a ragged batch back through a norm of an odd width
        {"name": "norm_grad 509x1001 f16", "op": "norm_grad", "dtype": "f16", "M": 509, "N": 1001, "p": 0.0, "residual": False},
        # back between two blocks: norm, the residual branch's gradient, dropout
        {"name": "norm_grad 16384x8192 p 0.1", "op": "norm_grad", "dtype": "bf16", "M": BIG_ROWS, "N": BIG_COLS, "p": 0.1, "residual": True},
        # a classifier's hidden layer with a small ragged batch
        {"name": "dropout 77x1001 f16 p 0.5", "op": "dropout", "dtype": "f16", "M": 77, "N": 1001, "p": 0.5, "residual": False},
        # the end of a feed-forward block over a long batch, onto the residual
        {"name": "dropout 16384x8192 bf16 p 0.1", "op": "dropout", "dtype": "bf16", "M": BIG_ROWS, "N": BIG_COLS, "p": 0.1, "residual": True},
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _features(rng, lo, hi):
    """A layer's width: a multiple of 64, of 8, or any number."""
    n = _spread(rng, lo, hi)
    to = rng.choice((64, 64, 8, 1))
    return max(lo, n // to * to)


def draw(rng):
    op = rng.choice(("quantize", "linear", "linear", "norm", "norm", "norm_grad", "dropout"))
    case = {"op": op, "dtype": rng.choice(("bf16", "f16"))}
    if op == "linear":
        while True:
            m, n, k = _spread(rng, 1, 32768), _features(rng, 64, 16384), _features(rng, 64, 16384)
            if m * n * k <= BIG_M * BIG_N * BIG_K and n * k <= BIG_N * BIG_K and m * max(n, k) <= BIG_M * BIG_N:
                break
        case.update({"M": m, "N": n, "K": k, "act": rng.choice(ACTS), "bias": rng.random() < 0.7, "residual": rng.random() < 0.5})
        return case
    n = _features(rng, 64, 16384)
    case.update({"M": _spread(rng, 1, BIG_ROWS * BIG_COLS // max(n, BIG_COLS)), "N": n})
    if op == "quantize":
        case["dtype"] = rng.choice(("bf16", "f16", "f32"))
    else:
        case.update({"p": rng.choice((0.0, 0.1, rng.uniform(0.01, 0.6))), "residual": rng.random() < 0.6})
    if op == "norm":
        case["out"] = rng.choice(("y", "q"))
    return case


def work(case):
    m, n, op = case["M"], case["N"], case["op"]
    cells = m * n
    wide = 4 if case["dtype"] == "f32" else 2
    if op == "quantize":
        # read, written in 8 bits with the scales, and back again
        return {"bytes": 2 * wide * cells + 2 * (cells + 4 * m), "flops": 0}
    if op == "linear":
        k = case["K"]
        extra = (2 * n if case["bias"] else 0) + (2 * cells if case["residual"] else 0)
        return {"bytes": m * k + n * k + 4 * (m + n) + 2 * cells + extra, "flops": 2 * m * n * k}
    held = case["residual"] or case["p"] > 0  # h is another tensor than x
    if op == "norm":
        out = 2 * cells if case["out"] == "y" else 2 * (cells + 4 * m) + 2 * cells  # 8 bits are read back for the comparison
        return {"bytes": 2 * cells + (2 * cells if case["residual"] else 0) + (2 * cells if held else 0) + out + 2 * n, "flops": 0}
    if op == "norm_grad":
        return {"bytes": 6 * cells + (2 * cells if case["residual"] else 0) + (2 * cells if case["p"] > 0 else 0) + 6 * n, "flops": 0}
    return {"bytes": 4 * cells + (2 * cells if case["residual"] else 0), "flops": 0}


# ---------------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------------
def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _activations(g, rows, cols, dtype):
    """Activations of a trained network: unit scale, with one feature in 128 much larger than the others."""
    scale = torch.where(torch.rand(cols, generator=g, device="cuda") < 1 / 128, 12.0, 1.0)
    return (_normal(g, rows, cols) * scale).to(dtype)


def _eight_bits(g, rows, cols, size):
    """A matrix as it was rounded to 8 bits: its largest value of a row is at 127, the rest within a few standard deviations."""
    q = (_normal(g, rows, cols) * 34).round().clamp(-127, 127).to(torch.int8)
    return q, size * (0.5 + torch.rand(rows, generator=g, device="cuda"))


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    op, m, n, dtype = case["op"], case["M"], case["N"], DTYPES[case["dtype"]]
    new = lambda rows, cols, t=dtype: torch.empty(rows, cols, dtype=t, device="cuda")  # noqa: E731
    s = {"case": dict(case), "seed": int(seed) * 1000003 + 17}
    if op == "quantize":
        s.update(x=_activations(g, m, n, dtype), q=new(m, n, torch.int8), scales=torch.empty(m, device="cuda"), out=new(m, n))
        return s
    if op == "linear":
        k = case["K"]
        s["x"], s["x_scales"] = _eight_bits(g, m, k, 1 / 34)
        s["w"], s["w_scales"] = _eight_bits(g, n, k, 1 / 34 / math.sqrt(k))
        s["bias"] = (_normal(g, n) * 0.1).to(dtype) if case["bias"] else None
        s["residual"] = _normal(g, m, n).to(dtype) if case["residual"] else None
        s["y"] = new(m, n)
        return s
    if op == "norm_grad":
        s.update(dy=(_normal(g, m, n) * 0.02).to(dtype), h=_activations(g, m, n, dtype), gamma=(1 + 0.1 * _normal(g, n)).to(dtype))
        s["residual"] = (_normal(g, m, n) * 0.02).to(dtype) if case["residual"] else None
        s.update(dh=new(m, n), dgamma=torch.empty(n, device="cuda"), dx=new(m, n) if case["p"] > 0 else None)
        return s
    s["x"] = _activations(g, m, n, dtype)
    s["residual"] = _activations(g, m, n, dtype) if case["residual"] else None
    if op == "dropout":
        s["y"] = new(m, n)
        return s
    s["gamma"] = (1 + 0.1 * _normal(g, n)).to(dtype)
    s["h"] = new(m, n) if case["residual"] or case["p"] > 0 else None
    s["y"] = new(m, n)
    if case["out"] == "q":
        s.update(q=new(m, n, torch.int8), scales=torch.empty(m, device="cuda"))
    return s


# ---------------------------------------------------------------------------------------------------------------------
# the plain form: elementary operations in 32 bits
# ---------------------------------------------------------------------------------------------------------------------
def _signed(v):
    """A 64-bit pattern as torch holds it."""
    return v - (1 << 64) if v >= 1 << 63 else v


GOLDEN, MIX_A, MIX_B = 0x9E3779B97F4A7C15, 0xBF58476D1CE4E5B9, 0x94D049BB133111EB
SALT = 0x64726F70


def _fold(z, bits):
    return z ^ ((z >> bits) & ((1 << (64 - bits)) - 1))


def _scramble(z):
    """The generator's finaliser on 64-bit patterns (int64, wrapping)."""
    z = _fold(z, 30) * _signed(MIX_A)
    z = _fold(z, 27) * _signed(MIX_B)
    return _fold(z, 31)


def _mixed(a, b):
    """The generator at counter b under seed a, a number of 64 bits."""
    z = (a + (b + 1) * GOLDEN) % 2**64
    z = (z ^ z >> 30) * MIX_A % 2**64
    z = (z ^ z >> 27) * MIX_B % 2**64
    return z ^ z >> 31


def _kept(seed, m, n, p):
    """(mask [m, n], scale of what is kept): 16 bits an element, four elements of a row to a 64-bit word."""
    cut = round(p * 65536)
    groups = -(-n // 4)
    at = torch.arange(1, m * groups + 1, device="cuda")
    words = _scramble(at * _signed(GOLDEN) + _signed(_mixed(seed, SALT)))
    parts = [((words >> (16 * i)) & 0xFFFF) >= cut for i in range(4)]
    return torch.stack(parts, 1).view(m, groups * 4)[:, :n], 65536 / (65536 - cut) if cut < 65536 else 0.0


def _dropped(v, seed, p):
    if p == 0:
        return v
    mask, scale = _kept(seed, v.shape[0], v.shape[1], p)
    return torch.where(mask, v * scale, 0.0)


def _rounded(v):
    """(integers as 32-bit floats, scales [rows]) of v rounded to 8 bits with one scale a row."""
    top = v.abs().amax(1, keepdim=True)
    return torch.round(v * (127 / top)), (top / 127).squeeze(1)


def _act(z, act):
    if act == "relu":
        return z.clamp_min(0)
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _plain(s):
    case = s["case"]
    op, dtype = case["op"], DTYPES[case["dtype"]]
    if op == "quantize":
        q, scales = _rounded(s["x"].float())
        return {"x": (q * scales.unsqueeze(1)).to(dtype), "scales": scales}
    if op == "linear":
        z = (s["x"].float() @ s["w"].float().t()) * s["x_scales"].unsqueeze(1) * s["w_scales"]
        if s["bias"] is not None:
            z = z + s["bias"].float()
        y = _act(z, case["act"])
        if s["residual"] is not None:
            y = y + s["residual"].float()
        return {"y": y.to(dtype)}
    if op == "dropout":
        y = _dropped(s["x"].float(), s["seed"], case["p"])
        if s["residual"] is not None:
            y = y + s["residual"].float()
        return {"y": y.to(dtype)}
    gamma = s["gamma"].float()
    if op == "norm":
        h = _dropped(s["x"].float(), s["seed"], case["p"])
        if s["residual"] is not None:
            h = h + s["residual"].float()
        y = h * torch.rsqrt((h * h).mean(1, keepdim=True) + EPS) * gamma
        out = {} if s["h"] is None else {"h": h.to(dtype)}
        if case["out"] == "y":
            return {**out, "y": y.to(dtype)}
        q, scales = _rounded(y)
        return {**out, "y": (q * scales.unsqueeze(1)).to(dtype), "scales": scales}
    h, dy = s["h"].float(), s["dy"].float()
    r = torch.rsqrt((h * h).mean(1, keepdim=True) + EPS)
    g, unit = dy * gamma, h * r
    dh = r * (g - unit * (g * unit).mean(1, keepdim=True))
    if s["residual"] is not None:
        dh = dh + s["residual"].float()
    out = {"dh": dh.to(dtype), "dgamma": (dy * unit).sum(0)}
    if s["dx"] is not None:
        out["dx"] = _dropped(dh, s["seed"], case["p"]).to(dtype)
    return out


# ---------------------------------------------------------------------------------------------------------------------
# the framework's operators
# ---------------------------------------------------------------------------------------------------------------------
_handle = None


def _context():
    """The program's one context, made before its first step."""
    global _handle
    if _handle is None:
        import paper_2009_09271_b200 as sc

        _handle = (sc, sc.Context(max_n=1))
    return _handle


def _own(s):
    sc, ctx = _context()
    case = s["case"]
    op = case["op"]
    if op == "quantize":
        ctx.sc_quantize(s["x"], s["q"], s["scales"])
        ctx.sc_dequantize(s["q"], s["scales"], s["out"])
        return {"x": s["out"], "scales": s["scales"]}
    if op == "linear":
        ctx.sc_linear_quantized(sc.ACTIVATIONS[case["act"]], s["x"], s["x_scales"], s["w"], s["w_scales"], s["y"], bias=s["bias"], residual=s["residual"])
        return {"y": s["y"]}
    if op == "dropout":
        ctx.sc_dropout(s["x"], s["y"], case["p"], s["seed"], residual=s["residual"])
        return {"y": s["y"]}
    if op == "norm":
        out = {} if s["h"] is None else {"h": s["h"]}
        if case["out"] == "y":
            ctx.sc_rms_norm(s["x"], s["gamma"], EPS, y=s["y"], residual=s["residual"], h=s["h"], p=case["p"], seed=s["seed"])
            return {**out, "y": s["y"]}
        ctx.sc_rms_norm(s["x"], s["gamma"], EPS, q=s["q"], scales=s["scales"], residual=s["residual"], h=s["h"], p=case["p"], seed=s["seed"])
        ctx.sc_dequantize(s["q"], s["scales"], s["y"])
        return {**out, "y": s["y"], "scales": s["scales"]}
    ctx.sc_rms_norm_grad(s["dy"], s["h"], s["gamma"], EPS, s["dh"], dgamma=s["dgamma"], residual=s["residual"], dx=s["dx"], p=case["p"], seed=s["seed"])
    out = {"dh": s["dh"], "dgamma": s["dgamma"]}
    return out if s["dx"] is None else {**out, "dx": s["dx"]}


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------------------------------------------------------------
# the definition in 64 bits
# ---------------------------------------------------------------------------------------------------------------------
def _splitmix(z):
    with np.errstate(over="ignore"):
        z = (z ^ (z >> np.uint64(30))) * np.uint64(MIX_A)
        z = (z ^ (z >> np.uint64(27))) * np.uint64(MIX_B)
        return z ^ (z >> np.uint64(31))


def _thinned64(v, seed, p):
    """Dropout with the generator's words made by unsigned arithmetic on the host, read as rows of 16-bit integers."""
    cut = round(p * 65536)
    if cut == 0:
        return v
    rows, cols = v.shape
    per_row = (cols + 3) // 4
    with np.errstate(over="ignore"):
        start = np.array([seed % 2**64], np.uint64) + np.uint64(SALT + 1) * np.uint64(GOLDEN)
        counters = np.arange(rows * per_row, dtype=np.uint64) + np.uint64(1)
        words = _splitmix(_splitmix(start)[0] + counters * np.uint64(GOLDEN))
    fields = words.astype("<u8").view("<u2").reshape(rows, per_row * 4)[:, :cols]
    gone = torch.from_numpy(np.ascontiguousarray(fields < cut)).to(v.device)
    return (v * (65536 / (65536 - cut))).masked_fill(gone, 0.0)


def _in_steps64(v):
    """(values in whole steps of the row's largest magnitude over 127, the steps)."""
    step = torch.linalg.vector_norm(v, ord=math.inf, dim=1, keepdim=True) / 127
    return torch.round(v / step) * step, step[:, 0]


def _act64(z, act):
    if act == "relu":
        return torch.relu(z)
    if act == "gelu":
        return z * torch.special.ndtr(z)
    if act == "gelu_tanh":
        return z * torch.sigmoid(math.sqrt(8 / math.pi) * (z + 0.044715 * z**3))
    return z * torch.sigmoid(z) if act == "silu" else z


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    branch = None if op == "quantize" or s["residual"] is None else s["residual"].double()
    if op == "quantize":
        x, step = _in_steps64(s["x"].double())
        return {"x": x, "scales": step}
    if op == "linear":
        z = torch.einsum("mk,nk->mn", s["x"].double() * s["x_scales"].double()[:, None], s["w"].double() * s["w_scales"].double()[:, None])
        if s["bias"] is not None:
            z += s["bias"].double()
        y = _act64(z, case["act"])
        return {"y": y if branch is None else y + branch}
    if op == "dropout":
        y = _thinned64(s["x"].double(), s["seed"], case["p"])
        return {"y": y if branch is None else y + branch}
    gamma = s["gamma"].double()
    if op == "norm":
        h = _thinned64(s["x"].double(), s["seed"], case["p"])
        if branch is not None:
            h = h + branch
        y = h / torch.sqrt(torch.einsum("mn,mn->m", h, h) / case["N"] + EPS)[:, None] * gamma
        out = {} if s["h"] is None else {"h": h}
        if case["out"] == "y":
            return {**out, "y": y}
        y, step = _in_steps64(y)
        return {**out, "y": y, "scales": step}
    h, dy = s["h"].double(), s["dy"].double()
    size = torch.sqrt(torch.einsum("mn,mn->m", h, h) / case["N"] + EPS)[:, None]
    pull = torch.einsum("mn,mn,n->m", dy, h, gamma)[:, None] / (case["N"] * size**3)
    dh = dy * gamma / size - h * pull
    if branch is not None:
        dh += branch
    out = {"dh": dh, "dgamma": torch.einsum("mn,mn->n", dy, h / size)}
    if s["dx"] is not None:
        out["dx"] = _thinned64(dh, s["seed"], case["p"])
    return out
