"""Cases that measure the training operators: a linear layer whose activations are kept in 8 bits, forward and backward.

Operators (``case["op"]``):

``checkpoint``   x is packed to 8 bits (groups of 32 features, a power-of-two scale each) and unpacked again
``act_grad``     dz = dy * act'(z^), db = column sums of dz, with z^ the 8-bit checkpoint of the pre-activation
``linear``       y = act(x W^T + b) + r, with the 8-bit checkpoint of z = x W^T + b on request
``grad_input``   dx = (dz W + r) * act'(z^)
``grad_weight``  dW = dz^T x^ in 32 bits, with x^ the 8-bit checkpoint of the layer's input

M counts tokens, K a layer's inputs, N its outputs.
"""
import math

import torch

own = False

GROUP = 32
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
# the range of a group's exponent: q * 2^e is a value of the type for every e in it
EXPONENTS = {"bf16": (-126, 122), "f16": (-24, 10)}
BIG_M, BIG_N, BIG_K = 8192, 16384, 4096
ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")


def listed():
    return [
        # a handful of tokens of an odd-sized layer: what a call costs when there is nothing to do
        {"name": "checkpoint 7x1000 f16", "op": "checkpoint", "dtype": "f16", "M": 7, "K": 1000},
        # the input of a wide layer over a long batch: bandwidth
        {"name": "checkpoint 16384x8192 bf16", "op": "checkpoint", "dtype": "bf16", "M": 16384, "K": 8192},
        # a classifier-sized hidden layer with a ragged batch
        {"name": "act_grad 1021x1000 f16 relu", "op": "act_grad", "dtype": "f16", "M": 1021, "N": 1000, "act": "relu"},
        # the hidden activations of a feed-forward block
        {"name": "act_grad 8192x16384 bf16 gelu", "op": "act_grad", "dtype": "bf16", "M": 8192, "N": 16384, "act": "gelu_tanh"},
        # one new token through a projection with its residual: latency and the weights' bandwidth
        {"name": "linear 1x4096x4096 bf16", "op": "linear", "dtype": "bf16", "M": 1, "N": 4096, "K": 4096,
         "act": "none", "bias": True, "residual": True, "keep": False},
        # a classifier head's sizes, with a small ragged batch and the checkpoint
        {"name": "linear 250x1000x512 f16 relu", "op": "linear", "dtype": "f16", "M": 250, "N": 1000, "K": 512,
         "act": "relu", "bias": True, "residual": False, "keep": True},
        # the widening half of a feed-forward block in training
        {"name": "linear 8192x16384x4096 gelu", "op": "linear", "dtype": "bf16", "M": BIG_M, "N": BIG_N, "K": BIG_K,
         "act": "gelu_tanh", "bias": True, "residual": False, "keep": True},
        # a ragged batch back through a classifier-sized layer and the activation below it
        {"name": "grad_input 509x1000x2048 f16", "op": "grad_input", "dtype": "f16", "M": 509, "N": 1000, "K": 2048,
         "act": "silu", "residual": False},
        # back through the widening half, onto the residual branch's gradient
        {"name": "grad_input 8192x16384x4096", "op": "grad_input", "dtype": "bf16", "M": BIG_M, "N": BIG_N, "K": BIG_K,
         "act": "none", "residual": True},
        # few tokens: the weight gradient's own bytes decide
        {"name": "grad_weight 64x4096x4096 f16", "op": "grad_weight", "dtype": "f16", "M": 64, "N": 4096, "K": 4096},
        # a long ragged batch into a small layer: few tiles, a long sum
        {"name": "grad_weight 32001x1000x1024", "op": "grad_weight", "dtype": "bf16", "M": 32001, "N": 1000, "K": 1024},
        # the widening half's weights
        {"name": "grad_weight 8192x16384x4096", "op": "grad_weight", "dtype": "bf16", "M": BIG_M, "N": BIG_N, "K": BIG_K},
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _features(rng, lo, hi):
    """A layer's width: a multiple of 64, of 8, or any number."""
    n = _spread(rng, lo, hi)
    to = rng.choice((64, 64, 8, 1))
    return max(lo, n // to * to)


def draw(rng):
    op = rng.choice(("checkpoint", "act_grad", "linear", "linear", "grad_input", "grad_weight"))
    case = {"op": op, "dtype": rng.choice(("bf16", "f16"))}
    if op in ("checkpoint", "act_grad"):
        width = _features(rng, 64, 16384)
        case.update({"M": _spread(rng, 1, 16384 * 8192 // max(width, 8192)), "K" if op == "checkpoint" else "N": width})
        if op == "act_grad":
            case["act"] = rng.choice(ACTS[1:])
        return case
    while True:
        n, k = _features(rng, 64, 16384), _features(rng, 64, 16384)
        m = _spread(rng, 1, 32768)
        if m * n * k <= BIG_M * BIG_N * BIG_K and n * k <= BIG_N * BIG_K and m * max(n, k) <= BIG_M * BIG_N:
            break
    case.update({"M": m, "N": n, "K": k})
    if op == "linear":
        case.update({"act": rng.choice(ACTS), "bias": rng.random() < 0.7, "residual": rng.random() < 0.5, "keep": rng.random() < 0.5})
    elif op == "grad_input":
        case.update({"act": rng.choice(ACTS), "residual": rng.random() < 0.5})
    return case


def work(case):
    m, op = case["M"], case["op"]
    kept = lambda rows, cols: rows * (cols + -(-cols // GROUP))  # noqa: E731
    if op == "checkpoint":
        return {"bytes": 4 * m * case["K"] + 2 * kept(m, case["K"]), "flops": 0}
    n = case["N"]
    if op == "act_grad":
        return {"bytes": 4 * m * n + kept(m, n) + 4 * n, "flops": 0}
    k, flops = case["K"], 2 * m * n * case["K"]
    if op == "linear":
        extra = (2 * n if case["bias"] else 0) + (2 * m * n if case["residual"] else 0)
        # a kept pre-activation is written by the layer, and read back into the type for the comparison
        extra += 2 * kept(m, n) + 2 * m * n if case["keep"] else 0
        return {"bytes": 2 * (m * k + n * k + m * n) + extra, "flops": flops}
    if op == "grad_input":
        extra = (2 * m * k if case["residual"] else 0) + (kept(m, k) if case["act"] != "none" else 0)
        return {"bytes": 2 * (m * n + n * k + m * k) + extra, "flops": flops}
    return {"bytes": 2 * m * n + kept(m, k) + 4 * n * k, "flops": flops}


# ---------------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------------
def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _activations(g, rows, cols, dtype):
    """Activations of a trained network: unit scale, with one feature in 128 much larger than the others."""
    scale = torch.where(torch.rand(cols, generator=g, device="cuda") < 1 / 128, 12.0, 1.0)
    return (_normal(g, rows, cols) * scale).to(dtype)


def _kept(g, rows, cols, kind):
    """A checkpoint as the forward pass left it: int8 values and one exponent byte per group of 32 features."""
    groups = -(-cols // GROUP)
    q = (_normal(g, rows, cols) * 42).round().clamp(-127, 127).to(torch.int8)
    e = torch.randint(-7, -2, (rows, groups), generator=g, device="cuda")
    return q, (e + 127).to(torch.uint8)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    kind, m = case["dtype"], case["M"]
    dtype = DTYPES[kind]
    op = case["op"]
    s = {"case": dict(case)}
    new = lambda rows, cols, t=dtype: torch.empty(rows, cols, dtype=t, device="cuda")  # noqa: E731
    groups = lambda cols: -(-cols // GROUP)  # noqa: E731
    if op == "checkpoint":
        k = case["K"]
        s.update(x=_activations(g, m, k, dtype), q=new(m, k, torch.int8), scales=new(m, groups(k), torch.uint8), out=new(m, k))
    elif op == "act_grad":
        n = case["N"]
        s["dy"] = (_normal(g, m, n) * 0.02).to(dtype)
        s["q"], s["scales"] = _kept(g, m, n, kind)
        s.update(dz=new(m, n), db=torch.empty(n, device="cuda"))
    elif op == "linear":
        n, k = case["N"], case["K"]
        s.update(x=_activations(g, m, k, dtype), w=(_normal(g, n, k) / math.sqrt(k)).to(dtype))
        s["bias"] = (_normal(g, n) * 0.1).to(dtype) if case["bias"] else None
        s["residual"] = _normal(g, m, n).to(dtype) if case["residual"] else None
        s["y"] = new(m, n)
        if case["keep"]:
            s.update(q=new(m, n, torch.int8), scales=new(m, groups(n), torch.uint8), z=new(m, n))
    elif op == "grad_input":
        n, k = case["N"], case["K"]
        s.update(dz=(_normal(g, m, n) * 0.02).to(dtype), w=(_normal(g, n, k) / math.sqrt(k)).to(dtype), dx=new(m, k))
        s["residual"] = (_normal(g, m, k) * 0.02).to(dtype) if case["residual"] else None
        if case["act"] != "none":
            s["q"], s["scales"] = _kept(g, m, k, kind)
    else:
        n, k = case["N"], case["K"]
        s["dz"] = (_normal(g, m, n) * 0.02).to(dtype)
        s["q"], s["scales"] = _kept(g, m, k, kind)
        s["dw"] = torch.empty(n, k, device="cuda")
    return s


# ---------------------------------------------------------------------------------------------------------------------
# the plain form: elementary operations in 32 bits
# ---------------------------------------------------------------------------------------------------------------------
def _grouped(v):
    """[rows, cols] as [rows, groups, 32], the last group filled with zeros."""
    pad = -v.shape[1] % GROUP
    if pad:
        v = torch.cat((v, v.new_zeros(v.shape[0], pad)), 1)
    return v.view(v.shape[0], -1, GROUP)


def _round_trip(v, kind):
    """v (32 bits) as the checkpoint of its type holds it."""
    lo, hi = EXPONENTS[kind]
    groups = _grouped(v)
    top = groups.abs().amax(2, keepdim=True)
    part, power = torch.frexp(top)  # top = part * 2^power, 1/2 <= part < 1
    e = (power - 7 + (part > 127 / 128).int()).clamp(lo, hi)
    most = torch.where(e == hi, 63.0, 127.0)
    q = torch.minimum(torch.maximum(torch.round(torch.ldexp(groups, -e)), -most), most)
    return torch.ldexp(q, e).view(v.shape[0], -1)[:, : v.shape[1]]


def _value(q, scales):
    """The stored values, in 32 bits."""
    return torch.ldexp(_grouped(q.float()), scales.int().unsqueeze(2) - 127).view(q.shape[0], -1)[:, : q.shape[1]]


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


def _slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * math.sqrt(0.5 / math.pi)
    if act == "gelu_tanh":
        t = torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * z * z)
    s = 1 / (1 + torch.exp(-z))
    return s * (1 + z * (1 - s))


def _plain(s):
    case = s["case"]
    kind, op = case["dtype"], case["op"]
    dtype = DTYPES[kind]
    if op == "checkpoint":
        return {"x": _round_trip(s["x"].float(), kind).to(dtype)}
    if op == "act_grad":
        dz = s["dy"].float() * _slope(_value(s["q"], s["scales"]), case["act"])
        return {"dz": dz.to(dtype), "db": dz.sum(0)}
    if op == "linear":
        z = s["x"].float() @ s["w"].float().t()
        if s["bias"] is not None:
            z = z + s["bias"].float()
        y = _act(z, case["act"])
        if s["residual"] is not None:
            y = y + s["residual"].float()
        out = {"y": y.to(dtype)}
        if case["keep"]:
            out["z"] = _round_trip(z, kind).to(dtype)
        return out
    if op == "grad_input":
        dx = s["dz"].float() @ s["w"].float()
        if s["residual"] is not None:
            dx = dx + s["residual"].float()
        if case["act"] != "none":
            dx = dx * _slope(_value(s["q"], s["scales"]), case["act"])
        return {"dx": dx.to(dtype)}
    return {"dw": s["dz"].float().t() @ _value(s["q"], s["scales"])}


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
    if op == "checkpoint":
        ctx.sc_checkpoint_pack(s["x"], s["q"], s["scales"])
        ctx.sc_checkpoint_unpack(s["q"], s["scales"], s["out"])
        return {"x": s["out"]}
    if op == "act_grad":
        ctx.sc_activation_grad(sc.ACTIVATIONS[case["act"]], s["dy"], s["q"], s["scales"], s["dz"], s["db"])
        return {"dz": s["dz"], "db": s["db"]}
    if op == "linear":
        act = sc.ACTIVATIONS[case["act"]]
        if not case["keep"]:
            ctx.sc_linear(act, s["x"], s["w"], s["y"], bias=s["bias"], residual=s["residual"])
            return {"y": s["y"]}
        ctx.sc_linear(act, s["x"], s["w"], s["y"], bias=s["bias"], residual=s["residual"], q=s["q"], scales=s["scales"])
        ctx.sc_checkpoint_unpack(s["q"], s["scales"], s["z"])
        return {"y": s["y"], "z": s["z"]}
    if op == "grad_input":
        if case["act"] == "none":
            ctx.sc_linear_grad_input(s["dz"], s["w"], s["dx"], residual=s["residual"])
        else:
            ctx.sc_linear_grad_input(s["dz"], s["w"], s["dx"], residual=s["residual"], act=sc.ACTIVATIONS[case["act"]],
                                     q=s["q"], scales=s["scales"])
        return {"dx": s["dx"]}
    ctx.sc_linear_grad_weight(s["dz"], s["dw"], q=s["q"], scales=s["scales"])
    return {"dw": s["dw"]}


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------------------------------------------------------------
# the definition in 64 bits
# ---------------------------------------------------------------------------------------------------------------------
def _stored64(q, scales):
    scale = torch.exp2(scales.double() - 127).repeat_interleave(GROUP, 1)[:, : q.shape[1]]
    return q.double() * scale


def _slope64(z, act):
    """Derivatives through the normal distribution and the logistic function."""
    if act == "relu":
        return torch.heaviside(z, torch.zeros((), dtype=z.dtype, device=z.device))
    if act == "gelu":
        return torch.special.ndtr(z) + z * torch.exp(-z.square() / 2) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":
        c = math.sqrt(8 / math.pi)
        s = torch.sigmoid(c * (z + 0.044715 * z**3))
        return s + z * s * (1 - s) * c * (1 + 0.134145 * z.square())
    s = torch.sigmoid(z)
    return s + z * s * (1 - s)


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
    kind, op = case["dtype"], case["op"]
    if op == "checkpoint":
        lo, hi = EXPONENTS[kind]
        x = s["x"].double()
        out = torch.empty_like(x)
        for at in range(0, x.shape[1], GROUP):
            part = x[:, at : at + GROUP]
            top = part.abs().max(1, keepdim=True).values
            e = torch.ceil(torch.log2(top / 127)).clamp(lo, hi)  # the power above, or one off where the logarithm rounds
            e = torch.where((top <= 127 * torch.exp2(e - 1)) & (e > lo), e - 1, e)
            e = torch.where((top > 127 * torch.exp2(e)) & (e < hi), e + 1, e)
            most = torch.where(e == hi, 63.0, 127.0).double()
            out[:, at : at + GROUP] = torch.clamp(torch.round(part / torch.exp2(e)), -most, most) * torch.exp2(e)
        return {"x": out}
    if op == "act_grad":
        dz = s["dy"].double() * _slope64(_stored64(s["q"], s["scales"]), case["act"])
        return {"dz": dz, "db": dz.sum(0)}
    if op == "linear":
        z = torch.einsum("mk,nk->mn", s["x"].double(), s["w"].double())
        if s["bias"] is not None:
            z += s["bias"].double()
        y = _act64(z, case["act"])
        if s["residual"] is not None:
            y += s["residual"].double()
        # a value at the edge of two steps of the checkpoint goes either way with the last bit of z
        return {"y": y, "z": None} if case["keep"] else {"y": y}
    if op == "grad_input":
        dx = torch.einsum("mn,nk->mk", s["dz"].double(), s["w"].double())
        if s["residual"] is not None:
            dx += s["residual"].double()
        if case["act"] != "none":
            dx *= _slope64(_stored64(s["q"], s["scales"]), case["act"])
        return {"dx": dx}
    return {"dw": torch.einsum("mn,mk->nk", s["dz"].double(), _stored64(s["q"], s["scales"]))}
