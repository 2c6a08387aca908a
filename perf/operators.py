"""The calls of the 8-bit operators whose time is followed from change to change.

A network whose weights and activations are held in 8-bit integers, one scale
for each row, runs these around every one of its matrix products:

- ``gemm_i8``: the product of int8 activations (tokens x K, a scale for each
  token) with int8 weights (channels x K, a scale for each channel);
- ``rmsnorm_i8``: the root-mean-square norm before it, with the residual's
  addition, whose output is written in 8 bits with a scale for each token;
- ``gated_i8``: the gated activation between two products, act(gate) * up,
  written the same way;
- ``quantize_i8``: any matrix's rows to 8 bits and scales (the weights, once,
  and activations that no other operator makes).

What an operator writes in 8 bits is read back here by ``dequantize_i8``, as
a program does that goes on with it in floating point: a pass of the last
three is the operator and the reading back of what it wrote.

``own`` chooses between those calls and the same operators in their plain
form, elementary torch operations in 32 bits.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-6


# ------------------------------------------------------------------ the cases

def _gemm(name, M, N, K, out, bias=False, slack=0):
    return {"name": name, "op": "gemm", "M": M, "N": N, "K": K, "out": out, "bias": bias, "slack": slack}


def _norm(name, M, N, dtype, residual=True, wide=False, slack=0):
    return {"name": name, "op": "norm", "M": M, "N": N, "dtype": dtype, "residual": residual, "wide": wide, "slack": slack}


def _gated(name, M, N, dtype, act):
    return {"name": name, "op": "gated", "M": M, "N": N, "dtype": dtype, "act": act}


def _quant(name, M, N, dtype, slack=0):
    return {"name": name, "op": "quant", "M": M, "N": N, "dtype": dtype, "slack": slack}


def listed():
    return [
        # a dense layer for the one token that is being generated: the weights are read once
        _gemm("gemm_token", 1, 4096, 4096, "bf16"),
        # the same layer for 32 sequences that generate together
        _gemm("gemm_dense_b32", 32, 4096, 4096, "f16"),
        # odd sizes, both operands slices of wider arrays whose rows start at any byte, with a bias
        _gemm("gemm_odd", 1021, 1531, 1777, "f32", bias=True, slack=3),
        # a dense layer over a prompt of 4096 tokens
        _gemm("gemm_4096", 4096, 4096, 4096, "bf16"),
        # the large square product: a wide layer over several prompts
        _gemm("gemm_8192", 8192, 8192, 8192, "bf16"),
        # the norm of one token: latency
        _norm("norm_token", 1, 4096, "bf16"),
        # rows of an odd length, no residual, from a wider fp32 array
        _norm("norm_odd", 777, 5003, "f32", residual=False, slack=3),
        # the norm of a long batch of prompts, weights kept in 32 bits
        _norm("norm_prompts", 8192, 4096, "bf16", wide=True),
        # the activation for 32 sequences that generate together
        _gated("gated_b32", 32, 11000, "f16", "gelu"),
        # the activation over prompts, gate and up the halves of one projection's output
        _gated("gated_prompts", 8192, 8192, "bf16", "silu"),
        # a small batch of activations of an odd width
        _quant("quant_odd", 96, 2049, "f16", slack=5),
        # a wide layer's weights, from 32 bits, when a program starts
        _quant("quant_weights", 8192, 8192, "f32"),
    ]


MOST_FLOPS = 3.0e11   # of a drawn case: below the largest listed ones
MOST_ELEMENTS = 3 << 24


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """Half of the sizes as they fall, odd ones among them, half rounded to a multiple of 64 or 16."""
    v = _log(rng, lo, hi)
    if rng.random() < 0.5:
        step = rng.choice([s for s in (64, 64, 16) if s <= max(v, 16)] or [16])
        v = max(step, int(round(v / step)) * step)
    return min(max(v, lo), hi)


def _draw_one(rng):
    op = rng.choice(["gemm", "gemm", "gemm", "norm", "norm", "gated", "quant"])
    # tokens: half of the calls generate (few of them), half work on prompts
    M = _log(rng, 1, 64) if rng.random() < 0.5 else _size(rng, 64, 8192)
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    slack = rng.choice([0, 0, 0, 16, 3])
    if op == "gemm":
        return {"op": op, "M": M, "N": _size(rng, 64, 16384), "K": _size(rng, 64, 16384), "out": dtype,
                "bias": rng.random() < 0.3, "slack": slack}
    N = _size(rng, 64, 16384)
    if op == "norm":
        return {"op": op, "M": M, "N": N, "dtype": dtype, "residual": rng.random() < 0.7, "wide": rng.random() < 0.5,
                "slack": slack}
    if op == "gated":
        return {"op": op, "M": M, "N": N, "dtype": dtype, "act": rng.choice(["silu", "silu", "gelu"])}
    return {"op": op, "M": M, "N": N, "dtype": dtype, "slack": slack}


def draw(rng):
    while True:
        c = _draw_one(rng)
        if c["op"] == "gemm":
            if 2 * c["M"] * c["N"] * c["K"] <= MOST_FLOPS and max(c["M"] * c["N"], c["N"] * c["K"], c["M"] * c["K"]) <= 1 << 27:
                return c
        elif c["M"] * c["N"] <= MOST_ELEMENTS:
            return c


def _read_type(case):
    """What the 8-bit values are read back in: the input's type.  The gated values
    go through an exponential, whose last bit can move a value across a rounding
    boundary: they are read back in 16 bits, as the next layer's activations are."""
    return "bf16" if case["op"] == "gated" and case["dtype"] == "f32" else case["dtype"]


def work(case):
    M, N = case["M"], case["N"]
    if case["op"] == "gemm":
        K = case["K"]
        return {"bytes": M * K + N * K + 4 * (M + N) + (4 * N if case["bias"] else 0) + M * N * SIZE[case["out"]],
                "flops": 2 * M * N * K}
    size = SIZE[case["dtype"]]
    bytes_ = M * N * (1 + SIZE[_read_type(case)]) + 4 * M  # the 8-bit values, what they are read back as, the scales
    if case["op"] == "norm":
        return {"bytes": bytes_ + M * N * size * (3 if case["residual"] else 1) + N * (4 if case["wide"] else size),
                "flops": M * N * (7 if case["residual"] else 6)}
    if case["op"] == "gated":
        return {"bytes": bytes_ + 2 * M * N * size, "flops": 8 * M * N}
    return {"bytes": bytes_ + M * N * size, "flops": 4 * M * N}


# ------------------------------------------------------------------ inputs

def _matrix(g, rows, cols, slack, dtype, scale=1.0):
    t = torch.randn((rows, cols + slack), generator=g, device="cuda")
    return t.mul_(scale).to(dtype)[:, :cols]


def _int8(g, rows, cols, slack, spread):
    """8-bit values as quantising a normal distribution gives them: the largest of a row near 127."""
    t = torch.randn((rows, cols + slack), generator=g, device="cuda")
    return t.mul_(spread).round_().clamp_(-127, 127).to(torch.int8)[:, :cols]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    M, N = case["M"], case["N"]
    if case["op"] == "gemm":
        K = case["K"]
        a, b = _int8(g, M, K, case["slack"], 32.0), _int8(g, N, K, case["slack"], 32.0)
        sa = (0.5 + torch.rand(M, generator=g, device="cuda")) / 32
        sb = (0.5 + torch.rand(N, generator=g, device="cuda")) / 32 * K ** -0.5
        bias = torch.randn(N, generator=g, device="cuda") * 0.1 if case["bias"] else None
        return {"case": case, "a": a, "b": b, "sa": sa, "sb": sb, "bias": bias}
    dtype = TYPES[case["dtype"]]
    if case["op"] == "norm":
        # a residual stream with a few channels that are larger than the rest
        x = _matrix(g, M, N, case["slack"], dtype, 0.5)
        big = 1 + 7 * (torch.rand(N, generator=g, device="cuda") < 0.01)
        r = (torch.randn((M, N), generator=g, device="cuda") * big).to(dtype) if case["residual"] else None
        w = 1 + 0.1 * torch.randn(N, generator=g, device="cuda")
        return {"case": case, "x": x, "r": r, "w": w if case["wide"] else w.to(dtype)}
    if case["op"] == "gated":
        p = _matrix(g, M, 2 * N, 0, dtype)  # the fused projection's output
        return {"case": case, "gate": p[:, :N], "up": p[:, N:]}
    return {"case": case, "x": _matrix(g, M, N, case["slack"], dtype)}


# ------------------------------------------------------------------ the framework's operators

def _run_own(state):
    import paper_1904_05347_amd as pk
    case = state["case"]
    if case["op"] == "gemm":
        return pk.gemm_i8(state["a"], state["b"], state["sa"], state["sb"], bias=state["bias"], dtype=TYPES[case["out"]])
    read = TYPES[_read_type(case)]
    if case["op"] == "norm":
        q, scale, h = pk.rmsnorm_i8(state["x"], state["w"], residual=state["r"], eps=EPS)
        values = pk.dequantize_i8(q, scale, dtype=read)
        return (values, scale, h) if case["residual"] else (values, scale)
    if case["op"] == "gated":
        q, scale = pk.gated_i8(state["gate"], state["up"], activation=case["act"])
    else:
        q, scale = pk.quantize_i8(state["x"])
    return pk.dequantize_i8(q, scale, dtype=read), scale


# ------------------------------------------------------------------ the plain forms

def _plain_rows(z):
    """(8-bit values, largest magnitude) of each row of fp32 z: round(z * (127 / max |z|))."""
    amax = z.abs().amax(dim=1, keepdim=True)
    return torch.round(z * (127.0 / amax)), amax


def run(state):
    if own:
        return _run_own(state)
    case = state["case"]
    if case["op"] == "gemm":
        c = torch.matmul(state["a"].float(), state["b"].float().t())
        c = c * (state["sa"][:, None] * state["sb"][None, :])
        if case["bias"]:
            c = c + state["bias"]
        return c.to(TYPES[case["out"]])
    read = TYPES[_read_type(case)]
    if case["op"] == "norm":
        h = state["x"]
        if case["residual"]:
            h = (h.float() + state["r"].float()).to(h.dtype)  # the residual stream as it is stored
        y = h.float()
        rms = torch.rsqrt((y * y).mean(dim=1, keepdim=True) + EPS)
        q, amax = _plain_rows(y * state["w"].float())
        scale = amax * rms / 127.0
        values = (q * scale).to(read)
        return (values, scale[:, 0], h) if case["residual"] else (values, scale[:, 0])
    if case["op"] == "gated":
        gate, up = state["gate"].float(), state["up"].float()
        if case["act"] == "silu":
            act = gate / (1.0 + torch.exp(-gate))
        else:
            act = 0.5 * gate * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (gate + 0.044715 * gate * gate * gate)))
        q, amax = _plain_rows(act * up)
    else:
        q, amax = _plain_rows(state["x"].float())
    scale = amax / 127.0
    return (q * scale).to(read), scale[:, 0]


# ------------------------------------------------------------------ from the definitions, in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "gemm":
        c = torch.empty((case["M"], case["N"]), dtype=torch.float64, device="cuda")
        b = s["b"].double().t().contiguous() * s["sb"].double()
        for i in range(0, case["M"], 2048):  # row blocks bound the memory
            c[i:i + 2048] = (s["a"][i:i + 2048].double() * s["sa"][i:i + 2048].double()[:, None]) @ b
        return c + s["bias"].double() if case["bias"] else c
    sums = None
    if case["op"] == "norm":
        h = s["x"].double()
        if case["residual"]:
            sums = h + s["r"].double()
            h = sums.to(s["x"].dtype).double()
        y = h * s["w"].double() / torch.sqrt(h.square().mean(dim=1, keepdim=True) + EPS)
    elif case["op"] == "gated":
        g, u = s["gate"].double(), s["up"].double()
        if case["act"] == "silu":
            y = g * torch.sigmoid(g) * u
        else:
            y = 0.5 * g * (1 + torch.tanh((2 / math.pi) ** 0.5 * (g + 0.044715 * g ** 3))) * u
    else:
        y = s["x"].double()
    scale = y.abs().amax(dim=1) / 127
    values = torch.round(y / scale[:, None]) * scale[:, None]
    return (values, scale) if sums is None else (values, scale, sums)
