"""Cases, plain forms and 64-bit definitions of the second half of a decoder layer in 8 bits.

Two operators: the linear layer on 8-bit integers with what stands around it in a layer (a root-mean-square norm before the
tokens are quantized; bias, activation and residual sum behind the product), and the gated feed-forward block (norm, gate
and up projection, activation, their product, quantized again, down projection, residual sum).  `run` computes them with
elementary torch operations in 32 bits while `own` is false and through paper_2410_13056_b200.serving while it is true.
"""
import math

import torch

own = False

_DT = {"bf16": torch.bfloat16, "fp16": torch.float16}
_EPS = 1e-5
_ACTS = ["none", "relu", "silu", "gelu", "gelu_tanh"]


# ---- cases ---------------------------------------------------------------------------------------------------

def _linear(name, n, d_in, d_out, dtype, act, bias, norm, residual):
    return {"name": name, "op": "linear", "n": n, "d_in": d_in, "d_out": d_out, "dtype": dtype, "act": act, "bias": bias, "norm": norm,
            "residual": residual}


def _gated(name, n, d_in, d_ff, d_out, dtype, act, bias, norm, residual):
    return {"name": name, "op": "gated", "n": n, "d_in": d_in, "d_ff": d_ff, "d_out": d_out, "dtype": dtype, "act": act, "bias": bias,
            "norm": norm, "residual": residual}


def listed():
    return [
        # one generated token through the output projection of an attention block, added to the layer's input
        _linear("linear one token, residual", 1, 4096, 4096, "bf16", "none", False, False, True),
        # a decoding batch through the norm and the up projection of a block without a gate
        _linear("linear batch 53, norm gelu", 53, 4096, 11008, "fp16", "gelu", True, True, False),
        # a chunk of a prompt through a down projection; neither size a multiple of a tile
        _linear("linear chunk 777, residual", 777, 11008, 4096, "bf16", "none", True, False, True),
        # prompts through the norm and an activated projection
        _linear("linear prompts 4000, norm silu", 4000, 4096, 11008, "bf16", "silu", False, True, False),
        # one stream generating: the time of the block for one token
        _gated("gated one token", 1, 4096, 11008, 4096, "bf16", "silu", False, True, True),
        # one stream, small layers: the time of the call itself counts
        _gated("gated one token, small", 1, 512, 1408, 512, "fp16", "silu", False, True, True),
        # five drafted tokens, sizes that fill no tile, biases, no norm of its own
        _gated("gated drafts 5, odd", 5, 2050, 5461, 2049, "fp16", "gelu_tanh", True, False, False),
        # a decoding batch through the largest layer
        _gated("gated batch 32, large", 32, 8192, 28672, 8192, "bf16", "silu", False, True, True),
        # a larger batch of streams
        _gated("gated batch 100", 100, 4096, 11008, 4096, "fp16", "silu", False, True, True),
        # a chunk of a prompt
        _gated("gated chunk 517", 517, 4096, 11008, 4096, "bf16", "gelu", False, True, True),
        # prompts of a common layer
        _gated("gated prompts 2048", 2048, 4096, 11008, 4096, "fp16", "silu", False, True, True),
        # whole prompts through the largest layer of the largest workload
        _gated("gated prompts 4096, large", 4096, 8192, 28672, 8192, "bf16", "silu", False, True, True),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["linear", "gated", "gated"])
    dtype, bias, norm, residual = rng.choice(["bf16", "fp16"]), rng.random() < 0.3, rng.random() < 0.7, rng.random() < 0.7
    round_up = 128 if rng.random() < 0.6 else 1  # most layers have round sizes
    while True:
        n = _log_int(rng, 1, 4096)
        d_in, d_ff = (-(-_log_int(rng, 512, most) // round_up) * round_up for most in (8192, 28672))
        if op == "linear":
            if rng.random() < 0.4:
                d_in, d_ff = d_ff, d_in
            if n * d_in * d_ff <= 4096 * 8192 * 28672:
                c = _linear("", n, d_in, d_ff, dtype, rng.choice(_ACTS), bias, norm, residual)
                break
        elif 3 * n * d_in * d_ff <= 3 * 4096 * 8192 * 28672:
            c = _gated("", n, d_in, d_ff, d_in, dtype, rng.choice(["silu", "silu"] + _ACTS), bias, norm, residual)
            break
    del c["name"]
    return c


# ---- inputs --------------------------------------------------------------------------------------------------

def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)


def _weight(g, d_out, d_in, bias, dt):
    """Codes (rows on 16 bytes), a scale per output channel, and the bias."""
    w = _randn(g, d_out, d_in) * (1.3 / math.sqrt(d_in))
    scale = w.abs().amax(1) * (1.0 / 127.0)
    codes = torch.zeros(d_out, (d_in + 15) // 16 * 16, dtype=torch.int8, device="cuda")
    codes[:, :d_in] = torch.round(w / scale[:, None]).to(torch.int8)
    return {"codes": codes[:, :d_in], "scale": scale, "bias": (0.1 * _randn(g, d_out)).to(dt) if bias else None}


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    dt, n, d_in, d_out = _DT[case["dtype"]], case["n"], case["d_in"], case["d_out"]
    # channels of very different size, one in a hundred far out, as a layer's input has them; the norm's weights are small there
    sigma = torch.exp(0.5 * _randn(g, d_in))
    far = torch.randperm(d_in, generator=g, device="cuda")[: max(1, d_in // 100)]
    sigma[far] *= 8.0
    x = (_randn(g, n, d_in) * sigma).to(dt)
    weight = (1.0 + 0.2 * _randn(g, d_in)).abs()
    weight[far] *= 0.3
    st = {"op": case["op"], "act": case["act"], "x": x, "norm": weight.to(dt) if case["norm"] else None, "residual": None}
    if case["residual"]:  # the layer's input: of a block that starts with its norm, the block's own
        st["residual"] = x if case["op"] == "gated" and d_out == d_in else _randn(g, n, d_out).to(dt)
    if case["op"] == "linear":
        st["w"] = _weight(g, d_out, d_in, case["bias"], dt)
    else:
        st["gate"], st["up"] = (_weight(g, case["d_ff"], d_in, case["bias"], dt) for _ in range(2))
        st["down"] = _weight(g, d_out, case["d_ff"], case["bias"], dt)
    return st


# ---- plain forms ---------------------------------------------------------------------------------------------

def _codes(x, norm):
    """Codes of the rows, as floats, and their scales."""
    v = x if norm is None else x * norm.float()
    scale = v.abs().amax(1, keepdim=True) * (1.0 / 127.0)
    inv = torch.where(scale > 0, torch.reciprocal(scale), torch.zeros_like(scale))
    codes = torch.round(v * inv).clamp(-127, 127)
    if norm is not None:
        scale = scale * torch.reciprocal(torch.sqrt((x * x).mean(1, keepdim=True) + _EPS))
    return codes, scale


def _product(codes, scale, w):
    z = (codes @ w["codes"].float().t()) * scale * w["scale"]
    return z if w["bias"] is None else z + w["bias"].float()


def _act(z, act):
    if act == "relu":
        return z.clamp(min=0)
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * torch.erfc(-math.sqrt(0.5) * z)
    if act == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)))
    return z


def _plain(st):
    dt = st["x"].dtype
    codes, scale = _codes(st["x"].float(), st["norm"])
    if st["op"] == "linear":
        y = _act(_product(codes, scale, st["w"]), st["act"])
    else:
        h = _act(_product(codes, scale, st["gate"]), st["act"]) * _product(codes, scale, st["up"])
        y = _product(*_codes(h.to(dt).float(), None), st["down"])  # h is a 16-bit value by the operator's definition
    if st["residual"] is not None:
        y = y + st["residual"].float()
    return {"y": y.to(dt)}


# ---- the framework's operators -------------------------------------------------------------------------------

def _own(st):
    from paper_2410_13056_b200 import serving

    if "layer" not in st:  # what a program makes once and keeps
        made = {k: serving.Int8Linear(st[k]["codes"], st[k]["scale"], st[k]["bias"]) for k in ("w", "gate", "up", "down") if k in st}
        st["layer"] = made["w"] if st["op"] == "linear" else serving.GatedMLP8(made["gate"], made["up"], made["down"], activation=st["act"])
    if st["op"] == "linear":
        return {"y": st["layer"](st["x"], activation=st["act"], residual=st["residual"], norm=st["norm"], eps=_EPS)}
    return {"y": st["layer"](st["x"], residual=st["residual"], norm=st["norm"], eps=_EPS)}


def run(state):
    return _own(state) if own else _plain(state)


# ---- what a pass cannot do without ---------------------------------------------------------------------------

def work(case):
    n, d_in, d_out = case["n"], case["d_in"], case["d_out"]
    gated = case["op"] == "gated"
    shapes = [(case["d_ff"], d_in), (case["d_ff"], d_in), (d_out, case["d_ff"])] if gated else [(d_out, d_in)]
    moved = 2 * n * (d_in + d_out) + sum(o * i + (6 if case["bias"] else 4) * o for o, i in shapes)
    if case["norm"]:
        moved += 2 * d_in
    if case["residual"] and not (gated and d_in == d_out):  # there it is x, read once
        moved += 2 * n * d_out
    return {"bytes": moved, "flops": 2 * n * sum(o * i for o, i in shapes)}


# ---- the definitions in 64 bits ------------------------------------------------------------------------------

def _rows64(x, weight):
    rms = 1.0
    if weight is not None:
        rms = torch.sqrt(torch.linalg.vecdot(x, x)[:, None] / x.shape[1] + _EPS)
        x = torch.mul(x, weight.double())
    step = x.abs().max(dim=1, keepdim=True).values / 127
    q = torch.where(step > 0, torch.round(x / step.clamp(min=1e-300)), torch.zeros_like(x))
    return q, step / rms


def _layer64(q, step, w):
    z = torch.matmul(q, w["codes"].double().T)
    z *= step
    z *= w["scale"].double()
    return z if w["bias"] is None else z.add_(w["bias"].double())


_ACT64 = {
    "none": lambda z: z,
    "relu": lambda z: torch.where(z > 0, z, torch.zeros_like(z)),
    "silu": lambda z: z * torch.sigmoid(z),
    "gelu": lambda z: z * torch.special.ndtr(z),
    "gelu_tanh": lambda z: z * torch.sigmoid(math.sqrt(8 / math.pi) * (z + 0.044715 * z ** 3)),
}


def exact(case, seed):
    st = prepare(case, seed)
    f = _ACT64[case["act"]]
    q, step = _rows64(st["x"].double(), st["norm"])
    if case["op"] == "linear":
        y = f(_layer64(q, step, st["w"]))
    else:
        h = f(_layer64(q, step, st["gate"])).mul_(_layer64(q, step, st["up"]))
        y = _layer64(*_rows64(h.to(st["x"].dtype).double(), None), st["down"])
    return {"y": y if st["residual"] is None else y + st["residual"].double()}
