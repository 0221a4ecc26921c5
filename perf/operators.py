"""What the 8-bit floating-point operators are measured on.

The format is e4m3 codes with one power-of-two scale (e8m0) for each block of 128 values of a row, or for each
block of 128 x 128 values of a weight.  The operators that make and read it:

  - quantize / dequantize: activations and gradients by rows, weights by tiles;
  - matmul: activations times a weight, and, with the same codes, a gradient times the transposed weight;
  - gated / gated_backward: the activation of a gated feed-forward block, its result in 8 bits for the next
    product, its two inputs kept in 8 bits and read back in the backward pass;
  - weight_grad: the gradient of a weight from the 8-bit input that the forward pass kept.

A case is one call.  Shapes are the projections of `inputs.py`'s decoder layer (4096 and 14336 features, 1024 for
keys and values) and of its largest single matrix (8192 x 28672); rows are tokens, from one to a long prefill.
With `own` false everything is computed by elementary torch operations in 32 bits.
"""
import math

import torch

own = False

BLOCK = 128
LARGEST = 448.0  # of e4m3


def listed():
    return [
        # a decoded token's hidden state on its way into a projection: what a call costs
        dict(name="quantize one token", op="quantize", rows=1, cols=4096, tile=False, dtype="bf16"),
        # the activations of a long prefill (or of a training batch)
        dict(name="quantize activations", op="quantize", rows=16384, cols=4096, tile=False, dtype="bf16"),
        # a weight read back from its 8-bit tiles
        dict(name="dequantize weight", op="dequantize", rows=14336, cols=4096, tile=True, dtype="bf16"),
        # a decoded token through the up projection: the weight's bytes
        dict(name="matmul one token", op="matmul", rows=1, inner=4096, outer=14336, transposed=False, dtype="bf16"),
        # a batch of decoded tokens through the down projection
        dict(name="matmul 33 tokens", op="matmul", rows=33, inner=14336, outer=4096, transposed=False, dtype="bf16"),
        # an ordinary prompt (an odd number of tokens) through the attention's output projection
        dict(name="matmul prompt", op="matmul", rows=1999, inner=4096, outer=4096, transposed=False, dtype="bf16"),
        # a training batch through the up projection
        dict(name="matmul training", op="matmul", rows=16384, inner=4096, outer=14336, transposed=False, dtype="bf16"),
        # the gradient of the same projection's input (the transposed weight), kept in 32 bits
        dict(name="matmul input gradient", op="matmul", rows=8192, inner=14336, outer=4096, transposed=True, dtype="f32"),
        # the middle of the feed-forward block of a training batch, with its checkpoints
        dict(name="gated training", op="gated", rows=16384, cols=14336, checkpoint=True, act="silu", dtype="bf16"),
        # its backward pass for a short batch
        dict(name="gated backward", op="gated_backward", rows=1999, cols=14336, act="silu", dtype="bf16"),
        # the gradient of the up projection's weight over a training batch
        dict(name="weight gradient training", op="weight_grad", rows=16384, inner=4096, outer=14336, dtype="f32"),
        # of a key projection's weight over a short batch (an odd number of tokens)
        dict(name="weight gradient short", op="weight_grad", rows=1001, inner=4096, outer=1024, dtype="bf16"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("quantize", "dequantize", "matmul", "matmul", "matmul", "matmul", "gated", "gated_backward",
                     "weight_grad", "weight_grad"))
    rows = _log_uniform(rng, 1, 16384)
    features = (1024, 4096, 8192, 14336)

    def size():  # a projection's width, or any
        return rng.choice(features) if rng.random() < 0.5 else _log_uniform(rng, 200, 14336)

    if op in ("quantize", "dequantize"):
        return dict(op=op, rows=rows, cols=size(), tile=rng.random() < 0.4, dtype=rng.choice(("bf16", "f32")))
    if op == "gated":
        return dict(op=op, rows=rows, cols=size(), checkpoint=rng.random() < 0.6, act=rng.choice(("silu", "gelu")),
                    dtype=rng.choice(("bf16", "bf16", "f32")) if rows <= 8192 else "bf16")
    if op == "gated_backward":
        return dict(op=op, rows=rows, cols=size(), act=rng.choice(("silu", "gelu")),
                    dtype=rng.choice(("bf16", "bf16", "f32")) if rows <= 8192 else "bf16")
    inner, outer = size(), size()
    rows = min(rows, 16384 * 4096 * 14336 // (inner * outer))
    if op == "matmul":
        if rng.random() < 0.3:  # single tokens, small batches
            rows = _log_uniform(rng, 1, 128)
        return dict(op=op, rows=rows, inner=inner, outer=outer, transposed=rng.random() < 0.4,
                    dtype=rng.choice(("bf16", "bf16", "f32")))
    return dict(op=op, rows=rows, inner=inner, outer=outer, dtype=rng.choice(("bf16", "f32")))


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


# ---- inputs ---------------------------------------------------------------------------

def _padded(rows, cols, dtype, unit):
    """An uninitialised matrix whose rows start on 16-byte boundaries."""
    return torch.empty((rows, -(-cols // unit) * unit), dtype=dtype, device="cuda")[:, :cols]


def _activations(g, rows, cols, dtype):
    """Tokens' features: normal, one channel in a thousand 20 times as large, the last of many tokens padding."""
    x = torch.randn((rows, cols), generator=g, device="cuda")
    x *= torch.where(torch.rand(cols, generator=g, device="cuda") < 0.001, 20.0, 1.0)
    if rows > 64:
        x[rows - rows // 50 - 1:] = 0.0
    out = _padded(rows, cols, dtype, 16)
    out.copy_(x)
    return out


def _weight(g, rows, cols):
    return torch.randn((rows, cols), generator=g, device="cuda") * 0.02


def _held(x, tile):
    """The codes and scales of a matrix as a program holds them: rows of codes on 16-byte boundaries, rows of
    scales on 4-byte boundaries."""
    q, s = _quantize(x, tile)
    codes = _padded(q.shape[0], q.shape[1], torch.uint8, 16)
    codes.copy_(q.view(torch.uint8))
    scales = _padded(s.shape[0], s.shape[1], torch.uint8, 4)
    scales.copy_(s.view(torch.uint8))
    return codes.view(torch.float8_e4m3fn), scales.view(torch.float8_e8m0fnu), tile


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    op, rows, state = case["op"], case["rows"], dict(case=case)
    if op in ("quantize", "dequantize"):
        x = _weight(g, rows, case["cols"]) if case["tile"] else _activations(g, rows, case["cols"], _dtype(case))
        if op == "quantize":
            state["x"] = _padded(rows, case["cols"], _dtype(case), 16).copy_(x)
        else:
            state["x"] = _held(x, case["tile"])
    elif op == "matmul":
        shape = (case["inner"], case["outer"]) if case["transposed"] else (case["outer"], case["inner"])
        state["a"] = _held(_activations(g, rows, case["inner"], torch.float32), False)
        state["b"] = _held(_weight(g, *shape), True)
    elif op == "gated":  # the two halves of one product's result
        both = _activations(g, rows, 2 * (-(-case["cols"] // 16) * 16), _dtype(case))
        half = both.shape[1] // 2
        state["gate"], state["up"] = both[:, :case["cols"]], both[:, half:half + case["cols"]]
    elif op == "gated_backward":
        state["dh"] = _activations(g, rows, case["cols"], _dtype(case))
        state["gate"] = _held(_activations(g, rows, case["cols"], torch.float32), False)
        state["up"] = _held(_activations(g, rows, case["cols"], torch.float32), False)
    else:
        state["dy"] = _activations(g, rows, case["outer"], torch.bfloat16)
        state["x"] = _held(_activations(g, rows, case["inner"], torch.float32), False)
    return state


# ---- the operators in plain form ---------------------------------------------------------

def _blocks(x, tile):
    """The matrix cut into blocks, with zeros behind its ends: [blocks down][rows each][blocks across][128]."""
    rows, cols = x.shape
    high = BLOCK if tile else 1
    down, across = -(-rows // high), -(-cols // BLOCK)
    if (down * high, across * BLOCK) != (rows, cols):
        x = torch.nn.functional.pad(x, (0, across * BLOCK - cols, 0, down * high - rows))
    return x.reshape(down, high, across, BLOCK)


def _quantize(x, tile):
    """Codes [rows][cols] and scales: the smallest power of two, from 2^-126, by which the block's largest finite
    magnitude is at most 448, 1 for a block without one; what is not finite has the code NaN."""
    rows, cols = x.shape
    b = _blocks(x.float(), tile)
    finite = torch.isfinite(b)
    amax = torch.where(finite, b.abs(), 0.0).amax(dim=(1, 3))
    mantissa, exponent = torch.frexp(amax)  # amax = mantissa 2^exponent, mantissa in [1/2, 1): 448 is 0.875 2^9
    e = torch.where(amax > 0, torch.clamp(exponent - 9 + (mantissa > 0.875).int(), min=-126), 0)
    q = torch.where(finite, torch.ldexp(b, -e[:, None, :, None]), math.nan)
    q = q.reshape(-1, q.shape[2] * BLOCK)[:rows, :cols].to(torch.float8_e4m3fn)
    return q, (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def _dequantize(held, to=torch.float32):
    codes, scales, tile = held
    b = _blocks(codes.to(to), tile)
    b = b * torch.exp2(scales.view(torch.uint8).to(to) - 127)[:, None, :, None]
    return b.reshape(-1, b.shape[2] * BLOCK)[:codes.shape[0], :codes.shape[1]]


def _act(g, act):
    if act == "silu":
        return g * torch.sigmoid(g)
    return 0.5 * g * (1 + torch.tanh(math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3)))


def _act_slope(g, act):
    if act == "silu":
        s = torch.sigmoid(g)
        return s * (1 + g * (1 - s))
    t = torch.tanh(math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3))
    return 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * g ** 2)


def _plain(state):
    case = state["case"]
    op = case["op"]
    if op == "quantize":
        return _quantize(state["x"], case["tile"])
    if op == "dequantize":
        return _dequantize(state["x"]).to(_dtype(case))
    if op == "matmul":
        a, b = _dequantize(state["a"]), _dequantize(state["b"])
        return (a @ (b if case["transposed"] else b.t())).to(_dtype(case))
    if op == "gated":
        gate, up = state["gate"].float(), state["up"].float()
        out = _quantize(_act(gate, case["act"]) * up, False)
        if case["checkpoint"]:
            out += _quantize(gate, False) + _quantize(up, False)
        return out
    if op == "gated_backward":
        dh, gate, up = state["dh"].float(), _dequantize(state["gate"]), _dequantize(state["up"])
        return (dh * up * _act_slope(gate, case["act"])).to(_dtype(case)), (dh * _act(gate, case["act"])).to(_dtype(case))
    return (state["dy"].float().t() @ _dequantize(state["x"])).to(_dtype(case))


# ---- the framework's -----------------------------------------------------------------------

def _own(state):
    from paper_2410_16926_b200 import pvq
    case = state["case"]
    op = case["op"]
    if op == "quantize":
        q = pvq.fp8_quantize(state["x"], tile=case["tile"])
        return q.codes, q.scales
    if op == "dequantize":
        return pvq.fp8_dequantize(pvq.Fp8Matrix(*state["x"]), dtype=_dtype(case))
    if op == "matmul":
        return pvq.fp8_matmul(pvq.Fp8Matrix(*state["a"]), pvq.Fp8Matrix(*state["b"]), transposed=case["transposed"],
                              dtype=_dtype(case))
    if op == "gated":
        if not case["checkpoint"]:
            h = pvq.fp8_gated(state["gate"], state["up"], act=case["act"])
            return h.codes, h.scales
        h, gate, up = pvq.fp8_gated(state["gate"], state["up"], act=case["act"], checkpoint=True)
        return h.codes, h.scales, gate.codes, gate.scales, up.codes, up.scales
    if op == "gated_backward":
        return pvq.fp8_gated_backward(state["dh"], pvq.Fp8Matrix(*state["gate"]), pvq.Fp8Matrix(*state["up"]), act=case["act"])
    return pvq.fp8_weight_grad(state["dy"], pvq.Fp8Matrix(*state["x"]), dtype=_dtype(case))


def run(state):
    return _own(state) if own else _plain(state)


# ---- what a pass cannot do without -----------------------------------------------------------

def work(case):
    op, rows = case["op"], case["rows"]
    size = 2 if case["dtype"] == "bf16" else 4

    def held(r, c, tile=False):  # bytes of codes and scales
        return r * c + (-(-r // BLOCK) if tile else r) * -(-c // BLOCK)

    if op in ("quantize", "dequantize"):
        n = rows * case["cols"]
        return dict(bytes=n * size + held(rows, case["cols"], case["tile"]), flops=2 * n)
    if op == "gated":
        n = rows * case["cols"]
        return dict(bytes=2 * n * size + (3 if case["checkpoint"] else 1) * held(rows, case["cols"]), flops=10 * n)
    if op == "gated_backward":
        n = rows * case["cols"]
        return dict(bytes=3 * n * size + 2 * held(rows, case["cols"]), flops=14 * n)
    inner, outer = case["inner"], case["outer"]
    flops = 2 * rows * inner * outer
    if op == "matmul":
        return dict(bytes=held(rows, inner) + held(outer, inner, True) + rows * outer * size, flops=flops)
    return dict(bytes=rows * outer * 2 + held(rows, inner) + outer * inner * size, flops=flops)


# ---- the same in 64 bits ---------------------------------------------------------------------

def _e4m3_64(v):
    """The nearest e4m3 value (ties to the even one) of numbers of magnitude up to 448."""
    _, e = torch.frexp(v)
    step = torch.ldexp(torch.ones_like(v), torch.clamp(e - 1, min=-6) - 3)
    return torch.round(v / step) * step  # (torch.round: halves to even)


def _codes_64(x, tile):
    rows, cols = x.shape
    high = BLOCK if tile else 1
    pad = torch.zeros((-(-rows // high) * high, -(-cols // BLOCK) * BLOCK), dtype=torch.float64, device=x.device)
    pad[:rows, :cols] = x
    pad = pad.view(pad.shape[0] // high, high, pad.shape[1] // BLOCK, BLOCK)
    top = pad.abs().amax(dim=(1, 3))
    scale = torch.exp2(torch.clamp(torch.ceil(torch.log2(top / LARGEST)), min=-126.0))
    scale = torch.where(top > 0, scale, torch.ones_like(scale))
    scale = torch.where(top / scale > LARGEST, scale * 2, torch.where((top > 0) & (top / scale <= LARGEST / 2) & (scale > 2.0 ** -126), scale / 2, scale))
    codes = _e4m3_64(pad / scale[:, None, :, None])
    return codes.view(-1, pad.shape[2] * BLOCK)[:rows, :cols], scale


def _values_64(held):
    codes, scales, tile = held
    scale = scales.double().repeat_interleave(BLOCK, dim=1)[:, :codes.shape[1]]
    if tile:
        scale = scale.repeat_interleave(BLOCK, dim=0)[:codes.shape[0]]
    return codes.double() * scale


def _gate_64(g, act):
    """The activation and its slope."""
    if act == "silu":
        sig = 1 / (1 + torch.exp(-g))
        return g * sig, sig + g * sig * (1 - sig)
    k = math.sqrt(2 / math.pi)
    inner = k * (g + 0.044715 * g * g * g)
    t = torch.tanh(inner)
    return g * (1 + t) / 2, (1 + t) / 2 + g / 2 * (1 - t * t) * k * (1 + 0.134145 * g * g)


def exact(case, seed):
    state = prepare(case, seed)
    op = case["op"]
    if op == "quantize":
        return _codes_64(state["x"].double(), case["tile"])
    if op == "dequantize":
        return _values_64(state["x"])
    if op == "matmul":
        a, b = _values_64(state["a"]), _values_64(state["b"])
        return torch.mm(a, b) if case["transposed"] else torch.mm(a, b.t())
    if op == "gated":
        gate, up = state["gate"].double(), state["up"].double()
        out = _codes_64(_gate_64(gate, case["act"])[0] * up, False)
        if case["checkpoint"]:
            out += _codes_64(gate, False) + _codes_64(up, False)
        return out
    if op == "gated_backward":
        value, slope = _gate_64(_values_64(state["gate"]), case["act"])
        dh = state["dh"].double()
        return dh * _values_64(state["up"]) * slope, dh * value
    return torch.mm(state["dy"].double().t(), _values_64(state["x"]))
