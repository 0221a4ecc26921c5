"""The 8-bit floating-point operators from their definitions, in 64 bits (NumPy), and how far the kernels may be off.

A half step of a type is eps / 2 of a value: 2^-8 (bf16), 2^-24 (fp32), 2^-4 (e4m3)."""
import numpy as np
import torch

HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def to64(t):
    return t.detach().to(torch.float64).cpu().numpy()


def e4m3(v):
    """Nearest e4m3 value, ties to even, of numbers up to 448 in magnitude."""
    _, e = np.frexp(v)
    step = np.ldexp(1.0, np.maximum(e - 1, -6) - 3)
    return np.round(v / step) * step


def half_step_e4m3(v):
    """Half the distance between e4m3 values around v (in units of the scale)."""
    _, e = np.frexp(v)
    return np.ldexp(0.5, np.maximum(e - 1, -6) - 3)


def spread(s, rows, cols, tile):
    """Scales of blocks -> of every value."""
    s = np.repeat(s, 128, axis=1)[:, :cols]
    return np.repeat(s, 128, axis=0)[:rows] if tile else s


def block_max(x, tile):
    rows, cols = x.shape
    high = 128 if tile else 1
    pad = np.zeros((-(-rows // high) * high, -(-cols // 128) * 128))
    pad[:rows, :cols] = np.where(np.isfinite(x), np.abs(x), 0.0)
    return pad.reshape(pad.shape[0] // high, high, pad.shape[1] // 128, 128).max(axis=(1, 3))


def scale_bytes(amax):
    """Smallest e >= -126 with amax <= 448 * 2^e, plus 127; 127 for blocks of zeros."""
    out = np.full(amax.shape, 127, dtype=np.int64)
    for i in np.ndindex(amax.shape):
        if amax[i] > 0:
            e = -126
            guess = int(np.floor(np.log2(amax[i]))) - 10
            e = max(e, guess)
            while amax[i] > 448.0 * 2.0 ** e:
                e += 1
            out[i] = e + 127
    return out


def quantize(x, tile):
    """(code values, scale bytes) of a float64 matrix."""
    b = scale_bytes(block_max(x, tile))
    s = spread(np.ldexp(1.0, b - 127), *x.shape, tile)
    with np.errstate(invalid="ignore"):
        return np.where(np.isfinite(x), e4m3(np.where(np.isfinite(x), x, 0.0) / s), np.nan), b


def values(q):
    """The values of an Fp8Matrix."""
    codes, scales, tile = q
    b = scales.view(torch.uint8).cpu().numpy().astype(np.int64)
    s = np.where(b == 255, np.nan, np.ldexp(1.0, np.where(b == 255, 0, b - 127)))
    return to64(codes) * spread(s, *codes.shape, tile)


def matmul_slack(a, b, inner_steps):
    """What sums in fp32 may lose: tensor cores add the products of 16 or 32 values at a time to the running sum, each such
    step and each of the additions inside one truncates at most 2^-23 of the magnitudes' sum."""
    return (inner_steps + 32) * 2.0 ** -23 * (np.abs(a) @ np.abs(b))


def argument(g, act):
    """w with act(g) = g * sigma(w), and its slope."""
    if act == "silu":
        return g, np.ones_like(g)
    k = 2.0 * np.sqrt(2.0 / np.pi)
    return k * (g + 0.044715 * g ** 3), k * (1.0 + 3.0 * 0.044715 * g ** 2)


def sigma(w):
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-w))


def activation(g, act):
    """Gelu too by sigma: (1 + tanh z) / 2 = sigma(2 z), where 1 + tanh z has no digits left in 64 bits from z = -19 down."""
    return g * sigma(argument(g, act)[0])


def slope(g, act):
    w, dw = argument(g, act)
    s = sigma(w)
    return s + g * s * (1.0 - s) * dw


def sigma_slack(g, act):
    """Relative error of sigma(w) in fp32: w has a handful of roundings (2^-24 each, of terms of w's size), so e^-w is off by
    |w| * 2^-22 and the exponential's own 2^-22; the sum and the reciprocal add 2^-23 each."""
    w, _ = argument(g, act)
    return (np.abs(w) + 3.0) * 2.0 ** -22
