"""Rows of the 8-bit floating-point operators that are as long as they may be: the last block's columns end at 2^31."""
import numpy as np
import pytest
import torch

import fp8_reference as ref
from paper_2410_16926_b200 import pvq

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16
COLS = [2 ** 31 - 127, 2 ** 31 - 100, 2 ** 31 - 72, 2 ** 31 - 1]
ENDS = 640  # columns looked at, at either end of a row: whole blocks, and the last one


def matrix(rows, cols, dtype, fill):
    """A matrix with the shortest allowed distance between its rows, and the bytes of all of it and 512 behind."""
    ld = -(-cols // 16) * 16
    size = dtype.itemsize
    raw = torch.empty(rows * ld * size + 512, dtype=torch.uint8, device="cuda")
    raw.fill_(fill)
    return raw[:rows * ld * size].view(dtype).view(rows, ld)[:, :cols], raw


def ends(t):
    first = -(-t.shape[1] // 128) * 128 - ENDS  # a block's first column
    return t[:, :ENDS], t[:, first:]


def untouched(raw, out, fill):
    """Between the rows and behind them."""
    rows, cols = out.shape
    size = out.element_size()
    lines = raw[:-512].view(rows, -1)
    return bool((lines[:, cols * size:] == fill).all()) and bool((raw[-512:] == fill).all())


def source(rows, cols, seed):
    """Ones, random at the ends of the rows, and large values wherever a row's end is overrun."""
    x, raw = matrix(rows, cols, BF16, 0x7f)  # (0x7f7f: 3.4e38)
    x.fill_(1.0)
    rng = np.random.default_rng(seed)
    for part in ends(x):
        part.copy_(torch.from_numpy(rng.standard_normal(tuple(part.shape)).astype(np.float32)))
    x[1:, :128] *= 1000.0
    return x


def same(codes, scales, x64, tile):
    want, b = ref.quantize(x64, tile)
    assert np.array_equal(ref.to64(codes), want) and np.array_equal(scales.view(torch.uint8).cpu().numpy(), b)


def of_8_bits(rows, cols, tile=False):
    codes, raw_codes = matrix(rows, cols, torch.uint8, 0xa5)
    scales = torch.full((1 if tile else rows, 2 ** 24), 0xa5, dtype=torch.uint8, device="cuda")
    return pvq.Fp8Matrix(codes.view(torch.float8_e4m3fn), scales.view(torch.float8_e8m0fnu), tile), raw_codes


@pytest.mark.parametrize("cols", COLS)
@pytest.mark.parametrize("tile", [False, True])
def test_quantize_and_dequantize(cols, tile):
    x = source(2, cols, 1)
    q, raw = of_8_bits(2, cols, tile)
    pvq.fp8_quantize(x, tile=tile, out=q)
    assert untouched(raw, q.codes, 0xa5)
    blocks = ENDS // 128
    for i, part in enumerate(ends(x)):
        scales = q.scales[:, :blocks] if i == 0 else q.scales[:, -blocks:]
        same(ends(q.codes)[i], scales, ref.to64(part), tile)
    out, raw = matrix(2, cols, BF16, 0xa5)
    pvq.fp8_dequantize(q, out=out)
    assert untouched(raw, out, 0xa5)
    for i, part in enumerate(ends(out)):
        scales = q.scales[:, :blocks] if i == 0 else q.scales[:, -blocks:]
        assert np.array_equal(ref.to64(part), ref.values(pvq.Fp8Matrix(ends(q.codes)[i], scales, tile)))


@pytest.mark.parametrize("cols", COLS)
def test_gated(cols):
    """As rows of the ends alone: a block knows nothing of the others."""
    gate, up = source(2, cols, 2), source(2, cols, 3)
    made = pvq.fp8_gated(gate, up, checkpoint=True)
    blocks = ENDS // 128
    for i in (0, 1):
        def cut(t):
            part = torch.zeros((2, ENDS), dtype=BF16, device="cuda")
            part[:, :ends(t)[i].shape[1]] = ends(t)[i]
            return part[:, :ends(t)[i].shape[1]]
        for q, want in zip(made, pvq.fp8_gated(cut(gate), cut(up), checkpoint=True)):
            assert torch.equal(ends(q.codes)[i].contiguous().view(torch.uint8), want.codes.contiguous().view(torch.uint8))
            scales = q.scales[:, :blocks] if i == 0 else q.scales[:, -blocks:]
            assert torch.equal(scales.contiguous().view(torch.uint8), want.scales.contiguous().view(torch.uint8))
    h, gate8, up8 = made
    del made, up, h
    outs = [matrix(2, cols, BF16, 0xa5) for _ in range(2)]
    pvq.fp8_gated_backward(gate, gate8, up8, out=[o for o, _ in outs])
    for out, raw in outs:
        assert untouched(raw, out, 0xa5)
    for i in (0, 1):
        part = [pvq.Fp8Matrix(torch.zeros((2, ENDS), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)[:, :ends(q.codes)[i].shape[1]],
                              torch.zeros((2, 8), dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu)[:, :blocks], False) for q in (gate8, up8)]
        for p, q in zip(part, (gate8, up8)):
            p.codes.view(torch.uint8).copy_(ends(q.codes)[i].view(torch.uint8))
            p.scales.view(torch.uint8).copy_((q.scales[:, :blocks] if i == 0 else q.scales[:, -blocks:]).view(torch.uint8))
        dh = torch.zeros((2, ENDS), dtype=BF16, device="cuda")[:, :ends(gate)[i].shape[1]]
        dh.copy_(ends(gate)[i])
        for (out, _), want in zip(outs, pvq.fp8_gated_backward(dh, *part)):
            assert torch.equal(ends(out)[i], want)
