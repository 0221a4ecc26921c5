"""The 8-bit floating-point operators without a GPU: what their entry points refuse, and the definitions the GPU tests
compare with."""
import ctypes as C

import numpy as np
import pytest
import torch

import fp8_reference as ref
from paper_2410_16926_b200 import pvq

INVALID, UNSUPPORTED, ALIGN = 1, 2, 3
P = 1 << 20  # an aligned address; the checks come before anything is read


def desc(rows=4, cols=256, ld_codes=256, ld_scales=4, tile=0, codes=P, scales=P):
    return pvq.Fp8Desc(codes, scales, rows, cols, ld_codes, ld_scales, tile)


BAD = [(dict(codes=None), INVALID), (dict(scales=None), INVALID), (dict(rows=0), INVALID), (dict(cols=0), INVALID), (dict(rows=-1), INVALID),
       (dict(tile=2), INVALID), (dict(ld_codes=240), INVALID), (dict(ld_scales=1), INVALID), (dict(codes=P + 8), ALIGN),
       (dict(ld_codes=264), ALIGN), (dict(scales=P + 2), ALIGN), (dict(ld_scales=6), ALIGN), (dict(rows=1 << 31), UNSUPPORTED),
       (dict(rows=1 << 30), UNSUPPORTED), (dict(ld_codes=1 << 36), UNSUPPORTED), (dict(rows=1, cols=1 << 31, ld_codes=1 << 31, ld_scales=1 << 24), UNSUPPORTED)]


@pytest.mark.parametrize("bad,status", BAD)
def test_matrices_are_checked(bad, status):
    L = pvq.lib()
    q, good = C.byref(desc(**bad)), C.byref(desc())
    cols = bad.get("cols", 256)
    ld = max(cols, 256)
    assert L.pvq_fp8_quantize(P, 1, ld, q, None) == status
    assert L.pvq_fp8_dequantize(q, P, 1, ld, None) == status
    assert L.pvq_fp8_matmul(q, good, 0, P, 1, 8, None, None) == status
    assert L.pvq_fp8_matmul(good, q, 0, P, 1, 8, None, None) == status
    assert L.pvq_fp8_gated(P, ld, P, ld, 1, 0, q, None, None, None) == status
    assert L.pvq_fp8_gated(P, 256, P, 256, 1, 0, good, q, good, None) == status
    assert L.pvq_fp8_gated(P, 256, P, 256, 1, 0, good, good, q, None) == status
    assert L.pvq_fp8_gated_backward(P, 256, 1, q, good, 0, P, 256, P, 256, None) == status
    assert L.pvq_fp8_gated_backward(P, 256, 1, good, q, 0, P, 256, P, 256, None) == status
    assert L.pvq_fp8_weight_grad(P, 64, 64, q, P, 0, ld, None, 0, None, None) == status
    assert L.pvq_fp8_quantize(P, 1, 256, None, None) == INVALID
    assert L.pvq_fp8_matmul(good, None, 0, P, 1, 8, None, None) == INVALID


@pytest.mark.parametrize("p,dtype,ld,status", [(None, 1, 256, INVALID), (P, 2, 256, INVALID), (P, 1, 248, INVALID), (P + 8, 1, 256, ALIGN),
                                               (P, 1, 260, ALIGN), (P, 0, 258, ALIGN), (P, 1, 1 << 36, UNSUPPORTED)])
def test_values_are_checked(p, dtype, ld, status):
    L = pvq.lib()
    q, w = C.byref(desc()), C.byref(desc(rows=256))
    t = C.byref(desc(rows=256, tile=1))
    assert L.pvq_fp8_quantize(p, dtype, ld, q, None) == status
    assert L.pvq_fp8_dequantize(q, p, dtype, ld, None) == status
    assert L.pvq_fp8_matmul(q, w, 0, p, dtype, ld, None, None) == status
    assert L.pvq_fp8_matmul(q, t, 1, p, dtype, ld, None, None) == status
    assert L.pvq_fp8_gated(p, ld, P, 256, dtype, 0, q, None, None, None) == status
    assert L.pvq_fp8_gated_backward(p, ld, dtype, q, q, 0, P, 256, P, 256, None) == status
    assert L.pvq_fp8_weight_grad(P, 64, 64, q, p, dtype, ld, None, 0, None, None) == status
    if dtype == 1:
        assert L.pvq_fp8_gated(P, 256, p, ld, dtype, 0, q, None, None, None) == status
        assert L.pvq_fp8_gated_backward(P, 256, dtype, q, q, 0, p, ld, P, 256, None) == status
        assert L.pvq_fp8_gated_backward(P, 256, dtype, q, q, 0, P, 256, p, ld, None) == status
        assert L.pvq_fp8_weight_grad(p, 256, ld, q, P, dtype, 256, None, 0, None, None) == status


def test_what_does_not_fit_together_is_refused():
    L = pvq.lib()
    q, t = C.byref(desc()), C.byref(desc(tile=1))
    other = C.byref(desc(rows=5))
    assert L.pvq_fp8_matmul(q, C.byref(desc(cols=250)), 0, P, 1, 8, None, None) == INVALID
    assert L.pvq_fp8_matmul(q, t, 1, P, 1, 256, None, None) == INVALID                       # 256 columns, 4 rows
    assert L.pvq_fp8_matmul(q, q, 2, P, 1, 8, None, None) == INVALID
    assert L.pvq_fp8_matmul(q, C.byref(desc(rows=256)), 1, P, 1, 256, None, None) == UNSUPPORTED   # scales by rows
    for act in (-1, 2):
        assert L.pvq_fp8_gated(P, 256, P, 256, 1, act, q, None, None, None) == INVALID
        assert L.pvq_fp8_gated_backward(P, 256, 1, q, q, act, P, 256, P, 256, None) == INVALID
    for args in ((t, None, None), (q, t, q), (q, q, t), (q, q, None), (q, None, q), (q, other, q), (q, q, other)):
        assert L.pvq_fp8_gated(P, 256, P, 256, 1, 0, *args, None) == INVALID
    for args in ((t, t), (q, t), (q, other), (other, q)):
        assert L.pvq_fp8_gated_backward(P, 256, 1, *args, 0, P, 256, P, 256, None) == INVALID
    assert L.pvq_fp8_weight_grad(P, 0, 64, q, P, 0, 256, None, 0, None, None) == INVALID
    big = C.byref(desc(rows=4096, cols=4096, ld_codes=4096, ld_scales=32))
    need = L.pvq_fp8_weight_grad_workspace(4096, 4096, 4096)
    assert need == 4096 * 4096 * 2
    assert L.pvq_fp8_weight_grad(P, 4096, 4096, big, P, 0, 4096, P, need - 1, None, None) == 4
    assert L.pvq_fp8_weight_grad(P, 4096, 4096, big, P, 0, 4096, P + 8, need, None, None) == ALIGN
    assert [L.pvq_fp8_weight_grad_workspace(*a) for a in ((0, 4096, 4096), (4096, 0, 4096), (4096, 4096, 0), (1, 1, 1))] == [0, 0, 0, 0]
    assert L.pvq_fp8_weight_grad(P, 1 << 31, 1 << 31, q, P, 0, 256, None, 0, None, None) == UNSUPPORTED


def test_scale_row_stride():
    L = pvq.lib()
    assert [L.pvq_fp8_scale_row_stride(c) for c in (-1, 0, 1, 128, 129, 512, 513, 14336)] == [0, 0, 4, 4, 4, 4, 8, 112]


def test_the_binding_refuses_what_is_not_on_the_gpu_or_of_another_type():
    x = torch.zeros(4, 128)
    codes, scales = torch.zeros(4, 128, dtype=torch.uint8), torch.zeros(4, 1, dtype=torch.uint8)
    q = pvq.Fp8Matrix(codes.view(torch.float8_e4m3fn), scales.view(torch.float8_e8m0fnu), False)
    for call in (lambda: pvq.fp8_quantize(x), lambda: pvq.fp8_dequantize(q), lambda: pvq.fp8_matmul(q, q), lambda: pvq.fp8_gated(x, x),
                 lambda: pvq.fp8_gated_backward(x, q, q), lambda: pvq.fp8_weight_grad(x.bfloat16(), q)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        pvq.fp8_quantize(x.double())
    with pytest.raises(TypeError):
        pvq.fp8_quantize(3)
    with pytest.raises(TypeError):
        pvq.fp8_matmul(q, q, dtype=torch.float16)
    with pytest.raises(ValueError):
        pvq.fp8_gated(x, x, act="relu")
    with pytest.raises(ValueError):
        pvq.fp8_gated_backward(x, q._replace(tile=True), q)
    with pytest.raises(ValueError):
        pvq.fp8_quantize(x, tile=True, out=q)


def test_the_reference_rounds_as_the_format_says():
    v = np.concatenate([np.linspace(-448, 448, 9001), np.ldexp(1.0, -np.arange(4, 14)), -np.ldexp(3.0, -np.arange(8, 14)), [0.0]])
    assert np.array_equal(ref.e4m3(v), ref.to64(torch.from_numpy(v).to(torch.float32).to(torch.float8_e4m3fn)))
    assert list(ref.scale_bytes(np.array([0.0, 448.0, 449.0, 224.0, 225.0, 1.0, 2.0 ** -149, 3e38]))) == [127, 127, 128, 126, 127, 119, 1, 247]


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_the_slopes_are_those_of_the_activations(act):
    g = np.linspace(-12, 12, 4001)
    e = 1e-5
    diff = (ref.activation(g + e, act) - ref.activation(g - e, act)) / (2 * e)
    # a central difference is off by e^2 / 6 times the third derivative (below 2), and by the values' roundings over e
    assert np.all(np.abs(diff - ref.slope(g, act)) < 1e-10 + 12 * 2.0 ** -52 / e)
    # and the activations those of include/pvq.h
    as_stated = g / (1 + np.exp(-g)) if act == "silu" else g * (1 + np.tanh(np.sqrt(2 / np.pi) * (g + 0.044715 * g ** 3))) / 2
    assert np.allclose(ref.activation(g, act), as_stated, rtol=1e-12, atol=1e-14)
