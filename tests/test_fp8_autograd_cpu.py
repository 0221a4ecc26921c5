"""The 8-bit floating-point calls record nothing for autograd, and say so (the refusal comes before that of tensors off the GPU)."""
import pytest
import torch

from paper_2410_16926_b200 import pvq


def calls():
    x = torch.zeros(4, 128)
    leaf = torch.zeros(4, 128, requires_grad=True)
    q = pvq.Fp8Matrix(torch.zeros(4, 128, dtype=torch.uint8).view(torch.float8_e4m3fn), torch.zeros(4, 1, dtype=torch.uint8).view(torch.float8_e8m0fnu), False)
    codes = leaf.to(torch.float8_e4m3fn)
    assert codes.requires_grad
    of_leaf = q._replace(codes=codes)
    return [lambda: pvq.fp8_quantize(leaf), lambda: pvq.fp8_quantize(leaf * 2), lambda: pvq.fp8_dequantize(of_leaf), lambda: pvq.fp8_matmul(of_leaf, q),
            lambda: pvq.fp8_gated(leaf, x), lambda: pvq.fp8_gated_backward(leaf, q, q), lambda: pvq.fp8_weight_grad(leaf.bfloat16(), q)]


@pytest.mark.parametrize("i", range(7))
def test_what_requires_a_gradient_is_refused(i):
    call = calls()[i]
    with pytest.raises(ValueError, match="requires a gradient"):
        call()
    with torch.no_grad(), pytest.raises(ValueError, match="CUDA"):
        call()
