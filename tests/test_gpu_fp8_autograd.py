"""The 8-bit floating-point calls and autograd: refusals, a torch.autograd.Function made of them, outputs that count as changed."""
import pytest
import torch

from paper_2410_16926_b200 import pvq

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


def normal(rows, cols, seed):
    return torch.randn((rows, cols), generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda", dtype=BF16)


class Projection(torch.autograd.Function):
    """x times an 8-bit weight transposed, x kept in 8 bits for the weight's gradient."""

    @staticmethod
    def forward(ctx, x, weight):
        xq, wq = pvq.fp8_quantize(x), pvq.fp8_quantize(weight, tile=True)
        ctx.save_for_backward(*xq[:2], *wq[:2])
        return pvq.fp8_matmul(xq, wq)

    @staticmethod
    def backward(ctx, dy):
        x, sx, w, sw = ctx.saved_tensors
        dx = pvq.fp8_matmul(pvq.fp8_quantize(dy), pvq.Fp8Matrix(w, sw, True), transposed=True)
        return dx, pvq.fp8_weight_grad(dy, pvq.Fp8Matrix(x, sx, False), dtype=BF16)


def test_a_function_of_these_calls():
    x, w, dy = normal(100, 256, 1).requires_grad_(), normal(384, 256, 2).requires_grad_(), normal(100, 384, 3)
    Projection.apply(x, w).backward(dy)
    with torch.no_grad():
        xq, wq = pvq.fp8_quantize(x), pvq.fp8_quantize(w, tile=True)
        assert torch.equal(w.grad, pvq.fp8_weight_grad(dy, xq, dtype=BF16))
        assert torch.equal(x.grad, pvq.fp8_matmul(pvq.fp8_quantize(dy), wq, transposed=True))
    with pytest.raises(ValueError, match="requires a gradient"):
        pvq.fp8_quantize(x)
    assert torch.equal(pvq.fp8_quantize(x.detach()).codes.view(torch.uint8), xq.codes.view(torch.uint8))


def test_outputs_count_as_changed():
    x, dy = normal(40, 256, 4), normal(40, 128, 5)
    q, w = pvq.fp8_quantize(x), pvq.fp8_quantize(normal(128, 256, 6), tile=True)
    versions = [t._version for t in (x, *q[:2], *w[:2], dy)]
    empty = lambda r, c, t: torch.empty((r, c), device="cuda", dtype=t)  # noqa: E731
    codes, scales = empty(40, 256, torch.uint8), empty(40, 4, torch.uint8)
    dgate, dup = empty(40, 256, BF16), empty(40, 256, BF16)
    for outs, call in (([codes, scales], lambda: pvq.fp8_quantize(x, out=(codes.view(torch.float8_e4m3fn), scales[:, :2].view(torch.float8_e8m0fnu)))),
                       ([dgate], lambda: pvq.fp8_dequantize(q, out=dgate)),
                       ([dgate, dup], lambda: pvq.fp8_gated_backward(x, q, q, out=(dgate, dup))),
                       ([dgate[:, :128]], lambda: pvq.fp8_matmul(q, w, out=dgate[:, :128])),
                       ([dup[:128 // 4]], lambda: pvq.fp8_weight_grad(dy[:, :32], q, dtype=BF16, out=dup[:32]))):
        before = [o._version for o in outs]
        call()
        assert [o._version for o in outs] == [v + 1 for v in before]
    assert [t._version for t in (x, *q[:2], *w[:2], dy)] == versions
    # what was saved for a backward pass and then written into is noticed
    a = normal(40, 256, 7).requires_grad_()
    b = normal(40, 256, 8)
    y = (a * b).sum()
    pvq.fp8_dequantize(q, out=b)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()
    with torch.inference_mode():
        out = torch.empty((40, 256), device="cuda", dtype=BF16)
        pvq.fp8_dequantize(q, out=out)
    pvq.fp8_dequantize(q, out=out)


def test_an_output_that_requires_a_gradient_is_refused():
    q = pvq.fp8_quantize(normal(40, 256, 4))
    out = torch.empty((40, 256), device="cuda", dtype=BF16, requires_grad=True)
    with pytest.raises(ValueError, match="requires a gradient"):
        pvq.fp8_dequantize(q, out=out)
    with torch.no_grad():
        pvq.fp8_dequantize(q, out=out)
    assert torch.equal(out.detach(), pvq.fp8_dequantize(q))
