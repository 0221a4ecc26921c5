"""fp32 results of 8-bit products over sums of any length, whichever kernel makes them."""
import pytest
import torch

from paper_2410_16926_b200 import pvq

pytestmark = pytest.mark.gpu

F32 = torch.float32


def operands(rows, inner, outer, transposed, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    make = lambda r, c: torch.randn((r, -(-c // 16) * 16), generator=g, device="cuda")[:, :c]  # noqa: E731
    return pvq.fp8_quantize(make(rows, inner)), pvq.fp8_quantize(make(*((inner, outer) if transposed else (outer, inner))), tile=True)


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("rows,inner,outer", [(1, 65600, 130), (2, 200000, 130), (16, 131075, 300), (20, 128256, 264), (33, 262144, 128), (64, 200000, 200),
                                              (100, 150001, 520), (128, 128256, 1024)])
def test_few_rows(rows, inner, outer, transposed):
    """Sums in tensor memory lose 8e-8 of themselves for every 1024 values, 6.5e-7 over the 8192 of a run, and the runs of
    a part, at most 32 here, are added in fp32, 2^-24 of the sum each and of either sign: together below 1e-6."""
    a, b = operands(rows, inner, outer, transposed, inner)
    va, vb = (pvq.fp8_dequantize(q, dtype=F32).double() for q in (a, b))
    want = va @ (vb if transposed else vb.t())
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = pvq.fp8_matmul(a, b, transposed=transposed, dtype=F32, status=status)
    assert int(status.item()) == 0
    assert float((got.double() - want).norm()) <= 1e-6 * float(want.norm())
    assert torch.equal(pvq.fp8_matmul(a, b, transposed=transposed, dtype=F32), got)


def test_the_longest_sum():
    """2^31 - 100 values, ones and twos of either sign in places that are known: the sum is a whole number."""
    inner = 2 ** 31 - 100
    ld = -(-inner // 16) * 16
    codes = torch.zeros((3, ld), dtype=torch.uint8, device="cuda")
    scales = torch.full((3, 2 ** 24), 127, dtype=torch.uint8, device="cuda")
    places = torch.tensor([0, 127, 128, 2 ** 28 - 1, 2 ** 28, 2 ** 30 + 5, inner - 65, inner - 1], device="cuda")
    for row, code in ((0, 0x38), (1, 0x40), (2, 0xb8)):  # 1, 2, -1
        codes[row, places[row:]] = code
    codes[:, inner:] = 0x7e  # (behind the end: 448)
    q = pvq.Fp8Matrix(codes[:, :inner].view(torch.float8_e4m3fn), scales.view(torch.float8_e8m0fnu), False)
    want = torch.tensor([[8, 14, -6], [14, 28, -12], [-6, -12, 6]], dtype=F32, device="cuda")
    assert torch.equal(pvq.fp8_matmul(q, q, dtype=F32), want)
    assert torch.equal(pvq.fp8_matmul(q, q), want.bfloat16())
