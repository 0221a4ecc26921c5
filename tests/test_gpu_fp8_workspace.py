"""The weight gradient's workspace as seen from Python: it can be declined, and where there is no memory for it the call goes on."""
import pytest
import torch

from paper_2410_16926_b200 import pvq

pytestmark = pytest.mark.gpu

ROWS, INNER, OUTER = 8192, 4096, 2048
WORKSPACE = 2 * ROWS * INNER


@pytest.fixture(scope="module")
def operands():
    g = torch.Generator(device="cuda").manual_seed(1)
    dy = torch.randn((ROWS, OUTER), generator=g, device="cuda", dtype=torch.bfloat16)
    return dy, pvq.fp8_quantize(torch.randn((ROWS, INNER), generator=g, device="cuda", dtype=torch.bfloat16))


def most(call):
    """What a call holds at most beyond what is held already."""
    torch.cuda.synchronize()
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    result = call()
    return result, torch.cuda.max_memory_allocated() - before


def test_declined(operands):
    dy, x = operands
    assert pvq.lib().pvq_fp8_weight_grad_workspace(ROWS, INNER, OUTER) == WORKSPACE
    out = torch.empty((OUTER, INNER), device="cuda")
    with_it, held = most(lambda: pvq.fp8_weight_grad(dy, x))
    assert held >= WORKSPACE + out.numel() * 4
    got, held = most(lambda: pvq.fp8_weight_grad(dy, x, out=out, workspace=False))
    assert held == 0 and got is out and torch.equal(out, with_it)


def test_no_memory_for_it(operands):
    dy, x = operands
    want = pvq.fp8_weight_grad(dy, x)
    out = torch.empty_like(want)
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    total = torch.cuda.mem_get_info()[1]
    torch.cuda.set_per_process_memory_fraction((torch.cuda.memory_reserved() + (4 << 20)) / total)
    try:
        with pytest.raises(torch.OutOfMemoryError):
            torch.empty(WORKSPACE, dtype=torch.uint8, device="cuda")
        pvq.fp8_weight_grad(dy, x, out=out)
    finally:
        torch.cuda.set_per_process_memory_fraction(1.0)
    assert torch.equal(out, want)
