"""Copies or scales of the 8-bit products and weight gradients that never arrive: every wait is bounded, the call ends, its status word says so,
what was not computed is NaN, nothing else is written, and the same call goes through afterwards.  On the bounds-checked build (in a child
process), which leaves them out where the status word asks for it, some stages into the call, and then waits for a short while only."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CHILD = """
import sys, time
import torch
from paper_2410_16926_b200 import pvq
op, rows, inner, outer, transposed, dtype, workspace = eval(sys.argv[1])
COPIES, SECOND, SCALES = -2 ** 31, 1 << 30, 1 << 29
dtype = torch.bfloat16 if dtype == "bf16" else torch.float32
g = torch.Generator(device="cuda").manual_seed(1)
make = lambda r, c, t: torch.randn((r, -(-c // 16) * 16), generator=g, device="cuda", dtype=t)[:, :c]
L = pvq.lib()
if op == "matmul":
    a = pvq.fp8_quantize(make(rows, inner, torch.bfloat16))
    b = pvq.fp8_quantize(make(*((inner, outer) if transposed else (outer, inner)), torch.bfloat16), tile=True)
    shape = (rows, outer)
    call = lambda out, status: pvq.fp8_matmul(a, b, transposed=transposed, dtype=dtype, out=out, status=status)
else:
    dy, x = make(rows, outer, torch.bfloat16), pvq.fp8_quantize(make(rows, inner, torch.bfloat16))
    assert (L.pvq_fp8_weight_grad_workspace(rows, inner, outer) > 0) == workspace
    shape = (outer, inner)
    call = lambda out, status: pvq.fp8_weight_grad(dy, x, dtype=dtype, out=out, status=status)
whole = torch.empty((shape[0] + 2, -(-shape[1] // 8) * 8 + 16), device="cuda", dtype=dtype)
out = whole[1:-1, :shape[1]]
def run(bits):
    status = torch.full((1,), bits, dtype=torch.int32, device="cuda")
    whole.fill_(77.0)
    torch.cuda.synchronize()
    began = time.time()
    call(out, status)
    torch.cuda.synchronize()
    took = time.time() - began
    got = out.clone()
    out.fill_(77.0)
    assert bool((whole == 77.0).all()), "written outside"
    return got, int(status.item()) & 0xffffffff, took
want, status, _ = run(0)
assert status == 0 and bool(torch.isfinite(want).all())
for name, bits in (("copies", COPIES), ("second", SECOND), ("scales", SCALES)):
    got, status, took = run(bits)
    bits &= 0xffffffff
    lost = torch.isnan(got)
    assert bool((lost | (got == want)).all()), (name, "neither right nor NaN")
    over = status != bits
    assert status == (bits | pvq.STATUS_STAGING_TIMEOUT if over else bits) and over == bool(lost.any()), (name, hex(status))
    print("RESULT", name, "over" if over else "through", "%.3f of the values lost, %.3f s" % (float(lost.float().mean()), took))
    assert took < 5.0
    again, status, _ = run(0)
    assert status == 0 and torch.equal(again, want), (name, "the next call")
print("done")
"""

BF16, F32 = "bf16", "f32"
# what ends early when copies, those of every second block of a cluster, or scales are left out
ALL, ONE_BLOCK, NO_SCALES = ("copies", "second", "scales"), ("copies", "scales"), ("copies", "second")


def run_child(case, ends):
    from paper_2410_16926_b200 import build
    env = dict(os.environ, PVQ_B200_LIB=build.build(debug=True), PYTHONPATH=ROOT)
    r = subprocess.run([sys.executable, "-c", CHILD, repr(case)], cwd=ROOT, env=env, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "done" in r.stdout, (r.stdout + r.stderr)[-3000:]
    print(r.stdout)
    over = tuple(line.split()[1] for line in r.stdout.splitlines() if line.startswith("RESULT") and line.split()[2] == "over")
    assert over == ends, r.stdout


@pytest.mark.parametrize("rows,inner,outer,transposed,dtype,ends", [
    (3, 14336, 300, False, BF16, ALL), (16, 14336, 4096, True, F32, ALL), (3, 4096, 16384, False, F32, ONE_BLOCK), (20, 14336, 2000, False, F32, ALL),
    (40, 28672, 1000, True, BF16, ALL), (64, 14336, 4096, False, BF16, ALL), (100, 14336, 515, False, F32, ALL), (128, 4096, 18000, True, BF16, ONE_BLOCK)])
def test_few_rows(rows, inner, outer, transposed, dtype, ends):
    run_child(("matmul", rows, inner, outer, transposed, dtype, None), ends)


@pytest.mark.parametrize("rows,inner,outer,transposed,dtype", [
    (1300, 2560, 2100, False, BF16), (1300, 2560, 2100, True, F32), (5000, 300, 5003, False, BF16), (5000, 300, 5003, False, F32), (2000, 20000, 4000, False, F32)])
def test_many_rows(rows, inner, outer, transposed, dtype):
    run_child(("matmul", rows, inner, outer, transposed, dtype, None), ALL)


@pytest.mark.parametrize("rows,inner,outer,dtype,workspace,ends", [
    (1001, 4096, 1024, BF16, False, ALL), (200, 5003, 5001, F32, False, ALL), (2000, 4096, 4096, F32, True, NO_SCALES), (500, 5003, 5001, BF16, True, NO_SCALES),
    (2100, 2500, 2100, F32, True, ALL), (700, 1500, 1500, BF16, False, ONE_BLOCK), (16384, 512, 500, F32, False, ALL), (4096, 300, 512, BF16, False, ALL)])
def test_weight_grad(rows, inner, outer, dtype, workspace, ends):
    run_child(("weight_grad", rows, inner, outer, None, dtype, workspace), ends)
