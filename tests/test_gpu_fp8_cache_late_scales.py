"""Scales of the 8-bit cache's pages that come late: nobody reads those of another tile in their place.  On the bounds-checked build (in a child
process), which holds back each tile's scales for a while, long after its keys are there, where the status word asks for it."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CHILD = """
import sys
import torch
from paper_2410_16926_b200 import pvq
heads, kv, n, length, seqs, causal = eval(sys.argv[1])
page, dim = 32, 64
per = -(-length // page)
g = torch.Generator(device="cuda").manual_seed(1)
rand = lambda *s: torch.randn(s, generator=g, device="cuda")
# every page a scale of its own
codes = [(rand(seqs * per, kv, page, dim) * 60).to(torch.float8_e4m3fn) for _ in range(2)]
scales = [torch.randint(127 - 12, 127 - 4, (seqs * per, kv), generator=g, device="cuda", dtype=torch.uint8).view(torch.float8_e8m0fnu) for _ in range(2)]
cache = pvq.Fp8Cache(*codes, *scales)
table = torch.arange(seqs * per, dtype=torch.int32, device="cuda").view(seqs, per)
lengths = torch.full((seqs,), length, dtype=torch.int32, device="cuda")
starts = torch.arange(seqs + 1, dtype=torch.int32, device="cuda") * n if n > 1 else None
q = rand(seqs * n, heads, dim).bfloat16()
LATE = 1 << 29
def run(bits):
    status = torch.full((1,), bits, dtype=torch.int32, device="cuda")
    out, lse = pvq.fp8_attention(q, cache, table, lengths, starts, causal=causal, lse=True, status=status)
    torch.cuda.synchronize()
    return out, lse, int(status.item())
want, want_lse, status = run(0)
assert status == 0 and bool(torch.isfinite(want).all())
for _ in range(3):
    out, lse, status = run(LATE)
    assert status == LATE, hex(status)
    assert torch.equal(out, want) and torch.equal(lse, want_lse), "%d rows differ" % int((out != want).any(dim=2).sum())
print("done")
"""


@pytest.mark.parametrize("heads,kv,n,length,seqs,causal", [
    (4, 4, 333, 1500, 12, False),   # items of 256 rows and of 77, in which one of the two tiles of rows has nothing to do
    (16, 16, 77, 1200, 20, True),   # ... in all items
    (8, 2, 100, 1023, 12, True),    # 256, 144: both tiles of rows work
    (2, 1, 400, 2000, 40, True),
    (8, 2, 1, 4000, 40, True), (32, 2, 2, 3000, 12, True), (4, 1, 1, 900, 1, True),  # few rows, shared by all blocks and in clusters
])
def test_scales_that_come_late(heads, kv, n, length, seqs, causal):
    from paper_2410_16926_b200 import build
    env = dict(os.environ, PVQ_B200_LIB=build.build(debug=True), PYTHONPATH=ROOT)
    r = subprocess.run([sys.executable, "-c", CHILD, repr((heads, kv, n, length, seqs, causal))], cwd=ROOT, env=env, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "done" in r.stdout, (r.stdout + r.stderr)[-3000:]
