"""Copies of every second thread block alone that never arrive: of a cluster the other blocks' parts are there, and still a row is right or NaN as a whole,
whichever block adds its dims up."""
import os
import subprocess
import sys

import pytest
from test_gpu_fp8_cache_timeout import CHILD, ROOT

pytestmark = pytest.mark.gpu

SECOND = CHILD.replace("run(-2 ** 31)", "run(1 << 30)").replace("0x80000000 |", "0x40000000 |")


@pytest.mark.parametrize("heads,kv,n,length,seqs", [(4, 1, 1, 12000, 1), (16, 2, 1, 6000, 12), (8, 8, 1, 9000, 2), (30, 2, 1, 4000, 30), (4, 4, 1, 1500, 74),
                                                    (8, 2, 1, 200000, 1), (8, 2, 8, 4000, 40), (8, 2, 64, 4000, 20), (8, 2, 100, 40000, 1)])
def test_copies_of_every_second_block(heads, kv, n, length, seqs):
    from paper_2410_16926_b200 import build
    assert SECOND.count("1 << 30") == 1 and SECOND.count("0x40000000") == 1
    env = dict(os.environ, PVQ_B200_LIB=build.build(debug=True), PYTHONPATH=ROOT)
    r = subprocess.run([sys.executable, "-c", SECOND, repr((heads, kv, n, length, seqs))], cwd=ROOT, env=env, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "done" in r.stdout, (r.stdout + r.stderr)[-3000:]
