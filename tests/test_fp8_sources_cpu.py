"""What can be seen of the 8-bit operators' kernels in their sources alone: the scopes of what blocks of a cluster tell one another."""
import os
import re

SOURCES = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2410_16926_b200", "csrc", "fp8")


def text(name):
    with open(os.path.join(SOURCES, name)) as f:
        return f.read()


def test_what_is_told_another_block_has_the_clusters_scope():
    """An arrival or a wait without a scope has the block's own: what was done before it need not be seen by another block.  What is
    handed over besides tensor memory (for which there are fences of its own) is the block's shared memory, released in front of
    the arrival."""
    found = [i for name in sorted(os.listdir(SOURCES)) for i in re.findall(r"mbarrier\.arrive[.\w:]*", text(name)) if "shared::cluster" in i]
    assert found and all(".relaxed.cluster" in i or ".release.cluster" in i for i in found), found
    for line, before in ((l, p) for name in ("fp8_matmul_many.cu", "fp8_weight_grad.cu") for p, l in zip(text(name).splitlines(), text(name).splitlines()[1:])):
        if "barrier_arrive_in(full_there + 8 * c)" in line:  # a converted stage
            assert "release_shared();" in before
    assert "release_shared();" in text("fp8_weight_grad.cu")


def test_a_pairs_waits_acquire_from_the_cluster():
    """In the kernels of pairs of blocks, every wait but that for copies that the block alone asked for; and both kinds of wait can."""
    mma = text("fp8_mma.cuh")
    for wait in ("try_wait", "test_wait"):
        assert len(re.findall(r"mbarrier\.%s\.parity\.relaxed\.cluster[^;]*;\\n\\t\"\s*\"fence\.acquire\.sync_restrict::shared::cluster\.cluster" % wait, mma)) == 1
    call = re.compile(r"\b(?:barrier_wait|warp_wait|barrier_passed|barrier_over)(<\w+>)?\((\w+)")
    many = call.findall(text("fp8_matmul_many.cu"))
    assert many and not [bar for scope, bar in many if not scope]
    grad = call.findall(text("fp8_weight_grad.cu"))
    assert grad and {bar for scope, bar in grad if not scope} == {"full_x"}
    assert {scope for scope, _ in many if scope} == {"<true>"} and {scope for scope, _ in grad if scope} == {"<PAIR>"}
