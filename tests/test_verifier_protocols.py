"""What the verifier's kernels rely on between warps and thread blocks, checked on the CPU against their source: faults of this kind show
themselves by chance or not at all when they run."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_20375_b200", "csrc")


def _kernel(source, name):
    """The text of a kernel without comments, from its name to the closing brace in the first column."""
    with open(os.path.join(CSRC, source)) as f:
        text = f.read()
    text = text[re.search(r"__global__[^;{]*\b" + name + r"\(", text).start():]
    return re.sub(r"//[^\n]*", "", text[:text.index("\n}\n")])


def test_the_walk_writes_to_other_blocks_once_they_have_begun():
    """Shared memory of another block of the cluster may be written when that block is known to run: every thread arrives at the cluster's
    barrier and waits for all before its first exchange.  The arrival comes before anything that takes time, so that the wait is short."""
    k = _kernel("verify.cu", "verify_kernel")
    first = re.search(r"\bexchange\((?!uint64_t)", k).start()  # (behind the definition of the lambda)
    arrive, wait = (k.find(f"barrier.cluster.{x}") for x in ("arrive", "wait"))
    assert 0 <= arrive < k.index("pdl_wait()") < wait < first
    # neither stands in a branch: the braces around them are the kernel's own
    for at in (arrive, wait):
        assert k[:at].count("{") - k[:at].count("}") == 1 + k[:at].count("namespace {")
