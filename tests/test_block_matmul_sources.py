"""Rules of the 8-bit product's kernels, checked on their text."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2511_13587_b200", "csrc")


def _code(name):
    with open(os.path.join(CSRC, name)) as f:
        return re.sub(r"//[^\n]*", "", f.read())


def test_every_launch_waits_for_those_before_it_and_then_reads():
    """What a launch before has written is visible behind the launch's own wait alone: it comes unconditionally, and ahead of every read."""
    for name in ("block_matmul.cu", "block_matmul_pair.cu"):
        code = _code(name)
        waits = [m.start() for m in re.finditer(r"pdl_wait\(\)", code)]
        assert len(waits) == 1 and re.search(r"[;{}]\s*$", code[:waits[0]]), name
        kernel = code[code.index("extern __shared__"):waits[0]]
        assert not re.search(r"tma_load|_scale\[|__ldg|p\.out\b", kernel), name
