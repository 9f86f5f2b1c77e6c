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


def test_the_pairs_producers_wait_for_the_last_stages_signals():
    """The MMAs of every stage signal a barrier in both CTAs; a producer waits there before it fills the stage again, and for the last fills of all
    before its CTA may leave."""
    code = _code("block_matmul_pair.cu")
    producer = code[code.index("Ring<kStages> st(1);"):code.index("else if (warp == 1)")]
    behind = producer[producer.index("st.next();"):]
    wait = re.search(r"for \(int i = max\(issued - kStages, 0\); i < issued && ok; \+\+i\) ok = warp_wait_or_abort\(&done_bar\[i % kStages\], "
                     r"\(i / kStages\) & 1, &s_abort\);", behind)
    assert wait and "rank" not in behind[:wait.start()]
    # the parity of fill i's completion, as the loop's ring has it when it waits for fill i ahead of fill i + kStages
    stages = int(re.search(r"kStages = (\d+)", code).group(1))
    at, par = 0, 1
    for fill in range(64):
        if fill >= stages:
            assert (at, par) == ((fill - stages) % stages, ((fill - stages) // stages) & 1)
        at += 1
        if at == stages:
            at, par = 0, par ^ 1


def test_loads_under_way_are_waited_for_whoever_gives_up():
    """The warp that waits for loads may give up when the one that asked for them has long been through: that one waits for its last fills in any case."""
    code = _code("block_matmul.cu")
    producer = code[code.index("if (warp == 0) {"):code.index("else if (warp == 1)")]
    depth, drained = 0, []
    for i, c in enumerate(producer):
        depth += (c == "{") - (c == "}")
        if producer.startswith("mbar_wait(&full_bar[i % stages], (i / stages) & 1)", i):
            drained.append(depth)
    assert drained == [1]                                     # the warp's own block: under no condition
    assert re.search(r"for \(int i = max\(issued - stages, 0\); i < issued; \+\+i\) mbar_wait", producer)
