"""Bounded waits of the prompt kernel, by reading its source: a run whose waits run out is not for a
GPU that others use, so what ends such a run is checked where it stands."""
import os
import re

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def source():
    with open(os.path.join(ROOT, "paper_2606_03910_gb300", "csrc", "attn_prompt.cu")) as f:
        return re.sub(r"//[^\n]*", "", f.read())


def softmax_branch():
    text = source()
    at = text.index('asm volatile("setmaxnreg.inc')
    return text[at:text.index("using Encode")]


def test_softmax_warps_meet_for_a_limited_time():
    """The softmax warps meet inside an item.  After a wait has run out each warp is told "no more
    items" whenever it asks, so some may be in an item and some have left: where they meet is a
    wait with a limit like the others, not a barrier of a number of threads."""
    text, body = source(), softmax_branch()
    assert not re.search(r"bar(rier)?\.(cta\.)?(sync|red)", text)
    meet = body[body.index("auto meet ="):]
    assert "wait(smem_addr(&sh.met), " in meet[:meet.index("};")]
    # only where every warp of the block ends do they all come together
    assert text.count("__syncthreads()") == 2
    assert text.index("__syncthreads()", text.index("__syncthreads()") + 1) > text.index("meet();")
