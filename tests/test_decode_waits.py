"""Waits of decode attention's kernels, by reading their source: what a missing one does depends on
the schedule, and a run whose waits run out is not for a GPU that others use."""
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def body(name):
    """The text of a function, from its name to its closing brace, without comments."""
    with open(os.path.join(ROOT, "paper_2606_03910_gb300", "csrc", "attn_decode.cu")) as f:
        text = re.sub(r"//[^\n]*", "", f.read())
    at = text.index(f" {name}(")
    return text[at:text.index("\n}\n", at)]


@pytest.mark.parametrize("kernel", ["join_kernel", "mass_kernel"])
def test_kernels_that_start_early_wait_before_they_end(kernel):
    """A grid that started before the one ahead of it in the stream was done, and of which no thread
    waits for that one, may itself be done first: what follows in the stream would then read outputs
    that are still being written.  So nothing returns before the wait, but for blocks that always
    have another beside them that does not."""
    before = re.split(r"(?<!let_)follow\(\);", body(kernel))
    assert len(before) == 2
    assert all(line.strip().startswith("if (blockIdx.y && ")
               for line in before[0].splitlines() if "return;" in line)


def test_giving_up_is_said_and_copies_land():
    """A wait that runs out sets the status itself: the thread that would say it for the block may
    have ended.  Nobody waits after that, the loading warp starts no further copies (a ring's place may
    still be in use, and a barrier takes no arrival before its turn), and the block stays until those
    in flight have had time to land in its shared memory."""
    wait = body("wait")
    gives_up = wait[wait.index("*late = 1"):]
    assert "flag_status(status, NETKV_DEV_ETIMEOUT)" in gives_up
    assert re.search(r"if \(\*late\) return;", wait)
    load = body("load_pages")
    loop = load[load.index("while ("):]
    assert "*late" in loop[:loop.index("{")]
    issue = loop[loop.index("wait("):]
    assert issue.index("if (!*late)") < issue.index("cp.async.bulk")
    kernel = body("decode_kernel")
    ends = [m.start() for m in re.finditer(r"return;", kernel)] + [len(kernel)]
    for end in ends:
        assert "settle(late);" in kernel[max(0, end - 60):end]
