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
