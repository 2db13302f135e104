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


def test_softmax_warps_leave_together():
    """The softmax warps meet at barriers inside an item.  After a wait has run out each warp is told
    "no more items" whenever it asks, so whether to take an item is a vote of them all, and no
    warp leaves the loop, or skips the item, before it."""
    body = softmax_branch()
    taken = body.index("items.next(")
    vote = body.index("all_softmax(")
    assert taken < vote < body.index("break;") and vote < body.index("continue;")
    # every barrier of the branch stands behind the vote
    assert body.index("sync_softmax(") > vote
    # and the vote is a barrier of all eight warps
    text = source()
    vote = text[text.index("bool all_softmax("):]
    assert "bar.red.and.pred p, 1, 256, " in vote[:vote.index("\n}\n")]
