"""How the chunk kernel's planning warp goes over sequences without new rows, by reading its source: other
warps wait for what it says next, so the way there may not grow with sequences that have nothing to do."""
from tests.test_chunk_waits import source


def test_idle_sequences_are_passed_together():
    """A run that has ended looks for no further sequence, and one that goes on finds it by a vote over a
    window of 32."""
    text = source()
    plan = text[text.index(" plan("):text.index(" read_pages(")]
    step = plan[plan.index("if (++kv_head < a.kv.heads) continue;"):plan.index("x.valid = 0;")]
    leave, vote = step.index("if (at >= end) break;"), step.index("__ballot_sync(~0u, mine.new_tokens != 0)")
    assert leave < vote < step.index("window(base + 32)") < step.index("pick(seq)")
    assert "++seq" not in step
