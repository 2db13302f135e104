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


def test_what_is_an_item_away_is_waited_for():
    """The planning warp waits through a whole item, and so do warps of a tile without rows beside a
    long one, for its next item and that one's scores.  2^31 - 1 keys are 2^24 steps of about 2,100
    clocks, so two seconds would end calls that are only long."""
    text = source()
    clocks = int(re.search(r"kStepClocks = (\d+)", text).group(1))
    assert clocks >= 20000
    assert "kItemPatience = kPatience + ((1ll << 31) / kKeys) * kStepClocks" in text
    for bar in ("item_full[at]", "begun", "s_full[t]"):
        waits = [text[m.start() - 20:m.start()] for m in re.finditer(re.escape(f"(smem_addr(&sh.{bar})"), text)]
        waits = [w for w in waits if re.search(r"wait(<\w+>)?$", w)]
        assert waits and all(w.endswith("wait<kItemPatience>") for w in waits), bar


def test_a_warp_decides_as_one():
    """Whether somebody has given up is read by each thread at its own time.  Threads of a warp that
    went different ways on it would wait for one another for ever, at the warp's barriers, shuffles
    and TMEM accesses: only the wait itself, and the end of the block, look at it thread by thread."""
    text = source()
    kernel = text[text.index("struct Items {"):]
    alone = [line.strip() for line in kernel.splitlines() if "*late" in line and "volatile int*" not in line]
    assert alone == ["if (*late) {", "if (lane == 0 && *late) flag_status(a.status, NETKV_DEV_ETIMEOUT);"]
    given_up = text[text.index("bool given_up("):]
    assert "__any_sync(~0u, *late)" in given_up[:given_up.index("\n}\n")]
    assert kernel.count("given_up(late)") == 5  # the next item, queries, keys and values, twice the plan


def test_no_loads_after_a_wait_has_run_out():
    """A ring's place may still be in use then, and its barrier takes no arrival before its turn: every
    load is behind a look at the flag that comes after the wait for its place."""
    text = source()
    load = text[text.index("items.next(sh, late)", text.index("uint32_t i = 0, cleared = 0")):]
    load = load[:load.index("warp == kSoftmaxWarps + 1")]
    for empty, expect in (("q_empty", "bar_expect(smem_addr(&sh.q_full)"), ("kv_empty[st]", "bar_expect(bar,")):
        wait = load.index(f"wait(smem_addr(&sh.{empty})")
        assert "given_up(late)" in load[wait:load.index(expect, wait)]
