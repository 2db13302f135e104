"""Bounded waits of the chunk kernel, by reading its source: a run whose waits run out is not for a GPU
that others use, so what ends such a run is checked where it stands."""
import os
import re

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def source():
    with open(os.path.join(ROOT, "paper_2606_03910_gb300", "csrc", "attn_chunk.cu")) as f:
        return re.sub(r"//[^\n]*", "", f.read())


def test_no_barrier_but_at_the_ends():
    """Warps that were told "no more items" after a wait has run out leave; where the others meet is a
    wait with a limit.  All come together only at the beginning and at the end."""
    text = source()
    assert not re.search(r"bar(rier)?\.(cta\.)?(sync|red)", text)
    kernel = text[text.index(" chunk_kernel("):text.index(" join_kernel(")]
    assert text.count("__syncthreads()") == kernel.count("__syncthreads()") == 2
    meet = text[text.index("auto meet ="):]
    assert "wait(AT(met), " in meet[:meet.index("};")]


def test_every_wait_is_limited():
    """The only look at a barrier that may not end is in wait(), which ends on the flag and on a limit,
    and says whether it has ended by itself."""
    text = source()
    wait = text[text.index("bool wait("):]
    wait = wait[:wait.index("\n}\n")]
    assert "if (*late) return false;" in wait and "clock64() - t0 > kLimit" in wait and "*late = 1;" in wait
    rest = text.replace(wait, "")
    assert "try_wait" not in rest and "while (true)" in rest
    clocks = int(re.search(r"kStepClocks = (\d+)", text).group(1))
    assert clocks >= 20000 and "kItemPatience = kPatience + ((1ll << 32) / kKeys) * kStepClocks" in text
    for bar in ("item_full[at]", "item_full[n % kItems]", "item_empty[n % kItems]"):
        waits = [text[m.start() - 20:m.start()] for m in re.finditer(re.escape(f"(AT({bar})"), text)]
        waits = [w for w in waits if re.search(r"wait(<\w+>)?$", w)]
        assert waits and all(w.endswith("wait<kItemPatience>") for w in waits), bar


def test_loops_over_items_end():
    """Each role's loop ends when an item is not valid, which next() and see() say after a wait has run
    out, and the planning warp's on the flag itself."""
    text = source()
    items = text[text.index("struct Items {"):text.index("struct Batches {")]
    assert items.count("given_up(late)") == 2
    for role in ("read_pages", "copy_values", "widen_tiles", "multiply", "softmax"):
        body = text[text.index(f" {role}("):]
        body = body[:body.index("\n}\n")]
        assert re.search(r"if \(!x\.valid\) break;|if \(!item\) break;|over = !x\.valid;", body), role
    plan = text[text.index(" plan("):text.index(" read_pages(")]
    assert "while (at < end && !given_up(late))" in plan


def test_no_copies_after_a_wait_has_run_out():
    """A ring's place may still be in use then: a copy, and a tile's stores, come only behind a wait for
    the place that has ended, for the whole warp alike."""
    text = source()
    copy = text[text.index(" copy_tile("):]
    copy = copy[:copy.index("\n}\n")]
    assert copy.index("wait(AT(codes_empty[st])") < copy.index("if (!__all_sync(~0u, ok)) return false;") \
        < copy.index("store_shared(") < copy.index("bar_expect(") < copy.index("cp.async.bulk.shared")
    widen = text[text.index(" widen_tiles("):]
    widen = widen[:widen.index("\n}\n")]
    assert widen.index("wait(AT(kv_empty[st])") < widen.index("if (!__all_sync(~0u, ok)) break;") \
        < widen.index("store_shared(")
    end = text[text.rindex("__syncthreads()"):]
    assert end.index("if (*late)") < end.index("tcgen05.dealloc") and "20000000ll" in end


def test_the_join_waits_before_it_ends():
    """It starts while the kernel before it ends: were its blocks to return without waiting, what follows
    in the stream could read outputs that are still being written."""
    text = source()
    join = text[text.index(" join_kernel("):]
    assert join.index("griddepcontrol.wait") < join.index("return;")


def test_only_items_with_keys_are_looked_ahead_for():
    """The pages' warp asks for items ahead before it says what it has of the present one, and an item's
    place comes back when the softmax is done with it: items without keys between two with some would
    stand for ever between them.  The planning warp deals with those itself."""
    text = source()
    plan = text[text.index(" plan("):text.index(" read_pages(")]
    assert re.search(r"if \(x\.steps\) publish\(x\);\s*else nothing_seen<", plan)
    assert plan.count("publish(x);") == 2  # and the last one, that says there are no more
    assert int(re.search(r"kItems = (\d+)", text).group(1)) >= 4  # the present one, two ahead, one behind


def test_what_stands_after_a_wait_has_run_out_is_not_an_address():
    """The planning warp leaves an item's place that may be in use, and page numbers are looked at only
    after the flag: both become addresses."""
    text = source()
    publish = text[text.index("auto publish ="):]
    publish = publish[:publish.index("};")]
    assert publish.index("wait<kItemPatience>(") < publish.index("if (!__all_sync(~0u, ok)) return;") \
        < publish.index("sh.item[n % kItems] = x;")
    values = text[text.index(" copy_values("):]
    values = values[:values.index("\n}\n")]
    assert values.index(".page[lane]") < values.index("if (given_up(late)) return;") < values.index("copy_tile<")
