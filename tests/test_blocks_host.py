"""The block pool's host side: what it refuses before any GPU work.  Pools on the CPU: no GPU here."""
import pytest

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def blocks():
    import __graft_entry__
    __graft_entry__.build()
    from paper_2606_03910_gb300 import blocks
    return blocks


def make(blocks, slots=3, pages=12, heads=2, dim=64, width=5, fmt="int8"):
    return blocks.BlockPool(pages, heads, dim, slots, width, fmt, device="cpu")


def state(pool):
    return list(pool.free), [list(p) for p in pool.page_of], list(pool.tokens), pool.table.tolist()


@pytest.mark.parametrize("other", [dict(heads=1), dict(heads=4), dict(dim=128), dict(fmt="e4m3"),
                                   dict(heads=1, dim=128)])
def test_move_between_unlike_pools(blocks, other):
    """Pages of another shape or format are neither written nor taken."""
    src, dst = make(blocks), make(blocks, **other)
    src.reserve([40, 0, 0])
    src.tokens[0] = 40
    before = state(dst)
    with pytest.raises(ValueError):
        blocks.move(src, 0, dst, 1)
    assert state(dst) == before


def rows(n, heads=2, dim=64):
    return torch.zeros((n, heads, dim), dtype=torch.float16)


def test_a_refused_append_changes_nothing(blocks):
    """Whatever the call behind it refuses (here: tensors of the host), the pool's pages are as before."""
    pool = make(blocks)
    pool.reserve([20, 0, 1])
    before = state(pool)
    for counts in ([30, 5, 0], [0, 0, 40]):
        with pytest.raises(TypeError):
            pool.append(rows(sum(counts)), rows(sum(counts)), counts)
        now = state(pool)
        assert now[:3] == before[:3] and sorted(now[0] + sum(now[1], [])) == list(range(12))
        assert [row[:len(p)] for row, p in zip(now[3], now[1])] == now[1]


@pytest.mark.parametrize("counts", [[16], [16, 16, 16, 16], [-1, 16, 16], [16, 16, 17], [1.5, 0, 0]])
def test_counts_that_do_not_fit(blocks, counts):
    """One count a slot, none below 0, and rows for all of them."""
    pool = make(blocks)
    before = state(pool)
    for call in (lambda: pool.append(rows(48), rows(48), counts),
                 lambda: pool.append(rows(64), rows(48), counts),
                 lambda: pool.read(rows(48), rows(48), counts)):
        with pytest.raises(ValueError):
            call()
        assert state(pool) == before
    if sum(counts) != 49:
        with pytest.raises(ValueError):
            pool.reserve(counts)
    assert state(pool) == before


def test_reserve_when_one_slot_has_more_than_it_needs(blocks):
    """Pages that a slot holds in advance are not another's."""
    pool = make(blocks)
    pool.reserve([80, 0, 0])
    with pytest.raises(MemoryError):
        pool.reserve([0, 80, 80])
    assert len(pool.free) == 7 and [len(p) for p in pool.page_of] == [5, 0, 0]
    pool.reserve([16, 80, 32])
    assert len(pool.free) == 0 and [len(p) for p in pool.page_of] == [5, 5, 2]


def test_move_of_a_slot_with_pages_in_advance(blocks, monkeypatch):
    """Pages that a slot holds beyond its tokens are neither copied nor counted, on either side, and a
    move that fails leaves the destination's pages as they were."""
    src, dst = make(blocks), make(blocks)
    src.reserve([60, 0, 0])
    src.tokens[0] = 20
    dst.reserve([0, 70, 0])
    copies = []
    monkeypatch.setattr(blocks.netkv, "netkv_copy_group_async", copies.extend)
    assert blocks.move(src, 0, dst, 1) == 2 * 2 * 2 * (16 * 64 + 4)
    assert len(copies) == 4 and dst.tokens == [0, 20, 0] and len(dst.page_of[1]) == 5

    def fail(copies):
        raise RuntimeError
    monkeypatch.setattr(blocks.netkv, "netkv_copy_group_async", fail)
    before = state(dst)
    with pytest.raises(RuntimeError):
        blocks.move(src, 0, dst, 2)
    assert state(dst)[:3] == before[:3]
